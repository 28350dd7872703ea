"""The keys of the draws of a layer in 8 bits, as far as the host sees them."""
import struct

import numpy as np
import pytest

import layer_reference as R
import paper_1610_02132_amd as q


def fields(d):
    return struct.unpack("=QIIIIQ", d.c())   # struct qsgd_draws


def test_fields_outside_their_words_wrap_as_in_params():
    """A seed or an iteration that a program counts down from 0, or past its word, names the same draws as in Params."""
    p = q.Params(n=1, s=1, d=1, seed=-1, stream_id=-2, iteration=2 ** 32 + 5).c()
    assert fields(q.Draws(seed=-1, stream_id=-2, iteration=2 ** 32 + 5, row_base=7)) == (p.seed, p.stream_id, p.iteration, 7, 0, 0)
    assert fields(q.Draws(seed=2 ** 64 + 3)) == (3, 0, 0, 0, 0, 0)
    assert fields(q.Draws(seed=np.int64(-1), iteration=np.int32(-1)))[0:3:2] == (2 ** 64 - 1, 2 ** 32 - 1)


@pytest.mark.parametrize("row_base", [-1, 2 ** 32, 2 ** 40])
def test_a_row_base_that_is_no_row_number_is_refused(row_base):
    with pytest.raises(ValueError, match="row_base"):
        q.Draws(row_base=row_base).c()
    assert fields(q.Draws(row_base=2 ** 32 - 1))[3] == 2 ** 32 - 1


def test_a_field_that_is_no_whole_number_is_refused():
    with pytest.raises(TypeError):
        q.Draws(seed=1.5).c()


@pytest.mark.parametrize("p", [0.1, 0.25, 0.5])
def test_one_name_for_dropout_and_levels_shifts_them(p):
    """Every draw there is, at every fraction of 256: kept elements that round by the mask's draw are p / 2 of a level too near to
    zero in the mean, those that round by draws of their own are not."""
    h = np.arange(65536)
    kept = h >= round(65536 * p)
    fraction = (np.arange(256) + 0.5) / 256
    up = (h + 0.5) / 65536 < fraction[:, None]
    same = (fraction - up[:, kept].mean(axis=1)).mean()      # the mask's draw once more
    apart = (fraction - up.mean(axis=1)).mean()
    assert abs(same - p / 2) < 1e-4 and abs(apart) < 2.0 ** -17


def blocks(seed, stream_id, iteration, rows, cols):
    """The generator's blocks that a call of the layer's operators takes."""
    return {(seed % 2 ** 64, b, r, stream_id % 2 ** 32, iteration) for r in range(rows) for b in range(-(-cols // 8))}


def test_the_headers_way_uses_no_block_twice():
    """Codec, dropouts and layers of several peers and steps; a dropout and its backward pass are one."""
    M, N, K, peers, layers, steps = 5, 24, 16, 6, 2, 3
    seen = set()

    def take(b):
        assert not seen & b
        seen.update(b)

    for step in range(steps):
        for peer in range(peers):
            for layer in range(layers):
                take(blocks(100 + layer, peer, step, M, N))                    # dropout
                take(blocks(200 + layer, 4 * peer + 3, step, M, K))            # x, forward
                for by, (rows, cols) in enumerate(((M, N), (N, K), (M, K))):   # dy, w, x, backward
                    take(blocks(200 + layer, 4 * peer + by, step, rows, cols))
                take({(300 + layer, i // 4, 0, peer, step) for i in range(N * K)})   # the codec, of a layer's gradient


def test_names_of_the_layers_gradients_wrap():
    """stream_id + 2 past its word is 0 or 1, for the reference's draws as for the library's."""
    d = q.Draws(seed=3, stream_id=2 ** 32 - 1)
    over = q.Draws(seed=3, stream_id=2 ** 32 + 1)
    assert (R.half_words(over, 2, 20) == R.half_words(q.Draws(seed=3, stream_id=1), 2, 20)).all()
    assert fields(d)[1] == 2 ** 32 - 1 and fields(over)[1] == 1
