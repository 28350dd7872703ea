"""The keys of the draws of a layer in 8 bits, as far as the host sees them."""
import struct

import numpy as np
import pytest

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
