"""The operators of a layer in 8 bits, as far as the host sees them: their draws' definition against the oracle's
generator, and properties of the kernels as they were built."""
import os

import numpy as np
import pytest

import layer_reference as R


@pytest.mark.parametrize("rows,cols,row_base", [(1, 1, 0), (3, 8, 0), (2, 21, 5), (4, 40, 2 ** 32 - 4)], ids=str)
def test_draws_are_blocks_of_the_oracles_generator(qo, rows, cols, row_base):
    from paper_1610_02132_amd import binding
    d = binding.Draws(seed=0xFEDCBA9876543210, stream_id=2 ** 32 - 1, iteration=9, row_base=row_base)
    got = R.half_words(d, rows, cols)
    for r in range(rows):
        for c in range(cols):
            block = qo.philox4x32_10([c // 8, row_base + r, d.stream_id, d.iteration], [d.seed & 0xFFFFFFFF, d.seed >> 32])
            word = int(block[c % 8 // 2])
            assert got[r, c] == (word >> 16 if c % 2 else word & 0xFFFF)


@pytest.mark.parametrize("p", [0.0, 0.1, 0.25, 1.0])
def test_share_of_dropped_draws(p):
    from paper_1610_02132_amd import binding
    h = R.half_words(binding.Draws(seed=3), 500, 400)
    share = float((h < np.rint(65536 * p)).mean())
    assert abs(share - p) <= 6 * np.sqrt(p * (1 - p) / h.size) + 2.0 ** -17


def test_kernels_keep_their_values_in_registers():
    from test_built_kernels import LIB, code_objects, kernels
    if not os.path.exists(LIB):
        pytest.skip("the library is not built")
    with open(LIB, "rb") as f:
        data = f.read()
    names = ("k_dropout", "k_quantize_rows", "k_quantize_columns", "k_product", "k_linear_few")
    seen = [(k[".name"], k[".private_segment_fixed_size"]) for elf in code_objects(data) for k in kernels(elf)
            if any(n in k[".name"] for n in names)]
    assert len(seen) >= 12 + 12 + 8 + 6
    assert not [s for s in seen if s[1]]
