"""The scratch of saki_paged_attention, on the host: what the kernels that may serve a call can write, no more."""
import ctypes as C

import pytest

from paper_2609_36601_b200 import binding


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("Q,G", [(1, 1), (1, 4), (1, 17), (4, 8), (7, 4), (8, 8), (17, 8), (32, 64)])
@pytest.mark.parametrize("D", [8, 64, 80, 96, 128, 136, 256])
def test_two_partial_results_for_every_row_of_a_block_on_each_sm(dtype, Q, G, D):
    i = binding.SakiAttnIn()
    i.B, i.Q, i.Hq, i.H, i.D, i.page_size, i.max_pages, i.n_pages, i.dtype, i.ld_table, i.scale = 64, Q, 2 * G, 2, D, 16, 400, 32, dtype, 400, 0.125
    got = binding.load_library().saki_paged_attention_scratch_bytes(C.byref(i))
    wide = 64 if D <= 64 else 128 if D <= 128 else 256           # columns, as the kernels round them up (float32 heads of 65 to 96: 96)
    rows = 128                                                   # eight warps of 16 rows
    assert 148 * 2 * 16 * (D + 2) * 4 <= got <= 148 * 2 * rows * (wide + 2) * 4 + (64 << 10)
