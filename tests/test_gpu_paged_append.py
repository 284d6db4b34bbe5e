"""laga_cache_append of many tokens: a wave has one or two of them, by their number, and a token's row is the same."""
import numpy as np
import pytest
import torch

from test_gpu_paged_cache import WIDTHS, append_inputs, i32, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("widths,d_c,dtype", [("v3", 512, "bf16"), ("v3", 1024, "bf16"), ("half", 416, "bf16"), ("small", 32, "bf16"),
                                              ("v3", 512, "fp32"), ("small", 64, "fp32")])
@pytest.mark.parametrize("T", [4095, 4096, 4097, 4098, 12001])
def test_a_call_of_all_tokens_is_calls_of_some(widths, d_c, dtype, T):
    import paper_2607_17644_amd as L
    page, dr = 16, WIDTHS[widths][1]
    lat, kpe, gam = append_inputs(T, d_c, dr, dtype, T, True)
    rng = np.random.default_rng(T)
    n_pages = -(-T // page) + 2
    slot = rng.permutation(n_pages * page)[:T]
    slot[5::17], slot[6::19] = -1, n_pages * page
    slot, position = i32(slot), i32(rng.integers(0, 200000, T))
    one, all_ = (torch.full((n_pages, page, d_c + dr), 7.0, dtype=lat.dtype, device="cuda") for _ in range(2))
    L.laga_cache_append(problem(T, 1, 16384, n_pages, page, widths, d_c, dtype), lat, kpe, position, slot, all_, gamma=gam)
    for i in range(0, T, 1000):
        j = min(T, i + 1000)
        L.laga_cache_append(problem(j - i, 1, 16384, n_pages, page, widths, d_c, dtype), lat[i:j], kpe[i:j], position[i:j].clone(),
                            slot[i:j].clone(), one, gamma=gam)
    torch.cuda.synchronize()
    assert torch.equal(one, all_) and one.isfinite().all() and (one != 7.0).any()
