"""laga_paged_attn where one worker's share of a row reaches past the page ids that it holds at a time: pages of one
key, and a few, under rows so long that a share has more than 512 of them."""
import pytest
import torch

from test_gpu_paged_attn import call, make
from test_gpu_paged_precision import exact

pytestmark = pytest.mark.gpu


# Shares of more than 16 tiles of 32 keys: 256 workers, 512 with d_c up to 256, per 32 heads (64 at 512 + 64 in bf16,
# whose ids are held by 128)
@pytest.mark.parametrize("widths,d_c,heads,dtype,page,lengths", [
    ("v3", 1024, 2, "bf16", 1, [140000]), ("small", 64, 3, "bf16", 1, [200000, 90001]), ("half", 256, 40, "bf16", 1, [143000]),
    ("v3", 512, 2, "fp32", 1, [140000]), ("small", 32, 2, "fp32", 1, [140000]), ("v3", 512, 4, "bf16", 1, [100001]), ("v3", 512, 70, "bf16", 1, [30000]),
    ("small", 64, 3, "bf16", 3, [850000])])
def test_shares_of_many_pages(widths, d_c, heads, dtype, page, lengths):
    """bf16 as in test_out_is_off_by_its_own_rounding. fp32: a score's sum of up to 1088 rounded products is off by about
    sqrt(1088) 2^-24 of a unit, 2^-19, and so is its weight, the exp2 and the sums of the weights by less: 2^-17 in norm."""
    x = make(lengths, page, widths, d_c, heads, dtype, seed=heads)
    out, lse = call(x)
    off = own = 0.0
    for t in range(len(lengths)):
        o, l, top = exact(x, t)
        off += float((out[t].double() - o).square().sum())
        own += float((o.to(torch.bfloat16).double() - o).square().sum() if dtype == "bf16" else o.square().sum())
        assert float((lse[t].double() - l).abs().max()) <= 2.0 ** -19 * (8 + top)
    print(f"out is off by {(off / own) ** 0.5:.3e}")
    assert off ** 0.5 <= (1.02 if dtype == "bf16" else 2.0 ** -17) * own ** 0.5
