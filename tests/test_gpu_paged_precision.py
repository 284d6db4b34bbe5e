"""How far laga_paged_attn's bf16 results are from the exact ones: out by its own rounding and next to nothing
more, whatever the spread of the scores, the number of heads and the rows beside it. Against the
formulas in fp64 on the GPU."""
import numpy as np
import pytest
import torch

from _util import f64
from test_gpu_paged_attn import call, make

pytestmark = pytest.mark.gpu


def exact(x, t):
    """Row t's output [heads, d_v], lse [heads] and largest |score|, the band as it is."""
    p = x["p"]
    n, dn, dc, dv = int(x["position"][t]) + 1, p.d_nope, p.d_c, p.d_v
    ids = torch.as_tensor(x["table"][x["request"][t]][:-(-n // p.page_size)].astype(np.int64), device="cuda")
    rows = x["cache"][ids].double().reshape(-1, x["cache"].shape[2])[:n]
    q, w = x["q"][t].double(), x["w"].double().reshape(dc, p.n_heads, dn + dv)
    out, lse, top = [], [], 0.0
    for h in range(p.n_heads):
        z = p.softmax_scale * ((rows[:, :dc] @ w[:, h, :dn].contiguous()) @ q[h, :dn] + rows[:, dc:] @ q[h, dn:])
        lse.append(torch.logsumexp(z, 0))
        out.append(torch.softmax(z, 0) @ (rows[:, :dc] @ w[:, h, dn:].contiguous()))
        top = max(top, float(z.abs().max()))
    return torch.stack(out), torch.stack(lse), top


# Scores of a standard deviation of 1, 4 and 12. One operand rounded to 8 bits (q W_k^T, the probabilities, the
# normalised sums) would move out by up to four roundings of its own at these spreads, as the covariance of scores
# and values under the softmax's weights has it (emulated: 3.3 for q W_k^T at 12). In two parts operands have 16
# bits, 2^8 times less: three of them make sqrt(1 + 3 (4 / 256)^2) = 1.0004 of out's own rounding. fp32 sums of n terms
# add about sqrt(n) 2^-25 of out (4e-6 for 20000 keys, to a rounding of 1.7e-3). 1.02 leaves room for both.
# lse: sums of up to n + 600 terms and one exp2 and log2 in fp32, 2^-19 of 8 + max |score|.
@pytest.mark.parametrize("gain", [1, 4, 12])
@pytest.mark.parametrize("widths,d_c,heads,lengths", [
    ("v3", 512, 4, [70000]), ("v3", 512, 16, [30000, 2000, 40001]), ("v3", 512, 40, [20000, 9, 21000]), ("v3", 512, 100, [16400, 64]),
    ("v3", 512, 16, [2000, 31, 700]), ("v3", 512, 64, [1500, 33]), ("v3", 512, 130, [900]), ("v3", 512, 2, [1] * 40 + [2, 3] * 20),
    ("v3", 1024, 5, [3000, 40]), ("v3", 256, 40, [2000, 5]), ("half", 128, 24, [3001, 70]), ("half", 512, 8, [2500]),
    ("small", 64, 16, [900, 31])])
def test_out_is_off_by_its_own_rounding(widths, d_c, heads, lengths, gain):
    x = make(lengths, 48, widths, d_c, heads, seed=heads)
    x["q"] = (x["q"].float() * gain).to(torch.bfloat16)
    out, lse = call(x)
    off = own = 0.0
    for t in range(len(lengths)):
        o, l, top = exact(x, t)
        off += float((out[t].double() - o).square().sum())
        own += float((o.to(torch.bfloat16).double() - o).square().sum())
        assert float((lse[t].double() - l).abs().max()) <= 2.0 ** -19 * (8 + top)
    print(f"out is off by {(off / own) ** 0.5:.4f} roundings")
    assert off ** 0.5 <= 1.02 * own ** 0.5


@pytest.mark.parametrize("heads", [4, 100])
def test_precision_does_not_depend_on_the_rows_beside(heads):
    """A row of 600 keys by itself and beside long ones: the same up to fp32 sums grouped otherwise."""
    x = make([600, 70000 if heads == 4 else 30000], 64, heads=heads, seed=3)
    x["q"] = (x["q"].float() * 8).to(torch.bfloat16)
    a = call(x)
    y = dict(x, position=x["position"].copy())
    y["position"][1] = -1
    b = call(y)
    o, l, top = exact(x, 0)
    for out, lse in (a, b):
        assert float((lse[0].double() - l).abs().max()) <= 2.0 ** -19 * (8 + top)
    # out: apart by a rounding where the sums' last bits decide it: fewer than one element in a hundred (each is within
    # 2^-8 of a step of the border with that probability, twice)
    differ = (f64(a[0][0]) != f64(b[0][0])).mean()
    print(f"{differ:.4f} of the elements differ")
    assert differ <= 0.01 and float((lse[0] - a[1][0]).abs().max()) <= 2.0 ** -18 * (8 + top)
