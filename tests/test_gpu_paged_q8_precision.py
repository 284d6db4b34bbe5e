"""How far laga_paged_attn_q8's bf16 results are from the exact ones: rounded once, from more than 16 bits. Against the
formulas in fp64 on the GPU, on the numbers that the cache stands for."""
import numpy as np
import pytest
import torch

from oracle import eight as E
from test_gpu_paged_q8 import call, make

pytestmark = pytest.mark.gpu


def exact(x, t):
    """Row t's output [heads, d_v], the band as it is."""
    p = x["p"]
    n, dn, dc, dv = int(x["position"][t]) + 1, p.d_nope, p.d_c, p.d_v
    ids = torch.as_tensor(x["table"][x["request"][t]][:-(-n // p.page_size)].astype(np.int64), device="cuda")
    size = torch.tensor(E.numbers(), device="cuda")
    rows = size[x["cache"].view(torch.uint8)[ids].long()].flatten(0, 1)[:n]
    power = 2.0 ** (x["scales"][ids].double().flatten(0, 1)[:n] - 127)
    rows = torch.cat((rows[:, :dc] * power[:, :1], rows[:, dc:] * power[:, 1:]), 1)
    q, w = x["q"][t].double(), x["w"].double().reshape(dc, p.n_heads, dn + dv)
    out = []
    for h in range(p.n_heads):
        z = p.softmax_scale * ((rows[:, :dc] @ w[:, h, :dn].contiguous()) @ q[h, :dn] + rows[:, dc:] @ q[h, dn:])
        out.append(torch.softmax(z, 0) @ (rows[:, :dc] @ w[:, h, dn:].contiguous()))
    return torch.stack(out)


# An output that is not the bf16 number nearest to the exact value lies, by what it was off before its rounding, from a
# border between two numbers; these are 2^-8 of it apart or more. With operands of 16 bits or more (a probability, the
# normalised sums before W_v: rounded by 2^-17 at most, a third of that rms) an output is off by sqrt(2) 2^-17 / sqrt(3) <
# 2^-17 of its size (the norm of its terms p_j v_j) rms, the fp32 sums of up to 2000 terms add sqrt(2000) 2^-25 < 2^-19. Of the outputs that are as large as
# their size at least, 0.8 of the rms in the mean of 2^-8 spacings: 2^-9 or 0.2 % are rounded the other way; where the sum is k
# times smaller than its size, k times as many. Outputs are close to normal with that size: over them min(1, 2^-9 / |v|) is
# 2^-9 0.8 (ln(2^9) + 0.1) in the mean, five times 0.2 %: 1 %. One operand of 11 bits (2^-12) would have 32 times as many.
@pytest.mark.parametrize("widths,d_c,heads,lengths", [
    ("v3", 512, 4, [2000, 31, 700]), ("v3", 512, 16, [9000]), ("v3", 512, 20, [1500, 40]), ("v3", 512, 40, [1200, 33]),
    ("v3", 512, 130, [900]), ("v3", 1024, 5, [2000, 40]), ("v3", 544, 9, [600]), ("v3", 256, 24, [2000, 5]), ("half", 256, 8, [1500]),
    ("half", 128, 40, [500, 70]), ("small", 64, 16, [900, 31])])
def test_out_is_rounded_once(widths, d_c, heads, lengths):
    x = make(lengths, 48, widths, d_c, heads, seed=heads)
    out, _ = call(x)
    differ = total = 0
    for t in range(len(lengths)):
        o = exact(x, t)
        differ += int((out[t] != o.to(torch.bfloat16)).sum())
        total += o.numel()
    print(f"{differ / total:.5f} of the outputs are not the nearest")
    assert differ <= 0.01 * total
