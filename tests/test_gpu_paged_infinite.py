"""Infinite elements in laga_paged_attn's cache and queries: a cached rotary key with an infinite element gives the
score that the definition gives, -infinity (the key has no weight) where the query's element has the other sign and
NaN rows where it has the same one or is zero; infinite queries and latents give NaN. Against the oracle's
explicit form in fp64."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from _util import f64
from test_gpu_paged_attn import call, make

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def put(x, r, j, element, value):
    """Cached position j of request r."""
    page = x["p"].page_size
    x["cache"][int(x["table"][r, j // page]), j % page, element] = value


def check(x, dtype, base=None):
    """NaN where the definition has NaN. Elsewhere out is off by its own rounding, u |out|, and next to it (16 bits in
    between: 2^-16, times at most 8 roundings of operands, of the mean of |v|, here below 4; fp32: sums of up to n + 600 terms,
    2^-19), lse by 2^-19 of 8 + max |score|, below 64."""
    p = x["p"]
    out, lse = call(x, base)
    with np.errstate(all="ignore"):
        ro, rl = O.attend(f64(x["q"]), f64(x["w"]), f64(x["cache"]), x["table"], x["position"], x["request"], d_c=p.d_c,
                          d_nope=p.d_nope, d_v=p.d_v, scale=p.softmax_scale, base=base)
    go, gl = f64(out), f64(lse)
    bad = np.isnan(ro).any(-1)
    assert np.isnan(ro[bad]).all() and np.isnan(go[bad]).all()
    assert np.isfinite(go[~bad]).all() and np.isfinite(gl[~bad]).all()
    near = 4 * (2.0 ** -13 if dtype == "bf16" else 2.0 ** -17)
    assert (np.abs(go - ro)[~bad] <= U[dtype] * np.abs(ro[~bad]) + near).all()
    assert (np.abs(gl - rl)[~bad] <= 2.0 ** -19 * 72).all()
    return bad


@pytest.mark.parametrize("dtype,widths,d_c,heads,n", [
    ("bf16", "v3", 512, 16, 500), ("bf16", "v3", 512, 100, 300), ("bf16", "v3", 1024, 4, 200), ("bf16", "v3", 256, 40, 200),
    ("bf16", "half", 128, 24, 100), ("bf16", "small", 64, 16, 70), ("fp32", "v3", 512, 8, 100), ("fp32", "small", 64, 4, 70)])
@pytest.mark.parametrize("base", [None, 10000.0])
def test_keys_of_no_weight(dtype, widths, d_c, heads, n, base):
    x = make([n, 40], 16, widths, d_c, heads, dtype, seed=heads)
    dn = x["p"].d_nope
    for j, e, v in ((0, 3, np.inf), (33, 3, np.inf), (n - 1, 3, np.inf), (39, 3, np.inf)):
        put(x, 0, j, d_c + e, v)
    put(x, 1, 7, d_c + 4, -np.inf)
    x["q"][:, 1, dn:] = x["q"][:, 1, dn:].abs().clamp(min=0.01)  # heads that surely have both kinds of rows
    x["q"][0, 2, dn:], x["q"][1, 2, dn:] = -1.0, 1.0
    if base is None:
        x["q"][0, 0, dn + 3] = 0.0
    bad = check(x, dtype, base)
    assert bad.any() and not bad.all()
    if base is None:
        assert bad[0, :3].tolist() == [True, True, False] and bad[1, 1:3].tolist() == [False, False]


@pytest.mark.parametrize("heads,n", [(4, 70000), (64, 40000), (100, 18000)])
def test_keys_of_no_weight_over_many_tiles(heads, n):
    """Whole tiles of them at the beginnings of shares, and a row's every key but one."""
    x = make([n, 600], 64, heads=heads, seed=2)
    x["q"][:, :, 128:] = -x["q"][:, :, 128:].abs().clamp(min=0.01)
    x["q"][:, 1, 128:] *= -1
    flat = x["cache"].view(-1, 576)
    rows = torch.as_tensor((x["table"][0][:-(-n // 64), None].astype(np.int64) * 64 + np.arange(64)).reshape(-1)[:n], device="cuda")
    flat[rows[: n // 2], 512 + 9] = float("inf")
    flat[rows[n // 2 + 100 :: 7], 512 + 5] = float("inf")
    rows = torch.as_tensor((x["table"][1][:10, None].astype(np.int64) * 64 + np.arange(64)).reshape(-1)[:600], device="cuda")
    flat[rows, 512] = float("inf")
    flat[rows[311], 512] = 1.0
    p, out, lse = x["p"], *call(x)
    w, q = x["w"].double().view(512, heads, 256), x["q"].double()
    for t, k in ((0, n), (1, 600)):
        ids = torch.as_tensor(x["table"][t][:-(-k // 64)].astype(np.int64), device="cuda")
        c = x["cache"][ids].double().reshape(-1, 576)[:k]
        for h in range(heads):
            z = p.softmax_scale * ((c[:, :512] @ w[:, h, :128].contiguous()) @ q[t, h, :128] + c[:, 512:] @ q[t, h, 128:])
            want = torch.softmax(z, 0) @ (c[:, :512] @ w[:, h, 128:].contiguous())
            if h == 1:
                assert want.isnan().all() and out[t, h].isnan().all()
                continue
            assert want.isfinite().all()
            # (as in check)
            assert ((out[t, h].double() - want).abs() <= U["bf16"] * want.abs() + 4 * 2.0 ** -13).all()
            assert abs(float(lse[t, h]) - float(torch.logsumexp(z, 0))) <= 2.0 ** -19 * 72


@pytest.mark.parametrize("dtype,heads", [("bf16", 4), ("bf16", 100), ("fp32", 4)])
def test_infinite_queries_and_latents(dtype, heads):
    """By the definition NaN: scores of both signs' infinities, or no weight times an infinite value."""
    x = make([300, 70, 50, 9], 16, heads=heads, dtype=dtype, seed=1)
    x["q"][0, 1, 5] = float("inf")
    x["q"][1, 2, 128 + 7] = float("-inf")
    put(x, 2, 33, 100, float("inf"))
    bad = check(x, dtype)
    assert bad[0, 1] and bad[1, 2] and bad[2].all() and bad.sum() == 2 + heads
