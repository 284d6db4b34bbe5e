"""laga_paged_attn on bf16 rows of 512 + 64 with so many keys that a worker has more than eight tiles
and a head block's waves take whole tiles: every number of heads, rows that workers share,
pages that end inside a tile, scores that jump late, what lies outside, and captured calls. Against the
formulas in fp64 on the GPU."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import paged as O
from _util import f64
from test_gpu_paged_attn import call, make
from test_gpu_paged_cache import i32

pytestmark = pytest.mark.gpu

U = 2.0 ** -8  # bf16, half a step, relative


def exact(x, t, base, offset):
    """Row t's output [heads, d_v] and lse [heads], and their bounds: with dx the rounding of x, at most
    U |x|, and sums of independent roundings within 6 U / sqrt(3) of the root of their squares,
      out: q W_k^T and the turned band (scale sum_c dqa_c cov(row_c, v)), the probabilities (sum_j dp_j v_jv), the
        normalised sum (sum_c do_c W_cv), itself once;
      lse: scale sum_c dqa_c mean(row_c);
    sums in fp32 of up to n terms, and exp2: 2^-18 of the mean of |v|; 2^-19 of 8 + max |z| for lse."""
    p = x["p"]
    n, dn, dc, dv = int(x["position"][t]) + 1, p.d_nope, p.d_c, p.d_v
    ids = torch.as_tensor(x["table"][x["request"][t]][:-(-n // p.page_size)].astype(np.int64), device="cuda")
    rows = x["cache"][ids].double().reshape(-1, x["cache"].shape[2])[:n]
    q = f64(x["q"][t])
    if base is not None:
        q[:, dn:] = O.producers.rope(q[None, None, :, dn:], np.array([offset + n - 1]), base)[0, 0]
    q, w, g = torch.as_tensor(q, device="cuda"), x["w"].double().reshape(dc, p.n_heads, dn + dv), 6 / 3.0 ** 0.5 * U
    out, lse, bo, bl = [], [], [], []
    for h in range(p.n_heads):
        wk, wv = w[:, h, :dn].contiguous(), w[:, h, dn:].contiguous()
        k, v = rows[:, :dc] @ wk, rows[:, :dc] @ wv
        z = p.softmax_scale * (k @ q[h, :dn] + rows[:, dc:] @ q[h, dn:])
        lse.append(torch.logsumexp(z, 0))
        pr = torch.softmax(z, 0)
        qa = torch.cat([wk @ q[h, :dn], q[h, dn:]])
        y, mean = pr @ v, pr @ rows
        out.append(y)
        cov = (rows * pr[:, None]).T.contiguous() @ v - mean[:, None] * y
        var = (p.softmax_scale * qa[:, None] * cov).square().sum(0) + (pr[:, None] * v).square().sum(0) + \
            (mean[:dc, None] * wv).square().sum(0)
        bo.append(U * y.abs() + g * var.sqrt() + 2.0 ** -18 * (pr @ v.abs()))
        bl.append(g * p.softmax_scale * (qa * mean).norm() + 2.0 ** -19 * (8 + z.abs().max()))
    return torch.stack(out), torch.stack(lse), torch.stack(bo), torch.stack(bl)


def check(x, base=None, offset=0, rows=None):
    a = call(x, base, offset)
    live = [t for t, n in enumerate(x["position"]) if n >= 0]
    for t in live if rows is None else rows:
        out, lse, bo, bl = exact(x, t, base, offset)
        do, dl = (a[0][t].double() - out).abs(), (a[1][t].double() - lse).abs()
        print(f"row {t}: out {(do / bo).max():.3f} of its bound, lse {(dl / bl).max():.3f}")
        assert (do <= bo).all() and (dl <= bl).all()
    pads = [t for t, n in enumerate(x["position"]) if n < 0]
    assert not a[0][pads].any() and a[1][pads].isneginf().all()
    return a


# A worker's tiles are more than eight with 2048 tiles (65536 keys) for up to 32 heads, 1024 for up to 64,
# 680 for up to 96, 512 for up to 128 (of each block of heads above that).
@pytest.mark.parametrize("heads,page,lengths", [
    (1, 64, [70001]), (16, 48, [30011, 20000, 15001, 4500, 33, 1]), (32, 1, [40000, 31007]), (17, 1000, [90000]),
    (33, 16, [17003, 21000]), (64, 64, [1500, 40001, 31, 32]), (65, 7, [12000, 13001, 5]), (96, 200, [30017]),
    (128, 64, [20011, 1, 640]), (100, 96, [16400, 999]), (130, 48, [8003, 4000, 2]), (300, 32, [9001])])
def test_heads_pages_and_lengths(heads, page, lengths):
    x = make(lengths, page, heads=heads, pad=2, seed=heads)
    a = check(x, base=10000.0, offset=3)
    b = call(x, base=10000.0, offset=3)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("heads,count,longest", [(8, 300, 600), (40, 150, 500), (128, 90, 500)])
def test_many_rows(heads, count, longest):
    """Rows of every length beside each other, whole and shared; some of them against the formulas."""
    rng = np.random.default_rng(heads)
    lengths = [int(v) for v in rng.integers(1, longest, count)]
    x = make(lengths, 16, heads=heads, fresh=1, pad=5, seed=heads)
    live = [t for t, n in enumerate(x["position"]) if n >= 0]
    check(x, base=10000.0, rows=live[::9])


def test_draft_tokens_of_one_request():
    x = make([20000, 30000, 400], 64, heads=20, fresh=3)
    check(x, base=10000.0)


@pytest.mark.parametrize("heads", [4, 128])
@pytest.mark.parametrize("gain", [30.0, 3000.0])
def test_scores_that_jump_late(heads, gain):
    """Keys in the middle and at the end of a share, of a row's last tile, too, whose scores are far above all before:
    more than the 64 powers of two that the first tile's maximum leaves room for, up to where all others vanish."""
    n = 70000 if heads == 4 else 18000
    x = make([n], 64, heads=heads, seed=7)
    flat = x["cache"][torch.as_tensor(x["table"][0][:-(-n // 64)].astype(np.int64), device="cuda")].clone()
    rows = flat.reshape(-1, flat.shape[2])
    w = x["w"].float().reshape(512, heads, -1)
    for i, j in enumerate((5000, 5001, n // 2 + 77, n - 1)):
        h = i % heads  # a row along head h's query: its score is about gain
        qa = torch.cat([w[:, h, :x["p"].d_nope] @ x["q"][0, h, :x["p"].d_nope].float(), x["q"][0, h, x["p"].d_nope:].float()])
        rows[j] = (qa * (gain * (1 + i % 2) / x["p"].softmax_scale / qa.square().sum())).to(torch.bfloat16)
    x["cache"][torch.as_tensor(x["table"][0][:-(-n // 64)].astype(np.int64), device="cuda")] = flat
    check(x)


@pytest.mark.parametrize("heads", [16, 64, 128])
def test_what_is_not_visible_is_not_read(heads):
    lengths = [40000, 33, 30011]
    x = make(lengths, 48, heads=heads, pad=1, width=900)
    a = call(x, base=10000.0)
    assert a[0].isfinite().all()
    seen = torch.zeros(x["cache"].shape[:2], dtype=torch.bool, device="cuda")
    for r, n in enumerate(lengths):
        seen[torch.as_tensor(x["table"][r][:n // 48].astype(np.int64), device="cuda")] = True
        if n % 48:
            seen[int(x["table"][r][n // 48]), :n % 48] = True
    x["cache"][~seen] = float("nan")
    for i, v in enumerate((-1, 2 ** 31 - 1, -2 ** 31)):
        x["table"][i, -(-lengths[i] // 48):] = v
    b = call(x, base=10000.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("heads", [16, 128])
@pytest.mark.parametrize("page", [20, 64])
def test_outside_is_nan_and_the_others_stay(heads, page):
    """A page outside the pool under a row, in a tile's middle too: NaN in that row, the others bit for bit
    (their tiles are shared out as before)."""
    lengths = [30000, 20000, 25000]
    x = make(lengths, page, heads=heads)
    a = call(x)
    y = dict(x, table=x["table"].copy())
    y["table"][1, 100], y["table"][2, (25000 - 1) // page] = x["p"].n_pages, -1
    b = call(y)
    assert torch.equal(a[0][0], b[0][0]) and torch.equal(a[1][0], b[1][0])
    assert b[0][1:].isnan().all() and b[1][1:].isnan().all()
    z = dict(x, cache=x["cache"].clone())
    z["cache"][x["table"][2, 100], 3, 7] = float("nan")
    c = call(z)
    assert torch.equal(a[0][:2], c[0][:2]) and c[0][2].isnan().all() and c[1][2].isnan().all()


@pytest.mark.parametrize("heads", [8, 128])
def test_pages_far_apart(heads):
    x = make([70000 if heads == 8 else 20000], 2048, heads=heads)
    a = call(x)
    n_pages, page, W = x["cache"].shape
    stride = (1 << 28) + 8  # from the 8th page on, offsets past 2^31 elements
    store = torch.empty(((n_pages - 1) * stride + page * W,), dtype=torch.bfloat16, device="cuda")
    far = store.as_strided(x["cache"].shape, (stride, W, 1))
    far.copy_(x["cache"])
    b = call(dict(x, cache=far, p=dataclasses.replace(x["p"], page_stride=stride)))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("heads", [16, 100])
def test_captured_at_growing_positions(heads):
    """One captured call, replayed with positions on either side of eight tiles per worker, between
    eager calls of the same: the same bits."""
    import paper_2607_17644_amd as L
    top = [45000, 30000]
    x = make(top, 64, heads=heads)
    p, table, request = x["p"], i32(x["table"]), i32(x["request"])
    position = i32(x["position"])
    ws = torch.empty(L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN), dtype=torch.uint8, device="cuda")
    out = torch.empty(p.shapes()["out"], dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(p.shapes()["lse"], device="cuda")

    def run():
        L.laga_paged_attn(p, x["q"], x["w"], x["cache"], table, position, row_request=request, rope_base=10000.0, out=out,
                          lse=lse, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for at in ([44999, 29999], [10, 31], [20000, -1], [44000, 7], [-1, -1], [44999, 29999]):
        position.copy_(torch.tensor(at, dtype=torch.int32))
        a = call(dict(x, position=np.array(at)), base=10000.0)
        out.fill_(float("nan")), lse.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a[0], out) and torch.equal(a[1], lse)
