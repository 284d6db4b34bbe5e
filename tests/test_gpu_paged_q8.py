"""A paged cache held in 8 bits through the C ABI, against the oracle in fp64: rows quantised as they are written (the
bytes have to be equal), read back (exactly), attended over, and decoding steps of all of them captured once."""
import ctypes
import dataclasses

import numpy as np
import pytest
import torch

from oracle import eight as E
from oracle import paged as O
from _util import f64
from test_gpu_paged_cache import WIDTHS, i32, pool, problem

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


def eight(x, d_c):
    """Numbers [..., d_c + d_rope] (fp32) as (cache, scales)."""
    out, exps = [], []
    for part in (x[..., :d_c], x[..., d_c:]):
        e = torch.ceil(torch.log2(part.abs().amax(-1, keepdim=True) / 448.0)).clamp(-100, 119)
        out.append((part / torch.exp2(e)).clamp(-448.0, 448.0).to(F8).view(torch.uint8))
        exps.append((e + 127).to(torch.uint8))
    return torch.cat(out, -1).view(F8), torch.cat(exps, -1).contiguous()


def make(lengths, page, widths="v3", d_c=512, heads=16, dtype="bf16", fresh=1, pad=0, spare=3, seed=0, width=None, spread=0.0):
    """A cache with the rows of requests of these lengths, fresh rows at the end of each; spread: the rows' own
    sizes are over 2^+-spread."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dn, dr, dv = WIDTHS[widths]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(seed)
    width = width or max(1, max(-(-n // page) for n in lengths))
    table, _, _ = pool(rng, lengths, width, page, spare)
    n_pages = sum(-(-n // page) for n in lengths) + spare
    x = torch.randn((n_pages, page, d_c + dr), generator=gen, device="cuda")
    size = torch.empty((n_pages, page, 2), device="cuda").uniform_(-spread - 0.5, spread + 0.5, generator=gen).exp2_()
    x[..., :d_c] *= size[..., :1]
    x[..., d_c:] *= size[..., 1:]
    cache, scales = eight(x, d_c)
    position = [n - fresh + i for n in lengths for i in range(fresh)]
    request = [r for r in range(len(lengths)) for _ in range(fresh)]
    at = np.linspace(0, len(position), pad).astype(int)
    position, request = np.insert(position, at, -1), np.insert(request, at, -1)
    q = torch.randn((len(position), heads, dn + dr), generator=gen, device="cuda").to(dt)
    w = (torch.randn((d_c, heads * (dn + dv)), generator=gen, device="cuda") * d_c ** -0.5).to(dt)
    p = problem(len(position), len(lengths), width, n_pages, page, widths, d_c, dtype, heads)
    return dict(p=p, q=q, w=w, cache=cache, scales=scales, table=table, position=position, request=request)


def call(x, base=None, offset=0, **kw):
    """The call, into outputs and a workspace that start as NaN, with guards behind them."""
    import paper_2607_17644_amd as L
    p = x["p"]
    nb = L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN_Q8)
    ws = torch.full((nb + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full(p.shapes()["out"], float("nan"), dtype=x["q"].dtype, device="cuda")
    lse = torch.full(p.shapes()["lse"], float("nan"), device="cuda")
    kw.setdefault("row_request", i32(x["request"]))
    L.laga_paged_attn_q8(p, x["q"], x["w"], x["cache"], x["scales"], i32(x["table"]), i32(x["position"]), rope_base=base,
                         position_offset=offset, out=out, lse=lse, workspace=ws[:nb], **kw)
    torch.cuda.synchronize()
    assert (ws[nb:] == 0xFF).all()
    return out, lse


def stands_for(x):
    return E.values(x["cache"].view(torch.uint8).cpu().numpy(), x["scales"].cpu().numpy(), x["p"].d_c)


def attend(x, base=None, offset=0):
    p = x["p"]
    return O.attend(f64(x["q"]), f64(x["w"]), stands_for(x), x["table"], x["position"], x["request"], d_c=p.d_c, d_nope=p.d_nope,
                    d_v=p.d_v, scale=p.softmax_scale, base=base, offset=offset)


def bounds(x, base, offset):
    """Bounds of |out - exact| and |lse - exact|, from the inputs; a sum of independent roundings u_i a_i is within
    6 / sqrt(3) |u a|_2. The roundings, each relative to its part:
      a score's operands (the query in two fp16 parts, 2^-22, and fp32 sums of up to 1088 + 128 terms, sqrt of their number times
        2^-24): 2^-18 of scale sum_c qa_c cov(c_c, v_v) for out, of scale sum_c qa_c mean(c_c) for lse
      a probability as an operand: fp16, 2^-12 (fp32: two parts, 2^-22, and sums as above: 2^-18) of p_j v_jv
      the normalised sums before W_v: two bf16 parts, 2^-17 (fp32: sums, 2^-18) of o_c W_cv
      out itself, outright: bf16 2^-8, fp32 2^-24
    exp2, log2 and the sums of the weights: 2^-18 of the weights' mean of |v|, 2^-19 of 8 + the largest score."""
    p, bf = x["p"], x["q"].dtype == torch.bfloat16
    dn, dc, page = p.d_nope, p.d_c, p.page_size
    q, w, cache = f64(x["q"]), f64(x["w"]), stands_for(x)
    bo, bl = np.zeros((p.rows, p.n_heads, p.d_v)), np.zeros((p.rows, p.n_heads))
    six = 6 / np.sqrt(3.0)
    u_z, u_p, u_o, u = 2.0 ** -18, 2.0 ** (-12 if bf else -18), 2.0 ** (-17 if bf else -18), 2.0 ** (-8 if bf else -24)
    for t in range(p.rows):
        n = int(x["position"][t]) + 1
        if n <= 0:
            continue
        rows = cache[x["table"][x["request"][t]][:-(-n // page)]].reshape(-1, cache.shape[2])[:n]
        qt = q[t].copy()
        if base is not None:
            qt[:, dn:] = O.producers.rope(q[None, t:t + 1, :, dn:], np.array([offset + n - 1]), base)[0, 0]
        for h in range(p.n_heads):
            wk = w[:, h * (dn + p.d_v):h * (dn + p.d_v) + dn]
            wv = w[:, h * (dn + p.d_v) + dn:(h + 1) * (dn + p.d_v)]
            qa = np.concatenate([wk @ qt[h, :dn], qt[h, dn:]])
            z = p.softmax_scale * (rows @ qa)
            pr = np.exp(z - z.max())
            pr /= pr.sum()
            v = rows[:, :dc] @ wv
            mean = pr @ rows
            cov = (rows * pr[:, None]).T @ v - np.outer(mean, pr @ v)
            var = (u_z * p.softmax_scale) ** 2 * ((qa[:, None] * cov) ** 2).sum(0) + u_p ** 2 * (pr[:, None] ** 2 * v ** 2).sum(0) + \
                u_o ** 2 * (mean[:dc, None] ** 2 * wv ** 2).sum(0)
            bo[t, h] = u * np.abs(pr @ v) + six * np.sqrt(var) + 2.0 ** -18 * (pr @ np.abs(v))
            bl[t, h] = six * u_z * p.softmax_scale * np.sqrt(((qa * mean) ** 2).sum()) + 2.0 ** -19 * (8 + np.abs(z).max())
    return bo, bl


def check(x, base=None, offset=0):
    out, lse = call(x, base, offset)
    ro, rl = attend(x, base, offset)
    bo, bl = bounds(x, base, offset)
    live = np.asarray(x["position"]) >= 0
    go, gl = f64(out), f64(lse)
    assert not go[~live].any() and np.isneginf(gl[~live]).all()
    do, dl = np.abs(go[live] - ro[live]), np.abs(gl[live] - rl[live])
    print(f"out {np.max(do / bo[live]):.3f} of its bound, lse {np.max(dl / bl[live]):.3f}")
    assert (do <= bo[live]).all() and (dl <= bl[live]).all()
    return out, lse


# ---------------------------------------------------------------- append
def append_inputs(tokens, page, widths, d_c, dtype, seed=0, spare=2):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dr = WIDTHS[widths][1]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn((tokens, d_c + dr), generator=gen, device="cuda")
    x *= torch.empty((tokens, 1), device="cuda").uniform_(-4, 4, generator=gen).exp2_()
    n_pages = -(-tokens // page) + spare
    slot = rng.permutation(n_pages * page)[:tokens]
    slot[rng.random(tokens) < 0.1] = -1
    p = problem(tokens, 1, 1 << 10, n_pages, page, widths, d_c, dtype)
    return dict(p=p, x=x.to(dt), gamma=torch.empty(d_c, device="cuda").uniform_(0.5, 1.5, generator=gen).to(dt), slot=slot,
                position=rng.integers(0, 1 << 17, tokens))


def append(y, joint=True, gamma=True, offset=0, base=10000.0, eps=1e-6, fill=0x2A, stream=None, cache=None, scales=None):
    import paper_2607_17644_amd as L
    p, d_c = y["p"], y["p"].d_c
    sh = p.shapes()
    cache = torch.full(sh["cache"], fill, dtype=torch.uint8, device="cuda").view(F8) if cache is None else cache
    scales = torch.full(sh["scales"], fill, dtype=torch.uint8, device="cuda") if scales is None else scales
    lat, kpe = y["x"][:, :d_c], y["x"][:, d_c:]
    if not joint:
        lat, kpe = lat.contiguous(), kpe.contiguous()
    L.laga_cache_append_q8(p, lat, kpe, i32(y["position"]), i32(y["slot"]), cache, scales, gamma=y["gamma"] if gamma else None,
                           eps=eps, rope_base=base, position_offset=offset, stream=stream)
    torch.cuda.synchronize()
    return cache.view(torch.uint8).cpu().numpy(), scales.cpu().numpy()


def check_append(y, **kw):
    """Bytes and scales equal to the definition's; and those that were not written as they were."""
    p = y["p"]
    got = append(y, **kw)
    start = np.full(p.shapes()["cache"], 0x2A, np.uint8), np.full(p.shapes()["scales"], 0x2A, np.uint8)
    x = f64(y["x"])
    # (eps as the call gets it: a float)
    want = E.append(x[:, :p.d_c], x[:, p.d_c:], y["position"], y["slot"], *start, gamma=f64(y["gamma"]) if kw.get("gamma", True) else None,
                    eps=float(np.float32(kw.get("eps", 1e-6))), base=kw.get("base", 10000.0), offset=kw.get("offset", 0))
    nan = (got[0] & 127) == 127
    assert np.array_equal(nan, (want[0] & 127) == 127)
    assert np.array_equal(got[0][~nan], want[0][~nan]) and np.array_equal(got[1], want[1])
    return got


@pytest.mark.parametrize("widths,d_c,dtype", [("v3", 512, "bf16"), ("v3", 1024, "bf16"), ("v3", 544, "fp32"), ("v3", 32, "bf16"),
                                              ("half", 416, "bf16"), ("half", 256, "fp32"), ("small", 64, "bf16"),
                                              ("small", 32, "fp32")])
@pytest.mark.parametrize("tokens,page", [(1, 1), (67, 48), (130, 7)])
def test_append(widths, d_c, dtype, tokens, page):
    y = append_inputs(tokens, page, widths, d_c, dtype, seed=tokens)
    check_append(y)
    check_append(y, joint=False, gamma=False, offset=3, base=500.0, eps=0.25)


def test_append_of_a_prompt():
    """Two tokens to a wave, one of them alone at the end."""
    check_append(append_inputs(4101, 64, "v3", 512, "bf16", seed=3))


@pytest.mark.parametrize("widths,d_c,dtype", [("v3", 1024, "fp32"), ("v3", 512, "bf16"), ("half", 416, "bf16"), ("small", 32, "fp32")])
def test_append_of_a_prompt_with_rows_and_weights_out_of_range(widths, d_c, dtype):
    """Two tokens to a wave: of a pair the one not finite, or a row of zeros, the other as ever; and weights that make every row
    infinite in places, or larger than a scale reaches."""
    y = append_inputs(4099, 48, widths, d_c, dtype, seed=d_c)
    x = y["x"]
    x[0, 1], x[3, 0], x[6], x[9], x[12, 2], x[15, d_c], x[18, d_c + 1] = (float(v) for v in ("inf", "nan", "0", "inf", "-inf", "inf", "nan"))
    check_append(y)
    y["gamma"][0] = 3e38
    check_append(y)
    y["gamma"][1], y["gamma"][2] = float("inf"), float("nan")
    check_append(y)


def test_append_at_the_edges_of_numbers():
    """Rows of zeros; a largest number that is 448 2^e, and the next one; numbers that are half-way between two; values that
    are not finite, alone and everywhere; magnitudes from 2^-140 to 2^127."""
    y = append_inputs(24, 16, "v3", 512, "fp32", seed=1)
    y["slot"] = np.arange(24)
    y["position"][:] = 0
    y["gamma"].fill_(1.0)
    x = y["x"]
    x[0] = 0.0
    # a row whose mean square is 1 exactly keeps its numbers (eps 0): 512 numbers +-1 with pairs (1 + a, sqrt(1 - ..)) avoided
    x[1, :512] = 1.0
    x[2, :512] = 0.0
    x[2, 0] = 1.75 * 2.0 ** 5
    x[3, 512:] = 0.0
    x[3, 512], x[3, 513], x[3, 514] = 448.0, 1.0625, 1.1875   # e = 0: ties to even
    x[4, 512:] = 0.0
    x[4, 512], x[4, 514] = float(np.nextafter(np.float32(448.0), np.float32(1e9))), 2.125
    x[5, 3], x[5, 520] = float("inf"), float("-inf")
    x[6, 3], x[6, 520] = float("nan"), float("nan")
    x[7] = float("nan")
    x[8, 512:] *= 2.0 ** -130
    x[9, 512:] = 3.0e38
    x[10, :512] *= 1e18
    x[11, :512] *= 1e-18
    x[12, 512:] = 2.0 ** -149
    x[13, 512:] = 0.0
    x[13, 512], x[13, 513:576] = 256.0, torch.linspace(-20, 20, 63, device="cuda")
    check_append(y)
    got, scales = append(y, eps=1e-6)
    assert (got[0, 0] == 0).all() and (scales[0, 0] == 27).all()
    assert (got[0, 7] & 127 == 127).all()


def test_append_writes_its_slots_alone():
    y = append_inputs(40, 16, "v3", 512, "bf16")
    y["slot"][:4] = [2 ** 31 - 1, -2 ** 31, y["p"].n_pages * 16, -5]
    check_append(y)


# ---------------------------------------------------------------- read
@pytest.mark.parametrize("widths,d_c,dtype", [("v3", 512, "bf16"), ("v3", 1024, "fp32"), ("half", 416, "bf16"), ("small", 32, "fp32"),
                                              ("small", 64, "bf16")])
@pytest.mark.parametrize("page,longest", [(1, 9), (48, 300), (64, 1)])
def test_read(widths, d_c, dtype, page, longest):
    import paper_2607_17644_amd as L
    rng = np.random.default_rng(page)
    lengths = [int(v) for v in rng.integers(1, longest + 1, 5)]
    x = make(lengths, page, widths, d_c, 1, dtype, spread=10.0, seed=page)
    request = np.repeat(np.arange(5), lengths)
    position = np.concatenate([np.arange(n) for n in lengths])
    order = rng.permutation(len(request))
    request, position = np.insert(request[order], 0, -1), np.insert(position[order], 0, -7)
    p = dataclasses.replace(x["p"], rows=len(request))
    c, k = L.laga_cache_read_q8(p, x["cache"], x["scales"], i32(x["table"]), i32(position), row_request=i32(request))
    wc, wk = E.read(x["cache"].view(torch.uint8).cpu().numpy(), x["scales"].cpu().numpy(), x["table"], position, request, d_c)
    assert np.array_equal(f64(c), wc) and np.array_equal(f64(k), wk)
    assert not c[0].any() and not k[0].any()


def test_read_many_rows_twice_and_outside():
    import paper_2607_17644_amd as L
    x = make([9000, 50], 64, heads=1)
    rng = np.random.default_rng(4)
    request, position = rng.integers(0, 2, 40000), rng.integers(0, 50, 40000)
    request[:20000], position[:20000] = 0, rng.integers(0, 9000, 20000)
    request[5], position[6], request[7] = 2, 64 * x["table"].shape[1], -1
    x["table"][1, 0] = x["p"].n_pages
    p = dataclasses.replace(x["p"], rows=40000)
    c, k = L.laga_cache_read_q8(p, x["cache"], x["scales"], i32(x["table"]), i32(position), row_request=i32(request))
    v = stands_for(x)
    bad = request == 1
    bad[[5, 6, 7]] = True
    want = v[x["table"][np.where(bad, 0, request), np.where(bad, 0, position) // 64], np.where(bad, 0, position) % 64]
    assert np.array_equal(f64(c)[~bad], want[~bad][:, :512]) and np.array_equal(f64(k)[~bad], want[~bad][:, 512:])
    assert c[torch.from_numpy(bad).cuda()].isnan().all() and k[torch.from_numpy(bad).cuda()].isnan().all()


def test_every_number_and_scale_comes_back():
    """All 256 bytes under the scales that an append writes, and the first and last that there are."""
    import paper_2607_17644_amd as L
    exps = [27, 28, 100, 126, 127, 128, 200, 246]
    p = problem(len(exps), 1, 1, 1, 8, "v3", 512, "fp32")
    cache = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(3)[:576].expand(1, 8, 576).contiguous().view(F8)
    scales = torch.tensor(exps, dtype=torch.uint8, device="cuda")[None, :, None].expand(1, 8, 2).contiguous()
    z = torch.zeros(8, dtype=torch.int32, device="cuda")
    at = torch.arange(8, dtype=torch.int32, device="cuda")
    want = E.values(cache.view(torch.uint8).cpu().numpy(), scales.cpu().numpy(), 512)[0]
    for q in (p, dataclasses.replace(p, dtype=L.DTYPE_BF16)):
        c, k = L.laga_cache_read_q8(q, cache, scales, z[:1, None], at, row_request=z)
        assert np.array_equal(f64(c), want[:, :512], equal_nan=True) and np.array_equal(f64(k), want[:, 512:], equal_nan=True)


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("widths,d_c,heads,dtype", [
    ("v3", 512, 16, "bf16"), ("v3", 512, 1, "bf16"), ("v3", 512, 33, "bf16"), ("v3", 512, 128, "bf16"),
    ("v3", 512, 130, "bf16"), ("v3", 256, 40, "bf16"), ("v3", 1024, 3, "bf16"), ("v3", 1024, 20, "bf16"), ("v3", 32, 5, "bf16"),
    ("v3", 544, 64, "bf16"), ("half", 128, 8, "bf16"), ("half", 416, 24, "bf16"), ("half", 512, 64, "bf16"),
    ("small", 64, 4, "bf16"), ("small", 32, 100, "bf16"), ("v3", 512, 16, "fp32"), ("v3", 512, 40, "fp32"), ("v3", 1024, 2, "fp32"),
    ("v3", 160, 70, "fp32"), ("half", 256, 7, "fp32"), ("half", 256, 20, "fp32"), ("small", 64, 4, "fp32"), ("small", 64, 20, "fp32")])
@pytest.mark.parametrize("page", [1, 48])
def test_widths(widths, d_c, heads, dtype, page):
    check(make([1, 31, 32, 33, 2, 97, 64, 65], page, widths, d_c, heads, dtype, pad=2), base=10000.0, offset=5)


@pytest.mark.parametrize("page", [7, 16, 64, 200])
@pytest.mark.parametrize("dtype,heads", [("bf16", 4), ("bf16", 40), ("fp32", 4)])
def test_pages_and_draft_tokens(page, dtype, heads):
    check(make([5, 130, 300, 64, 9], page, heads=heads, dtype=dtype, fresh=3, d_c=256))


@pytest.mark.parametrize("dtype,heads,n", [("bf16", 2, 9001), ("bf16", 20, 7000), ("bf16", 34, 4099), ("fp32", 2, 3001), ("bf16", 66, 2500)])
def test_one_long_row(dtype, heads, n):
    """One row over every worker: its parts are joined; again bit for bit."""
    x = make([n], 64, heads=heads, dtype=dtype)
    a = check(x, base=10000.0)
    b = call(x, base=10000.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_ragged_batch_with_long_and_short_rows():
    rng = np.random.default_rng(1)
    lengths = [int(v) for v in np.concatenate([rng.integers(1, 40, 60), [3000, 1, 2111, 32, 700]])]
    rng.shuffle(lengths)
    check(make(lengths, 16, heads=3, pad=7), base=10000.0)
    check(make(lengths, 16, heads=20, pad=7), base=10000.0)
    check(make(lengths, 16, heads=35, pad=1), base=10000.0)


@pytest.mark.parametrize("heads,dtype", [(4, "bf16"), (20, "bf16"), (40, "bf16"), (4, "fp32")])
def test_peaked_scores(heads, dtype):
    """Scores of +-60 and a key that takes all of a row: the running maximum moves late and far."""
    x = make([400, 50], 16, heads=heads, seed=3, dtype=dtype)
    x["q"] = (x["q"].float() * 12).to(x["q"].dtype)
    check(x)


@pytest.mark.parametrize("heads,dtype", [(4, "bf16"), (40, "bf16"), (4, "fp32")])
@pytest.mark.parametrize("spread", [3.0, 12.0])
def test_rows_of_many_sizes(heads, dtype, spread):
    """Scales over 2^+-spread, the latent's and the key's apart: small probabilities of large rows count."""
    x = make([300, 2000, 70], 16, heads=heads, seed=5, dtype=dtype, spread=spread)
    x["q"] = (x["q"].float() * 2.0 ** -spread).to(x["q"].dtype)
    check(x, base=10000.0)


def test_a_far_larger_row_of_no_weight_and_far_smaller_rows():
    """One key 2^60 times the others with a score that leaves it 2^-70 of the weight or none; and the others alone."""
    x = make([200, 64], 16, heads=8, seed=6)
    p = x["p"]
    at = (int(x["table"][0, 3]), 5)
    x["cache"][at] = x["cache"][at].float().abs().to(F8)
    # the key's band decides the scores: the latent's products are out of it
    x["q"][..., :p.d_nope] = 0.0
    x["q"][..., p.d_nope:] = -x["q"][..., p.d_nope:].abs()
    x["scales"][at][0] += 60
    for add in (3, 4):
        y = dict(x, scales=x["scales"].clone())
        y["scales"][at][1] += add
        check(y)


@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** 40])
def test_queries_of_any_size(size):
    """q scaled by a power of two and the softmax's scale by its inverse: the same bits."""
    x = make([100, 33], 16, heads=20, seed=8, dtype="fp32")
    a = call(x, base=10000.0)
    b = call(dict(x, q=x["q"] * size, p=dataclasses.replace(x["p"], softmax_scale=x["p"].softmax_scale / size)), base=10000.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_what_is_not_visible_is_not_read():
    """NaN behind a row's position, in unused pages and in the table's other entries' pages, and any
    scales there, change nothing, bit for bit."""
    for dtype, heads in (("bf16", 5), ("bf16", 20), ("bf16", 128), ("fp32", 5)):
        x = make([70, 33, 1, 500], 48, heads=heads, dtype=dtype, pad=1, width=20)
        a = call(x, base=10000.0)
        seen = torch.zeros(x["cache"].shape[:2], dtype=torch.bool, device="cuda")
        for r, n in enumerate([70, 33, 1, 500]):
            for j in range(n):
                seen[x["table"][r, j // 48], j % 48] = True
        x["cache"].view(torch.uint8)[~seen] = 0x7F
        x["scales"][~seen] = 255
        for i, v in enumerate((-1, 2 ** 31 - 1, -2 ** 31)):
            x["table"][i, 10:] = v
        b = call(x, base=10000.0)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_outside_is_nan_and_the_others_stay():
    for heads in (3, 20, 128):
        x = make([70, 33, 40, 500, 64, 9], 16, heads=heads, width=33)
        a = call(x)
        y = dict(x, table=x["table"].copy(), position=x["position"].copy(), request=x["request"].copy())
        y["table"][1, 0] = y["p"].n_pages   # a visible page past the pool
        y["table"][2, 2] = -5               # below it
        y["request"][4] = 6                 # no such request
        y["position"][5] = 33 * 16          # past the table
        b = call(y)
        bad = torch.tensor([1, 2, 4, 5], device="cuda")
        ok = torch.tensor([0, 3], device="cuda")
        assert b[0][bad].isnan().all() and b[1][bad].isnan().all()
        # (the tiles are shared out anew: equal up to the grouping of a row's sums)
        assert torch.allclose(a[0][ok].float(), b[0][ok].float(), atol=2e-2) and b[0][ok].isfinite().all()
        # nothing of a row in the pool
        y["table"][3, :] = -1
        c = call(y)
        assert c[0][3].isnan().all() and c[1][3].isnan().all()
        y["position"][:] = 2 ** 31 - 1
        assert call(y)[0].isnan().all()


@pytest.mark.parametrize("heads", [2, 20, 70])
def test_nan_in_a_visible_row_and_in_a_query(heads):
    x = make([70, 33, 300], 16, heads=heads)
    a = call(x)
    y = dict(x, cache=x["cache"].clone(), q=x["q"].clone())
    y["cache"].view(torch.uint8)[x["table"][0, 1], 3, 7] = 0xFF
    y["q"][2, 1, 5] = float("nan")
    y["q"][2, 0, 130] = float("inf")
    b = call(y)
    assert b[0][0].isnan().all() and b[1][0].isnan().all() and torch.equal(a[0][1], b[0][1])
    assert b[0][2, :2].isnan().all() and b[1][2, :2].isnan().all()
    assert torch.equal(a[0][2, 2:], b[0][2, 2:]) and torch.equal(a[1][2, 2:], b[1][2, 2:])


def test_no_rows_visible_at_all():
    x = make([5, 6, 7], 16, heads=4)
    x["position"][:] = -1
    out, lse = call(x, base=10000.0)
    assert not out.any() and lse.isneginf().all()


def test_row_request_left_out_and_lse_by_itself():
    import paper_2607_17644_amd as L
    from paper_2607_17644_amd import binding as B
    for heads in (4, 100):
        x = make([70, 33, 40], 16, heads=heads)
        a = call(x)
        b = call(x, row_request=None)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        # the C call without lse
        p = x["p"]
        ws = torch.empty(L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN_Q8), dtype=torch.uint8, device="cuda")
        out, table, pos = torch.empty_like(a[0]), i32(x["table"]), i32(x["position"])
        st = B._lib.laga_paged_attn_q8(ctypes.byref(p.c()), None, x["q"].data_ptr(), x["w"].data_ptr(), x["cache"].data_ptr(),
                                       x["scales"].data_ptr(), table.data_ptr(), None, pos.data_ptr(), out.data_ptr(), None,
                                       ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == 0 and torch.equal(out, a[0])


def test_pages_far_apart():
    """Page offsets past 2^32 bytes: the same bits read, attended over and written."""
    import paper_2607_17644_amd as L
    x = make([300, 70], 16, heads=3)
    a = call(x)
    n_pages, page, W = x["cache"].shape
    stride = (1 << 28) + 16
    store = torch.empty(((n_pages - 1) * stride + page * W,), dtype=torch.uint8, device="cuda")
    assert store.numel() > 1 << 32
    far = store.as_strided(x["cache"].shape, (stride, W, 1)).view(F8)
    far.view(torch.uint8).copy_(x["cache"].view(torch.uint8))
    p = dataclasses.replace(x["p"], page_stride=stride)
    b = call(dict(x, cache=far, p=p))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    request, position = i32([0] * 300), torch.arange(300, dtype=torch.int32, device="cuda")
    r, s = dataclasses.replace(x["p"], rows=300), dataclasses.replace(p, rows=300)
    c = L.laga_cache_read_q8(r, x["cache"], x["scales"], i32(x["table"]), position, row_request=request)
    d = L.laga_cache_read_q8(s, far, x["scales"], i32(x["table"]), position, row_request=request)
    assert torch.equal(c[0], d[0]) and torch.equal(c[1], d[1])
    y = append_inputs(300, 16, "v3", 512, "bf16")
    y["slot"] = np.random.default_rng(0).permutation(n_pages * 16)[:300]
    y["p"] = dataclasses.replace(y["p"], n_pages=n_pages)
    near = append(y)
    far.view(torch.uint8).fill_(0x2A)
    y["p"] = dataclasses.replace(y["p"], page_stride=stride)
    got = append(y, cache=far)
    assert np.array_equal(near[0], got[0]) and np.array_equal(near[1], got[1])


def test_another_stream():
    import paper_2607_17644_amd as L
    x = make([300, 70], 16, heads=3)
    y = append_inputs(67, 48, "v3", 512, "bf16")
    a, e = call(x), append(y)
    args = (dataclasses.replace(x["p"], rows=2), x["cache"], x["scales"], i32(x["table"]), i32([299, 3]))
    r = L.laga_cache_read_q8(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b, f = call(x, stream=side), append(y, stream=side)
    s = L.laga_cache_read_q8(*args, stream=side)
    with torch.cuda.stream(side):
        c = call(x)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[0], c[0])
    assert np.array_equal(e[0], f[0]) and np.array_equal(e[1], f[1])
    assert torch.equal(r[0], s[0]) and torch.equal(r[1], s[1])


def test_wrong_tensors_are_refused():
    import paper_2607_17644_amd as L
    x = make([70, 33], 16, heads=2)
    p, table, pos = x["p"], i32(x["table"]), i32(x["position"])
    ok = dict(cache=x["cache"], scales=x["scales"])
    for kw, match in ((dict(cache=x["cache"].view(torch.uint8)), "cache has dtype"), (dict(cache=x["cache"][:-1]), "cache has shape"),
                      (dict(scales=x["scales"].to(torch.int32)), "scales has dtype"), (dict(scales=x["scales"][..., 0]), "scales has shape"),
                      (dict(cache=torch.empty(x["cache"].shape[::-1], dtype=torch.uint8, device="cuda").permute(2, 1, 0).view(torch.uint8)), "cache"),
                      (dict(scales=x["scales"].cpu()), "device tensor")):
        with pytest.raises(ValueError, match=match):
            L.laga_paged_attn_q8(p, x["q"], x["w"], block_table=table, position=pos, **{**ok, **kw})
        if match != "device tensor":
            with pytest.raises(ValueError, match=match):
                L.laga_cache_read_q8(p, block_table=table, position=pos, **{**ok, **kw})
    with pytest.raises(ValueError, match="q has dtype"):
        L.laga_paged_attn_q8(p, x["q"].float(), x["w"], **ok, block_table=table, position=pos)
    with pytest.raises(L.LagaError, match="LAGA_ERR_WORKSPACE"):
        L.laga_paged_attn_q8(p, x["q"], x["w"], **ok, block_table=table, position=pos,
                             workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


# ---------------------------------------------------------------- together
def _server(heads=4, page=16, R=5, width=12, seed=0):
    """Buffers of a small server: one step is plan, append, attention; and the cache's last rows back."""
    import paper_2607_17644_amd as L
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n_pages, dt = 40, torch.bfloat16
    p = problem(R, R, width, n_pages, page, heads=heads)
    sh = p.shapes()
    s = {k: torch.zeros(sh[k], dtype=torch.int32, device="cuda")
         for k in ("lengths", "fresh", "free_count", "row_begin", "row_request", "position", "slot", "status")}
    s["table"] = torch.full(sh["block_table"], -1, dtype=torch.int32, device="cuda")
    s["free"] = torch.arange(n_pages, dtype=torch.int32, device="cuda").flip(0).contiguous()
    s["free_count"].fill_(n_pages)
    s["fresh"].fill_(1)
    s["cache"] = torch.zeros(sh["cache"], dtype=torch.uint8, device="cuda").view(F8)
    s["scales"] = torch.zeros(sh["scales"], dtype=torch.uint8, device="cuda")
    s["x"] = torch.randn((R, 576), generator=gen, device="cuda").to(dt)
    s["q"] = torch.randn(sh["q"], generator=gen, device="cuda").to(dt)
    s["w"] = (torch.randn(sh["w_kv_b"], generator=gen, device="cuda") / 22).to(dt)
    s["out"], s["lse"] = torch.zeros(sh["out"], dtype=dt, device="cuda"), torch.zeros(sh["lse"], device="cuda")
    s["c_kv"], s["k_pe"] = torch.zeros(sh["c_kv"], dtype=dt, device="cuda"), torch.zeros(sh["k_pe"], dtype=dt, device="cuda")
    s["ws_plan"] = torch.zeros(L.laga_paged_workspace_bytes(p, L.OP_PAGE_PLAN), dtype=torch.uint8, device="cuda")
    s["ws"] = torch.zeros(L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN_Q8), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        L.laga_page_plan(p, s["lengths"], s["fresh"], s["table"], s["free"], s["free_count"], lengths_out=s["lengths"],
                         free_count_out=s["free_count"], row_begin=s["row_begin"], row_request=s["row_request"],
                         position=s["position"], slot=s["slot"], status=s["status"], workspace=s["ws_plan"], stream=stream)
        L.laga_cache_append_q8(p, s["x"][:, :512], s["x"][:, 512:], s["position"], s["slot"], s["cache"], s["scales"], stream=stream)
        L.laga_paged_attn_q8(p, s["q"], s["w"], s["cache"], s["scales"], s["table"], s["position"], row_request=s["row_request"],
                             rope_base=10000.0, out=s["out"], lse=s["lse"], workspace=s["ws"], stream=stream)
        L.laga_cache_read_q8(p, s["cache"], s["scales"], s["table"], s["position"], row_request=s["row_request"], c_kv=s["c_kv"],
                             k_pe=s["k_pe"], stream=stream)

    return s, step


def _feed(s, i):
    """The step's inputs, written in place: a new token for each request, now and then none."""
    gen = torch.Generator(device="cuda").manual_seed(100 + i)
    s["x"].copy_(torch.randn(s["x"].shape, generator=gen, device="cuda"))
    s["q"].copy_(torch.randn(s["q"].shape, generator=gen, device="cuda"))
    s["fresh"].copy_(torch.tensor([1, i % 2, 1, int(i % 7 > 0), 1], dtype=torch.int32))


@pytest.mark.parametrize("heads", [4, 40])
def test_decoding_steps_captured_once(heads):
    """One captured step replayed for token after token, its lengths advancing on the device, with eager work and
    synchronisations between, equals the eager program at every step; the last step equals the oracle's."""
    names = ("lengths", "free_count", "table", "position", "slot", "scales", "out", "lse", "c_kv", "k_pe")
    e, eager = _server(heads)
    want = []
    for i in range(60):
        _feed(e, i)
        eager()
        torch.cuda.synchronize()
        assert int(e["status"]) == 0
        want.append({k: e[k].clone() for k in names} | {"cache": e["cache"].view(torch.uint8).clone()})
    g, step = _server(heads)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        _feed(g, 0)
        step(side)  # warm-up: the first token
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step(side)
    torch.cuda.synchronize()
    for i in range(1, 60):
        _feed(g, i)
        g["out"].fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in names:
            assert torch.equal(g[k], want[i][k]), (i, k)
        assert torch.equal(g["cache"].view(torch.uint8), want[i]["cache"]), i
    p = problem(5, 5, 12, 40, 16, heads=heads)
    x = dict(p=p, q=g["q"], w=g["w"], cache=g["cache"], scales=g["scales"], table=g["table"].cpu().numpy(),
             position=g["position"].cpu().numpy(), request=g["row_request"].cpu().numpy())
    check(x, base=10000.0)
    c, k = E.read(g["cache"].view(torch.uint8).cpu().numpy(), g["scales"].cpu().numpy(), x["table"], x["position"], x["request"], 512)
    assert np.array_equal(f64(g["c_kv"]), c) and np.array_equal(f64(g["k_pe"]), k)


def test_a_prompt_s_chunk_from_read_rows_and_served_rows_agree():
    """The rows read back through the training kernels (whole-sequence attention on c_kv and k_pe) against the same tokens
    served from the 8-bit cache: within the two kernels' own bars of 2e-2 for the same numbers."""
    import paper_2607_17644_amd as L
    n, heads = 200, 4
    x = make([n], 16, heads=heads, seed=2)
    p = dataclasses.replace(x["p"], rows=n)
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((n, heads, 192), generator=gen, device="cuda").to(torch.bfloat16)
    c, k = L.laga_cache_read_q8(p, x["cache"], x["scales"], i32(x["table"]), at, row_request=zero)
    so, sl = L.laga_paged_attn_q8(p, q, x["w"], x["cache"], x["scales"], i32(x["table"]), at, row_request=zero)
    t = L.Problem(1, n, heads, 512, 128, 64, 128, p.softmax_scale)
    kv = L.laga_reconstruct_kv(t, c[None], x["w"])
    out, lse = L.laga_attn_fwd(t, q[None], c[None], k[None], x["w"], kv=kv)
    torch.cuda.synchronize()
    assert (so.float() - out[0].float()).abs().max() < 4e-2
    assert (sl - lse[0].t()).abs().max() < 4e-2


def test_two_captured_calls_with_workspaces_of_their_own():
    made = [make([300, 40, 9], 16, heads=h, seed=h) for h in (4, 40)]
    import paper_2607_17644_amd as L
    runs = []
    for x in made:
        want = call(x, base=10000.0)
        p, table, pos, req = x["p"], i32(x["table"]), i32(x["position"]), i32(x["request"])
        ws = torch.empty(L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN_Q8), dtype=torch.uint8, device="cuda")
        out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(st), torch.cuda.graph(g, stream=st):
            L.laga_paged_attn_q8(p, x["q"], x["w"], x["cache"], x["scales"], table, pos, row_request=req, rope_base=10000.0, out=out,
                                 lse=lse, workspace=ws, stream=st)
        runs.append((g, st, out, lse, want, (table, pos, req, ws)))
    for _ in range(5):
        for g, st, out, *_ in runs:
            out.zero_()
            torch.cuda.synchronize()
        for g, st, *_ in runs:
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for _, _, out, lse, want, _ in runs:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("widths,d_c,heads,page,lengths", [("v3", 512, 4, 1, [100001]), ("v3", 512, 70, 1, [30000]), ("v3", 1024, 2, 1, [60000]),
                                                           ("small", 64, 3, 3, [150000]), ("half", 256, 20, 1, [70000])])
def test_shares_of_many_pages(widths, d_c, heads, page, lengths):
    """A worker's share of a row with more pages than a wave holds the ids of. Out's norm is off by its own rounding and a
    little, in fp64 on the GPU."""
    x = make(lengths, page, widths, d_c, heads, seed=heads)
    out, lse = call(x)
    p = x["p"]
    size = torch.tensor(E.numbers(), device="cuda")
    rows = size[x["cache"].view(torch.uint8)[i32(x["table"]).long()[0]].long()].reshape(-1, d_c + p.d_rope)[:lengths[0]]
    s = 2.0 ** (x["scales"][i32(x["table"]).long()[0]].double().reshape(-1, 2)[:lengths[0]] - 127)
    rows = torch.cat((rows[:, :d_c] * s[:, :1], rows[:, d_c:] * s[:, 1:]), 1)
    w = x["w"].double().view(d_c, heads, p.d_nope + p.d_v)
    off = own = 0.0
    for h in range(heads):
        q = x["q"][0, h].double()
        z = p.softmax_scale * (rows[:, :d_c] @ (w[:, h, :p.d_nope] @ q[:p.d_nope]) + rows[:, d_c:] @ q[p.d_nope:])
        l = torch.logsumexp(z, 0)
        o = (torch.exp(z - l) @ rows[:, :d_c]) @ w[:, h, p.d_nope:]
        off += float((out[0, h].double() - o).square().sum())
        own += float((o.to(torch.bfloat16).double() - o).square().sum())
        assert float((lse[0, h].double() - l).abs()) <= 2.0 ** -19 * (8 + float(z.abs().max()))
    print(f"out is off by {(off / own) ** 0.5:.4f} of its rounding")
    # p in fp16 adds an eighth of a rounding to each weight: sqrt(1 + 1/64), and the rest 2%
    assert off ** 0.5 <= 1.03 * own ** 0.5


def test_a_scale_of_nan():
    """Byte 255 is NaN, byte 0 is 2^-127, in the read and in the rows that see them."""
    import paper_2607_17644_amd as L
    x = make([40, 70], 16, heads=4)
    a = call(x)
    y = dict(x, scales=x["scales"].clone())
    y["scales"][int(x["table"][0, 1]), 3, 1] = 255
    b = call(y)
    assert b[0][0].isnan().all() and b[1][0].isnan().all() and torch.equal(a[0][1], b[0][1])
    y["scales"][int(x["table"][0, 1]), 3, 1] = 0
    check(y)
    p = dataclasses.replace(x["p"], rows=3)
    y["scales"][int(x["table"][0, 1]), 4, 0] = 255
    c, k = L.laga_cache_read_q8(p, x["cache"], y["scales"], i32(x["table"]), i32([20, 19, 18]), row_request=i32([0, 0, 0]))
    assert c[0].isnan().all() and not k[0].isnan().any() and (k[1].abs() <= 2.0 ** -118).all() and not c[1].isnan().any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_near_where_two_roundings_meet(dtype):
    """Many rows, so that numbers fall as near to the middle of two as single precision can tell, and largest numbers near
    the end of a scale; and rows of few different numbers, which meet there exactly."""
    y = append_inputs(3000, 16, "v3", 512, dtype, seed=11)
    gen = torch.Generator(device="cuda").manual_seed(3)
    some = torch.tensor([1.0, 1.0625, 1.125, 1.1875, -1.0625, 1.75, -1.75, 0.0], device="cuda")
    y["x"][:500] = some[torch.randint(0, 8, (500, 576), generator=gen, device="cuda")].to(y["x"].dtype)
    y["position"][:250] = 0
    y["position"][2000:] = np.arange(1000) * 131
    check_append(y)
    check_append(y, gamma=False, eps=0.0)
