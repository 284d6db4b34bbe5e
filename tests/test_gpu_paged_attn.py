"""laga_paged_attn against the oracle's explicit form in fp64, through the C ABI: head widths,
latent widths, types, pages that end inside a tile, rows of padding, what lies outside, long
rows split over the GPU, and a captured decoding step."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from _util import f64
from test_gpu_paged_cache import WIDTHS, i32, pool, problem

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}  # half a step, relative


def make(lengths, page, widths="v3", d_c=512, heads=16, dtype="bf16", fresh=1, pad=0, spare=3, seed=0, width=None):
    """A paged cache with the rows of requests of these lengths, and fresh rows at the end of each."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dn, dr, dv = WIDTHS[widths]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(seed)
    width = width or max(1, max(-(-n // page) for n in lengths))
    table, _, _ = pool(rng, lengths, width, page, spare)
    n_pages = sum(-(-n // page) for n in lengths) + spare
    cache = torch.randn((n_pages, page, d_c + dr), generator=gen, device="cuda").to(dt)
    position = [n - fresh + i for n in lengths for i in range(fresh)]
    request = [r for r in range(len(lengths)) for _ in range(fresh)]
    at = np.linspace(0, len(position), pad).astype(int)
    position, request = np.insert(position, at, -1), np.insert(request, at, -1)
    T = len(position)
    q = torch.randn((T, heads, dn + dr), generator=gen, device="cuda").to(dt)
    w = (torch.randn((d_c, heads * (dn + dv)), generator=gen, device="cuda") * d_c ** -0.5).to(dt)
    p = problem(T, len(lengths), width, n_pages, page, widths, d_c, dtype, heads)
    return dict(p=p, q=q, w=w, cache=cache, table=table, position=position, request=request)


def call(x, base=None, offset=0, **kw):
    """The call, into outputs and a workspace that start as NaN, with guards behind them."""
    import paper_2607_17644_amd as L
    p = x["p"]
    nb = L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN)
    ws = torch.full((nb + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full(p.shapes()["out"], float("nan"), dtype=x["q"].dtype, device="cuda")
    lse = torch.full(p.shapes()["lse"], float("nan"), device="cuda")
    kw.setdefault("row_request", i32(x["request"]))
    L.laga_paged_attn(p, x["q"], x["w"], x["cache"], i32(x["table"]), i32(x["position"]), rope_base=base,
                      position_offset=offset, out=out, lse=lse, workspace=ws[:nb], **kw)
    torch.cuda.synchronize()
    assert (ws[nb:] == 0xFF).all()
    return out, lse


def rounding(x, dtype, base, offset):
    """Bounds of |out - exact| and |lse - exact|, from the inputs. With half a step u: the error
    of a sum of independent roundings of parts a_i is within 6 u / sqrt(3) |a|_2 (uniform in
    +- u |a_i| at most, so a standard deviation of u |a_i| / sqrt(3); six of them). Parts:
      q W_k^T and the turned band, rounded to the element type: z_j moves by scale sum_c dqa_c c_jc, so
        out_v by scale sum_c dqa_c cov(c_c, v_v) under the softmax's weights, lse by scale sum_c dqa_c mean(c_c)
      the probabilities p_j as operands: sum_j dp_j v_jv
      the normalised sum before W_v: sum_c do_c W_cv
      out itself, once: u |out| outright.
    fp32: the sums are rounded at every step instead, of up to d_c + d_rope + n terms: sqrt of
    their number times as much, taken as 64 (4096 terms); exp2 and log2 add about 2^-20 relative."""
    p, u = x["p"], U[dtype]
    dn, dc, page = p.d_nope, p.d_c, p.page_size
    q, w = f64(x["q"]), f64(x["w"])
    bo, bl = np.zeros((p.rows, p.n_heads, p.d_v)), np.zeros((p.rows, p.n_heads))
    grow = 6 / np.sqrt(3.0) * (1.0 if dtype == "bf16" else 64.0)
    for t in range(p.rows):
        n = int(x["position"][t]) + 1
        if n <= 0:
            continue
        ids = torch.as_tensor(x["table"][x["request"][t]][:-(-n // page)].astype(np.int64), device="cuda")
        rows = f64(x["cache"][ids]).reshape(-1, x["cache"].shape[2])[:n]
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
            o = pr @ rows[:, :dc]
            var = (p.softmax_scale ** 2 * (qa[:, None] * cov) ** 2).sum(0) + (pr[:, None] ** 2 * v ** 2).sum(0) + \
                (o[:, None] ** 2 * wv ** 2).sum(0)
            bo[t, h] = u * np.abs(pr @ v) + grow * u * np.sqrt(var) + 2.0 ** -18 * (pr @ np.abs(v))
            bl[t, h] = grow * u * p.softmax_scale * np.sqrt(((qa * mean) ** 2).sum()) + 2.0 ** -19 * (8 + np.abs(z).max())
    return bo, bl


def check(x, dtype, base=None, offset=0):
    p = x["p"]
    out, lse = call(x, base, offset)
    ro, rl = O.attend(f64(x["q"]), f64(x["w"]), f64(x["cache"]), x["table"], x["position"], x["request"], d_c=p.d_c,
                      d_nope=p.d_nope, d_v=p.d_v, scale=p.softmax_scale, base=base, offset=offset)
    bo, bl = rounding(x, dtype, base, offset)
    live = np.asarray(x["position"]) >= 0
    go, gl = f64(out), f64(lse)
    assert not go[~live].any() and np.isneginf(gl[~live]).all()
    do, dl = np.abs(go[live] - ro[live]), np.abs(gl[live] - rl[live])
    print(f"out {np.max(do / bo[live]):.3f} of its bound, lse {np.max(dl / bl[live]):.3f}")
    assert (do <= bo[live]).all() and (dl <= bl[live]).all()
    return out, lse


@pytest.mark.parametrize("widths,d_c,heads,dtype", [
    ("v3", 512, 16, "bf16"), ("v3", 512, 1, "bf16"), ("v3", 512, 33, "bf16"), ("v3", 512, 128, "bf16"),
    ("v3", 512, 130, "bf16"), ("v3", 256, 40, "bf16"), ("v3", 1024, 3, "bf16"), ("v3", 32, 5, "bf16"),
    ("v3", 544, 64, "bf16"), ("half", 128, 8, "bf16"), ("half", 416, 24, "bf16"), ("half", 512, 64, "bf16"),
    ("small", 64, 4, "bf16"), ("small", 32, 100, "bf16"), ("v3", 512, 16, "fp32"), ("v3", 1024, 2, "fp32"),
    ("v3", 160, 70, "fp32"), ("half", 256, 7, "fp32"), ("small", 64, 4, "fp32")])
@pytest.mark.parametrize("page", [1, 48])
def test_widths(widths, d_c, heads, dtype, page):
    x = make([1, 31, 32, 33, 2, 97, 64, 65], page, widths, d_c, heads, dtype, pad=2)
    check(x, dtype, base=10000.0, offset=5)


@pytest.mark.parametrize("page", [7, 16, 64, 200])
@pytest.mark.parametrize("dtype,heads", [("bf16", 4), ("bf16", 40), ("fp32", 4)])
def test_pages_and_draft_tokens(page, dtype, heads):
    check(make([5, 130, 300, 64, 9], page, heads=heads, dtype=dtype, fresh=3, d_c=256), dtype, base=None)


@pytest.mark.parametrize("dtype,heads,n", [("bf16", 2, 9001), ("bf16", 34, 4099), ("fp32", 2, 3001), ("bf16", 66, 2500)])
def test_one_long_row(dtype, heads, n):
    """One row over every worker: its parts are joined; again bit for bit."""
    x = make([n], 64, heads=heads, dtype=dtype)
    a = check(x, dtype, base=10000.0)
    b = call(x, base=10000.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_ragged_batch_with_long_and_short_rows():
    rng = np.random.default_rng(1)
    lengths = [int(v) for v in np.concatenate([rng.integers(1, 40, 60), [3000, 1, 2111, 32, 700]])]
    rng.shuffle(lengths)
    check(make(lengths, 16, heads=3, pad=7), "bf16", base=10000.0)
    check(make(lengths, 16, heads=35, pad=1), "bf16", base=10000.0)


def test_peaked_scores():
    """Scores of +-60 and a key that takes all of a row: the running maximum moves late and far."""
    for heads in (4, 40):
        x = make([400, 50], 16, heads=heads, seed=3)
        x["q"] = (x["q"].float() * 12).to(torch.bfloat16)
        check(x, "bf16")


def test_what_is_not_visible_is_not_read():
    """NaN and infinity behind a row's position, in unused pages and in the table's other entries'
    pages change nothing, bit for bit."""
    for dtype, heads in (("bf16", 5), ("bf16", 128), ("fp32", 5)):
        x = make([70, 33, 1, 500], 48, heads=heads, dtype=dtype, pad=1, width=20)
        a = call(x, base=10000.0)
        seen = torch.zeros(x["cache"].shape[:2], dtype=torch.bool, device="cuda")
        for r, n in enumerate([70, 33, 1, 500]):
            for j in range(n):
                seen[x["table"][r, j // 48], j % 48] = True
        x["cache"][~seen] = float("nan")
        x["cache"][~seen] = torch.where(torch.rand_like(x["cache"][~seen].float()) < 0.5, float("inf"), float("nan")).to(
            x["cache"].dtype)
        for i, v in enumerate((-1, 2 ** 31 - 1, -2 ** 31)):
            x["table"][i, 10:] = v
        b = call(x, base=10000.0)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_outside_is_nan_and_the_others_stay():
    for heads in (3, 128):
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
        y["request"][0], y["position"][0] = -1, 0
        assert call(y)[0][0].isnan().all()
        y["position"][:] = 2 ** 31 - 1
        assert call(y)[0].isnan().all()


def test_nan_in_a_visible_row_and_infinite_queries():
    x = make([70, 33], 16, heads=2)
    a = call(x)
    y = dict(x, cache=x["cache"].clone())
    y["cache"][x["table"][0, 1], 3, 7] = float("nan")
    b = call(y)
    assert b[0][0].isnan().all() and b[1][0].isnan().all() and torch.equal(a[0][1], b[0][1])


def test_no_rows_visible_at_all():
    x = make([5, 6, 7], 16, heads=4)
    x["position"][:] = -1
    out, lse = call(x, base=10000.0)
    assert not out.any() and lse.isneginf().all()


def test_row_request_left_out_and_lse_by_itself():
    import ctypes
    import paper_2607_17644_amd as L
    from paper_2607_17644_amd import binding as B
    x = make([70, 33, 40], 16, heads=4)
    a = call(x)
    b = call(x, row_request=None)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # the C call without lse
    p = x["p"]
    ws = torch.empty(L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN), dtype=torch.uint8, device="cuda")
    out, table, pos = torch.empty_like(a[0]), i32(x["table"]), i32(x["position"])
    st = B._lib.laga_paged_attn(ctypes.byref(p.c()), None, x["q"].data_ptr(), x["w"].data_ptr(), x["cache"].data_ptr(),
                                table.data_ptr(), None, pos.data_ptr(), out.data_ptr(), None, ws.data_ptr(), ws.numel(),
                                torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(out, a[0])


def test_pages_far_apart():
    """Page offsets past 2^32 elements give the same bits."""
    x = make([300, 70], 16, heads=3)
    a = call(x)
    n_pages, page, W = x["cache"].shape
    stride = (1 << 28) + 8
    store = torch.empty(((n_pages - 1) * stride + page * W,), dtype=torch.bfloat16, device="cuda")
    far = store.as_strided(x["cache"].shape, (stride, W, 1))
    far.copy_(x["cache"])
    import dataclasses
    b = call(dict(x, cache=far, p=dataclasses.replace(x["p"], page_stride=stride)))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_another_stream():
    import paper_2607_17644_amd as L
    x = make([300, 70], 16, heads=3)
    a = call(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = call(x, stream=side)
    with torch.cuda.stream(side):
        c = call(x)
    assert torch.equal(a[0], b[0]) and torch.equal(a[0], c[0])
    del L


def _server(heads=4, page=16, R=5, width=12, d_model=64, dtype="bf16", seed=0):
    """Buffers of a small server: one step is plan, append, attention and W_o."""
    import paper_2607_17644_amd as L
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n_pages = 40
    dt = torch.bfloat16
    p = problem(R, R, width, n_pages, page, heads=heads, dtype=dtype)
    sh = p.shapes()
    s = {k: torch.zeros(sh[k], dtype=torch.int32, device="cuda")
         for k in ("lengths", "fresh", "free_count", "row_begin", "row_request", "position", "slot", "status")}
    s["table"] = torch.full(sh["block_table"], -1, dtype=torch.int32, device="cuda")
    s["free"] = torch.arange(n_pages, dtype=torch.int32, device="cuda").flip(0).contiguous()
    s["free_count"].fill_(n_pages)
    s["fresh"].fill_(1)
    s["cache"] = torch.zeros(sh["cache"], dtype=dt, device="cuda")
    s["x"] = torch.randn((R, 576), generator=gen, device="cuda").to(dt)
    s["q"] = torch.randn(sh["q"], generator=gen, device="cuda").to(dt)
    s["w"] = (torch.randn(sh["w_kv_b"], generator=gen, device="cuda") / 22).to(dt)
    s["gamma"] = torch.ones(512, dtype=dt, device="cuda")
    s["w_o"] = torch.randn((heads * 128, d_model), generator=gen, device="cuda").to(dt)
    s["out"], s["lse"] = torch.zeros(sh["out"], dtype=dt, device="cuda"), torch.zeros(sh["lse"], device="cuda")
    s["y"] = torch.zeros((R, d_model), dtype=dt, device="cuda")
    s["ws_plan"] = torch.zeros(L.laga_paged_workspace_bytes(p, L.OP_PAGE_PLAN), dtype=torch.uint8, device="cuda")
    s["ws"] = torch.zeros(L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN), dtype=torch.uint8, device="cuda")
    po = L.OutProj(R, heads, 128, d_model)

    def step(stream=None):
        L.laga_page_plan(p, s["lengths"], s["fresh"], s["table"], s["free"], s["free_count"], lengths_out=s["lengths"],
                         free_count_out=s["free_count"], row_begin=s["row_begin"], row_request=s["row_request"],
                         position=s["position"], slot=s["slot"], status=s["status"], workspace=s["ws_plan"],
                         stream=stream)
        L.laga_cache_append(p, s["x"][:, :512], s["x"][:, 512:], s["position"], s["slot"], s["cache"],
                            gamma=s["gamma"], stream=stream)
        L.laga_paged_attn(p, s["q"], s["w"], s["cache"], s["table"], s["position"], row_request=s["row_request"],
                          rope_base=10000.0, out=s["out"], lse=s["lse"], workspace=s["ws"], stream=stream)
        L.laga_out_proj_fwd(po, s["out"], s["w_o"], y=s["y"], stream=stream)

    return s, step


def _feed(s, i):
    """The step's inputs, written in place: a new token for each request, now and then none."""
    gen = torch.Generator(device="cuda").manual_seed(100 + i)
    s["x"].copy_(torch.randn(s["x"].shape, generator=gen, device="cuda"))
    s["q"].copy_(torch.randn(s["q"].shape, generator=gen, device="cuda"))
    s["fresh"].copy_(torch.tensor([1, i % 2, 1, int(i % 7 > 0), 1], dtype=torch.int32))


def test_decoding_steps_captured_once():
    """One captured step replayed for token after token, its lengths advancing on the device, with
    eager work and synchronisations between, equals the eager program at every step."""
    names = ("lengths", "free_count", "table", "position", "slot", "cache", "out", "lse", "y")
    e, eager = _server()
    want = []
    for i in range(70):
        _feed(e, i)
        eager()
        torch.cuda.synchronize()
        assert int(e["status"]) == 0
        want.append({k: e[k].clone() for k in names})
    g, step = _server()
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
    for i in range(1, 70):
        _feed(g, i)
        g["out"].fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in names:
            assert torch.equal(g[k], want[i][k]), (i, k)


def test_two_captured_steps_with_workspaces_of_their_own():
    a, step_a = _server(seed=1)
    b, step_b = _server(heads=40, seed=2)
    for s, step in ((a, step_a), (b, step_b)):
        for i in range(20):
            _feed(s, i)
            step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs = []
    for (s, step), st in zip(((a, step_a), (b, step_b)), streams):
        s["fresh"].zero_()
        st.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(st), torch.cuda.graph(g, stream=st):
            s["position"].copy_(s["lengths"] - 1)
            import paper_2607_17644_amd as L
            p = problem(5, 5, 12, 40, 16, heads=s["q"].shape[1])
            L.laga_paged_attn(p, s["q"], s["w"], s["cache"], s["table"], s["position"], rope_base=10000.0, out=s["out"],
                              lse=s["lse"], workspace=s["ws"], stream=st)
        graphs.append(g)
    want = []
    for s, g in zip((a, b), graphs):
        g.replay()
        torch.cuda.synchronize()
        want.append((s["out"].clone(), s["lse"].clone()))
    for _ in range(5):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s, (o, l) in zip((a, b), want):
            assert torch.equal(s["out"], o) and torch.equal(s["lse"], l)


@pytest.mark.parametrize("heads", [16, 64])
def test_served_rows_are_the_trained_block_s(heads):
    """The producers and the whole-sequence attention against the served rows of the same tokens: within
    the two kernels' own bounds (each is held to the oracle by the framework's bar of 2e-2)."""
    import laga_inputs as LI
    import paper_2607_17644_amd as L
    from _util import to_dev
    w = LI.WORKLOADS["v3_shard_s4096"].replace(seq_len=333, n_heads=heads)
    y, x = LI.make_prologue_inputs(w), LI.make_inputs(w, with_dout=False)
    lat, kpe, q, gam, wkv = (to_dev(v, "bf16") for v in (y["latent_raw"], y["kpe_raw"], y["q"], y["gamma"], x["w_kv_b"]))
    pp = L.Problem(1, 333, heads, 512, 128, 64, 128, w.scale)
    qr = q.clone()
    c, k, _ = L.laga_prologue_fwd(pp, lat, kpe, q=qr, gamma=gam)
    kv = L.laga_reconstruct_kv(pp, c, wkv)
    out, lse = L.laga_attn_fwd(pp, qr, c, k, wkv, kv=kv)
    # the same tokens served: 300 as a prompt, the rest one at a time; every row attends
    p = problem(333, 1, 24, 30, 16, heads=heads)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    table, free = z(1, 24) - 1, torch.arange(30, dtype=torch.int32, device="cuda")
    lengths, count = z(1), z(1) + 30
    cache = torch.zeros((30, 16, 576), dtype=torch.bfloat16, device="cuda")
    for n in [300] + [1] * 33:
        at = int(lengths)
        ps = problem(n, 1, 24, 30, 16, heads=heads)
        _, _, _, _, pos, slot, status = L.laga_page_plan(ps, lengths, z(1) + n, table, free, count, lengths_out=lengths,
                                                         free_count_out=count)
        assert int(status) == 0
        L.laga_cache_append(ps, lat[0, at:at + n], kpe[0, at:at + n], pos, slot, cache, gamma=gam)
    so, sl = L.laga_paged_attn(p, q[0].contiguous(), wkv, cache, table, torch.arange(333, dtype=torch.int32, device="cuda"),
                               row_request=z(333), rope_base=10000.0)
    torch.cuda.synchronize()
    assert (so.float() - out[0].float()).abs().max() < 4e-2
    assert (sl - lse[0].t()).abs().max() < 4e-2


@pytest.mark.parametrize("widths,d_c,heads", [("v3", 512, 24), ("v3", 1024, 5), ("half", 128, 64), ("small", 32, 40)])
@pytest.mark.parametrize("count,longest", [(24, 1), (24, 4), (1500, 3)])
def test_lse_of_short_rows_is_held_in_fp32(widths, d_c, heads, count, longest):
    """The lse of a row with one key is its score, sum_c qa_c row_c over d_nope, then d_c + d_rope terms: fp32 sums of
    N terms are within sqrt(N) 2^-24 of their value in the mean, for any roundings that do not lean one way."""
    rng = np.random.default_rng(5)
    lengths = [int(v) for v in rng.integers(1, longest + 1, count)]
    x = make(lengths, 16, widths, d_c, heads, seed=9)
    p = x["p"]
    lse = f64(call(x, base=10000.0, offset=2)[1])
    _, want = O.attend(f64(x["q"]), f64(x["w"]), f64(x["cache"]), x["table"], x["position"], x["request"], d_c=d_c,
                       d_nope=p.d_nope, d_v=p.d_v, scale=p.softmax_scale, base=10000.0, offset=2)
    off = np.linalg.norm(lse - want) / np.linalg.norm(want)
    print(f"{off:.2e}")
    assert off <= np.sqrt(p.d_nope + d_c + p.d_rope) * 2.0 ** -24


@pytest.mark.parametrize("d_c,heads,count,dtype", [(512, 16, 521, "bf16"), (1024, 128, 6, "bf16"), (256, 2, 700, "fp32")])
def test_products_of_many_rows(d_c, heads, count, dtype):
    """More blocks of rows than workgroups take at once, and the widest latent with many heads; rows of padding
    between."""
    rng = np.random.default_rng(2)
    check(make([int(v) for v in rng.integers(1, 5, count)], 16, d_c=d_c, heads=heads, dtype=dtype, pad=9), dtype, base=10000.0)
