"""laga_page_plan, laga_page_release and laga_cache_append against the oracle, through the C ABI.
Plans are whole numbers and have to be equal; cache rows that are not written keep their bits."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from _util import f64

pytestmark = pytest.mark.gpu

WIDTHS = {"v3": (128, 64, 128), "half": (64, 32, 64), "small": (32, 16, 32)}


def problem(rows, requests, width, n_pages, page, widths="v3", d_c=512, dtype="bf16", heads=2, page_stride=0):
    import paper_2607_17644_amd as L
    dn, dr, dv = WIDTHS[widths]
    return L.Paged(rows, requests, width, n_pages, page, heads, d_c, dn, dr, dv, (dn + dr) ** -0.5,
                   L.DTYPE_BF16 if dtype == "bf16" else L.DTYPE_FP32, page_stride)


def i32(x):
    return torch.tensor(np.ascontiguousarray(x), dtype=torch.int32, device="cuda")


def pool(rng, lengths, width, page, spare):
    """A table that holds lengths and a stack of the other pages."""
    have = [-(-n // page) for n in lengths]
    n_pages = sum(have) + spare
    ids, at = rng.permutation(n_pages), 0
    table = np.full((len(lengths), width), -1)
    for r, n in enumerate(have):
        table[r, :n] = ids[at:at + n]
        at += n
    free = np.full(n_pages, -7)
    free[:n_pages - at] = ids[at:]
    return table, free, n_pages - at


def run_plan(lengths, fresh, table, free, count, rows, page, in_place=False):
    import paper_2607_17644_amd as L
    p = problem(rows, len(lengths), table.shape[1], len(free), page)
    dl, dt, dc = i32(lengths), i32(table), i32([count])
    df = i32(free)
    kw = dict(lengths_out=dl, free_count_out=dc) if in_place else {}
    names = ("lengths_out", "free_count_out", "row_begin", "row_request", "position", "slot", "status")
    for k in names:
        kw.setdefault(k, torch.full(p.shapes()[k], -99, dtype=torch.int32, device="cuda"))
    ws = torch.full((L.laga_paged_workspace_bytes(p, L.OP_PAGE_PLAN) + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    got = L.laga_page_plan(p, dl, i32(fresh), dt, df, dc, workspace=ws[:-64], **kw)
    torch.cuda.synchronize()
    assert (ws[-64:] == 0x5A).all() and torch.equal(df, i32(free))
    res = {k: v.cpu().numpy() for k, v in zip(names, got)}
    res["block_table"] = dt.cpu().numpy()
    ref = O.plan(lengths, fresh, table, free, count, rows, page)
    for k in ref:
        assert np.array_equal(res[k].reshape(-1), np.asarray(ref[k]).reshape(-1)), (k, ref["status"])
    return ref


# 4096 requests fit the sums' one turn and the search in LDS; more rows than 8192: two launches
@pytest.mark.parametrize("R,page,chunk,pad", [(1, 1, 1, 0), (1, 64, 5000, 3), (2, 7, 40, 0), (63, 16, 1, 0),
                                              (64, 64, 1, 5), (65, 1, 3, 1), (1000, 32, 700, 1001), (4096, 16, 1, 0),
                                              (4097, 16, 2, 0), (9000, 5, 3, 11), (300, 48, 9000, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan(R, page, chunk, pad, in_place):
    rng = np.random.default_rng(R * 1000 + page)
    lengths = rng.integers(0, 10 * page + 2, R)
    lengths[rng.random(R) < 0.2] = 0
    fresh = np.where(rng.random(R) < 0.15, 0, np.where(rng.random(R) < 20 / (20 + R), rng.integers(1, chunk + 1, R), 1))
    fresh[-1] = chunk
    width = int(max(-(-(n + f) // page) for n, f in zip(lengths, fresh)))
    spare = int(sum(-(-(n + f) // page) for n, f in zip(lengths, fresh))) + 1
    table, free, count = pool(rng, lengths, width, page, spare)
    assert run_plan(lengths, fresh, table, free, count, int(fresh.sum()) + pad, page, in_place)["status"] == 0


def test_plan_takes_the_last_page_and_the_last_row_and_no_tokens():
    table = np.full((3, 4), -1)
    assert run_plan([0, 0, 0], [16, 16, 0], table, np.arange(8)[::-1], 8, 32, 4)["free_count_out"] == 0
    assert run_plan([0, 0, 0], [0, 0, 0], table, np.arange(8), 0, 1, 4)["status"] == 0


@pytest.mark.parametrize("rows", [40, 20000])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_is_all_or_nothing(rows, in_place):
    rng = np.random.default_rng(3)
    lengths = np.array([3, 0, 8, 5])
    table, free, count = pool(rng, lengths, 6, 4, 9)
    big = 2 ** 31 - 1
    for ln, fr, cnt, r, code in ((lengths, [1, 2, 3, rows], count, rows, None), (lengths, [1, 2, 17, 0], count, rows, 2),
                                 (lengths, [9, 9, 9, 9], count, rows, 4 if rows > 36 else None),
                                 (lengths, [1, 1, -1, 1], count, rows, 8), ([3, -2, 8, 5], [1, 1, 1, 1], count, rows, 8),
                                 (lengths, [1, 1, 1, 1], -1, rows, 8), (lengths, [1, 1, 1, 1], len(free) + 1, rows, 8),
                                 (lengths, [big, big, big, big], count, rows, None), ([big] * 4, [big] * 4, count, rows, None),
                                 (lengths, [8, 8, 8, 8], count, 5, None)):
        ref = run_plan(ln, fr, table, free, cnt, r, 4, in_place)
        assert ref["status"] != 0 and (code is None or ref["status"] == code)


@pytest.mark.parametrize("R,page,every,width", [(1, 1, 1, 5), (3, 7, 2, 9), (64, 64, 9, 128), (2000, 16, 2, 200),
                                                (4100, 3, 1, 7), (9, 16, 1, 2000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_release(R, page, every, width, in_place):
    import paper_2607_17644_amd as L
    rng = np.random.default_rng(R)
    lengths = rng.integers(0, width * page + 1, R)
    drop = (np.arange(R) % every == 0) * rng.integers(1, 9, R)
    table, free, count = pool(rng, lengths, width, page, 13)
    p = problem(1, R, width, len(free), page)

    def go(lengths, count, code):
        dl, dc, df, dt = i32(lengths), i32([count]), i32(free), i32(table)
        kw = dict(lengths_out=dl, free_count_out=dc) if in_place else {}
        lo, co, st = L.laga_page_release(p, dl, i32(drop), dt, df, dc, **kw)
        torch.cuda.synchronize()
        ref = O.release(lengths, drop, table, free, count, page)
        assert ref["status"] == int(st) and (st != 0) == code
        assert np.array_equal(lo.cpu().numpy(), ref["lengths_out"]) and int(co) == ref["free_count_out"]
        assert np.array_equal(df.cpu().numpy(), ref["free_pages"]) and torch.equal(dt, i32(table))

    go(lengths, count, False)
    go(lengths, len(free), lengths[0] > 0)  # no room on the stack
    bad = lengths.copy()
    bad[-1] = -1
    go(bad, count, True)
    bad[-1] = width * page + 1
    go(bad, count, True)


def append_inputs(T, d_c, d_rope, dtype, seed, joint):
    rng = np.random.default_rng(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    lat = rng.standard_normal((T, d_c)) * np.exp(rng.uniform(np.log(0.1), np.log(10.0), (T, 1)))
    x = torch.from_numpy(np.concatenate([lat, rng.standard_normal((T, d_rope))], 1)).to(dt).cuda()
    gamma = torch.from_numpy(rng.uniform(0.5, 1.5, d_c)).to(dt).cuda()
    if joint:
        return x[:, :d_c], x[:, d_c:], gamma
    return x[:, :d_c].contiguous(), x[:, d_c:].contiguous(), gamma


# A stored value is off by its own rounding, u |x| with u = eps / 2, and by the fp32 arithmetic before it:
# a norm of up to 1024 terms and three products (below 2^-20 |x| together), a rotation of two
# products with sine and cosine of an angle formed in fp64 and rounded once (|a| <= pi: 2^-23
# absolute; with the products and the sum below 2^-21 (|x0| + |x1|)).
U = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


@pytest.mark.parametrize("widths,d_c", [("v3", 512), ("v3", 1024), ("v3", 32), ("half", 416), ("small", 64)])
@pytest.mark.parametrize("T,page,joint,gamma", [(1, 1, True, True), (5, 7, True, False), (70, 16, False, True),
                                                (1100, 64, True, True)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append(widths, d_c, T, page, joint, gamma, dtype):
    import paper_2607_17644_amd as L
    dr = WIDTHS[widths][1]
    lat, kpe, gam = append_inputs(T, d_c, dr, dtype, T, joint)
    rng = np.random.default_rng(T + page)
    n_pages = -(-T // page) + 3
    slot = rng.permutation(n_pages * page)[:T]
    # padding and slots outside the pool store nothing
    slot[3::7] = -1
    slot[4::9] = n_pages * page
    slot[5::11] = 2 ** 31 - 1
    slot[2::13] = -2 ** 31
    position = rng.integers(0, 200000, T)
    cache = torch.randn((n_pages, page, d_c + dr), device="cuda").to(lat.dtype)
    before = cache.clone()
    p = problem(T, 1, 8192, n_pages, page, widths, d_c, dtype)
    L.laga_cache_append(p, lat, kpe, i32(position), i32(slot), cache, gamma=gam if gamma else None, eps=1e-5,
                        rope_base=5000.0, position_offset=77)
    torch.cuda.synchronize()
    ref = O.append(f64(lat), f64(kpe), position, slot, f64(before), f64(gam) if gamma else None, 1e-5, 5000.0, 77)
    keep = np.ones(n_pages * page, bool)
    keep[slot[(slot >= 0) & (slot < n_pages * page)]] = False
    keep = torch.from_numpy(keep).cuda().view(n_pages, page)
    assert torch.equal(cache[keep], before[keep])
    got = f64(cache)
    pair = np.zeros_like(ref)
    k = np.abs(ref[..., d_c:]).reshape(*ref.shape[:2], -1, 2)
    pair[..., d_c:] = np.repeat(np.hypot(k[..., 0], k[..., 1]), 2, -1)
    assert (np.abs(got - ref) <= U[dtype] * np.abs(ref) + 2.0 ** -20 * np.abs(ref) + 2.0 ** -20 * pair + 1e-30).all()


def test_append_to_pages_far_apart():
    """Page offsets past 2^32 elements (a pool that holds other layers' pages between)."""
    import paper_2607_17644_amd as L
    page, n_pages, d_c, dr, T = 16, 40, 512, 64, 33
    stride = (1 << 27) + 8
    store = torch.empty(((n_pages - 1) * stride + page * (d_c + dr),), dtype=torch.bfloat16, device="cuda")
    cache = store.as_strided((n_pages, page, d_c + dr), (stride, d_c + dr, 1))
    cache.zero_()
    lat, kpe, gam = append_inputs(T, d_c, dr, "bf16", 5, True)
    slot = np.random.default_rng(1).permutation(n_pages * page)[:T]
    slot[:2] = [n_pages * page - 1, 0]
    p = problem(T, 1, 4, n_pages, page, page_stride=stride)
    L.laga_cache_append(p, lat, kpe, i32(np.arange(T)), i32(slot), cache, gamma=gam)
    near = torch.zeros((n_pages, page, d_c + dr), dtype=torch.bfloat16, device="cuda")
    L.laga_cache_append(problem(T, 1, 4, n_pages, page), lat, kpe, i32(np.arange(T)), i32(slot), near, gamma=gam)
    torch.cuda.synchronize()
    assert torch.equal(cache, near) and near.abs().sum() > 0


def test_append_is_the_prologue_row():
    """The rows of laga_prologue_fwd, bit for bit."""
    import paper_2607_17644_amd as L
    T, page = 100, 16
    lat, kpe, gam = append_inputs(T, 512, 64, "bf16", 9, False)
    pp = L.Problem(1, T, 2, 512, 128, 64, 128, 0.07)
    c, k, _ = L.laga_prologue_fwd(pp, lat[None], kpe[None], gamma=gam, position_offset=9)
    cache = torch.zeros((7, page, 576), dtype=torch.bfloat16, device="cuda")
    L.laga_cache_append(problem(T, 1, 8, 7, page), lat, kpe, i32(np.arange(T)), i32(np.arange(T)), cache, gamma=gam,
                        position_offset=9)
    torch.cuda.synchronize()
    assert torch.equal(cache.view(-1, 576)[:T], torch.cat((c[0], k[0]), -1))


def test_binding_refusals():
    import paper_2607_17644_amd as L
    lat, kpe, gam = append_inputs(8, 512, 64, "bf16", 5, True)
    cache = torch.zeros((4, 16, 576), dtype=torch.bfloat16, device="cuda")
    p, s = problem(8, 1, 4, 4, 16), i32(np.arange(8))
    for bad in (dict(lat=lat[:7]), dict(lat=lat.float()), dict(kpe=kpe.t()), dict(s=s.long()), dict(s=s.cpu()),
                dict(cache=cache[:, :, :512]), dict(cache=cache[:, ::2]), dict(cache=cache.float())):
        a = dict(dict(lat=lat, kpe=kpe, s=s, cache=cache), **bad)
        with pytest.raises(ValueError):
            L.laga_cache_append(p, a["lat"], a["kpe"], s, a["s"], a["cache"])
    with pytest.raises(L.LagaError) as e:  # a column slice that starts off the 16-byte grid
        wide = torch.zeros((8, 520), dtype=torch.bfloat16, device="cuda")
        L.laga_cache_append(p, wide[:, 4:516], kpe, s, s, cache)
    assert e.value.status == 4
    with pytest.raises(ValueError):
        L.laga_page_plan(p, i32([1]), i32([1, 2]), i32([[1] * 4]), i32([0] * 4), i32([1]))
