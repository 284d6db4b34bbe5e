"""The serving calls without a GPU: the rule that shares out tiles, and what the C ABI and the
binding refuse before any launch."""
import ctypes
import dataclasses
import os
import subprocess

import pytest
import torch

import paper_2607_17644_amd as L
from paper_2607_17644_amd import binding as B
from paper_2607_17644_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
P = L.Paged(rows=8, requests=4, table_width=16, n_pages=100, page_size=64, n_heads=16, d_c=512, d_nope=128, d_rope=64,
            d_v=128, softmax_scale=0.072)
FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: validation fails first
OFF = ctypes.c_void_p(0x10008)
CFG = B._CPrologue(1e-6, 10000.0, 0)
BIG = 1 << 40


def test_shares_of_tiles(tmp_path):
    exe = str(tmp_path / "paged_tiles")
    r = subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I",
                        os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                        os.path.join(HERE, "host", "paged_tiles.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


def replaced(**kw):
    return ctypes.byref(dataclasses.replace(P, **kw).c())


def call(name, p, ptr=FAKE, ws=FAKE, nbytes=BIG, cfg=ctypes.byref(CFG)):
    """One entry point with one kind of pointer. (With arguments that are all good it would launch
    on these addresses: every use here has one that is refused.)"""
    lib = B._lib
    if name == "plan":
        return lib.laga_page_plan(p, *[ptr] * 12, ws, nbytes, None)
    if name == "release":
        return lib.laga_page_release(p, *[ptr] * 8, ws, nbytes, None)
    if name == "append":
        return lib.laga_cache_append(p, cfg, ptr, 512, ptr, ptr, 64, ptr, ptr, ptr, None)
    return lib.laga_paged_attn(p, cfg, *[ptr] * 8, ws, nbytes, None)


NAMES = ("plan", "release", "append", "attn")
BAD = [(2, kw) for kw in (dict(rows=0), dict(requests=-1), dict(table_width=0), dict(n_pages=0), dict(page_size=0),
                          dict(n_heads=0), dict(d_c=-32), dict(softmax_scale=float("nan")), dict(softmax_scale=0.0),
                          dict(page_stride=64 * 576 - 8), dict(page_stride=-8))] + \
      [(3, kw) for kw in (dict(d_nope=64), dict(d_c=48), dict(d_c=2048), dict(dtype=5), dict(reserved=1),
                          dict(rows=1 << 31), dict(rows=BIG), dict(requests=BIG), dict(table_width=BIG),
                          dict(n_pages=BIG), dict(page_size=BIG), dict(n_heads=BIG), dict(n_heads=1024),
                          dict(n_pages=1 << 25), dict(table_width=(1 << 24) + 1), dict(requests=1 << 27),
                          dict(rows=1 << 27), dict(rows=1 << 26, table_width=17), dict(rows=1 << 22, table_width=1),
                          dict(rows=1 << 20, table_width=1, n_heads=128), dict(page_stride=64 * 576 + 4),
                          dict(page_stride=1 << 41))]


@pytest.mark.parametrize("code,kw", BAD)
def test_sizes_are_refused(code, kw):
    p = replaced(**kw)
    for name in NAMES:
        assert call(name, p) == code, name
    for op in (L.OP_PAGE_PLAN, L.OP_PAGED_ATTN):
        assert B._lib.laga_paged_workspace_bytes(p, op) == 0


def test_pointers_and_workspace_are_refused():
    lib, p = B._lib, replaced()
    for name in NAMES:
        assert call(name, None) == 1, name
        assert call(name, p, ptr=None) == 1, name
        assert call(name, p, ptr=OFF) == 4, name
    for op, names in ((L.OP_PAGE_PLAN, ("plan", "release")), (L.OP_PAGED_ATTN, ("attn",))):
        need = lib.laga_paged_workspace_bytes(p, op)
        assert need > 0 and need % 256 == 0
        for name in names:
            assert call(name, p, ws=None) == 5, name
            assert call(name, p, ws=OFF) == 4, name
            assert call(name, p, nbytes=need - 1) == 5, name
    assert lib.laga_paged_workspace_bytes(p, 0) == 0 and lib.laga_paged_workspace_bytes(None, 3) == 0
    # every required pointer by itself
    for i in range(12):
        a = [FAKE] * 12
        a[i] = None
        assert lib.laga_page_plan(p, *a, FAKE, BIG, None) == 1, i
        a[i] = OFF
        assert lib.laga_page_plan(p, *a, FAKE, BIG, None) == 4, i
    for i in (0, 1, 2, 3, 5, 6):
        a = [FAKE] * 8
        a[i] = None
        assert lib.laga_paged_attn(p, None, *a, FAKE, BIG, None) == 1, i
    # more rows than requests need row_request
    a = [FAKE] * 8
    a[4] = None
    assert lib.laga_paged_attn(p, None, *a, FAKE, BIG, None) == 2


def test_rotation_and_strides_are_refused():
    lib, p = B._lib, replaced()
    assert lib.laga_cache_append(p, None, FAKE, 512, FAKE, FAKE, 64, FAKE, FAKE, FAKE, None) == 1
    for bad in (B._CPrologue(-1.0, 1e4, 0), B._CPrologue(1e-6, 1.0, 0), B._CPrologue(1e-6, float("inf"), 0),
                B._CPrologue(1e-6, 1e4, -1), B._CPrologue(1e-6, 1e4, (1 << 53) - 1000)):
        assert call("append", p, cfg=ctypes.byref(bad)) == 2
        assert call("attn", p, cfg=ctypes.byref(bad)) == 2
    for ls, ks, code in ((511, 64, 2), (512, 63, 2), (0, 64, 2), (516, 64, 3), (512, 68, 3), (BIG, 64, 3)):
        assert lib.laga_cache_append(p, ctypes.byref(CFG), FAKE, ls, FAKE, FAKE, ks, FAKE, FAKE, FAKE, None) == code


def test_binding_refuses_host_tensors():
    i32 = {k: torch.zeros(v, dtype=torch.int32) for k, v in P.shapes().items()
           if k in ("lengths", "fresh", "drop", "block_table", "free_pages", "free_count", "position", "slot")}
    f = {k: torch.zeros(P.shapes()[k], dtype=torch.bfloat16) for k in ("cache", "q", "w_kv_b", "latent_raw", "kpe_raw")}
    with pytest.raises(ValueError, match="device tensor"):
        L.laga_page_plan(P, i32["lengths"], i32["fresh"], i32["block_table"], i32["free_pages"], i32["free_count"])
    with pytest.raises(ValueError, match="device tensor"):
        L.laga_page_release(P, i32["lengths"], i32["drop"], i32["block_table"], i32["free_pages"], i32["free_count"])
    with pytest.raises(ValueError, match="device tensor"):
        L.laga_cache_append(P, f["latent_raw"], f["kpe_raw"], i32["position"], i32["slot"], f["cache"])
    with pytest.raises(ValueError, match="device tensor"):
        L.laga_paged_attn(P, f["q"], f["w_kv_b"], f["cache"], i32["block_table"], i32["position"])
    with pytest.raises(TypeError, match="lengths"):
        L.laga_page_plan(P, None, i32["fresh"], i32["block_table"], i32["free_pages"], i32["free_count"])


def test_a_problem_follows_its_fields():
    p = dataclasses.replace(P)
    assert p.shapes()["q"] == (8, 16, 192) and p == P
    need = L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN)
    p.rows, p.n_heads = 9, 32
    assert p.shapes()["q"] == (9, 32, 192) and p.shapes()["lse"] == (9, 32) and p != P
    assert L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN) > need
    p.d_c = 48
    assert L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN) == 0
