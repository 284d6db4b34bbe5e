"""The serving calls on a cache in 8 bits without a GPU: what the C ABI and the binding refuse before any launch."""
import ctypes
import dataclasses

import pytest
import torch

import paper_2607_17644_amd as L
from paper_2607_17644_amd import binding as B
from test_paged_host import BAD, BIG, CFG, FAKE, OFF, P, replaced


def call(name, p, ptr=FAKE, ws=FAKE, nbytes=BIG, cfg=ctypes.byref(CFG)):
    """One entry point with one kind of pointer. (Every use here has an argument that is refused.)"""
    lib = B._lib
    if name == "append":
        return lib.laga_cache_append_q8(p, cfg, ptr, 512, ptr, ptr, 64, ptr, ptr, ptr, ptr, None)
    if name == "read":
        return lib.laga_cache_read_q8(p, *[ptr] * 7, None)
    return lib.laga_paged_attn_q8(p, cfg, *[ptr] * 9, ws, nbytes, None)


NAMES = ("append", "read", "attn")


@pytest.mark.parametrize("code,kw", BAD + [(3, dict(page_stride=64 * 576 + 8)), (3, dict(page_stride=1 << 40))])
def test_sizes_are_refused(code, kw):
    p = replaced(**kw)
    for name in NAMES:
        assert call(name, p) == code, name
    assert B._lib.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN_Q8) == 0


def test_pointers_and_workspace_are_refused():
    lib, p = B._lib, replaced()
    for name in NAMES:
        assert call(name, None) == 1, name
        assert call(name, p, ptr=None) == 1, name
        assert call(name, p, ptr=OFF) == 4, name
    need = lib.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN_Q8)
    assert need > 0 and need % 256 == 0
    assert call("attn", p, ws=None) == 5 and call("attn", p, ws=OFF) == 4 and call("attn", p, nbytes=need - 1) == 5
    # every required pointer by itself
    cfg = ctypes.byref(CFG)
    for i, bad, code in [(i, None, 1) for i in (0, 2, 3, 4, 5, 6)] + [(i, OFF, 4) for i in range(7)]:
        a = [FAKE] * 7  # latent, gamma, kpe, position, slot, cache, scales
        a[i] = bad
        assert lib.laga_cache_append_q8(p, cfg, a[0], 512, a[1], a[2], 64, *a[3:], None) == code, i
    for i, bad, code in [(i, None, 1) for i in (0, 1, 2, 4, 5, 6)] + [(i, OFF, 4) for i in range(7)]:
        a = [FAKE] * 7
        a[i] = bad
        assert lib.laga_cache_read_q8(p, *a, None) == code, i
    for i, bad, code in [(i, None, 1) for i in (0, 1, 2, 3, 4, 6, 7)] + [(i, OFF, 4) for i in range(9)]:
        a = [FAKE] * 9
        a[i] = bad
        assert lib.laga_paged_attn_q8(p, None, *a, FAKE, BIG, None) == code, i
    # more rows than requests need row_request
    a = [FAKE] * 9
    a[5] = None
    assert lib.laga_paged_attn_q8(p, None, *a, FAKE, BIG, None) == 2
    assert lib.laga_cache_read_q8(p, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, None) == 2


def test_rotation_and_strides_are_refused():
    lib, p = B._lib, replaced()
    assert lib.laga_cache_append_q8(p, None, FAKE, 512, FAKE, FAKE, 64, FAKE, FAKE, FAKE, FAKE, None) == 1
    for bad in (B._CPrologue(-1.0, 1e4, 0), B._CPrologue(1e-6, 1.0, 0), B._CPrologue(1e-6, float("inf"), 0),
                B._CPrologue(1e-6, 1e4, -1), B._CPrologue(1e-6, 1e4, (1 << 53) - 1000)):
        assert call("append", p, cfg=ctypes.byref(bad)) == 2
        assert call("attn", p, cfg=ctypes.byref(bad)) == 2
    for ls, ks, code in ((511, 64, 2), (512, 63, 2), (0, 64, 2), (516, 64, 3), (512, 68, 3), (BIG, 64, 3)):
        assert lib.laga_cache_append_q8(p, ctypes.byref(CFG), FAKE, ls, FAKE, FAKE, ks, FAKE, FAKE, FAKE, FAKE, None) == code


def test_binding_refuses_host_tensors():
    z = {k: torch.zeros(v, dtype=torch.int32) for k, v in P.shapes().items() if k in ("block_table", "position", "slot")}
    f = {k: torch.zeros(P.shapes()[k], dtype=torch.bfloat16) for k in ("q", "w_kv_b", "latent_raw", "kpe_raw")}
    cache = torch.zeros(P.shapes()["cache"], dtype=torch.uint8).view(torch.float8_e4m3fn)
    scales = torch.zeros(P.shapes()["scales"], dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensor"):
        L.laga_cache_append_q8(P, f["latent_raw"], f["kpe_raw"], z["position"], z["slot"], cache, scales)
    with pytest.raises(ValueError, match="device tensor"):
        L.laga_cache_read_q8(P, cache, scales, z["block_table"], z["position"])
    with pytest.raises(ValueError, match="device tensor"):
        L.laga_paged_attn_q8(P, f["q"], f["w_kv_b"], cache, scales, z["block_table"], z["position"])
    with pytest.raises(TypeError, match="cache"):
        L.laga_cache_read_q8(P, None, scales, z["block_table"], z["position"])


def test_workspace_grows_with_rows_and_heads():
    need = L.laga_paged_workspace_bytes(P, L.OP_PAGED_ATTN_Q8)
    # the queries, their blocks' maxima and whole rows in fp32
    assert need >= 4 * 8 * 16 * (576 + 5 + 512)
    assert L.laga_paged_workspace_bytes(dataclasses.replace(P, rows=9, n_heads=100), L.OP_PAGED_ATTN_Q8) > need
