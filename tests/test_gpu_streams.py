"""Calls on a stream that is not the current one (stream=): what they allocate is allocated on that stream, so that
no block of theirs is given out to other work while they run; and the results are those of the current stream."""
import pytest
import torch

import laga_inputs as LI
from _util import dev_inputs, problem_for, to_dev
from test_gpu_paged_attn import make
from test_gpu_paged_cache import append_inputs, i32, problem

pytestmark = pytest.mark.gpu


def block_stream(t):
    """The stream that a tensor's memory was allocated on."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's")


def on_both(call, monkeypatch):
    """call(stream): its tensors on the current stream and on another; every allocation on the other's. (The inputs
    are the caller's: made before, and kept.)"""
    want = call(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    seen, empty = [], torch.empty

    def spy(*args, **kw):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kw)

    with monkeypatch.context() as m:
        m.setattr(torch, "empty", spy)
        got = call(side)
    torch.cuda.synchronize()
    assert seen and set(seen) == {side.cuda_stream}
    for a, b in zip(want, got):
        assert torch.equal(a, b) and block_stream(b) == side.cuda_stream


def test_training_calls(monkeypatch):
    import paper_2607_17644_amd as L
    w = LI.WORKLOADS["v3_train_s16384"].replace(seq_len=200, n_heads=2)
    d, p = dev_inputs(w, LI.make_inputs(w)), problem_for(w)
    on_both(lambda s: (L.laga_reconstruct_kv(p, d["c_kv"], d["w_kv_b"], stream=s),), monkeypatch)
    kv = L.laga_reconstruct_kv(p, d["c_kv"], d["w_kv_b"])
    on_both(lambda s: L.laga_attn_fwd(p, d["q"], d["c_kv"], d["k_pe"], d["w_kv_b"], kv=kv, stream=s), monkeypatch)
    # (by position, too)
    on_both(lambda s: L.laga_attn_fwd(p, d["q"], d["c_kv"], d["k_pe"], d["w_kv_b"], kv, None, None, None, s), monkeypatch)
    out, lse = L.laga_attn_fwd(p, d["q"], d["c_kv"], d["k_pe"], d["w_kv_b"], kv=kv)
    args = (p, d["q"], d["c_kv"], d["k_pe"], d["w_kv_b"], kv, out, lse, d["dout"])
    on_both(lambda s: L.laga_attn_bwd(*args, stream=s), monkeypatch)
    on_both(lambda s: L.laga_attn_bwd_noalloc(*args, stream=s), monkeypatch)


def test_projection_and_producers(monkeypatch):
    import paper_2607_17644_amd as L
    x = {k: to_dev(v, "bf16") for k, v in LI.make_out_proj_inputs(64, 4, 128, 256).items()}
    po = L.OutProj(64, 4, 128, 256)
    on_both(lambda s: (L.laga_out_proj_fwd(po, x["out"], x["w_o"], stream=s),), monkeypatch)
    on_both(lambda s: L.laga_out_proj_bwd(po, x["out"], x["w_o"], x["dy"], stream=s), monkeypatch)
    lat, kpe, gam = append_inputs(100, 512, 64, "bf16", 9, False)
    pp = L.Problem(1, 100, 2, 512, 128, 64, 128, 0.07)
    on_both(lambda s: L.laga_prologue_fwd(pp, lat[None], kpe[None], gamma=gam, stream=s), monkeypatch)
    c, k, rstd = L.laga_prologue_fwd(pp, lat[None], kpe[None], gamma=gam)
    dc, dk = c.float(), k.float()
    on_both(lambda s: L.laga_prologue_bwd(pp, lat[None], rstd, dc, dk, gamma=gam, stream=s), monkeypatch)


def test_serving_calls(monkeypatch):
    import paper_2607_17644_amd as L
    p = problem(6, 3, 4, 12, 16)
    # (the table and the stack are written in place, with the same values each time)
    lengths, fresh, drop, table = i32([3, 0, 16]), i32([1, 2, 3]), i32([0, 1, 1]), i32([[1] * 4] * 3)
    free, count = i32(list(range(12))), i32([9])
    on_both(lambda s: L.laga_page_plan(p, lengths, fresh, table, free, count, stream=s), monkeypatch)
    on_both(lambda s: L.laga_page_release(p, lengths, drop, table, free, count, stream=s), monkeypatch)
    x = make([300, 70], 16, heads=3)
    table, position, request = i32(x["table"]), i32(x["position"]), i32(x["request"])
    on_both(lambda s: L.laga_paged_attn(x["p"], x["q"], x["w"], x["cache"], table, position, row_request=request,
                                        rope_base=10000.0, stream=s), monkeypatch)


def test_an_output_dropped_on_the_current_stream_is_kept_until_its_work_is_done():
    """The caller's own work on an output, on the current stream, before it drops it: the block is not given out to
    the call's stream before that work is done."""
    import paper_2607_17644_amd as L
    x = make([300, 70], 16, heads=3)
    table, position = i32(x["table"]), i32(x["position"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, _ = L.laga_paged_attn(x["p"], x["q"], x["w"], x["cache"], table, position, stream=side)
    at = out.data_ptr()
    torch.cuda.current_stream().wait_stream(side)
    big = torch.ones((8192, 8192), device="cuda")
    for _ in range(40):  # some milliseconds
        big = (big @ big).clamp(max=1.0)
    kept = out + 0
    del out
    with torch.cuda.stream(side):
        again = torch.empty(kept.shape, dtype=kept.dtype, device="cuda")
    assert again.data_ptr() != at
    torch.cuda.synchronize()
    want, _ = L.laga_paged_attn(x["p"], x["q"], x["w"], x["cache"], table, position)
    assert torch.equal(kept, want)
