"""Pins of oracle.paged: hand-written steps, conservation of pages, and its rows against the
whole-sequence oracles."""
import numpy as np
import pytest

import laga_inputs as LI
from oracle import absorbed, laga, paged, producers


def test_plan_of_a_hand_written_step():
    # pages of 4; request 0 has 3 tokens (page 7), request 1 none, request 2 has 8 (pages 1, 5)
    table = np.array([[7, -1, -1], [-1, -1, -1], [1, 5, -1]])
    free = [0, 2, 3, 4, 6, -1, -1, -1]
    o = paged.plan([3, 0, 8], [2, 0, 1], table, free, 5, rows=5, page=4)
    assert o["status"] == 0 and o["free_count_out"] == 3 and o["lengths_out"] == [5, 0, 9]
    assert o["block_table"].tolist() == [[7, 6, -1], [-1, -1, -1], [1, 5, 4]]
    assert o["row_begin"] == [0, 2, 2, 3]
    assert o["row_request"] == [0, 0, 2, -1, -1] and o["position"] == [3, 4, 8, -1, -1]
    assert o["slot"] == [7 * 4 + 3, 6 * 4, 4 * 4, -1, -1]
    # all or nothing, each reason
    for args, code in ((([3, 0, 8], [2, 1, 3], table, free, 5, 5), paged.PLAN_ROWS),
                       (([3, 0, 8], [2, 0, 5], table, free, 5, 9), paged.PLAN_TABLE),
                       (([3, 0, 8], [2, 0, 1], table, free, 1, 9), paged.PLAN_PAGES),
                       (([3, -1, 8], [2, 0, 1], table, free, 5, 9), paged.PLAN_INVALID),
                       (([3, 0, 8], [2, 0, 1], table, free, 9, 9), paged.PLAN_INVALID)):
        o = paged.plan(*args, page=4)
        assert o["status"] == code and o["row_begin"] == [0] * 4 and set(o["slot"]) == {-1}
        assert o["block_table"].tolist() == table.tolist() and o["lengths_out"] == args[0]


@pytest.mark.parametrize("page", [1, 3, 16])
def test_pages_are_conserved_over_random_steps(page):
    rng = np.random.default_rng(page)
    R, n_pages, width = 6, 40, 12
    table, free, count, lengths = np.full((R, width), -1), list(rng.permutation(n_pages)), n_pages, [0] * R
    for _ in range(60):
        fresh = rng.integers(0, 3 * page, R)
        o = paged.plan(lengths, fresh, table, free, count, rows=200 * page, page=page)
        if o["status"] == 0:
            live = [s for s in o["slot"] if s >= 0]
            assert len(live) == len(set(live)) == fresh.sum()
        else:
            assert o["free_count_out"] == count
        table, count, lengths = o["block_table"], o["free_count_out"], o["lengths_out"]
        drop = rng.random(R) < 0.2
        o = paged.release(lengths, drop, table, free, count, page)
        assert o["status"] == 0
        free, count, lengths = o["free_pages"], o["free_count_out"], o["lengths_out"]
        held = [int(table[r, j]) for r in range(R) for j in range(-(-lengths[r] // page))]
        assert sorted(held + free[:count]) == list(range(n_pages))


def _cached(w, page, seed=0):
    """A one-sequence workload with its rows in a paged cache."""
    rng = np.random.default_rng(seed)
    x = LI.make_inputs(w)
    n_pages = -(-w.seq_len // page) + 2
    ids = rng.permutation(n_pages)
    cache = rng.standard_normal((n_pages, page, w.d_c + w.d_rope))
    for j in range(w.seq_len):
        cache[ids[j // page], j % page] = np.concatenate([x["c_kv"][0, j], x["k_pe"][0, j]])
    return x, cache, ids[None]


@pytest.mark.parametrize("page", [1, 7, 32])
def test_attend_is_the_row_of_the_whole_sequence(page):
    w = LI.WORKLOADS["tiny_fp32"].replace(seq_len=50)
    x, cache, table = _cached(w, page)
    kw = dict(n_heads=w.n_heads, d_nope=w.d_nope, d_v=w.d_v, scale=w.scale)
    ro, rl = laga.attn_fwd(x["q"], x["c_kv"], x["k_pe"], x["w_kv_b"], **kw)
    ao, al = absorbed.absorbed_fwd(x["q"], x["c_kv"], x["k_pe"], x["w_kv_b"], **kw)
    pos = [0, 1, 30, 31, 32, 49, -1]
    o, l = paged.attend(x["q"][0][pos], x["w_kv_b"], cache, table, pos, [0] * len(pos), d_c=w.d_c, d_nope=w.d_nope,
                        d_v=w.d_v, scale=w.scale)
    np.testing.assert_allclose(o[:-1], ro[0][pos[:-1]], rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(o[:-1], ao[0][pos[:-1]], rtol=1e-9, atol=1e-12)
    np.testing.assert_allclose(l[:-1], rl[0].T[pos[:-1]], rtol=1e-12)
    np.testing.assert_allclose(l[:-1], al[0].T[pos[:-1]], rtol=1e-9)
    assert not o[-1].any() and np.isneginf(l[-1]).all()


def test_append_then_attend_is_prologue_then_attention():
    w = LI.WORKLOADS["tiny_fp32"].replace(seq_len=21)
    y = LI.make_prologue_inputs(w)
    page, n_pages = 8, 5
    o = paged.plan([0], [21], np.full((1, 3), -1), list(range(n_pages)), n_pages, rows=21, page=page)
    cache = paged.append(y["latent_raw"][0], y["kpe_raw"][0], o["position"], o["slot"],
                         np.zeros((n_pages, page, w.d_c + w.d_rope)), gamma=y["gamma"], offset=3)
    c, k, q, _ = producers.prologue_forward(y["latent_raw"], y["kpe_raw"], y["q"], w.d_nope, y["gamma"], 1e-6, 1e4, 3)
    rows = paged.gather(cache, o["block_table"][0], 21)
    np.testing.assert_allclose(rows, np.concatenate([c[0], k[0]], -1), rtol=1e-12, atol=1e-14)
    wkv = LI.make_inputs(w)["w_kv_b"]
    ro, rl = laga.attn_fwd(q, c, k, wkv, n_heads=w.n_heads, d_nope=w.d_nope, d_v=w.d_v, scale=w.scale)
    po, pl = paged.attend(y["q"][0], wkv, cache, o["block_table"], o["position"], o["row_request"], d_c=w.d_c,
                          d_nope=w.d_nope, d_v=w.d_v, scale=w.scale, base=1e4, offset=3)
    np.testing.assert_allclose(po, ro[0], rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(pl, rl[0].T, rtol=1e-10)


def test_what_lies_outside_is_nan():
    w = LI.WORKLOADS["tiny_fp32"].replace(seq_len=20)
    x, cache, table = _cached(w, 8)
    table = np.array([[table[0, 0], -1, table[0, 2]]])
    kw = dict(d_c=w.d_c, d_nope=w.d_nope, d_v=w.d_v, scale=w.scale)
    o, l = paged.attend(x["q"][0][:4], x["w_kv_b"], cache, table, [7, 8, 24, 3], [0, 0, 0, 5], **kw)
    assert np.isfinite(o[0]).all() and np.isnan(o[1:]).all() and np.isnan(l[1:]).all()
