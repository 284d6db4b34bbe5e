"""A laga.Paged that calls have used is copied and pickled as any dataclass, and the copy has its own fields."""
import copy
import dataclasses
import pickle

import pytest

import paper_2607_17644_amd as L

P = L.Paged(rows=8, requests=4, table_width=16, n_pages=100, page_size=64, n_heads=16, d_c=512, d_nope=128, d_rope=64,
            d_v=128, softmax_scale=0.072, page_stride=64 * 576 + 8)


@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, lambda p: pickle.loads(pickle.dumps(p)), dataclasses.replace])
def test_a_used_problem_is_copied(again):
    p = dataclasses.replace(P)
    need = L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN)
    q = again(p)
    assert q == p and q is not p and dataclasses.asdict(q) == dataclasses.asdict(p)
    assert L.laga_paged_workspace_bytes(q, L.OP_PAGED_ATTN) == need
    q.n_heads = 64
    assert L.laga_paged_workspace_bytes(q, L.OP_PAGED_ATTN) > need == L.laga_paged_workspace_bytes(p, L.OP_PAGED_ATTN)
    assert p.shapes()["q"] == (8, 16, 192) and q.shapes()["q"] == (8, 64, 192)
