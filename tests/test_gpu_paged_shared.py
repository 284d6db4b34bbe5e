"""laga_paged_attn where several rows read the same pages: successive rows of one request, and rows of requests
whose tables name the same pages."""
import dataclasses

import numpy as np
import pytest
import torch

from test_gpu_paged_attn import call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,lengths", [(4, [40000, 30000]), (40, [20000, 21000]), (100, [9000, 12000]), (16, [300, 70])])
def test_rows_of_one_request_and_of_two_with_its_pages(heads, lengths):
    """Each request's row twice, as two rows of it and as rows of two requests with equal tables, side by side and
    apart: the order of tiles, and so every bit, is the same (by position and request alone)."""
    x = make(lengths, 64, heads=heads, seed=heads)
    table, q = x["table"], x["q"]
    one = dict(x, table=table, q=q[[0, 0, 1, 1]].contiguous(), position=x["position"][[0, 0, 1, 1]], request=np.array([0, 0, 1, 1]),
               p=dataclasses.replace(x["p"], rows=4))
    two = dict(one, table=table[[0, 0, 1, 1]].copy(), request=np.arange(4), p=dataclasses.replace(x["p"], rows=4, requests=4))
    a, b, c = call(one, base=10000.0), call(two, base=10000.0), call(two, base=10000.0, row_request=None)
    for i in range(2):
        assert torch.equal(a[i], b[i]) and torch.equal(a[i], c[i])
    # (a request's two rows are cut into shares at other places)
    assert torch.allclose(a[0][0].float(), a[0][1].float(), rtol=2.0 ** -7, atol=2.0 ** -7) and a[0].isfinite().all()


def test_padding_between_the_rows_of_a_request():
    x = make([30000, 9], 48, heads=8, fresh=3, pad=4)
    a = call(x)
    live = [t for t, n in enumerate(x["position"]) if n >= 0]
    y = dict(x, q=x["q"][live].contiguous(), position=x["position"][live], request=x["request"][live],
             p=dataclasses.replace(x["p"], rows=len(live)))
    b = call(y)
    assert torch.equal(a[0][live], b[0]) and torch.equal(a[1][live], b[1])
