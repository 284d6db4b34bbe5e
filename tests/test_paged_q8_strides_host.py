"""A pool in 8 bits whose strides are not the call's is refused by its strides, by the binding, without a GPU."""
import dataclasses

import pytest
import torch

from paper_2607_17644_amd import binding as B
from test_paged_host import P

F8 = torch.float8_e4m3fn


def test_a_pool_with_other_strides_is_refused():
    n, page, width = P.shapes()["cache"]
    good = torch.zeros((n, page, width), dtype=torch.uint8)
    assert B._cache_at(P, good.view(F8), -1, F8) == good.data_ptr()
    turned = torch.zeros((n, width, page), dtype=torch.uint8).transpose(1, 2).view(F8)
    wider = torch.zeros((n, page, width + 16), dtype=torch.uint8)[..., :width].view(F8)
    apart = torch.zeros((n, page + 1, width), dtype=torch.uint8)[:, :page].view(F8)
    for t in (turned, wider, apart):
        assert t.shape == good.shape
        with pytest.raises(ValueError, match="cache has strides"):
            B._cache_at(P, t, -1, F8)
    # pages apart by what the problem says are not
    assert B._cache_at(dataclasses.replace(P, page_stride=(page + 1) * width), apart, -1, F8) == apart.data_ptr()
    with pytest.raises(ValueError, match="cache has strides"):
        B._cache_at(dataclasses.replace(P, page_stride=(page + 1) * width), good.view(F8), -1, F8)
