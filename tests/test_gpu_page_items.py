"""laga_page_release of nearly 2^31 pages at once, and of one page of more than 2^30 requests each."""
import pytest
import torch

from test_gpu_paged_cache import problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,width", [(32767, 65535), ((1 << 30) + 77, 1)])
def test_release_of_the_largest_pools(R, width):
    import paper_2607_17644_amd as L
    n = R * width
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GiB")
    ids = lambda: torch.arange(n, dtype=torch.int32, device="cuda")
    p = problem(1, R, width, n, 1)
    lengths = torch.full((R,), width, dtype=torch.int32, device="cuda")
    free, count = torch.full((n,), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    drop = torch.ones((R,), dtype=torch.int32, device="cuda")
    left, count, status = L.laga_page_release(p, lengths, drop, ids().view(R, width), free, count, lengths_out=lengths)
    torch.cuda.synchronize()
    assert int(status) == 0 and int(count) == n and not left.any()
    assert torch.equal(free, ids())
