"""laga_paged_attn_q8: rows beside others that are outside the table or the pool, and a prompt's chunk over its cached prefix,
held to the bounds of every other row."""
import numpy as np
import pytest
import torch

from _util import f64
from test_gpu_paged_q8 import attend, bounds, call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,dtype", [(3, "bf16"), (20, "bf16"), (40, "bf16"), (128, "bf16"), (3, "fp32"), (40, "fp32")])
def test_rows_beside_bad_ones(heads, dtype):
    """Shares are laid out anew around the bad rows: no tile of another row is left out or taken twice."""
    x = make([70, 33, 40, 500, 64, 9, 2000], 16, heads=heads, dtype=dtype, width=125)
    x["table"][1, 0] = x["p"].n_pages  # a visible page past the pool
    x["table"][2, 2] = -5              # below it
    x["request"][4] = 7                # no such request
    x["position"][5] = 125 * 16        # past the table
    bad = np.isin(np.arange(7), [1, 2, 4, 5])
    out, lse = call(x, base=10000.0)
    assert out[torch.from_numpy(bad).cuda()].isnan().all() and lse[torch.from_numpy(bad).cuda()].isnan().all()
    y = dict(x, position=np.where(bad, -1, x["position"]))
    (ro, rl), (bo, bl) = attend(y, 10000.0), bounds(y, 10000.0, 0)
    assert (np.abs(f64(out) - ro) <= bo)[~bad].all() and (np.abs(f64(lse) - rl) <= bl)[~bad].all()


@pytest.mark.parametrize("heads,dtype", [(4, "bf16"), (20, "bf16"), (40, "bf16"), (4, "fp32")])
def test_a_prompt_s_chunk_over_its_prefix(heads, dtype):
    """Sixty new tokens of each of two prompts, a row each, over what is cached of them (nothing, of the second)."""
    check(make([200, 60], 16, heads=heads, dtype=dtype, fresh=60, pad=2), base=10000.0, offset=3)
