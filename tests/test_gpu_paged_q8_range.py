"""laga_paged_attn_q8 over the range that the format has: powers of two that leave the scores as they are leave the results
as they are, bit for bit."""
import dataclasses

import pytest
import torch

from test_gpu_paged_q8 import call, check, eight, make

pytestmark = pytest.mark.gpu

FORMS = [(4, "bf16"), (20, "bf16"), (40, "bf16"), (130, "bf16"), (4, "fp32"), (24, "fp32"), (64, "fp32")]


def moved(x, q_nope=0, q_rope=0, latent=0, key=0, scale=0):
    """x with these powers of two on the query's parts, the cache's two scales and the softmax's scale (all exact)."""
    dn, s = x["p"].d_nope, x["scales"].int()
    s[..., 0] += latent
    s[..., 1] += key
    assert int(s.min()) >= 0 and int(s.max()) < 255
    q = torch.cat((x["q"][..., :dn] * 2.0 ** q_nope, x["q"][..., dn:] * 2.0 ** q_rope), -1)
    return dict(x, q=q, scales=s.to(torch.uint8), p=dataclasses.replace(x["p"], softmax_scale=x["p"].softmax_scale * 2.0 ** scale))


def same(a, b, power=0):
    assert a[0].isfinite().all() and a[1].isfinite().all()
    assert torch.equal(a[0], (b[0].double() * 2.0 ** -power).to(a[0].dtype)) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("heads,dtype", FORMS)
@pytest.mark.parametrize("d_c", [512, 1024])
def test_large_keys_under_a_small_softmax_scale(heads, dtype, d_c):
    """The band alone decides: keys of 2^126, products of the scaled query with them past fp32's range, scores of a few."""
    x = make([300, 31, 70], 16, heads=heads, dtype=dtype, seed=heads, d_c=d_c)
    x["q"][..., :x["p"].d_nope] = 0.0
    same(call(x, base=10000.0), call(moved(x, q_rope=-70, key=130, scale=-60), base=10000.0))


@pytest.mark.parametrize("heads,dtype", FORMS)
@pytest.mark.parametrize("d_c", [512, 1024])
def test_the_largest_latents(heads, dtype, d_c):
    """Rows of one tile (the sums of more than a few such numbers pass fp32's range themselves): latents of up to 2^127."""
    x = make([32, 1, 20], 16, heads=heads, dtype=dtype, seed=heads, d_c=d_c)
    same(call(x), call(moved(x, q_nope=-62, q_rope=-62, latent=124, key=124, scale=-62)), 124)


@pytest.mark.parametrize("heads,dtype", FORMS)
def test_small_numbers_under_large_queries(heads, dtype):
    x = make([300, 31, 70], 16, heads=heads, dtype=dtype, seed=heads)
    same(call(x), call(moved(x, q_nope=50, q_rope=50, latent=-70, key=-70, scale=20)), -70)


@pytest.mark.parametrize("heads,dtype", FORMS)
@pytest.mark.parametrize("power", [12, -12, 50, -80])
def test_the_query_s_two_parts_have_sizes_of_their_own(heads, dtype, power):
    x = make([300, 31, 70], 16, heads=heads, dtype=dtype, seed=heads)
    y = moved(x, q_rope=power, key=-power)
    same(check(x, base=10000.0) if heads < 64 else call(x, base=10000.0), call(y, base=10000.0))


@pytest.mark.parametrize("widths,d_c,heads,dtype", [("v3", 512, 4, "bf16"), ("v3", 512, 20, "bf16"), ("v3", 512, 40, "fp32"), ("v3", 1024, 3, "fp32"),
                                                    ("half", 416, 24, "bf16"), ("small", 64, 4, "fp32")])
@pytest.mark.parametrize("power", [6, 12])
def test_columns_of_many_sizes(widths, d_c, heads, dtype, power):
    """Every second number of the latents smaller by 2^power, and what the query has for it larger: their products count alike."""
    x = make([200, 31, 70], 16, widths, d_c, heads, dtype, seed=d_c)
    p = x["p"]
    v = x["cache"].float()
    v[..., :d_c] *= torch.exp2(x["scales"][..., :1].float() - 127)
    v[..., d_c:] *= torch.exp2(x["scales"][..., 1:].float() - 127)
    v[..., :d_c:2] *= 2.0 ** -power
    cache, scales = eight(v, d_c)
    w = x["w"].clone().view(d_c, heads, p.d_nope + p.d_v)
    w[::2, :, :p.d_nope] *= 2.0 ** power
    check(dict(x, cache=cache, scales=scales, w=w.view(d_c, -1)))
