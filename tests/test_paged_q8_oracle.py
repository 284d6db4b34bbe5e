"""The oracle of a cache in 8 bits: its numbers by hand and against torch's own e4m3, the scale's rule, rows."""
import numpy as np
import torch

from oracle import eight as E
from oracle import paged as O


def test_numbers():
    n = E.numbers()
    assert n[0] == 0 and n[1] == 2.0 ** -9 and n[7] == 7 * 2.0 ** -9 and n[8] == 2.0 ** -6 and n[0x38] == 1.0
    assert n[126] == 448.0 and np.isnan(n[127]) and np.isnan(n[255]) and n[0xb8] == -1.0 and np.signbit(n[128])
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(n, t, equal_nan=True)


def test_the_scale_is_the_least_that_holds_the_largest():
    assert [E.exponent(x) for x in (448.0, 448.0001, 1.75, 1.7500001, 3.5, 0.0, 2.0 ** -300, 1e300)] == \
        [0, 1, -8, -7, -7, -100, -100, 119]


def test_quantise_rounds_to_the_nearest_even():
    # scale 1: the largest is in (224, 448]
    x = np.array([448.0, 1.0, 1.0625, 1.1875, 1.06250001, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, np.nan, -np.inf])
    b, e = E.quantise(x)
    assert e == 0
    assert b.tolist() == [126, 0x38, 0x38, 0x3a, 0x39, 128, 0, 2, 127, 127]
    rng = np.random.default_rng(0)
    y = rng.normal(size=4096).astype(np.float32)
    b, e = E.quantise(y)
    want = torch.from_numpy(y * np.float32(2.0 ** -e)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert e == int(np.ceil(np.log2(np.abs(y).max() / 448.0))) and np.array_equal(b, want)
    assert np.abs(E.numbers()[b] * 2.0 ** e - y).max() <= 2.0 ** -4 * np.abs(y).max()


def test_rows_and_what_they_stand_for():
    rng = np.random.default_rng(1)
    lat, kpe = rng.normal(size=(3, 64)), 30 * rng.normal(size=(3, 16))
    cache, scales = np.full((2, 4, 80), 9, np.uint8), np.full((2, 4, 2), 7, np.uint8)
    c, s = E.append(lat, kpe, [5, 0, 9], [6, -1, 0], cache, scales, gamma=np.full(64, 2.0))
    want = O.append(lat, kpe, [5, 0, 9], [6, -1, 0], np.zeros((2, 4, 80)), gamma=np.full(64, 2.0))
    v = E.values(c, s, 64)
    for p, r in ((1, 2), (0, 0)):
        assert np.abs(v[p, r, :64] - want[p, r, :64]).max() <= 2.0 ** -4 * np.abs(want[p, r, :64]).max()
        assert np.abs(v[p, r, 64:] - want[p, r, 64:]).max() <= 2.0 ** -4 * np.abs(want[p, r, 64:]).max()
        assert s[p, r, 1] > s[p, r, 0]
    keep = np.ones((2, 4), bool)
    keep[1, 2] = keep[0, 0] = False
    assert (c[keep] == 9).all() and (s[keep] == 7).all()
    table = np.array([[1, 0], [5, -1]])
    ck, kp = E.read(c, s, table, [2, 4, -1, 0, 9, 1], [0, 0, 0, 1, 0, -1], 64)
    assert np.array_equal(ck[0], v[1, 2, :64]) and np.array_equal(kp[1], v[0, 0, 64:])
    assert not ck[2].any() and all(np.isnan(ck[i]).all() for i in (3, 4, 5))
