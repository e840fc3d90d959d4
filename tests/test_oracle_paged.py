"""Pins of the rotation, 4-bit and paged-cache oracle (oracle/paged.py), on the CPU."""
import numpy as np
import pytest

from oracle import decode as dec
from oracle import paged

F = 10000.0 ** (-np.arange(0, 16, 2) / 16)   # 8 pairs


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_goes_by_the_distance(interleaved):
    g = np.random.default_rng(1)
    q, k = g.normal(size=(2, 32))
    for p, s in ((0, 0), (5, 3), (1000, 17), (-4, 9)):
        a, b = (paged.rotate(x, y, F, 1.0, interleaved) for x, y in ((q, p), (k, s)))
        assert np.isclose(np.linalg.norm(a), np.linalg.norm(q), rtol=1e-13)
        assert np.array_equal(a[16:], q[16:])
        far = paged.rotate(q, p + 77, F, 1.0, interleaved) @ paged.rotate(k, s + 77, F, 1.0, interleaved)
        assert np.isclose(a @ b, far, rtol=0, atol=1e-11)
    assert np.array_equal(paged.rotate(q, 0, F, 1.0, interleaved), q)


def test_rotation_closed_forms():
    x = np.zeros(32)
    x[0] = 1.0
    y = paged.rotate(x, 3, F, 2.0, False)       # pair (0, 8), frequency 1
    assert np.allclose(y[[0, 8]], [2 * np.cos(3), 2 * np.sin(3)], atol=1e-15) and np.count_nonzero(y) == 2
    y = paged.rotate(x, 3, F, 2.0, True)        # pair (0, 1)
    assert np.allclose(y[[0, 1]], [2 * np.cos(3), 2 * np.sin(3)], atol=1e-15) and np.count_nonzero(y) == 2


@pytest.mark.parametrize("interleaved", [False, True])
def test_back_is_the_gradient(interleaved):
    """Against central differences of <y, g>, exact for a linear map up to rounding."""
    gen = np.random.default_rng(2)
    x, grad = gen.normal(size=(2, 32))
    want = paged.rotate(grad, 11, F, 1.3, interleaved, back=True)
    for i in range(32):
        e = np.zeros(32)
        e[i] = 0.5
        up, down = (paged.rotate(x + s * e, 11, F, 1.3, interleaved) @ grad for s in (1, -1))
        assert np.isclose(up - down, want[i], rtol=0, atol=1e-13)


def test_codes_are_the_nearest_and_ties_go_to_even():
    # one unit block: the largest value fixes 2^0
    v = np.array([6.9, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, 0.26, 0.74, 5.01, 6.0, -6.5, 0.0] * 2)
    c, s = paged.to_codes(v)
    assert s.tolist() == [127]
    want = [6, 0, 1, 1, 2, 2, 4, 4, 0, -4, 0.5, 0.5, 6, 6, -6, 0] * 2
    assert paged.from_codes(c, s).tolist() == want
    for top, e in ((7.0, 1), (6.999, 0), (3.5, 0), (3.49, -1), (14.0, 2), (0.0, -125), (7 * 2.0 ** -130, -125)):
        v = np.zeros(32)
        v[5] = top
        assert paged.to_codes(v)[1][0] == e + 127, top
    for bad in (np.nan, np.inf, -np.inf):
        v = np.ones(64)
        v[40] = bad
        c, s = paged.to_codes(v)
        x = paged.from_codes(c, s)
        assert np.all(x[:32] == 1) and np.all(np.isnan(x[32:]))


def test_codes_error_and_idempotence():
    """A value is off by at most half a step of its range: 2^e / 4 below 2 2^e, 2^e / 2
    below 4 2^e, 2^e above; what the codes stand for codes to itself."""
    v = np.random.default_rng(3).normal(size=(50, 64)) * 3
    c, s = paged.to_codes(v)
    x = paged.from_codes(c, s)
    unit = np.repeat(2.0 ** (s.astype(float) - 127), 32, -1)
    half = np.where(np.abs(v) < 2 * unit, 0.25, np.where(np.abs(v) < 4 * unit, 0.5, 1.0)) * unit
    assert np.all(np.abs(x - v) <= half)
    assert np.array_equal(paged.from_codes(*paged.to_codes(x)), x)


def test_pages_hold_what_a_dense_cache_holds():
    g = np.random.default_rng(4)
    B, H, page, d, lens = 3, 2, 16, 32, [0, 17, 40]
    table = np.array([[4, -1, 99], [7, 2, -1], [0, 6, 1]])
    pool = g.normal(size=(2, 8, H, page, d))
    c = paged.Cache(pool[0], pool[1], table)
    dense = np.zeros((2, B, H, 48, d))
    for b in range(B):
        for p in range(lens[b]):
            at = c.place(b, p)
            dense[0, b, :, p], dense[1, b, :, p] = c.k[at[0], :, at[1]], c.v[at[0], :, at[1]]
    new = g.normal(size=(2, B, H, d))
    for b in range(B):
        c.write(b, lens[b], new[0, b], new[1, b])
    q = g.normal(size=(B, 4, d))
    O, L, A, S = c.attend(q, [x + 1 for x in lens], 0.3)
    ref = dec.decode_step(q, dense[0], dense[1], lens, 0.3, new[0], new[1])
    assert np.allclose(O, ref["O"], atol=1e-13) and np.allclose(L, ref["L"], atol=1e-13)
    assert np.all(A >= np.abs(O) - 1e-15)
    assert c.place(0, 16) is None and c.place(0, 32) is None and c.place(0, 48) is None and c.place(0, -1) is None
    O, L, _, _ = c.attend(q, [0, 0, 0], 0.3)
    assert np.all(O == 0) and np.all(L == -np.inf)
