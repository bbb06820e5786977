"""The oracle of the paged-cache operators on its own: the 4-bit form and the layouts (no GPU needed)."""
import numpy as np
import pytest

from oracle import paged as P


def test_encode4_against_all_values():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((64, 64)) * np.exp(rng.uniform(-12, 9, (64, 1)))
    x[3, :32] = 0
    c, s = P.encode4(x)
    y = P.decode4(c, s)
    assert np.isfinite(y).all() and (y[3, :32] == 0).all()
    for r in range(64):
        for g in range(2):
            a, b = x[r, 32 * g:32 * g + 32], y[r, 32 * g:32 * g + 32]
            step = 2.0 ** (int(s[r, g]) - 127)
            top = np.abs(a).max()
            assert top == 0 or 3.5 * step < top <= 7 * step
            near = np.abs(np.abs(a)[:, None] - P.LEVELS[:8] * step).min(axis=1)
            assert np.array_equal(np.abs(np.abs(a) - np.abs(b)), near)


@pytest.mark.parametrize("x, want", [(0.25, 0), (0.75, 1), (1.25, 1), (1.75, 2), (2.5, 2), (3.5, 4), (5, 4), (7, 6), (-0.75, -1), (0.26, 0.5), (6.5, 6)])
def test_ties_go_to_the_even_code(x, want):
    g = np.zeros((1, 32))
    g[0, 0], g[0, 1] = 7.0, x
    c, s = P.encode4(g)
    assert s[0, 0] == 127 and P.decode4(c, s)[0, 1] == want


def test_exponents_end_where_values_leave_the_halves():
    g = np.zeros((3, 32))
    g[0, 0], g[1, 0], g[2, 0] = 1e9, 1e-9, 2.0 ** -24
    c, s = P.encode4(g)
    y = P.decode4(c, s)
    assert list(s[:, 0]) == [P.E_MAX + 127, P.E_MIN + 127, P.E_MIN + 127]
    assert y[0, 0] == 6 * 2.0 ** 13 == P.half(y)[0, 0] and y[1, 0] == 0 and y[2, 0] == 2.0 ** -24 == P.half(y)[2, 0]
    for bad in (np.nan, np.inf, -np.inf):
        g[0, 5] = bad
        assert np.isnan(P.decode4(*P.encode4(g))[0]).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("bits", [16, 4])
def test_put_and_get_are_inverse_and_places_are_apart(hd, bits):
    rng = np.random.default_rng(1)
    nb, nkv = 3, 2
    c = P.Cache(np.zeros(P.cache_bytes(nb, nkv, hd, bits), dtype=np.uint8), nb, nkv, hd, bits)
    want = {}
    for s in rng.permutation(nb * 16):
        k, v = rng.standard_normal((2, nkv, hd))
        c.put(int(s), k, v)
        want[int(s)] = (k, v)
    for s, (k, v) in want.items():
        for a, b in zip(c.get(s), (k, v)):
            assert np.array_equal(a, P.decode4(*P.encode4(b)) if bits == 4 else P.half(b))
    before = c.data.copy()
    c.put(-1, *want[0])
    c.put(nb * 16, *want[0])
    assert np.array_equal(before, c.data)


def test_visible():
    assert list(P.visible(9, 3, 2)) == [0, 1, 7, 8, 9] and list(P.visible(3, 0, 0)) == [0, 1, 2, 3]
    assert list(P.visible(2, 1, 0)) == [2] and list(P.visible(-1, 4, 4)) == [] and list(P.visible(4, 9, 3)) == [0, 1, 2, 3, 4]
