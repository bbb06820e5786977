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


@pytest.mark.parametrize("name", ["mini_norm", "mini_window", "mini_kv4", "mini_long", "mini_long_moe"])
def test_three_forms_of_the_model_agree(name):
    """Dense, cached and paged evaluation of the models with per-head norms, windows and 4-bit caches."""
    import synth
    from oracle import model as M
    cfg = dict(synth.model_config(name), vocab=97, d_model=64, d_ffn=32, n_layers=2)
    if "window" in cfg:
        cfg.update(window=7, sinks=2)
    W = M.Weights(cfg, synth.make_weights(cfg, 7, std=0.2, gain_jitter=0.3))
    toks = np.random.default_rng(8).integers(0, 97, 24)
    dense = M.forward_dense(cfg, W, toks)
    m = M.CachedModel(cfg, W)
    step = [m.step(toks[:9])] + [m.step(toks[i:i + 1]) for i in range(9, 24)]
    assert np.allclose(step, dense[8:], rtol=1e-9, atol=1e-9)
    kv = M.PagedKV(cfg, 4, 16)
    table = [2, 0]
    out = M.paged_forward(cfg, W, kv, toks, np.arange(24), [table[p // 16] * 16 + p % 16 for p in range(24)], [0] * 24, [table], [23])
    assert np.allclose(out[0], dense[-1], rtol=1e-9, atol=1e-9)


@pytest.mark.parametrize("window, sinks", [(0, 0), (5, 0), (5, 3), (1, 0)])
def test_attention_against_a_dense_mask(window, sinks):
    rng = np.random.default_rng(3)
    n, nq, nkv, hd = 21, 4, 2, 64
    c = P.Cache(np.zeros(P.cache_bytes(3, nkv, hd, 16), dtype=np.uint8), 3, nkv, hd, 16)
    table = np.array([[2, 0]])
    for j in range(n):
        c.put(int(table[0, j // 16]) * 16 + j % 16, *rng.standard_normal((2, nkv, hd)))
    q = rng.standard_normal((6, nq, hd))
    out, _ = P.attention(q, c, table, [n], [0, 6], window, sinks, 0.3)
    K, V = (np.stack([c.get(int(table[0, j // 16]) * 16 + j % 16)[i] for j in range(n)]) for i in (0, 1))
    for t in range(6):
        p = n - 6 + t
        for h in range(nq):
            s = 0.3 * K[:, h // 2] @ q[t, h]
            hidden = np.array([j > p or (window and j <= p - window and j >= sinks) for j in range(n)], dtype=bool)
            s[hidden] = -np.inf
            e = np.exp(s - s.max())
            assert np.allclose(out[t, h], e @ V[:, h // 2] / e.sum())
