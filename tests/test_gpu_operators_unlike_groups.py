"""Scores over a 4-bit cache where groups of 32 dimensions differ by many powers of two, in queries and keys: every product counts in 32 bits."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from tests.test_gpu_operators import make_batch, no_error_of_earlier_tests, run_attention  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd, powers", [(64, [8, -12]), (64, [-12, 8]), (128, [8, -12, 0, -6]), (128, [-12, -6, 8, 0]), (128, [0, 8, -6, -12])])
@pytest.mark.parametrize("runs", [[1, 1], [5, 3], [60, 40]])
def test_queries_and_keys_of_unlike_groups(runs, hd, powers):
    nq, nkv = 4, 2
    cache, c, tables, lens, cu, q = make_batch([150, 70], runs, nq, nkv, hd, 4, seed=71)
    rng = np.random.default_rng(72)
    scale = np.repeat(2.0 ** np.array(powers), 32)
    q = (rng.standard_normal(q.shape) * scale / np.sqrt(hd)).astype(np.float16)
    for s, n in enumerate(lens):
        for j in range(n):
            c.put(int(tables[s, j // 16]) * 16 + j % 16, rng.standard_normal((nkv, hd)) / scale, rng.standard_normal((nkv, hd)))
    cache.data.copy_(torch.from_numpy(c.data))
    got = run_attention(cache, tables, lens, cu, q, max(runs))
    want, spread = P.attention(q.astype(np.float64), c, tables, lens, cu)
    # A score: hd products added in 32 bits, off by hd 2^-24 of the sum of |q| |k| over the groups of 32; and each group of the query to within 2^-25 of its
    # largest, times the sum of 32 magnitudes of the key (at most 6 |k|): 3 2^-24 of the same. Twice (numerator and sum), then as for other scores:
    # a probability's rounding to a half, its bottom, the output's rounding
    groups = lambda x: np.linalg.norm(x.reshape(*x.shape[:-1], -1, 32), axis=-1)      # noqa: E731
    kept = [c.get(int(tables[s, j // 16]) * 16 + j % 16) for s, n in enumerate(lens) for j in range(n)]
    K, V = np.stack([k for k, _ in kept]), np.stack([v for _, v in kept])
    qk = (groups(q.astype(np.float64)).reshape(-1, hd // 32).max(axis=0) * groups(K).reshape(-1, hd // 32).max(axis=0)).sum()
    delta = 2 * ((hd + 3) * 2.0 ** -24 * qk + 2.0 ** -21) + 2.0 ** -11
    assert delta < 2.0 ** -9
    off = np.abs(got - want) > delta * spread + 2.0 ** -11 * np.abs(want) + 2.0 ** -25 * (1 + 150 * np.abs(V).max())
    assert not off.any(), (np.argwhere(off)[:5], got[off][:5], want[off][:5])


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("runs", [[1, 1], [3, 2], [60, 40]])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_query_that_is_not_finite_gives_nan_and_leaves_others_alone(bad, runs, hd):
    """In each group of its dimensions in turn."""
    nq, nkv = 4, 2
    cache, c, tables, lens, cu, q = make_batch([150, 70], runs, nq, nkv, hd, 4, seed=73)
    clean = run_attention(cache, tables, lens, cu, q, max(runs))
    for d in range(7, hd, 16):
        x = q.copy()
        x[0, 1, d] = bad
        got = run_attention(cache, tables, lens, cu, x, max(runs))
        assert np.isnan(got[0, 1]).all()
        got[0, 1] = clean[0, 1]
        assert np.array_equal(got, clean)
