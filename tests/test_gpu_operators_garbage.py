"""Attention over a cache whose hidden and unused places hold anything at all: bytes of uninitialised memory, not only infinities and NaN."""
import copy

import numpy as np
import pytest
import torch

from tests.test_gpu_operators import check_attention, make_batch, no_error_of_earlier_tests, run_attention  # noqa: F401

pytestmark = pytest.mark.gpu


def litter(c, lens, runs, tables, window, sinks, scales, seed):
    """Random bytes in every place of the cache that no query sees; in 4 bits with scale bytes of the given range."""
    rng = np.random.default_rng(seed)
    kept = np.zeros(16 * c.n_blocks, dtype=bool)
    for s, n in enumerate(lens):
        for j in range(n):
            first = n - runs[s]                      # the first query's position: of all of them it sees farthest back
            if 0 <= tables[s, j // 16] < c.n_blocks and (not window or j > first - window or j < sinks):
                kept[tables[s, j // 16] * 16 + j % 16] = True
    for slot in np.flatnonzero(~kept):
        b, o, hd = slot // 16, slot % 16, c.hd
        if c.bits == 16:
            c.k.view(np.uint16)[b, :, o] = rng.integers(0, 1 << 16, (c.nkv, hd))
            c.v.view(np.uint16)[b, :, :, o] = rng.integers(0, 1 << 16, (c.nkv, hd))
            continue
        g = np.arange(hd // 32) * 16 + o
        c.kc[b, :, o * (hd // 2):(o + 1) * (hd // 2)] = rng.integers(0, 256, (c.nkv, hd // 2))
        c.vc[b][:, c._value_at(o)] = rng.integers(0, 256, (c.nkv, hd // 2))
        c.ks[b][:, g] = rng.integers(scales[0], scales[1] + 1, (c.nkv, hd // 32))
        c.vs[b][:, g] = rng.integers(scales[0], scales[1] + 1, (c.nkv, hd // 32))


@pytest.mark.parametrize("bits, scales", [(16, (0, 255)), (4, (0, 255)), (4, (141, 254)), (4, (141, 141))])
@pytest.mark.parametrize("runs", [[1, 1, 1, 1], [5, 3, 1, 2], [70, 90, 1, 3]])
@pytest.mark.parametrize("window, sinks", [(0, 0), (37, 3)])
@pytest.mark.parametrize("hd, nq, nkv", [(64, 4, 2), (128, 8, 2)])
def test_what_hidden_places_hold_does_not_matter(hd, nq, nkv, window, sinks, runs, bits, scales):
    cache, c, tables, lens, cu, q = make_batch([250, 97, 33, 7], runs, nq, nkv, hd, bits, seed=51, width=20)
    tables[0, 3] = -1                                # (keys of no block: another block is read in its place)
    tables[1, 5] = c.n_blocks
    dirty = copy.deepcopy(c.data)
    litter(type(c)(dirty, c.n_blocks, nkv, hd, bits), lens, runs, tables, window, sinks, scales, 52)
    cache.data.copy_(torch.from_numpy(dirty))
    got = run_attention(cache, tables, lens, cu, q, max(runs), window, sinks)
    check_attention(got, cache, c, tables, lens, cu, q, window, sinks)
