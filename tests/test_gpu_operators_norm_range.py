"""Per-head norms of rows whose squares leave the range of 32 bits: the norm of a row does not depend on the row's scale."""
import numpy as np
import pytest
import torch

import paper_2604_07609_amd as B
from oracle import paged as P
from tests.test_gpu_operators import TYPES, dev, new_cache, no_error_of_earlier_tests, oracle_cache, rope_table  # noqa: F401

pytestmark = pytest.mark.gpu

POWERS = [-38, -31, -21, -17, -13, -3, 0, 9, 17, 18, 19, 20, 30, 37]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -20, 1e-30])
def test_rows_of_any_scale(eps, hd, dtype, bits):
    nq, nkv = 3, 3
    powers = [p for p in POWERS if dtype != "half" or -5 <= p <= 3]
    T = len(powers) + 2
    rng = np.random.default_rng(61)
    x = np.clip(rng.standard_normal((T, 3 * nq, hd)), -3, 3)
    x[:len(powers)] *= 10.0 ** np.array(powers, dtype=np.float64)[:, None, None]
    if dtype != "half":
        x[-2, :, 5] *= 1e25                          # one element alone; and unlike heads in one token
        x[-1] *= 10.0 ** rng.integers(-30, 30, (3 * nq, 1)).astype(np.float64)
    x = torch.from_numpy(x).to(TYPES[dtype])
    gains = [(1 + 0.2 * rng.standard_normal(hd)).astype(np.float32) for _ in range(2)]
    table, pos = rope_table(T, hd), np.arange(T)
    cache = new_cache(1 + T // 16, nkv, hd, bits)
    want = oracle_cache(cache)
    q, k, v = (m.contiguous() for m in x.cuda().split(nq, 1))
    v = torch.ones_like(v)
    out = torch.zeros(T, nq, hd, dtype=torch.float16, device="cuda")
    B.qk_norm_rope(q, k, v, dev(np.int32(pos)), dev(np.int32(pos)), dev(table), cache, out, *(dev(g) for g in gains), eps=eps,
                   stream=torch.cuda.current_stream().cuda_stream)
    xd, e32 = x.double().numpy(), float(np.float32(eps))
    wq, wk = (P.norm_rope(m, g.astype(np.float64), e32, table, pos) for m, g in ((xd[:, :nq], gains[0]), (xd[:, nq:2 * nq], gains[1])))
    got = oracle_cache(cache)
    for t in range(T):
        want.put(t, wk[t], np.ones((nkv, hd)))
    # (the tolerance of the store's other tests: 2^-16 of the row's largest in 32 bits, with room for twice that, then one rounding to halves)
    pairs = [(out.double().cpu().numpy(), wq)]
    if bits == 4:
        assert np.array_equal(got.data, want.data)
    else:
        pairs.append((np.stack([got.get(t)[0] for t in range(T)]), wk))
    for a, b in pairs:
        b = np.clip(b, -65504, 65504)
        assert np.isfinite(a).all()
        off = np.abs(a - b) > 2.0 ** -11 * np.abs(b) + 2.0 ** -15 * np.abs(b).max(axis=-1, keepdims=True) + 2.0 ** -25
        assert not off.any(), (np.argwhere(off)[:5], a[off][:5], b[off][:5])
