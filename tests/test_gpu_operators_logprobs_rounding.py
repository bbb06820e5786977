"""Log probabilities: how far they may be off, counted from the roundings that the sums have."""
import numpy as np
import pytest

from oracle import logprobs as L
from tests.test_gpu_operators import no_error_of_earlier_tests  # noqa: F401
from tests.test_gpu_operators_logprobs import EPS, call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temperature", [False, True])
@pytest.mark.parametrize("dtype", ["float", "bf16"])
@pytest.mark.parametrize("R, V", [(1, 128256), (3, 50257), (9, 24601), (300, 32000)])
def test_log_probabilities_are_as_near_as_their_roundings(R, V, dtype, temperature):
    x, rng = make(R, V, dtype, seed=V + R)
    tokens = np.concatenate((x.float().argmax(1, keepdim=True).cpu().numpy(), rng.integers(0, V, (R, 4))), 1)
    inverse = np.float32(1 / rng.uniform(0.5, 1.5, R)) if temperature else None
    got = call(x, tokens, inverse=inverse)["logprobs"].astype(np.float64)
    x = x.double().cpu().numpy()
    # y = x c - M is rounded once, c = log2(e) / T twice, which is as if d = z - max were off by three of its roundings, and by those of the 2 that M may lie below the
    # largest; 2^y by 2^-23. A term is then added to four others of its lane's tile, two more sums, those of the tiles after it, 64 lanes', four waves' and the parts'; wherever M
    # rises, a factor (its exponent, which is once more part of d, its power of two, the product), as many times as a wave has tiles at most
    tiles = V // 4096 + 2
    for r in range(R):
        o = L.row(x[r], 1.0 if inverse is None else float(inverse[r]))
        seen = o["p"] > 0
        spread = (o["p"][seen] * np.abs(o["d"][seen])).sum()
        log_sum = np.log(np.exp(o["d"]).sum())
        off = EPS * (4 * spread + 4 + 6 + tiles + 3 * tiles + 6 + 12 + 9)
        for a, t in zip(got[r], tokens[r]):
            # the token's own y, the logarithm (2 of its last place) and the difference times ln 2
            tol = off + EPS * (3 * abs(o["d"][t]) + 2 + 4 * log_sum + 2 * abs(o["logp"][t]))
            assert abs(a - o["logp"][t]) <= tol, (r, t, a, o["logp"][t], tol)
