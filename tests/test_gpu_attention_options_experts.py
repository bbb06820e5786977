"""An engine with experts and a 4-bit cache at once. Every token takes all of its experts, so that no choice hangs on logits that the codes move."""
import numpy as np
import pytest

import synth
from tests import parity
from tests.test_gpu_attention_options import tokens_of
from tests.test_gpu_parity import sampled

pytestmark = pytest.mark.gpu

# 8 %: what a 4-bit cache moves a logits row of two layers by at most (derived beside the dense engines' tests). The experts' weights add to it: a router
# logit (about 0.45 here: 512 terms of 0.02) moves by those 4.4 % of itself, 0.02, its weight by as much of itself, and the sum of the experts'
# outputs, half of the residual stream, by 1 % of the row. sqrt(4.4^2 + 1^2) 1.35 + 2 = 8.1 %
RTOL = 9e-2


@pytest.mark.parametrize("window, qk_norm", [(0, 0), (80, 1)])
def test_stepwise(lib, monkeypatch, window, qk_norm):
    cfg = dict(synth.model_config("mini_long_moe"), n_experts=4, n_active=4, kv_bits=4, window=window, sinks=16 if window else 0, qk_norm=qk_norm)
    eng = synth.engine_config("mini_long_moe")
    raw = synth.make_weights(cfg, 201, gain_jitter=0.1)
    blob = synth.pack_blob(cfg, raw)
    monkeypatch.setattr(parity, "ROUTE_MARGIN", 2 * RTOL)      # (the order of two experts: each one's logit moves by at most that of the largest)
    reqs = sampled(synth.make_workload("mini", cfg["vocab"], 301, n_requests=9), 201)
    toks = {}
    worst = parity.stepwise_check(lib, cfg, eng, raw, blob, reqs, rtol=RTOL, tokens_out=toks)
    print("worst relative logit error", worst)
    ev, _, st = parity.run_engine(lib, cfg, eng, blob, reqs)
    assert tokens_of(ev) == toks and st["free_blocks"] == eng["kv_num_blocks"]
    assert st["kv_bytes"] == cfg["n_layers"] * lib.kv_cache_bytes(eng["kv_num_blocks"], cfg["n_kv_heads"], cfg["head_dim"], 4)


def test_a_router_that_chooses(lib):
    """Sixteen experts, four of them taken: the loop and its single iterations agree, with graphs and without."""
    cfg = dict(synth.model_config("mini_long_moe"), kv_bits=4)
    eng = synth.engine_config("mini_long_moe")
    blob = synth.pack_blob(cfg, synth.make_weights(cfg, 202, gain_jitter=0.1))
    reqs = sampled(synth.make_workload("mini", cfg["vocab"], 302, n_requests=9), 202)
    want = tokens_of(parity.run_engine(lib, cfg, eng, blob, reqs)[0])
    assert sorted(want) == list(range(len(reqs))) and all(len(want[t]) == r["max_new_tokens"] for t, r in enumerate(reqs))
    assert all(0 <= x < cfg["vocab"] for row in want.values() for x in row)
    assert tokens_of(parity.run_engine(lib, cfg, eng, blob, reqs, window=1)[0]) == want
    assert tokens_of(parity.run_engine(lib, cfg, eng, blob, reqs, flags=lib.FLAG_NO_GRAPH)[0]) == want
    assert np.unique(np.concatenate([np.array(r) for r in want.values()])).size > 8
