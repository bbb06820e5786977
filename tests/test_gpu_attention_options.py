"""Engines with per-head norms, a sliding window with sinks, a 4-bit cache: every iteration against the oracle, in every mode of the
scheduler, and the free-running loop against the iteration-by-iteration run."""
import numpy as np
import pytest

import synth
from tests import parity
from tests.test_gpu_parity import setup, sampled, _fixed_prompts
from tests.test_gpu_speculative import free_run, repetitive_requests

pytestmark = pytest.mark.gpu

# Halves: the engine's tolerance. 4 bits: keys and values reach the coder with errors of about 2^-10 of their group's largest magnitude
# (activations are halves), and the borders between codes are 14 in twice that magnitude: about 14 2^-10 = 1.4 % of the
# elements take the neighbouring code, a step of 1/7 of that magnitude on average, 0.4 of it being an element's mean size: sqrt(0.014)
# 0.15 / 0.4 = 4.4 % of the norm of a key or value, of which half reaches the residual stream. Keys and values do so independently, in
# both layers: sqrt(4) 2.2 % = 4.4 % of a logits row typically; up to 1.35 times that in the worst of a hundred rows (their errors are sums over
# few heads and scatter by a third), and the engine's 2 %: 8 %. The oracle itself, its input moved by 2^-10, moves by 2 to 3.7 %
# here, and 4-bit caches move logits by 11 to 22 % against halves.
RTOL = {16: 2e-2, 4: 8e-2}


def rtol(cfg):
    return RTOL[cfg.get("kv_bits", 16)]


def tokens_of(ev):
    got = {}
    for rid, idx, tok in sorted((int(x["request_id"]), int(x["index"]), int(x["token"])) for x in ev):
        got.setdefault(rid, []).append(tok)
    return got


@pytest.mark.parametrize("name, seed", [("mini_norm", 181), ("mini_window", 182), ("mini_kv4", 183), ("mini_long", 184), ("mini_long_moe", 193)])
def test_stepwise(lib, name, seed):
    cfg, eng, raw, blob = setup(name, seed)
    reqs = sampled(synth.make_workload("mini", cfg["vocab"], seed + 100, n_requests=9), seed)
    toks = {}
    worst = parity.stepwise_check(lib, cfg, eng, raw, blob, reqs, rtol=rtol(cfg), tokens_out=toks)
    print(name, "worst relative logit error", worst)
    ev, _, st = parity.run_engine(lib, cfg, eng, blob, reqs)
    assert tokens_of(ev) == toks and st["free_blocks"] == eng["kv_num_blocks"]
    assert st["kv_bytes"] == cfg["n_layers"] * lib.kv_cache_bytes(eng["kv_num_blocks"], cfg["n_kv_heads"], cfg["head_dim"], cfg.get("kv_bits", 16))


@pytest.mark.parametrize("name, seed", [("mini_window", 185), ("mini_kv4", 186), ("mini_long", 187), ("mini_long_moe", 194)])
def test_long_prompts_and_contexts(lib, name, seed):
    """Prompts of up to 600 tokens: the workgroups' shared tiles, contexts beyond the window, sequences shared by workgroups."""
    cfg, eng, raw, blob = setup(name, seed)
    worst = parity.stepwise_check(lib, cfg, eng, raw, blob, _fixed_prompts(cfg, [600, 17, 1, 333, 90], 5, seed), rtol=rtol(cfg))
    print(name, "long prompts: worst relative logit error", worst)


@pytest.mark.parametrize("mode", ["chunked_prefill", "preemption", "prefix_cache"])
@pytest.mark.parametrize("name", ["mini_norm", "mini_long"])
def test_with_the_scheduler_extensions(lib, name, mode):
    cfg, eng, raw, blob = setup(name, 188)
    reqs = synth.make_workload("mini", cfg["vocab"], 288, n_requests=10)
    eng = dict(eng, max_seq_len=160, max_prefill_tokens=256, max_batch=6, kv_num_blocks=96)
    if mode == "chunked_prefill":
        eng = dict(eng, chunked_prefill=True, max_prefill_tokens=48)
    elif mode == "preemption":
        eng = dict(eng, preemption=True, kv_num_blocks=14, max_batch=4)
        for r in reqs:
            r["prompt"] = r["prompt"][:40]
    else:
        eng = dict(eng, prefix_cache=True, kv_num_blocks=40)
        reqs = synth.with_shared_prefixes(reqs, cfg["vocab"], 388, n_prefixes=2, prefix_len=(16, 50), share=0.8)
        reqs = [dict(r, prompt=r["prompt"][: eng["max_seq_len"] - r["max_new_tokens"] - 1]) for r in reqs]
    worst = parity.stepwise_check(lib, cfg, eng, raw, blob, reqs, rtol=rtol(cfg))
    print(name, "with", mode, ": worst relative logit error", worst)


@pytest.mark.parametrize("name, k", [("mini_norm", 4), ("mini_kv4", 7), ("mini_long", 7)])
def test_speculative(lib, name, k):
    """Drafts: up to 15 rows of a kv head (one tile), 32 of 64-wide and of 128-wide heads (several)."""
    cfg, eng, raw, blob = setup(name, 189)
    eng = dict(eng, speculative=k, max_seq_len=160, max_prefill_tokens=256, max_batch=6, kv_num_blocks=96)
    reqs = repetitive_requests(cfg, eng, 189, 9)
    worst, toks = parity.stepwise_check_speculative(lib, cfg, eng, raw, blob, reqs, rtol=rtol(cfg))
    got, st = free_run(lib, cfg, eng, blob, reqs)
    print(name, "k", k, "worst relative logit error", worst, "drafted", st["spec_drafted"], "accepted", st["spec_accepted"])
    assert got == toks


def test_a_window_beyond_every_context_changes_nothing_but_rounding(lib):
    cfg, eng, raw, blob = setup("mini_gqa128", 190)
    reqs = _fixed_prompts(cfg, [100, 37, 60], 4, 190)
    for more in (dict(window=4096, sinks=3), dict(kv_bits=16)):
        parity.stepwise_check(lib, dict(cfg, **more), eng, raw, blob, reqs, rtol=2e-2)


def test_options_that_do_not_fit_are_refused(lib):
    cfg, eng, raw, blob = setup("mini_gqa", 191)
    for bad in (dict(kv_bits=8), dict(sinks=4), dict(window=1 << 31), dict(window=8, dtype=0), dict(kv_bits=4, dtype=0), dict(qk_norm=1)):
        with pytest.raises(lib.BlinkError):
            lib.Engine(dict(cfg, **bad), eng, blob)


def test_no_graph_and_phase_times(lib):
    """Kernels enqueued one by one, and phase 3 (norms, rotation, storage) has a kernel of its own."""
    cfg, eng, raw, blob = setup("mini_long", 192)
    reqs = _fixed_prompts(cfg, [50, 20], 4, 192)
    want = tokens_of(parity.run_engine(lib, cfg, eng, blob, reqs)[0])
    assert tokens_of(parity.run_engine(lib, cfg, eng, blob, reqs, flags=lib.FLAG_NO_GRAPH)[0]) == want
    e = lib.Engine(cfg, eng, blob, flags=lib.FLAG_EXIT_WHEN_IDLE)
    try:
        for phase in (3, 4, 12):
            e.submit(reqs[0]["prompt"], 3)
            e.time_phase(phase)
            e.run(3)
            e.wait()
            assert (e.phase_times_ms()[:3] > 0).all() == (phase != 12)
            e.stop()
    finally:
        e.shutdown()
