"""Which stream the operators' calls go to where none is given: the one that their tensors are used on."""
import numpy as np
import pytest
import torch

import paper_2604_07609_amd as B
from paper_2604_07609_amd import binding as M
from tests.test_gpu_operators import check_attention, dev, make_batch, no_error_of_earlier_tests, oracle_cache, rope_table  # noqa: F401


class Handle:
    cuda_stream = 4711


@pytest.mark.parametrize("given, want", [(None, 4711), (0, 0), (99, 99)])
def test_the_current_stream_of_the_device_unless_one_is_given(monkeypatch, given, want):
    asked = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: asked.append(device) or Handle)
    assert M._stream(given, torch.zeros(1), 3) == want
    assert asked == ([3] if given is None else [])


def test_other_libraries_tensors_go_to_the_null_stream():
    assert M._stream(None, object(), 0) == 0


def check_results(cache, x, place, turned, out, back, tables, lens, cu):
    now = oracle_cache(cache)
    for i, s in enumerate(place):
        k, v = now.get(int(s))
        assert np.array_equal(back[0][i].double().cpu().numpy(), k) and np.array_equal(back[1][i].double().cpu().numpy(), v)
        if cache.desc.bits == 16:
            assert np.array_equal(v, x[i, -cache.n_kv_heads:].half().double().numpy())       # the values that came late
    assert bool(turned.any())
    check_attention(out.double().cpu().numpy(), cache, now, tables, lens, cu, turned.cpu().numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("captured", [False, True])
def test_calls_follow_the_work_that_makes_their_inputs(bits, captured):
    """A decode step on a stream of the caller's that is busy when it is called, or that is being captured."""
    S, nq, nkv, hd = 3, 4, 2, 64
    cache, _, tables, lens, cu, _ = make_batch([40, 17, 90], [1] * S, nq, nkv, hd, bits, seed=81)
    x = torch.from_numpy(np.random.default_rng(82).standard_normal((S, nq + 2 * nkv, hd)).astype(np.float32))
    place = np.int32([tables[s, (n - 1) // 16] * 16 + (n - 1) % 16 for s, n in enumerate(lens)])
    slots, pos, table, source = dev(place), dev(np.int32(lens - 1)), dev(rope_table(100, hd)), x.cuda()
    batch = dev(tables), dev(lens), dev(cu)
    qkv = torch.zeros_like(source)
    q, k, v = qkv.split((nq, nkv, nkv), 1)
    turned, out = (torch.zeros(S, nq, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    back = [torch.zeros(S, nkv, hd, dtype=torch.float16, device="cuda") for _ in range(2)]
    work = torch.zeros(B.attention_workspace_bytes(nq, cache, S), dtype=torch.uint8, device="cuda")
    busy, product = torch.randn(4096, 4096, device="cuda"), torch.zeros(4096, 4096, device="cuda")

    def step():
        B.qk_norm_rope(q, k, v, pos, slots, table, cache, turned, q_scale=0.125)
        B.kv_cache_read(cache, slots, *back)
        B.paged_attention(turned, cache, *batch, out, work)

    torch.mm(busy, busy, out=product)
    torch.cuda.synchronize()
    if captured:
        qkv.copy_(source)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for _ in range(3):
            out.zero_()
            turned.zero_()
            g.replay()
            torch.cuda.synchronize()
            check_results(cache, x, place, turned, out, back, tables, lens, cu)
        return
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(20):
            torch.mm(busy, busy, out=product)
        qkv.copy_(source)
        step()
        torch.cuda.current_stream().synchronize()
    check_results(cache, x, place, turned, out, back, tables, lens, cu)
