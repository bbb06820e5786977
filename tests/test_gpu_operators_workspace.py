"""One workspace for calls of any shapes, one after the other: every call leaves it so that any other one can use it."""
import numpy as np
import pytest
import torch

import paper_2604_07609_amd as B
from tests.test_gpu_operators import check_attention, dev, make_batch, no_error_of_earlier_tests  # noqa: F401

pytestmark = pytest.mark.gpu

ZEROS = 8192      # the bytes of a workspace that hold zeros before and after every call


def shapes(hd, bits):
    """Batches whose plans differ: their results in the workspace, their counters, the workgroups that share them."""
    rng = np.random.default_rng(31)
    yield "prompt in parts", make_batch([2500], [60], 8, 2, hd, bits, seed=32), 60, {}
    yield "many single tokens", make_batch([int(x) for x in rng.integers(150, 260, 100)], [1] * 100, 8, 2, hd, bits, seed=33), 1, {}
    yield "drafts", make_batch([2600, 40, 1900], [4, 4, 1], 16, 4, hd, bits, seed=34), 4, {}
    yield "prompts and single tokens", make_batch([700, 90, 300, 1200], [150, 1, 300, 1], 8, 2, hd, bits, seed=35), 300, dict(window=200, sinks=3)
    yield "one context", make_batch([9000], [1], 8, 8, hd, bits, seed=36), 1, {}
    yield "few sequences, many heads", make_batch([300, 0, 500, 620], [1] * 4, 48, 48, hd, bits, seed=37), 1, {}


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hd", [64, 128])
def test_calls_of_different_shapes_share_a_workspace(hd, bits):
    batches = list(shapes(hd, bits))
    size = max(B.attention_workspace_bytes(b[5].shape[1], b[0], len(b[3]), max_q) for _, b, max_q, _ in batches)
    shared = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")       # what is behind the zeros does not matter
    shared[:ZEROS] = 0
    alone = {}
    for name, b, max_q, mask in batches:
        fresh = torch.zeros(B.attention_workspace_bytes(b[5].shape[1], b[0], len(b[3]), max_q), dtype=torch.uint8, device="cuda")
        alone[name] = attend(b, max_q, mask, fresh)
        check_attention(alone[name].double().cpu().numpy(), *b, **mask)
    order = list(range(len(batches)))
    for turn in range(3):                            # each shape behind different ones
        for i in order[turn:] + order[:turn] + order[::-1]:
            name, b, max_q, mask = batches[i]
            got = attend(b, max_q, mask, shared)
            assert not shared[:ZEROS].any(), name
            assert torch.equal(got, alone[name]), name


def attend(b, max_q, mask, workspace):
    cache, _, tables, lens, cu, q = b
    out = torch.full(q.shape, 9.0, dtype=torch.float16, device="cuda")
    B.paged_attention(dev(q), cache, dev(tables), dev(lens), dev(cu), out, workspace, max_q=max_q, stream=torch.cuda.current_stream().cuda_stream, **mask)
    return out


def test_a_chunk_and_a_long_context_of_one_sequence():
    """4 bits, one sequence in both calls: a prompt chunk's results, then more workgroups with results in groups."""
    nq, nkv, hd, few = 32, 8, 128, 40
    cache, c, _, _, _, _ = make_batch([few * 16], [1], nq, nkv, hd, 4, seed=41, spare=0)
    rng = np.random.default_rng(42)
    tables = rng.integers(0, few, (1, 4096)).astype(np.int32)
    q = (rng.standard_normal((64, nq, hd)) / np.sqrt(hd)).astype(np.float16)
    work = torch.zeros(B.attention_workspace_bytes(nq, cache, 1, 64), dtype=torch.uint8, device="cuda")
    chunk = (cache, c, tables, np.int32([4000]), np.int32([0, 64]), q)
    one = (cache, c, tables, np.int32([65531]), np.int32([0, 1]), q[:1])
    for _ in range(2):
        attend(chunk, 64, {}, work)
        got = attend(one, 1, {}, work)
        assert not work[:ZEROS].any()
        check_attention(got.double().cpu().numpy(), *one)
    alone = attend(chunk, 64, {}, torch.zeros_like(work))
    assert torch.equal(attend(chunk, 64, {}, work), alone)


def test_the_size_covers_every_smaller_call():
    """The documented size does not shrink with a larger max_q or more sequences, for any head count."""
    for nkv, nq in ((1, 1), (8, 32), (1, 64), (1024, 1024)):
        for hd in (64, 128):
            for bits in (16, 4):
                cache = B.KVCache(torch.empty(B.kv_cache_bytes(1, nkv, hd, bits), dtype=torch.uint8, device="cuda"), 1, nkv, hd, bits)
                for n in (1, 2, 64, 1024):
                    sizes = [B.attention_workspace_bytes(nq, cache, n, m) for m in (1, 2, 5, 33, 300, 1 << 20)]
                    assert all(a >= ZEROS for a in sizes)
                    for a, b in zip(sizes, sizes[1:]):
                        assert a <= b
                assert B.attention_workspace_bytes(nq, cache, 1, 300) <= B.attention_workspace_bytes(nq, cache, 1024, 300)
