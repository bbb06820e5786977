"""The operators for many continuations of one prompt, as they are used together, and on streams, in graphs and over caches where they could get in each other's way."""
import numpy as np
import pytest
import torch

import paper_2604_07609_amd as B
from tests.test_gpu_operators import check_attention, dev, new_cache, no_error_of_earlier_tests, oracle_cache, rope_table  # noqa: F401
from tests.test_gpu_operators_logprobs import call, check as check_logprobs, make as make_logits
from tests.test_gpu_operators_shared import make_groups, repeated, run_shared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("captured", [False, True])
def test_continuations_of_one_prompt(bits, captured):
    """A prompt of 77 tokens stored once in two layers, its last block forked for five of six continuations, then decode steps: store, attention of the
    group, a product with an output matrix, the log probability and rank of every sequence's token and the alternatives; the likeliest token goes on, the sequences' scores
    with it. Captured: a step is a graph that moves its own lengths and places."""
    layers, S, prompt, steps, nq, nkv, hd, V, k = 2, 6, 77, 24, 8, 2, 64, 1003, 4
    rng = np.random.default_rng(31)
    width = (prompt + steps + 15) // 16
    common = prompt // 16
    blocks = common + S * (width - common)
    order = rng.permutation(blocks + 2)
    tables = np.zeros((S, width), dtype=np.int32)
    tables[:, :common] = order[:common]
    tables[:, common:] = order[common:blocks].reshape(S, -1)
    caches = [new_cache(blocks + 2, nkv, hd, bits) for _ in range(layers)]
    rope = dev(rope_table(prompt + steps, hd))
    embed = torch.from_numpy((rng.standard_normal((layers, V, (nq + 2 * nkv) * hd))).astype(np.float16)).cuda()
    head = torch.from_numpy((0.3 * rng.standard_normal((V, nq * hd))).astype(np.float16)).cuda()
    split = lambda m: (x.unflatten(-1, (-1, hd)) for x in m.split((nq * hd, nkv * hd, nkv * hd), -1))      # noqa: E731
    # the prompt, by its first continuation's table
    ids = torch.from_numpy(rng.integers(0, V, prompt)).cuda()
    place = dev(np.int32([tables[0, j // 16] * 16 + j % 16 for j in range(prompt)]))
    first = []
    for c, e in zip(caches, embed):
        turned, out = (torch.zeros(prompt, nq, hd, dtype=torch.float16, device="cuda") for _ in range(2))
        B.qk_norm_rope(*split(e[ids]), dev(np.arange(prompt, dtype=np.int32)), place, rope, c, turned, q_scale=hd ** -0.5)
        work = torch.zeros(B.attention_workspace_bytes(nq, c, 1, prompt), dtype=torch.uint8, device="cuda")
        B.paged_attention(turned, c, dev(tables[:1]), dev(np.int32([prompt])), dev(np.int32([0, prompt])), out, work, max_q=prompt)
        first.append(out)
    # every token of it scored
    logits = first[-1][:-1].flatten(1).float() @ head.float().T
    got = call(logits, ids[1:, None].cpu().numpy())
    check_logprobs(got, logits, ids[1:, None].cpu().numpy())
    # its last block for the others
    B.kv_cache_copy(caches, dev(np.full(S - 1, tables[0, common], dtype=np.int32)), dev(tables[1:, common].copy()))
    for c in caches:
        x = c.data.view(2 if bits == 16 else 1, blocks + 2, -1)
        assert (x[:, tables[1:, common].tolist()] == x[:, [int(tables[0, common])]]).all()

    token = torch.from_numpy(rng.integers(0, V, S).astype(np.int32)).cuda()
    lens, pos = dev(np.full(S, prompt, dtype=np.int32)), dev(np.full(S, prompt - 1, dtype=np.int32))
    t, cu, starts, shared = dev(tables), dev(np.arange(S + 1, dtype=np.int32)), dev(np.int32([0, S])), dev(np.int32([common * 16]))
    turned, outs = (torch.zeros(layers, S, nq, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    size = max(B.shared_attention_workspace_bytes(nq, caches[0], S, 1, S), B.token_logprobs_workspace_bytes(S, V, n_given=1, k=k))
    work = torch.zeros(size, dtype=torch.uint8, device="cuda")          # (one for all of them in turn)
    logits, score = torch.zeros(S, V, device="cuda"), torch.zeros(S, device="cuda")
    given = torch.zeros(S, 1, dtype=torch.int32, device="cuda")
    got = dict(logprobs=torch.zeros(S, 1, device="cuda"), ranks=torch.zeros(S, 1, dtype=torch.int32, device="cuda"), entropy=torch.zeros(S, device="cuda"),
               top_ids=torch.zeros(S, k, dtype=torch.int32, device="cuda"), top_logprobs=torch.zeros(S, k, device="cuda"))
    rows = torch.arange(S, device="cuda")

    def step():
        lens.add_(1); pos.add_(1)
        slots = (t[rows, (pos // 16).long()] * 16 + pos % 16).int()
        for i, c in enumerate(caches):
            B.qk_norm_rope(*split(embed[i][token.long()]), pos, slots, rope, c, turned[i], q_scale=hd ** -0.5)
            B.shared_attention(turned[i], c, t, lens, cu, starts, shared, outs[i], work, share_all=True)
        torch.mm(outs.sum(0, dtype=torch.float16).flatten(1).float(), head.float().T, out=logits)
        given.copy_(((token + 1) % V)[:, None])
        B.token_logprobs(logits, work, tokens=given, **got)
        score.add_(got["top_logprobs"][rows, rows % k])
        token.copy_(got["top_ids"][rows, rows % k])         # (continuations that differ)

    run = step
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        keep = [x.clone() for x in (lens, pos, token, score, *(c.data for c in caches))]
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for x, y in zip((lens, pos, token, score, *(c.data for c in caches)), keep):
            x.copy_(y)
        run = g.replay
    total = np.zeros(S)
    for i in range(steps):
        run()
        torch.cuda.synchronize()
        now = np.full(S, prompt + i + 1, dtype=np.int32)
        assert np.array_equal(lens.cpu().numpy(), now)
        for c, q, o in zip(caches, turned, outs):
            check_attention(o.double().cpu().numpy(), c, oracle_cache(c), tables, now, np.arange(S + 1, dtype=np.int32), q.cpu().numpy())
        check_logprobs({n: v.cpu().numpy() for n, v in got.items()}, logits, given.cpu().numpy(), k)
        total += [got["top_logprobs"][s, s % k].double().item() for s in range(S)]
        assert np.array_equal(token.cpu().numpy(), [got["top_ids"][s, s % k].item() for s in range(S)])
    assert np.allclose(score.double().cpu().numpy(), total, rtol=steps * 2.0 ** -24, atol=0)      # (terms of one sign)
    assert len(set(token.cpu().numpy().tolist())) > 1


@pytest.mark.parametrize("bits", [16, 4])
def test_groups_that_gain_beside_groups_that_do_not(bits):
    """Without share_all: a group with long shared keys, which goes together, and small ones, which are taken apart."""
    b, starts, shared, max_q = repeated([(12000, [(12030, 1)] * 40), (64, [(70, 1), (100, 1)]), (640, [(700, 2)])], 6, 2, 64, bits)
    got = run_shared(b, starts, shared, max_q, share_all=False)
    check_attention(got, *b)
    assert np.array_equal(got, run_shared(b, starts, shared, max_q, share_all=False))


@pytest.mark.parametrize("bits", [16, 4])
def test_groups_beyond_four_gib(bits):
    """Blocks at both ends of a cache of 5 GiB: a group's shared ones at its end, by tiles of few rows and by steps of prompt items."""
    nkv, hd, members = 64, 128, 5
    blocks = (5 << 30) // B.kv_cache_bytes(1, nkv, hd, bits)
    far = B.KVCache(torch.zeros(B.kv_cache_bytes(blocks, nkv, hd, bits), dtype=torch.uint8, device="cuda"), blocks, nkv, hd, bits)
    for m in (2, 12):
        b, starts, shared, max_q = make_groups([(64, [(64 + members, members)] * m)], nkv, nkv, hd, bits, seed=m)
        near, c, tables, lens, cu, q = b
        n = near.desc.n_blocks
        place = np.concatenate((np.arange(n // 2), np.arange(blocks - (n - n // 2), blocks)))           # of the small cache's blocks
        far.data.view(2 if bits == 16 else 1, blocks, -1)[:, place.tolist()] = near.data.view(2 if bits == 16 else 1, n, -1)
        got = run_shared((far, None, np.int32(place[tables]), lens, cu, q), starts, shared, max_q)
        assert np.array_equal(got, run_shared(b, starts, shared, max_q))
        check_attention(got, *b)


def test_rows_of_logits_beyond_four_gib():
    V, R = 40000, 40
    stride = (5 << 30) // 4 // R
    x = torch.zeros(R * stride, device="cuda").view(R, stride)[:, :V]
    rng = np.random.default_rng(40)
    x.copy_(torch.from_numpy(rng.standard_normal((R, V)).astype(np.float32)))
    tokens = rng.integers(0, V, (R, 2))
    check_logprobs(call(x, tokens, 3), x, tokens, 3)


def test_two_graphs_in_flight_with_a_workspace_each():
    b, starts, shared, max_q = make_groups([(200, [(220, 1), (230, 1), (205, 1)]), (64, [(90, 1), (80, 1)])], 8, 2, 64, 4, seed=41)
    cache, c, tables, lens, cu, q = b
    logits, rng = make_logits(30, 5000, "half", 42)
    tokens = rng.integers(0, 5000, (30, 1))
    args, t = [dev(x) for x in (q, tables, lens, cu, starts, shared)], dev(np.int32(tokens))
    runs = []
    for i in range(2):
        work = [torch.zeros(B.shared_attention_workspace_bytes(8, cache, 5, 2, 5), dtype=torch.uint8, device="cuda"),
                torch.zeros(B.token_logprobs_workspace_bytes(30, 5000, k=5), dtype=torch.uint8, device="cuda")]
        outs = dict(logprobs=torch.zeros(30, 1, device="cuda"), ranks=torch.zeros(30, 1, dtype=torch.int32, device="cuda"), entropy=torch.zeros(30, device="cuda"),
                    top_ids=torch.zeros(30, 5, dtype=torch.int32, device="cuda"), top_logprobs=torch.zeros(30, 5, device="cuda"))
        out = torch.zeros(q.shape, dtype=torch.float16, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.shared_attention(args[0], cache, *args[1:], out, work[0], share_all=True)
            B.token_logprobs(logits, work[1], tokens=t, **outs)
        runs.append((g, torch.cuda.Stream(), out, outs, work))
    torch.cuda.synchronize()
    for _ in range(20):
        for g, st, *_ in runs:
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for _, _, out, outs, work in runs:
        check_attention(out.double().cpu().numpy(), *b)
        check_logprobs({n: v.cpu().numpy() for n, v in outs.items()}, logits, tokens, 5)
        assert not work[0][:8192].any() and not work[1][:8192].any()


@pytest.mark.parametrize("captured", [False, True])
def test_calls_follow_the_work_that_makes_their_inputs(captured):
    """On the caller's stream, busy when it is called, or being captured; no stream is named."""
    b, starts, shared, max_q = make_groups([(100, [(110, 1), (130, 1)])], 4, 2, 64, 16, seed=43)
    cache, c, tables, lens, cu, q = b
    logits, rng = make_logits(9, 3000, "float", 44)
    tokens = rng.integers(0, 3000, (9, 1))
    source, x = dev(q), logits.clone()
    late_q, late_x = torch.zeros_like(source), torch.zeros_like(x)
    args, t = [dev(y) for y in (tables, lens, cu, starts, shared)], dev(np.int32(tokens))
    out, work = torch.zeros_like(source), torch.zeros(B.shared_attention_workspace_bytes(4, cache, 2, 1, 2), dtype=torch.uint8, device="cuda")
    logprobs, room = torch.zeros(9, 1, device="cuda"), torch.zeros(B.token_logprobs_workspace_bytes(9, 3000), dtype=torch.uint8, device="cuda")
    blocks = dev(np.int32([int(tables[0, 0])])), torch.full((1,), -1, dtype=torch.int32, device="cuda")
    to = cache.desc.n_blocks - 1
    assert to not in tables
    busy, product = torch.randn(4096, 4096, device="cuda"), torch.zeros(4096, 4096, device="cuda")

    def step():
        for _ in range(3):
            torch.mm(busy, busy, out=product)
        late_q.copy_(source); late_x.copy_(x); blocks[1].fill_(to)
        B.kv_cache_copy(cache, *blocks)
        B.shared_attention(late_q, cache, *args, out, work, share_all=True)
        B.token_logprobs(late_x, room, tokens=t, logprobs=logprobs)

    torch.mm(busy, busy, out=product)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    if captured:
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=st):
            step()
        g.replay()
        torch.cuda.synchronize()
    else:
        with torch.cuda.stream(st):
            step()
        st.synchronize()
    check_attention(out.double().cpu().numpy(), *b)
    check_logprobs(dict(logprobs=logprobs.cpu().numpy()), x, tokens)
    v = cache.data.view(2, cache.desc.n_blocks, -1)
    assert torch.equal(v[:, to], v[:, int(tables[0, 0])])


def test_workspaces_that_are_too_small_or_not_aligned():
    b, starts, shared, max_q = make_groups([(100, [(110, 1), (130, 1)])], 4, 2, 64, 16, seed=45)
    need = B.shared_attention_workspace_bytes(4, b[0], 2, 1, 2)
    exact = torch.zeros(need, dtype=torch.uint8, device="cuda")
    check_attention(run_shared(b, starts, shared, max_q, workspace=exact), *b)
    for bad in (torch.zeros(need // 2, dtype=torch.uint8, device="cuda"), torch.zeros(need + 64, dtype=torch.uint8, device="cuda")[64:]):
        with pytest.raises(B.BlinkError, match="workspace"):
            run_shared(b, starts, shared, max_q, workspace=bad)
    # the size holds for smaller calls too, and grows with each number
    sizes = [B.shared_attention_workspace_bytes(4, b[0], *n) for n in ((2, 1, 2, 1), (3, 1, 2, 1), (3, 2, 2, 1), (3, 2, 40, 1), (3, 2, 40, 20), (3, 2, 4000, 2000))]
    assert sizes == sorted(sizes)
    # (rows of 9000: three workgroups each, whose results are joined; a row of 4096 or less is one's, and takes nothing but the counters)
    logits = torch.zeros(4, 9000, device="cuda")
    need = B.token_logprobs_workspace_bytes(4, 9000, k=2)
    assert need >= B.token_logprobs_workspace_bytes(4, 9000, k=1) and need >= B.token_logprobs_workspace_bytes(3, 9000, n_given=0, k=2)
    ids, lp = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    for bad in (torch.zeros(8192, dtype=torch.uint8, device="cuda"), torch.zeros(need + 64, dtype=torch.uint8, device="cuda")[64:]):
        with pytest.raises(B.BlinkError, match="workspace"):
            B.token_logprobs(logits, bad, top_ids=ids, top_logprobs=lp)
