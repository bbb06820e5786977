"""The paged-cache operators against the fp64 oracle: norms, rotation and storage; attention with a window and sinks; 16 and 4 bits."""
import numpy as np
import pytest
import torch

import paper_2604_07609_amd as B
from oracle import paged as P

pytestmark = pytest.mark.gpu

TYPES = {"float": torch.float32, "half": torch.float16, "bf16": torch.bfloat16}
GARBAGE = 0xFF      # halves of it are NaN, scales of it not a number


@pytest.fixture(autouse=True, scope="module")
def no_error_of_earlier_tests():
    """Tests of the host path leave an error behind on purpose; torch would take it for its own."""
    B.load_library().hipGetLastError()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def rope_table(rows, hd):
    ang = np.arange(rows)[:, None] * 10000.0 ** (-2.0 * np.arange(hd // 2) / hd)
    return np.stack((np.cos(ang), np.sin(ang)), axis=-1).astype(np.float32)


def new_cache(n_blocks, nkv, hd, bits):
    data = torch.full((P.cache_bytes(n_blocks, nkv, hd, bits),), GARBAGE, dtype=torch.uint8, device="cuda")
    return B.KVCache(data, n_blocks, nkv, hd, bits)


def oracle_cache(c):
    d = c.desc
    return P.Cache(c.data.cpu().numpy().copy(), d.n_blocks, d.n_kv_heads, d.head_dim, d.bits)


# ---- storage -----------------------------------------------------------------------------------------------------------------

def check_store(T, nq, nkv, hd, bits, dtype, norm, slots, positions, n_blocks, seed=0, q_scale=0.125, change=None):
    rng = np.random.default_rng(seed)
    eps = 2.0 ** -20
    width = (nq + 2 * nkv) * hd
    qkv = torch.from_numpy((rng.standard_normal((T, width)) * np.exp(0.5 * rng.standard_normal(width))).astype(np.float32)).to(TYPES[dtype])
    if change is not None:
        change(qkv)
    x = qkv.double().numpy()
    xq, xk, xv = (m.reshape(T, -1, hd) for m in np.split(x, [nq * hd, (nq + nkv) * hd], axis=1))
    gains = [(1 + 0.2 * rng.standard_normal(hd)).astype(np.float32) if norm else None for _ in range(2)]
    rows = 300
    table = rope_table(rows, hd)
    cache = new_cache(n_blocks, nkv, hd, bits)
    want = oracle_cache(cache)
    q, k, v = (m.unflatten(-1, (-1, hd)) for m in qkv.cuda().split((nq * hd, nkv * hd, nkv * hd), -1))
    out = torch.full((T, nq, hd), 7.0, dtype=torch.float16, device="cuda")
    B.qk_norm_rope(q, k, v, dev(np.int32(positions)), dev(np.int32(slots)), dev(table), cache, out, *(None if g is None else dev(g) for g in gains),
                   eps=eps, q_scale=q_scale, stream=torch.cuda.current_stream().cuda_stream)
    got_q = out.double().cpu().numpy()
    got = oracle_cache(cache)
    safe = np.clip(positions, 0, rows - 1)
    eps32 = float(np.float32(eps))
    with np.errstate(invalid="ignore"):
        wq = P.norm_rope(xq, None if gains[0] is None else gains[0].astype(np.float64), eps32, table, safe) * float(np.float32(q_scale))
        wk = P.norm_rope(xk, None if gains[1] is None else gains[1].astype(np.float64), eps32, table, safe)
    # 32 bits: the norm's sum of hd squares and its root are off by less than (hd / 2 + 8) 2^-24 of the value, the products and the
    # sum of a rotation by 6 roundings of its two terms; all of it below 2^-16 of the row's largest. Then one rounding to halves:
    # 2^-11 of the value, or half a step of the smallest ones, 2^-25
    def near(a, b):
        top = np.abs(b).max(axis=-1, keepdims=True)
        fine = np.isfinite(b)
        assert np.array_equal(np.isnan(a), np.isnan(b))
        with np.errstate(invalid="ignore"):
            off = np.abs(a - b) > 2.0 ** -11 * np.abs(b) + 2.0 ** -15 * top + 2.0 ** -25
        assert not (off & fine).any(), (np.argwhere(off & fine)[:5], a[off & fine][:5], b[off & fine][:5])

    for t in range(T):
        if not 0 <= positions[t] < rows:
            assert (got_q[t] == 7.0).all()
            continue
        near(got_q[t], P.half(wq[t]).astype(np.float64) if not np.isfinite(wq[t]).all() else wq[t])
        want.put(int(slots[t]), wk[t], xv[t])
    if bits == 4:
        assert np.array_equal(got.data, want.data)      # codes and scales, and everything else untouched
        return
    assert np.array_equal(got.v.view(np.uint16), want.v.view(np.uint16))
    written = np.zeros((n_blocks, 16), dtype=bool)
    for t in range(T):
        if 0 <= positions[t] < rows and 0 <= slots[t] < 16 * n_blocks:
            written[slots[t] // 16, slots[t] % 16] = True
            near(got.k[slots[t] // 16, :, slots[t] % 16].astype(np.float64), wk[t])
    at = written[:, None, :, None]
    assert (got.k.view(np.uint16)[np.broadcast_to(~at, got.k.shape)] == 0xFFFF).all()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("hd, nq, nkv", [(64, 6, 2), (128, 4, 1), (64, 5, 5), (128, 32, 8)])
@pytest.mark.parametrize("norm", [True, False])
def test_store_a_run_that_begins_inside_a_block(hd, nq, nkv, dtype, bits, norm):
    T = 45
    blocks = [5, 2, 7, 0]
    pos = np.arange(T) + 3
    check_store(T, nq, nkv, hd, bits, dtype, norm, [blocks[p // 16] * 16 + p % 16 for p in pos], pos, 8)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("T", [1, 2, 31, 33, 130, 700])
def test_store_tokens_anywhere(T, bits):
    rng = np.random.default_rng(T)
    slots = rng.permutation(50 * 16)[:T]
    check_store(T, 4, 2, 64, bits, "bf16", True, slots, rng.integers(0, 300, T), 50, seed=T)


@pytest.mark.parametrize("bits", [16, 4])
def test_store_many_tokens_take_the_large_groups(bits):
    T, rng = 8300, np.random.default_rng(5)
    starts, slots = rng.permutation(530)[:T // 16 + 1] * 16, []
    for i in range(T):
        slots.append(int(starts[i // 16]) + i % 16)
    check_store(T, 8, 8, 64, bits, "half", False, slots, rng.integers(0, 300, T), 530, seed=3)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hd", [64, 128])
def test_store_skips_padding_and_bad_places(bits, hd):
    slots = [3, -1, 16, 17, 18, 19, 20, 4 * 16, 2 ** 31 - 1, -2 ** 31, 40, 41, 42, 43, 5, 63]
    pos = [0, 1, 299, 300, -1, 2 ** 31 - 1, 7, 8, 9, 10, 20, 21, 22, 23, -2 ** 31, 5]
    check_store(len(slots), 4, 2, hd, bits, "float", True, slots, pos, 4)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", ["float", "half"])
def test_store_infinities_nan_zeros_and_large_values(bits, dtype):
    def change(qkv):
        hd, nq, nkv = 64, 4, 2
        k0, v0 = nq * hd, (nq + nkv) * hd
        qkv[0, 5] = float("nan")
        qkv[1, k0 + 7] = float("inf")
        qkv[2, v0 + 40] = float("nan")
        qkv[3, v0 + 3] = float("-inf") if bits == 4 else -60000.0
        qkv[4, k0:k0 + 64] = 0
        qkv[5, v0:v0 + 64] = 0
        qkv[6, v0:v0 + 32] *= 30000 if dtype == "half" else 1e9
        qkv[7, v0:v0 + 32] *= 1e-6
        qkv[8, v0 + 1] = -0.0
    check_store(9, 4, 2, 64, bits, dtype, False, np.arange(9) + 16, np.arange(9), 3, change=change)
    check_store(9, 4, 2, 64, bits, dtype, True, np.arange(9) + 16, np.arange(9), 3, change=change)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hd", [64, 128])
def test_read_gives_what_is_stored(bits, hd):
    rng = np.random.default_rng(2)
    cache = new_cache(6, 3, hd, bits)
    c = oracle_cache(cache)
    slots = rng.permutation(96)[:50]
    for s in slots:
        c.put(int(s), *rng.standard_normal((2, 3, hd)))
    cache.data.copy_(torch.from_numpy(c.data))
    ask = np.concatenate((slots, [-1, 96, 2 ** 31 - 1, -2 ** 31]))
    k, v = (torch.full((len(ask), 3, hd), 5.0, dtype=torch.float16, device="cuda") for _ in range(2))
    B.kv_cache_read(cache, dev(np.int32(ask)), k, v, stream=torch.cuda.current_stream().cuda_stream)
    k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
    for i, s in enumerate(slots):
        assert np.array_equal(k[i], c.get(int(s))[0]) and np.array_equal(v[i], c.get(int(s))[1])
    assert (k[50:] == 5).all() and (v[50:] == 5).all()


# ---- attention -----------------------------------------------------------------------------------------------------------------

def make_batch(lens, runs, nq, nkv, hd, bits, seed=0, extra_rows=0, spare=3, width=None, unlike=False):
    """A filled cache (places of no token hold garbage), queries and tables."""
    rng = np.random.default_rng(seed)
    need = [(n + 15) // 16 for n in lens]
    width = width or max(max(need), 1)
    n_blocks = sum(need) + spare
    order = rng.permutation(n_blocks)
    tables, at = np.full((len(lens), width), -1, dtype=np.int32), 0
    cache = new_cache(n_blocks, nkv, hd, bits)
    c = oracle_cache(cache)
    for s, n in enumerate(lens):
        tables[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
        kv = rng.standard_normal((2, n, nkv, hd)) * (np.exp(rng.uniform(-3, 3, (2, n, nkv, 1))) if unlike else 1.0)
        for j in range(n):
            c.put(int(tables[s, j // 16]) * 16 + j % 16, kv[0, j], kv[1, j])
    cache.data.copy_(torch.from_numpy(c.data))
    cu = np.concatenate(([0], np.cumsum(runs))).astype(np.int32)
    q = (rng.standard_normal((int(cu[-1]) + extra_rows, nq, hd)) / np.sqrt(hd)).astype(np.float16)
    return cache, c, tables, np.int32(lens), cu, q


def run_attention(cache, tables, lens, cu, q, max_q, window=0, sinks=0, scale=1.0, workspace=None, stream=None, fill=9.0):
    if workspace is None:
        workspace = torch.zeros(B.attention_workspace_bytes(q.shape[1], cache, len(lens), max_q), dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, fill, dtype=torch.float16, device="cuda")
    B.paged_attention(dev(q), cache, dev(tables), dev(lens), dev(cu), out, workspace, max_q=max_q, window=window, sinks=sinks, scale=scale,
                      stream=torch.cuda.current_stream().cuda_stream)
    counters = (len(lens) * cache.desc.n_kv_heads + 2) * 4      # (and more)
    assert not workspace[:counters].any()
    return out.double().cpu().numpy()


def check_attention(got, cache, c, tables, lens, cu, q, window=0, sinks=0, scale=1.0, fill=9.0):
    want, spread = P.attention(q.astype(np.float64), c, tables, lens, cu, window, sinks, scale)
    hd = q.shape[2]
    # scores: hd products in 32 bits of at most |q| |k| in all: off by hd 2^-24 of that; a probability by as much (twice: numerator and
    # sum), by its rounding to a half, 2^-11, and at the bottom of the halves by 2^-25 of the largest. Then the output's rounding
    K = np.nan_to_num(np.abs(np.stack([c.get(s)[0] for s in range(16 * c.n_blocks)])), nan=0.0, posinf=0.0)
    V = np.nan_to_num(np.abs(np.stack([c.get(s)[1] for s in range(16 * c.n_blocks)])), nan=0.0, posinf=0.0)
    qk = np.linalg.norm(q.astype(np.float64), axis=-1).max() * np.linalg.norm(K, axis=-1).max() * scale
    delta = 2 * (hd * 2.0 ** -24 * qk + 2.0 ** -21) + 2.0 ** -11
    T = cu[-1]
    a, b = got[:T], want[:T]
    assert np.array_equal(np.isnan(a), np.isnan(b)), np.argwhere(np.isnan(a) != np.isnan(b))[:5]
    inf = np.isinf(b)
    assert np.array_equal(a[inf], np.sign(b[inf]) * 65504.0)       # (outputs saturate)
    fine = np.isfinite(b)
    with np.errstate(invalid="ignore"):
        tol = delta * np.where(np.isfinite(spread[:T]), spread[:T], 0) + 2.0 ** -11 * np.abs(b) + 2.0 ** -25 * (1 + int(max(lens.max(), 1)) * V.max())
        off = (np.abs(a - b) > tol) & fine
    assert not off.any(), (np.argwhere(off)[:5], a[off][:5], b[off][:5], tol[off][:5])
    assert (got[T:] == fill).all()


CASES = [
    # lens, queries of each, window, sinks
    ([1], [1], 0, 0),
    ([16], [1], 0, 0),
    ([17, 1, 640, 33, 0, 300], [1, 1, 1, 1, 1, 1], 0, 0),
    ([17, 1, 640, 33, 0, 300], [1, 1, 1, 1, 1, 1], 40, 5),
    ([500, 100, 90], [1, 1, 1], 1, 0),
    ([500, 100, 90], [1, 1, 1], 1, 40),
    ([500, 100], [1, 1], 64, 16),
    ([300, 4, 90], [4, 4, 2], 50, 3),
    ([300, 8, 0, 90], [8, 8, 0, 1], 0, 0),
    ([200, 150], [150, 150], 0, 0),
    ([333, 70], [70, 70], 33, 7),
    ([333, 70, 5, 64], [130, 70, 1, 64], 100, 0),
    ([400, 300, 0, 20, 129], [1, 300, 1, 3, 100], 90, 70),
    ([700], [65], 0, 0),
]


@pytest.mark.parametrize("lens, runs, window, sinks", CASES)
@pytest.mark.parametrize("hd, nq, nkv", [(64, 6, 2), (128, 4, 1), (64, 3, 3), (128, 16, 2)])
@pytest.mark.parametrize("bits", [16, 4])
def test_attention(lens, runs, window, sinks, hd, nq, nkv, bits):
    b = make_batch(lens, runs, nq, nkv, hd, bits, seed=len(lens) + nq, extra_rows=2, unlike=True)
    got = run_attention(*b[:1], *b[2:], max_q=max(runs), window=window, sinks=sinks)
    check_attention(got, *b, window=window, sinks=sinks)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("nq, nkv", [(24, 1), (12, 1), (20, 4), (33, 1)])
def test_attention_group_sizes(nq, nkv, bits):
    b = make_batch([100, 40, 7], [1, 2, 7], nq, nkv, 64, bits, seed=nq)
    check_attention(run_attention(*b[:1], *b[2:], max_q=7, window=30, sinks=1, scale=0.7), *b, window=30, sinks=1, scale=0.7)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n, q", [(3000, 1), (3000, 4), (2500, 60)])
def test_attention_split_along_the_keys(n, q, bits):
    b = make_batch([n], [q], 4, 1, 64, bits, seed=7)
    check_attention(run_attention(*b[:1], *b[2:], max_q=q), *b)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("lens, runs", [([40000], [1]), ([23000, 100, 9000], [3, 1, 1])])
def test_attention_of_more_results_than_one_workgroup_adds_up(lens, runs, bits):
    """Contexts that dozens of workgroups share: their results are added up in groups. (The table repeats a few blocks: what is
    compared is long, the cache is not.)"""
    nkv, nq, hd, few = 2, 6, 64, 40
    cache, c, _, _, _, _ = make_batch([few * 16], [1], nq, nkv, hd, bits, seed=17, spare=0)
    rng = np.random.default_rng(18)
    width = (max(lens) + 15) // 16
    tables = rng.integers(0, few, (len(lens), width)).astype(np.int32)
    cu = np.concatenate(([0], np.cumsum(runs))).astype(np.int32)
    q = (rng.standard_normal((int(cu[-1]), nq, hd)) / 8).astype(np.float16)
    got = run_attention(cache, tables, np.int32(lens), cu, q, max(runs))
    check_attention(got, cache, c, tables, np.int32(lens), cu, q)
    assert np.array_equal(got, run_attention(cache, tables, np.int32(lens), cu, q, max(runs)))


@pytest.mark.parametrize("bits", [16, 4])
def test_attention_large_and_equal_scores(bits):
    """Scores far from zero, of both signs, and all equal: the running maximum moves at every step, or never."""
    b = make_batch([200, 200], [1, 70], 4, 1, 64, bits, seed=8)
    for f in (40.0, 0.0):
        q = (b[5] * f).astype(np.float16)
        b2 = (*b[:5], q)
        check_attention(run_attention(b[0], *b2[2:], max_q=70), *b2)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("runs", [[1, 1], [5, 3], [60, 80]])
@pytest.mark.parametrize("window, sinks", [(0, 0), (21, 2)])
def test_attention_strange_values_reach_only_the_rows_that_see_them(runs, window, sinks, bits):
    """Keys and values that are infinite or NaN, inside the contexts: rows whose mask hides them do not change."""
    hd, nkv = 64, 2
    cache, c, tables, lens, cu, q = make_batch([90, 85], runs, 4, nkv, hd, bits, seed=9)
    rng = np.random.default_rng(10)
    for s, j, what in ((0, 89, np.inf), (0, 60, -np.inf), (0, 40, np.nan), (1, 84, np.nan), (1, 30, np.inf)):
        k, v = rng.standard_normal((2, nkv, hd))
        v[1, 11 + s] = what
        c.put(int(tables[s, j // 16]) * 16 + j % 16, k, v)
    if bits == 16:
        c.v[tables[1, 50 // 16], 0, 3, 50 % 16] = np.float16(np.inf)     # (the operator saturates; a caller's own cache may hold one)
        c.v[tables[0, 70 // 16], 0, 3, 70 % 16] = np.float16(-np.inf)
    k, v = rng.standard_normal((2, nkv, hd))
    k[0, 5] = np.nan
    c.put(int(tables[1, 2]) * 16, k, v)
    cache.data.copy_(torch.from_numpy(c.data))
    got = run_attention(cache, tables, lens, cu, q, max(runs), window, sinks)
    check_attention(got, cache, c, tables, lens, cu, q, window, sinks)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("runs", [[1, 1, 1], [3, 2, 1], [70, 90, 1]])
def test_attention_bad_tables_and_lengths(runs, bits):
    """Block ids outside the cache hide their keys; lengths and offsets that do not fit are cut to the tensors."""
    cache, c, tables, lens, cu, q = make_batch([100, 90, 40], runs, 4, 2, 64, bits, seed=11, extra_rows=3)
    tables[0, 2], tables[1, 0], tables[2, 1] = -1, 2 ** 31 - 1, cache.desc.n_blocks
    got = run_attention(cache, tables, lens, cu, q, max(runs))
    check_attention(got, cache, c, tables, lens, cu, q)
    lens2 = np.int32([2 ** 31 - 1, -5, 40])                  # longer than the table; negative
    got = run_attention(cache, tables, lens2, cu, q, max(runs))
    wide = np.int32([tables.shape[1] * 16, 0, 40])
    check_attention(got, cache, c, tables, wide, cu, q)
    cu2 = np.int32([-3, cu[1], cu[2], 2 ** 31 - 1])         # the last sequence to the end of q, the first from its beginning
    assert np.isfinite(run_attention(cache, tables, lens, cu2, q, max(runs))[:cu[2]]).all()
    back = np.int32([5, 2, 1, 0])                           # runs of negative length: nothing is written
    assert (run_attention(cache, tables, lens, back, q, max(runs)) == 9.0).all()


def test_attention_beyond_max_q_is_not_computed():
    b = make_batch([60, 50], [5, 2], 4, 2, 64, 16, seed=12)
    got = run_attention(*b[:1], *b[2:], max_q=3)
    assert (got[3:5] == 9.0).all()
    full = run_attention(*b[:1], *b[2:], max_q=5)
    check_attention(full, *b)
    assert np.allclose(got[:3], full[:3], atol=1e-2) and np.allclose(got[5:], full[5:], atol=1e-2)


def test_strided_rows_and_another_stream():
    """Queries and outputs inside wider rows; work on a stream of the caller's, one workspace for calls in a row."""
    cache, c, tables, lens, cu, q = make_batch([70, 33], [1, 1], 4, 2, 64, 4, seed=13)
    wide_q, wide_o = torch.zeros(2, 9, 64, dtype=torch.float16, device="cuda"), torch.full((2, 7, 64), 3.0, dtype=torch.float16, device="cuda")
    wide_q[:, 2:6] = dev(q)
    work = torch.zeros(B.attention_workspace_bytes(4, cache, 2), dtype=torch.uint8, device="cuda")
    args = [dev(x) for x in (tables, lens, cu)]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        B.paged_attention(wide_q[:, 2:6], cache, *args, wide_o[:, 1:5], work, stream=st.cuda_stream)
    st.synchronize()
    o = wide_o.cpu().numpy()
    check_attention(o[:, 1:5].astype(np.float64), cache, c, tables, lens, cu, q)
    assert (o[:, :1] == 3).all() and (o[:, 5:] == 3).all()


@pytest.mark.parametrize("bits", [16, 4])
def test_store_and_attention_together_in_a_graph(bits):
    """A decode step as it is served: store the new token, attend to the cache, captured once and replayed as positions move on."""
    S, nq, nkv, hd, eps = 5, 8, 2, 128, 2.0 ** -20
    rng = np.random.default_rng(14)
    lens0 = np.int32([31, 15, 90, 1, 47])
    cache, c, tables, _, cu, _ = make_batch([n + 20 for n in lens0], [1] * S, nq, nkv, hd, bits, seed=14)
    table = rope_table(200, hd)
    gq, gk = ((1 + 0.2 * rng.standard_normal(hd)).astype(np.float32) for _ in range(2))
    qkv = torch.zeros(S, (nq + 2 * nkv) * hd, dtype=torch.bfloat16, device="cuda")
    q, k, v = (m.unflatten(-1, (-1, hd)) for m in qkv.split((nq * hd, nkv * hd, nkv * hd), -1))
    lens, pos, slots = dev(lens0), dev(lens0 - 1), dev(np.zeros(S, np.int32))
    fixed = dev(table), dev(gq), dev(gk), dev(tables), dev(cu)
    turned, out = (torch.zeros(S, nq, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    work = torch.zeros(B.attention_workspace_bytes(nq, cache, S), dtype=torch.uint8, device="cuda")

    def step():
        st = torch.cuda.current_stream().cuda_stream
        B.qk_norm_rope(q, k, v, pos, slots, fixed[0], cache, turned, fixed[1], fixed[2], eps=eps, q_scale=hd ** -0.5, stream=st)
        B.paged_attention(turned, cache, fixed[3], lens, fixed[4], out, work, window=24, sinks=2, stream=st)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(6):
        now = lens0 + i
        x = torch.from_numpy(rng.standard_normal((S, qkv.shape[1])).astype(np.float32)).bfloat16()
        qkv.copy_(x)
        place = np.int32([tables[s, (now[s] - 1) // 16] * 16 + (now[s] - 1) % 16 for s in range(S)])
        lens.copy_(torch.from_numpy(now)); pos.copy_(torch.from_numpy(now - 1)); slots.copy_(torch.from_numpy(place))
        c = oracle_cache(cache)
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        xd = x.double().numpy().reshape(S, -1, hd)
        wk = P.norm_rope(xd[:, nq:nq + nkv], gk.astype(np.float64), eps, table, now - 1)
        for s in range(S):
            c.put(int(place[s]), wk[s], xd[s, nq + nkv:])
        got = oracle_cache(cache)
        if bits == 4:
            assert np.array_equal(got.data, c.data)
        # (attention against the cache and the queries as they are: each operator's own tolerance holds)
        check_attention(out.double().cpu().numpy(), cache, got, tables, now, cu, turned.cpu().numpy(), window=24, sinks=2)
        eager = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(eager, out)


def test_two_graphs_in_flight_with_a_workspace_each():
    b = make_batch([900, 700, 30], [1, 1, 1], 8, 2, 64, 4, seed=15)
    cache, c, tables, lens, cu, q = b
    args = [dev(x) for x in (q, tables, lens, cu)]
    graphs, outs, streams = [], [], []
    work = [torch.zeros(B.attention_workspace_bytes(8, cache, 3), dtype=torch.uint8, device="cuda") for _ in range(2)]
    for i in range(2):
        out = torch.zeros(q.shape, dtype=torch.float16, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.paged_attention(args[0], cache, *args[1:], out, work[i], stream=torch.cuda.current_stream().cuda_stream)
        graphs.append(g); outs.append(out); streams.append(torch.cuda.Stream())
    torch.cuda.synchronize()
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    check_attention(outs[0].double().cpu().numpy(), *b)


def test_results_do_not_depend_on_the_rest_of_the_batch_by_more_than_rounding():
    one = make_batch([300], [1], 4, 1, 128, 4, seed=16)
    a = run_attention(*one[:1], *one[2:], max_q=1)
    again = run_attention(*one[:1], *one[2:], max_q=1)
    assert np.array_equal(a, again)
    check_attention(a, *one)


@pytest.mark.parametrize("bits", [16, 4])
def test_more_prompts_than_workgroups_with_strange_values(bits):
    """Workgroups that take several prompts one after the other; in some of those, values that are not finite and not seen by all."""
    S, n, nq, nkv, hd = 96, 130, 8, 8, 64
    cache, c, tables, lens, cu, q = make_batch([n] * S, [n] * S, nq, nkv, hd, bits, seed=20)
    rng = np.random.default_rng(21)
    for s in range(0, S, 5):
        j, g = int(rng.integers(0, n)), int(rng.integers(0, nkv))
        k, v = rng.standard_normal((2, nkv, hd))
        v[g, 7] = (np.inf, -np.inf, np.nan)[s % 3]
        c.put(int(tables[s, j // 16]) * 16 + j % 16, k, v)
        if bits == 16 and s % 3 < 2:
            c.v[tables[s, j // 16], g, 7, j % 16] = np.float16((np.inf, -np.inf)[s % 3])
    cache.data.copy_(torch.from_numpy(c.data))
    got = run_attention(cache, tables, lens, cu, q, n, 50, 3)
    check_attention(got, cache, c, tables, lens, cu, q, 50, 3)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hd, window, sinks", [(128, 200, 20), (64, 0, 0), (64, 333, 1)])
def test_chunks_of_several_items_behind_a_context(hd, window, sinks, bits):
    b = make_batch([1500, 901, 64], [1300, 500, 1], 8, 2, hd, bits, seed=22)
    got = run_attention(*b[:1], *b[2:], max_q=1300, window=window, sinks=sinks)
    check_attention(got, *b, window=window, sinks=sinks)


@pytest.mark.parametrize("bits", [16, 4])
def test_the_largest_number_of_sequences(bits):
    rng = np.random.default_rng(23)
    lens = [int(x) for x in rng.integers(0, 70, 1024)]
    runs = [1] * 1024
    lens[700], runs[700] = 300, 290
    b = make_batch(lens, runs, 2, 1, 64, bits, seed=23)
    for max_q in (290, 1):                               # (max_q 1: of the long one, the first)
        got = run_attention(*b[:1], *b[2:], max_q=max_q, window=40, sinks=2)
        if max_q == 1:
            at = int(b[4][700])
            assert (got[at + 1:at + 290] == 9.0).all()
            keep = np.r_[0:at + 1, at + 290:len(got)]
            assert np.allclose(got[keep], full[keep], atol=1e-2)
        else:
            check_attention(got, *b, window=40, sinks=2)
            full = got


def test_more_sequences_are_refused():
    b = make_batch([1], [1], 2, 1, 64, 16, seed=24)
    lens, cu, tables = np.ones(1025, np.int32), np.arange(1026, dtype=np.int32), np.zeros((1025, 1), np.int32)
    with pytest.raises(RuntimeError):
        run_attention(b[0], tables, lens, cu, np.zeros((1025, 2, 64), np.float16), 1, workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("bits", [16, 4])
def test_places_behind_4_gib_of_cache(bits):
    """The same tokens in a small cache and in one whose blocks lie beyond 32 bits of bytes: the same results, to the bit."""
    nq, nkv, hd = 16, 8, 128
    lens, runs = np.int32([100, 300, 33]), [1, 200, 3]
    need = (lens + 15) // 16
    few, many = int(need.sum()), 150000 if bits == 16 else 320000      # 9.8 and 5.6 GB
    caches = [B.KVCache(torch.empty(P.cache_bytes(n, nkv, hd, bits), dtype=torch.uint8, device="cuda"), n, nkv, hd, bits) for n in (few, many)]
    T = int(lens.sum())
    g = torch.Generator().manual_seed(25)
    q, k, v = (torch.randn(T, n, hd, generator=g).cuda() for n in (nq, nkv, nkv))
    pos = dev(np.concatenate([np.arange(n) for n in lens]).astype(np.int32))
    table = dev(rope_table(300, hd))
    rng = np.random.default_rng(25)
    results = []
    for cache, n in zip(caches, (few, many)):
        cache.data[:1 << 20].fill_(GARBAGE)
        blocks = (rng.permutation(few) if n == few else n - 1 - 7 * rng.permutation(few)).astype(np.int32)
        tables = np.zeros((3, int(need.max())), np.int32)
        tables[0, :need[0]], tables[1, :need[1]], tables[2, :need[2]] = np.split(blocks, np.cumsum(need)[:-1])
        slots = np.concatenate([tables[s, np.arange(m) // 16] * 16 + np.arange(m) % 16 for s, m in enumerate(lens)]).astype(np.int32)
        turned = torch.empty(T, nq, hd, dtype=torch.float16, device="cuda")
        st = torch.cuda.current_stream().cuda_stream
        B.qk_norm_rope(q, k, v, pos, dev(slots), table, cache, turned, q_scale=hd ** -0.5, stream=st)
        back = torch.zeros(2, T, nkv, hd, dtype=torch.float16, device="cuda")
        B.kv_cache_read(cache, dev(slots), back[0], back[1], stream=st)
        last = np.concatenate([np.arange(e - r, e) for e, r in zip(np.cumsum(lens), runs)])
        rows = turned[dev(last)].contiguous()
        cu = dev(np.concatenate(([0], np.cumsum(runs))).astype(np.int32))
        one = dev(np.int32([0, 1, 2, 3]))
        outs = []
        for qq, c, max_q in ((rows, cu, max(runs)), (rows[:3].contiguous(), one, 1)):
            out = torch.zeros_like(qq)
            work = torch.zeros(B.attention_workspace_bytes(nq, cache, 3, max_q), dtype=torch.uint8, device="cuda")
            B.paged_attention(qq, cache, dev(tables), dev(lens), c, out, work, max_q=max_q, stream=st)
            outs.append(out)
        torch.cuda.synchronize()
        results.append([turned.clone(), back, *outs])
    assert bool(torch.isfinite(results[0][2]).all()) and float(results[0][3].abs().max()) > 0
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [16, 4])
def test_prompts_and_single_tokens_in_a_graph(bits):
    """A mixed batch and one long prompt whose keys are cut into parts (two kernels), captured and replayed beside eager calls of their own."""
    mixed = make_batch([400, 90, 300, 5], [150, 1, 300, 1], 8, 2, 64, bits, seed=26)
    long = make_batch([2500], [60], 8, 2, 64, bits, seed=27)
    calls = []
    for b, max_q in ((mixed, 300), (long, 60)):
        args = [dev(x) for x in (b[5], *b[2:5])]
        out = torch.zeros(b[5].shape, dtype=torch.float16, device="cuda")
        works = [torch.zeros(B.attention_workspace_bytes(8, b[0], len(b[3]), max_q), dtype=torch.uint8, device="cuda") for _ in range(2)]
        calls.append((b, args, out, works, max_q))

    def step(which):
        for b, args, out, works, max_q in calls:
            B.paged_attention(args[0], b[0], *args[1:], out, works[which], max_q=max_q, window=70, sinks=4, stream=torch.cuda.current_stream().cuda_stream)

    step(0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(0)
    for _ in range(4):
        for c in calls:
            c[2].zero_()
        g.replay()
        torch.cuda.synchronize()
        first = [c[2].clone() for c in calls]
        step(1)
        torch.cuda.synchronize()
        for (b, _, out, _, _), x in zip(calls, first):
            assert torch.equal(x, out)
            check_attention(x.double().cpu().numpy(), *b, window=70, sinks=4)
