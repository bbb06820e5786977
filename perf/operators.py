"""Operators of long-context attention, as cases for measurement: queries and keys normed per head, rotated and stored
into a paged cache in one pass, and attention over that cache with a sliding window and first tokens that stay
visible, the cache held in half precision or in 4 bits.

Where `own` is false everything here is elementary torch operations. The 4-bit form is the microscaling one: e2m1 codes
with one power-of-two scale (exponent + 127 in a byte, 255: not a number) for every 32 neighbouring dimensions of a
token's key or value. The exponent is the one that puts the group's largest magnitude into (3.5, 7], within
[-23, 13] so that every value is a half; the codes are the nearest ones, ties to the even code.
"""
import math

import torch

own = False

# the type of the projections that come in
TYPES = {"half": torch.float16, "bf16": torch.bfloat16, "float": torch.float32}
EPS = 2.0 ** -20            # exact in 32 bits
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BETWEEN = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))   # borders of the codes; True: a tie goes up


def listed():
    w = lambda name, **k: dict(name=name, op="store", **k)      # noqa: E731
    a = lambda name, **k: dict(name=name, op="attend", **k)     # noqa: E731
    return [
        # one decoding sequence, 32 query and 8 kv heads of 128: nothing but latency
        w("store_one_token", tokens=1, nq=32, nkv=8, hd=128, dtype="float", bits=16, norm=True, run=1),
        # a decode iteration of a full batch, the head counts of the mixture-of-experts shape
        w("store_decode_256", tokens=256, nq=32, nkv=4, hd=128, dtype="bf16", bits=16, norm=True, run=1),
        # the longest prefill iteration, two prompts that begin inside a block
        w("store_prompt_8191", tokens=8191, nq=32, nkv=8, hd=128, dtype="half", bits=16, norm=True, run=4093),
        # the same iteration into 4 bits
        w("store4_prompt_8191", tokens=8191, nq=32, nkv=8, hd=128, dtype="half", bits=4, norm=True, run=4093),
        # a decode iteration of a model of 64-wide heads without shared kv heads, no norms: rotation and storage alone
        w("store4_decode_61", tokens=61, nq=16, nkv=16, hd=64, dtype="bf16", bits=4, norm=False, run=1),
        # one conversation behind its window
        a("window_one_sequence", seqs=1, q=1, lo=1037, hi=1037, nq=32, nkv=8, hd=128, bits=16, window=512, sinks=4, pad=0),
        # a full batch of ragged conversations, most of them longer than the window, some slots of the batch unused
        a("window_decode_256", seqs=256, q=1, lo=40, hi=5120, nq=32, nkv=8, hd=128, bits=16, window=1024, sinks=4, pad=3),
        # two prompts that prefill, queries far behind the first keys
        a("window_prompt_2x4000", seqs=2, q=4000, lo=4000, hi=4000, nq=32, nkv=8, hd=128, bits=16, window=1024, sinks=4, pad=0),
        # one long conversation with all its keys: the work is split along the keys
        a("four_bit_one_sequence", seqs=1, q=1, lo=65531, hi=65531, nq=32, nkv=4, hd=128, bits=4, window=0, sinks=0, pad=0),
        # a decode iteration at long contexts: what a 4-bit cache is for
        a("four_bit_decode_128", seqs=128, q=1, lo=3000, hi=16384, nq=32, nkv=8, hd=128, bits=4, window=0, sinks=0, pad=0),
        # drafted tokens checked together, 64-wide heads, window and 4 bits at once
        a("four_bit_drafts_48", seqs=48, q=5, lo=9, hi=5120, nq=16, nkv=2, hd=64, bits=4, window=2048, sinks=16, pad=1),
        # a chunk of a long prompt over its 4-bit cache
        a("four_bit_chunk_2048", seqs=1, q=2048, lo=16384, hi=16384, nq=32, nkv=8, hd=128, bits=4, window=0, sinks=0, pad=0),
    ]


def draw(rng):
    def spread(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))

    hd = rng.choice((64, 128, 128))
    nkv = rng.choice((1, 2, 4, 8, 16)) if hd == 64 else rng.choice((1, 2, 4, 8))
    nq = nkv * rng.choice((1, 2, 3, 4, 6, 8))
    bits = rng.choice((16, 4))
    if rng.random() < 0.35:
        tokens = spread(1, 8191 * 40 // max(40, nq + nkv))
        return dict(op="store", tokens=tokens, nq=nq, nkv=nkv, hd=hd, dtype=rng.choice(tuple(TYPES)), bits=bits,
                    norm=rng.random() < 0.7, run=1 if rng.random() < 0.5 else spread(1, tokens))
    kind = rng.choice(("decode", "decode", "drafts", "prompt"))
    sinks = rng.choice((0, 1, 4, 16, 77))
    window = rng.choice((0, spread(1, 4096), spread(16, 4096)))
    if kind == "prompt":
        q = spread(9, 2048)
        hi = q + (0 if rng.random() < 0.5 else spread(1, 8192))
        seqs = max(1, min(rng.randint(1, 4), 2048 * 8192 // (q * hi)))
    else:
        q = 1 if kind == "decode" else rng.randint(2, 8)
        hi = spread(max(1, q), 16384)
        seqs = min(spread(1, 256), max(1, 128 * 16384 // hi), max(1, 48 * 8 * 5120 // (q * hi)) if q > 1 else 256)
    lo = q if rng.random() < 0.5 and q <= hi else hi
    if not window:
        sinks = 0
    return dict(op="attend", seqs=seqs, q=q, lo=lo, hi=hi, nq=nq, nkv=nkv, hd=hd, bits=bits, window=window, sinks=sinks, pad=rng.choice((0, 0, 1)))


# ---- the cache: blocks of 16 tokens -------------------------------------------------------------------------------------
# 16 bits: halves, keys [block][kv head][token][dim], then values [block][kv head][dim][token].
# 4 bits: a record per block and kv head, 17 bytes per dimension: the keys' codes [token][dim / 2], the values' codes
# [token / 4][16][token % 4][hd / 32], where the pair (j, m) holds the dimensions 2 (j hd / 32 + m) and the next, then the keys' and
# the values' scales [dim / 32][token]. The lower half of a byte is the lower dimension.

def _bytes(blocks, nkv, hd, bits):
    return blocks * nkv * (hd * 64 if bits == 16 else hd * 17)


def _parts16(data, blocks, nkv, hd):
    kv = data.view(torch.float16).view(2, blocks, nkv, 16 * hd)
    return kv[0].unflatten(-1, (16, hd)), kv[1].unflatten(-1, (hd, 16))


def _parts4(data, blocks, nkv, hd):
    rec = data.view(blocks, nkv, hd * 17)
    return (rec[..., :8 * hd].unflatten(-1, (16, hd // 2)), rec[..., 8 * hd:16 * hd].unflatten(-1, (4, 16, 4, hd // 32)),
            rec[..., 16 * hd:16 * hd + hd // 2].unflatten(-1, (hd // 32, 16)), rec[..., 16 * hd + hd // 2:].unflatten(-1, (hd // 32, 16)))


def _codes(x):
    """x [..., hd] -> (bytes [..., hd / 2], scale bytes [..., hd / 32])."""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    m, e = torch.frexp(top)                                         # top = m 2^e, m in [0.5, 1)
    e = (e - 3 + (m > 0.875).to(e.dtype)).clamp(-23, 13)
    e = torch.where(top == 0, torch.full_like(e, -23), e)
    y = torch.ldexp(g, -e.unsqueeze(-1))
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    code += a > 0.25
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    fine = torch.isfinite(g).all(-1)
    code = torch.where(fine.unsqueeze(-1), code | (torch.signbit(g).to(torch.uint8) << 3), torch.zeros_like(code))
    code = code.flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | (code[..., 1] << 4), torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)


def _values(code, scale):
    """The inverse, in 32 bits."""
    lut = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=code.device)
    v = torch.stack((lut[(code & 15).long()], lut[(code >> 4).long()]), -1).flatten(-2).unflatten(-1, (-1, 32))
    s = torch.exp2(scale.float() - 127.0)
    s = torch.where(scale == 255, torch.full_like(s, math.nan), s)
    return (v * s.unsqueeze(-1)).flatten(-2)


def _put(data, blocks, nkv, hd, bits, block, off, k, v):
    """Stores k, v [token][kv head][hd] (in 32 or 64 bits) at (block, off)."""
    if bits == 16:
        kc, vc = _parts16(data, blocks, nkv, hd)
        kc[block, :, off] = k.clamp(-65504, 65504).to(torch.float16)
        vc[block, :, :, off] = v.clamp(-65504, 65504).to(torch.float16)
        return
    kc, vc, ks, vs = _parts4(data, blocks, nkv, hd)
    code, scale = _codes(k)
    kc[block, :, off] = code
    ks[block, :, :, off] = scale
    code, scale = _codes(v)
    vc[block, :, off // 4, :, off % 4] = code.unflatten(-1, (16, hd // 32))
    vs[block, :, :, off] = scale


def _get(data, blocks, nkv, hd, bits, block, off):
    """k, v [...][kv head][hd] in 32 bits of the tokens at (block, off)."""
    if bits == 16:
        kc, vc = _parts16(data, blocks, nkv, hd)
        return kc[block, :, off].float(), vc[block, :, :, off].float()
    kc, vc, ks, vs = _parts4(data, blocks, nkv, hd)
    return (_values(kc[block, :, off], ks[block, :, :, off]),
            _values(vc[block, :, off // 4, :, off % 4].flatten(-2), vs[block, :, :, off]))


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _lens(case):
    """Context lengths, those of unused batch slots (0) at the end."""
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    return [hi if n == 1 else int(round(lo * (hi / lo) ** (((i * 7919) % n) / (n - 1)))) for i in range(n)] + [0] * case["pad"]


def _table(rows, hd, device):
    inv = 500000.0 ** (-torch.arange(0, hd, 2, dtype=torch.float64, device=device) / hd)
    ang = torch.arange(rows, dtype=torch.float64, device=device)[:, None] * inv
    return torch.stack((ang.cos(), ang.sin()), -1).float()


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=dev)      # noqa: E731
    nq, nkv, hd, bits = case["nq"], case["nkv"], case["hd"], case["bits"]
    if case["op"] == "store":
        T, run = case["tokens"], case["run"]
        # runs of neighbouring positions, each from its own place on; blocks in any order
        first = torch.randint(0, 4096, ((T + run - 1) // run,), generator=g, device=dev)
        pos = (first[:, None] + torch.arange(run, device=dev)).flatten()[:T]
        per = (run + 15) // 16 + 1
        blocks = first.numel() * per + 5
        where = torch.randperm(blocks, generator=g, device=dev)
        seq = torch.arange(T, device=dev) // run
        slots = where[seq * per + pos // 16 - first[seq] // 16] * 16 + pos % 16
        # one matrix of the fused projection: channels of unlike size, as projections have
        qkv = (rand(T, (nq + 2 * nkv) * hd) * torch.exp(0.5 * rand((nq + 2 * nkv) * hd))).to(TYPES[case["dtype"]])
        q, k, v = (x.unflatten(-1, (-1, hd)) for x in qkv.split((nq * hd, nkv * hd, nkv * hd), -1))
        data = torch.zeros(_bytes(blocks, nkv, hd, bits), dtype=torch.uint8, device=dev)
        return dict(case=case, q=q, k=k, v=v, positions=pos.int(), slots=slots.int(), table=_table(4096 + run, hd, dev), data=data, blocks=blocks,
                    q_gain=1 + 0.2 * rand(hd) if case["norm"] else None, k_gain=1 + 0.2 * rand(hd) if case["norm"] else None,
                    out=torch.zeros(T, nq, hd, dtype=torch.float16, device=dev))
    lens = _lens(case)
    S, M = len(lens), case["q"]
    runs = [min(M, n) if n else 1 for n in lens]                    # tokens of each sequence; an unused slot has one without keys
    width = (max(lens) + 15) // 16
    blocks = sum((n + 15) // 16 for n in lens) + 3
    order = torch.randperm(blocks, generator=g, device=dev).tolist()
    rows, at = [], 0
    for n in lens:
        m = (n + 15) // 16
        rows.append(order[at:at + m] + [0] * (width - m))
        at += m
    data = torch.zeros(_bytes(blocks, nkv, hd, bits), dtype=torch.uint8, device=dev)
    scale = torch.exp(0.3 * rand(nkv, hd))
    for b in range(0, blocks, 2048):                                # keys and values of every place of the pool
        n = min(2048, blocks - b)
        t = torch.arange(n * 16, device=dev)
        _put(data, blocks, nkv, hd, bits, b + t // 16, t % 16, rand(n * 16, nkv, hd) * scale, rand(n * 16, nkv, hd) * scale)
    T = sum(runs)
    cu = [0]
    for n in runs:
        cu.append(cu[-1] + n)
    whole = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)        # noqa: E731
    return dict(case=case, q=(rand(T, nq, hd) / math.sqrt(hd)).half(), data=data, blocks=blocks, tables=whole(rows), lens=whole(lens), cu=whole(cu), max_q=M,
                out=torch.zeros(T, nq, hd, dtype=torch.float16, device=dev))


# ---- one pass ---------------------------------------------------------------------------------------------------------------

def _turn(x, gain, table, positions, scale):
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    cs = table[positions.long()].to(x.dtype)[:, None]
    a, b = x.chunk(2, -1)
    c, s = cs[..., 0], cs[..., 1]
    return torch.cat((a * c - b * s, b * c + a * s), -1) * scale


def _store(st):
    case = st["case"]
    hd, nkv, bits, blocks = case["hd"], case["nkv"], case["bits"], st["blocks"]
    q = _turn(st["q"].float(), st["q_gain"], st["table"], st["positions"], hd ** -0.5)
    st["out"].copy_(q.clamp(-65504, 65504))
    # the keys' codes lie next to borders: 64 bits
    k = _turn(st["k"].to(torch.float64 if bits == 4 else torch.float32), st["k_gain"], st["table"], st["positions"], 1.0)
    slots = st["slots"].long()
    _put(st["data"], blocks, nkv, hd, bits, slots // 16, slots % 16, k, st["v"].float())
    if bits == 16:
        return st["out"], st["data"].view(torch.float16)
    k, v = _get(st["data"], blocks, nkv, hd, bits, slots // 16, slots % 16)
    return st["out"], k.half(), v.half()


def _attend(st):
    case = st["case"]
    nq, nkv, hd, window, sinks, M = (case[n] for n in ("nq", "nkv", "hd", "window", "sinks", "q"))
    lens, cu = st["lens"].long(), st["cu"].long()
    S, L = lens.numel(), st["tables"].shape[1] * 16
    G = nq // nkv
    dev = lens.device
    # the positions that some query of a sequence may see
    if window and sinks + window + M - 1 < L:
        at = torch.cat((torch.arange(sinks, device=dev).expand(S, -1), lens[:, None] + torch.arange(1 - window - M, 0, device=dev)), 1)
        once = torch.cat((torch.ones(sinks, dtype=torch.bool, device=dev).expand(S, -1), at[:, sinks:] >= sinks), 1)
    else:
        at = torch.arange(L, device=dev).expand(S, -1)
        once = torch.ones_like(at, dtype=torch.bool)
    there = once & (at >= 0) & (at < lens[:, None])
    safe = torch.where(there, at, 0)
    k, v = _get(st["data"], st["blocks"], nkv, hd, case["bits"], st["tables"].long().gather(1, safe // 16), safe % 16)    # [S, keys, nkv, hd]
    k, v = (torch.where(there[:, :, None, None], x, 0.0).transpose(1, 2).contiguous() for x in (k, v))
    i = torch.arange(M, device=dev)
    mine = i < (cu[1:] - cu[:-1])[:, None]
    row = torch.where(mine, cu[:-1, None] + i, 0)
    pos = lens[:, None] - (cu[1:] - cu[:-1])[:, None] + i
    seen = there[:, None, :] & (at[:, None, :] <= pos[:, :, None])
    if window:
        seen = seen & ((at[:, None, :] > pos[:, :, None] - window) | (at[:, None, :] < sinks))
    q = st["q"].float()[row].view(S, M, nkv, G, hd).permute(0, 2, 1, 3, 4).reshape(S, nkv, M * G, hd)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).view(S, nkv, M, G, -1)
    s = torch.where(seen[:, None, :, None, :], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(S, nkv, M * G, -1), v).view(S, nkv, M, G, hd)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(S, M, nq, hd)
    st["out"][row[mine]] = o[mine].clamp(-65504, 65504).half()
    return st["out"]


def run(state):
    case = state["case"]
    if not own:
        return _store(state) if case["op"] == "store" else _attend(state)
    import paper_2604_07609_amd as B
    # what a serving program keeps from call to call: the cache's description and a workspace
    if "cache" not in state:
        state["cache"] = B.KVCache(state["data"], state["blocks"], case["nkv"], case["hd"], bits=case["bits"])
        if case["op"] == "attend":
            n = B.attention_workspace_bytes(case["nq"], state["cache"], state["lens"].numel(), state["max_q"])
            state["workspace"] = torch.zeros(n, dtype=torch.uint8, device="cuda")
    cache, stream = state["cache"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "attend":
        B.paged_attention(state["q"], cache, state["tables"], state["lens"], state["cu"], state["out"], state["workspace"], max_q=state["max_q"],
                          window=case["window"], sinks=case["sinks"], stream=stream)
        return state["out"]
    B.qk_norm_rope(state["q"], state["k"], state["v"], state["positions"], state["slots"], state["table"], cache, state["out"],
                   q_gain=state["q_gain"], k_gain=state["k_gain"], eps=EPS, q_scale=case["hd"] ** -0.5, stream=stream)
    if case["bits"] == 16:
        return state["out"], state["data"].view(torch.float16)
    if "k_out" not in state:
        state["k_out"] = torch.empty(case["tokens"], case["nkv"], case["hd"], dtype=torch.float16, device="cuda")
        state["v_out"] = torch.empty_like(state["k_out"])
    B.kv_cache_read(cache, state["slots"], state["k_out"], state["v_out"], stream=stream)
    return state["out"], state["k_out"], state["v_out"]


# ---- what a pass cannot do without --------------------------------------------------------------------------------------------

def work(case):
    nq, nkv, hd, bits = case["nq"], case["nkv"], case["hd"], case["bits"]
    per_key = nkv * (4 * hd if bits == 16 else 17 * hd // 16)        # bytes of a token's key and value
    if case["op"] == "store":
        T, size = case["tokens"], TYPES[case["dtype"]].itemsize
        read = T * (nq + 2 * nkv) * hd * size + T * (8 + 4 * hd)     # projections; position, slot, a row of the table
        wrote = T * nq * hd * 2 + T * per_key + (T * nkv * hd * 4 if bits == 4 else 0)
        return dict(bytes=read + wrote, flops=T * (nq + nkv) * hd * 8)
    W, Z, M = case["window"], case["sinks"], case["q"]
    keys = pairs = tokens = 0
    for n in _lens(case):
        m, w = min(M, n), W or n
        tokens += m if n else 1
        pairs += sum(min(p + 1, w) + min(Z, max(0, p + 1 - w)) for p in range(n - m, n))
        keys += min(n, w + m - 1) + min(Z, max(0, n - (w + m - 1))) if n else 0
    return dict(bytes=tokens * nq * hd * 4 + keys * per_key + 4 * len(_lens(case)) + keys // 4, flops=4 * hd * nq * pairs)


# ---- from the definitions, in 64 bits -------------------------------------------------------------------------------------------

def _exact_four(x):
    """The values that groups of 32 of x [..., hd] stand for once stored in 4 bits, by search among all of them."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = g.abs().max(-1).values
    e = torch.full_like(top, -23)
    for n in range(-22, 14):
        e = torch.where(top > 3.5 * 2.0 ** n, torch.full_like(top, n), e)
    y = g * 2.0 ** -e[..., None]
    out = torch.zeros_like(y)
    for i, (edge, up) in enumerate(BETWEEN):
        out = torch.where(y.abs() >= edge if up else y.abs() > edge, torch.full_like(y, LEVELS[i + 1]), out)
    return (out * y.sign() * 2.0 ** e[..., None]).reshape(x.shape)


def exact(case, seed):
    st = prepare(case, seed)
    nq, nkv, hd, bits, blocks = case["nq"], case["nkv"], case["hd"], case["bits"], st["blocks"]
    if case["op"] == "store":
        def turned(x, gain):
            x = x.double()
            if gain is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / hd + EPS).sqrt() * gain.double()
            z = torch.complex(x[..., :hd // 2], x[..., hd // 2:]) * torch.view_as_complex(st["table"].double())[st["positions"].long()][:, None]
            return torch.cat((z.real, z.imag), -1)

        q, k, v = turned(st["q"], st["q_gain"]) / math.sqrt(hd), turned(st["k"], st["k_gain"]), st["v"].double()
        if bits == 4:
            return q, _exact_four(k), _exact_four(v)
        pool = torch.zeros(2, blocks, nkv, 16 * hd, dtype=torch.float64, device=q.device)
        slots = st["slots"].long()
        pool[0].view(blocks, nkv, 16, hd).permute(0, 2, 1, 3)[slots // 16, slots % 16] = k
        pool[1].view(blocks, nkv, hd, 16).permute(0, 3, 1, 2)[slots // 16, slots % 16] = v
        return q, pool.flatten()
    # every sequence by itself, 256 queries at a time
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=st["out"].device)
    cu, W, Z, G = st["cu"].tolist(), case["window"], case["sinks"], nq // nkv
    for s, n in enumerate(st["lens"].tolist()):
        if not n:
            continue
        at = torch.arange(n, device=out.device)
        block = st["tables"][s].long()[at // 16]
        if bits == 16:
            pool = st["data"].view(torch.float16).view(2, blocks, nkv, 16 * hd)
            k = pool[0].view(blocks, nkv, 16, hd).permute(0, 2, 1, 3)[block, at % 16].double()
            v = pool[1].view(blocks, nkv, hd, 16).permute(0, 3, 1, 2)[block, at % 16].double()
        else:
            rec = st["data"].view(blocks, nkv, 17 * hd)[st["tables"][s].long()[:(n + 15) // 16]].long()         # [blocks, nkv, bytes]
            two = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float64, device=out.device)
            kv = []
            for part in (0, 1):
                c = rec[..., 8 * hd * part:8 * hd * (part + 1)]
                if part:
                    c = c.reshape(-1, nkv, 4, 16, 4, hd // 32).permute(0, 1, 2, 4, 3, 5)
                c = c.reshape(-1, nkv, 16, hd // 2)
                x = torch.stack((two[c % 16], two[c // 16]), -1).reshape(-1, nkv, 16, hd)
                e = rec[..., 16 * hd + hd // 2 * part:16 * hd + hd // 2 * (part + 1)].reshape(-1, nkv, hd // 32, 16).transpose(2, 3)
                x = x * (2.0 ** (e.double() - 127)).repeat_interleave(32, -1)
                kv.append(x.permute(0, 2, 1, 3).reshape(-1, nkv, hd)[:n])
            k, v = kv
        k, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
        for t in range(cu[s], cu[s + 1], 256):
            end = min(t + 256, cu[s + 1])
            pos = n - (cu[s + 1] - torch.arange(t, end, device=out.device))
            q = st["q"][t:end].double().view(-1, nkv, G, hd).permute(1, 0, 2, 3).reshape(nkv, -1, hd)
            a = torch.matmul(q, k).view(nkv, end - t, G, n)
            hidden = at > pos[:, None]
            if W:
                hidden |= (at <= pos[:, None] - W) & (at >= Z)
            a = torch.softmax(a.masked_fill(hidden[None, :, None, :], -math.inf), -1)
            out[t:end] = torch.matmul(a.view(nkv, -1, n), v).view(nkv, end - t, G, hd).permute(1, 0, 2, 3).reshape(end - t, nq, hd)
    return out
