"""Operators for many continuations of one prompt, as cases for measurement: blocks of a paged cache copied where a
continuation begins inside one, attention over a paged cache of which the sequences of a group share the first blocks, and
log probabilities of given tokens with their ranks, the entropy and the most probable tokens.

Where `own` is false everything here is elementary torch operations. A cache of 4 bits holds e2m1 codes with one power-of-two
scale (exponent + 127 in a byte) for every 32 neighbouring dimensions of a token's key or value.
"""
import math

import torch

own = False

TYPES = {"half": torch.float16, "bf16": torch.bfloat16, "float": torch.float32}      # of the logits
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    c = lambda name, **k: dict(name=name, op="copy", **k)           # noqa: E731
    a = lambda name, **k: dict(name=name, op="attend", **k)         # noqa: E731
    p = lambda name, **k: dict(name=name, op="logprobs", **k)       # noqa: E731
    return [
        # eight continuations of one prompt begin inside its last block: that block for seven of them, in all 32 layers
        c("fork_7_in_32_layers", layers=32, copies=7, blocks=64, nkv=8, hd=128, bits=16),
        # a beam search of 64 sequences reorders: contexts move, one layer of a 4-bit cache at a time, and are read back
        c("reorder_4_bit", layers=1, copies=2039, blocks=4096, nkv=4, hd=128, bits=4),
        # four samples of one question: nothing but latency
        a("share_1x4", groups=1, seqs=4, ragged=False, shared=1040, spread=1, lo=3, hi=60, q=1, nq=32, nkv=8, hd=128, bits=16, pad=0),
        # sixteen prompts with eight samples each
        a("share_16x8", groups=16, seqs=8, ragged=False, shared=4000, spread=8, lo=16, hi=512, q=1, nq=32, nkv=8, hd=128, bits=16, pad=0),
        # a full batch behind one long system prompt, some slots of the batch unused
        a("share_1x253", groups=1, seqs=253, ragged=False, shared=8200, spread=1, lo=17, hi=1000, q=1, nq=32, nkv=8, hd=128, bits=16, pad=3),
        # questions with four or fewer answers of nine tokens to be scored, heads that share no kv head
        a("choices_40x4_of_9", groups=40, seqs=4, ragged=True, shared=1500, spread=5, lo=9, hi=9, q=9, nq=16, nkv=16, hd=64, bits=16, pad=0),
        # an agent's long context in 4 bits, tried 64 times
        a("share4_1x64", groups=1, seqs=64, ragged=False, shared=32771, spread=1, lo=40, hi=2000, q=1, nq=32, nkv=4, hd=128, bits=4, pad=0),
        # drafted tokens checked for up to sixteen samples of each of six prompts
        a("share4_drafts_6x16_of_5", groups=6, seqs=16, ragged=True, shared=6000, spread=2, lo=5, hi=300, q=5, nq=32, nkv=8, hd=128, bits=4, pad=1),
        # one sequence's token with five alternatives: nothing but latency
        p("logprobs_1", rows=1, vocab=32000, dtype="float", given=1, k=5, temperature=False, masked=0.0, padding=0, wide=0),
        # a decode iteration of a full batch, sampled with temperatures
        p("logprobs_256", rows=256, vocab=128256, dtype="float", given=1, k=20, temperature=True, masked=0.0, padding=0, wide=0),
        # every token of a prompt's chunk scored, halves, rows of a wider matrix, without alternatives
        p("logprobs_prompt_1021", rows=1021, vocab=151936, dtype="bf16", given=1, k=0, temperature=False, masked=0.0, padding=13, wide=64),
        # answers given as single letters: five tokens per row, an odd vocabulary of which a grammar forbids much
        p("logprobs_letters_61", rows=61, vocab=24601, dtype="half", given=5, k=3, temperature=False, masked=0.7, padding=2, wide=0),
    ]


def draw(rng):
    def spread(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))

    op = rng.choice(("copy", "attend", "attend", "attend", "logprobs", "logprobs"))
    if op == "logprobs":
        vocab = spread(900, 160000)
        rows = spread(1, max(1, min(4096, 33 * 10 ** 6 // vocab)))
        return dict(op=op, rows=rows, vocab=vocab, dtype=rng.choice(tuple(TYPES)), given=rng.choice((0, 1, 1, 2, 7)), k=rng.choice((0, 1, 5, 20, 64)),
                    temperature=rng.random() < 0.4, masked=rng.choice((0.0, 0.0, 0.5, 0.98)), padding=rng.randint(0, rows // 3), wide=rng.choice((0, 0, 1, 64)))
    hd = rng.choice((64, 128, 128))
    nkv = rng.choice((1, 2, 4, 8, 16)) if hd == 64 else rng.choice((1, 2, 4, 8))
    bits = rng.choice((16, 16, 4))
    if op == "copy":
        layers = rng.choice((1, 2, 8, 32))
        blocks = spread(4, 8192 // layers)
        return dict(op=op, layers=layers, copies=spread(1, blocks // 2), blocks=blocks, nkv=nkv, hd=hd, bits=bits)
    nq = nkv * rng.choice((1, 2, 3, 4, 6, 8))
    q = rng.choice((1, 1, 1, 2, 5, 8, 17))
    shared = spread(30, 32768)
    most = 256 * 8200 * 8 * 128 // ((shared + 500) * nkv * hd * q)                  # sequences
    groups = spread(1, max(1, min(64, most)))
    seqs = spread(1, max(1, min(256 // groups, most // groups)))
    lo = spread(q, q + 100)
    return dict(op=op, groups=groups, seqs=seqs, ragged=rng.random() < 0.4, shared=shared, spread=rng.choice((1, 2, 8)), lo=lo, hi=max(lo, spread(lo, 1000)), q=q,
                nq=nq, nkv=nkv, hd=hd, bits=bits, pad=rng.choice((0, 0, 2)))


# ---- the cache: blocks of 16 tokens -------------------------------------------------------------------------------------
# 16 bits: halves, keys [block][kv head][token][dim], then values [block][kv head][dim][token].
# 4 bits: a record per block and kv head, 17 bytes per dimension: the keys' codes [token][dim / 2], the values' codes
# [token / 4][16][token % 4][hd / 32], where the pair (j, m) holds the dimensions 2 (j hd / 32 + m) and the next, then the keys' and
# the values' scales [dim / 32][token]. The lower half of a byte is the lower dimension.

def _bytes(blocks, nkv, hd, bits):
    return blocks * nkv * (hd * 64 if bits == 16 else hd * 17)


def _filled(blocks, nkv, hd, bits, g, scale):
    """A cache in which every place of the pool holds a token."""
    dev = scale.device
    if bits == 16:
        kv = torch.randn(2, blocks, nkv, 16 * hd, generator=g, device=dev)
        k, v = kv[0].view(blocks, nkv, 16, hd), kv[1].view(blocks, nkv, hd, 16)
        k *= scale[:, None, :]
        v *= scale[:, :, None]
        return kv.half().view(torch.uint8).flatten()
    # codes of numbers whose largest lies in the upper two steps of its scale, and scales around one
    rec = torch.randint(0, 256, (blocks, nkv, 17 * hd), generator=g, device=dev, dtype=torch.uint8)
    rec[..., 16 * hd:] = torch.randint(123, 127, (blocks, nkv, hd), generator=g, device=dev, dtype=torch.uint8)
    return rec.flatten()


def _values(code, scale):
    """code bytes [..., hd / 2], scale bytes [..., hd / 32] -> [..., hd] in 32 bits."""
    lut = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=code.device)
    v = torch.stack((lut[(code & 15).long()], lut[(code >> 4).long()]), -1).flatten(-2).unflatten(-1, (-1, 32))
    return (v * torch.exp2(scale.float() - 127.0).unsqueeze(-1)).flatten(-2)


def _get(data, blocks, nkv, hd, bits, block, off):
    """k, v [...][kv head][hd] in 32 bits of the tokens at (block, off)."""
    if bits == 16:
        kv = data.view(torch.float16).view(2, blocks, nkv, 16 * hd)
        return kv[0].unflatten(-1, (16, hd))[block, :, off].float(), kv[1].unflatten(-1, (hd, 16))[block, :, :, off].float()
    rec = data.view(blocks, nkv, hd * 17)
    kc, vc = rec[..., :8 * hd].unflatten(-1, (16, hd // 2)), rec[..., 8 * hd:16 * hd].unflatten(-1, (4, 16, 4, hd // 32))
    ks, vs = rec[..., 16 * hd:16 * hd + hd // 2].unflatten(-1, (hd // 32, 16)), rec[..., 16 * hd + hd // 2:].unflatten(-1, (hd // 32, 16))
    return _values(kc[block, :, off], ks[block, :, :, off]), _values(vc[block, :, off // 4, :, off % 4].flatten(-2), vs[block, :, :, off])


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _batch(case):
    """(shared tokens and sequences of every group, all sequences' lengths; unused slots of the batch (0) at the end)."""
    n, top, groups, lens = case["groups"], case["shared"], [], []
    for g in range(n):
        size = 1 + (g * 7919 + case["seqs"] - 1) % case["seqs"] if case["ragged"] else case["seqs"]
        groups.append((max(1, int(round(top * case["spread"] ** (-(g * 31 % n) / max(1, n - 1))))), size))
    total, i = sum(s for _, s in groups), 0
    for shared, size in groups:
        for _ in range(size):
            lens.append(shared + int(round(case["lo"] * (case["hi"] / case["lo"]) ** (((i * 7919) % total) / max(1, total - 1)))))
            i += 1
    return groups, lens + [0] * case["pad"]


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=dev)          # noqa: E731
    whole = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)    # noqa: E731
    if case["op"] == "logprobs":
        R, V, G = case["rows"], case["vocab"], case["given"]
        # some rows are sure of a few tokens, others of none
        x = rand(R, V + case["wide"]) * (1.0 + 2.0 * torch.rand(R, 1, generator=g, device=dev))
        likely = torch.randint(0, V, (R, 4), generator=g, device=dev)
        x.scatter_add_(1, likely, 14.0 * torch.rand(R, 1, generator=g, device=dev).expand(R, 4) * torch.rand(R, 4, generator=g, device=dev))
        if case["masked"]:
            x[torch.rand(R, V + case["wide"], generator=g, device=dev) < case["masked"]] = -math.inf
            x.scatter_(1, likely, rand(R, 4))
        tokens = torch.randint(0, V, (R, G), generator=g, device=dev)
        if G:
            tokens[:, 0] = likely[:, 0]
            tokens[R - case["padding"]:] = -1
        return dict(case=case, logits=x.to(TYPES[case["dtype"]])[:, :V], tokens=tokens.int(), inverse=1.0 / (0.5 + torch.rand(R, generator=g, device=dev)) if case["temperature"] else None)
    nkv, hd, bits = case["nkv"], case["hd"], case["bits"]
    scale = torch.exp(0.3 * rand(nkv, hd))
    if case["op"] == "copy":
        where = torch.randperm(case["blocks"], generator=g, device=dev)
        n, few = case["copies"], max(1, case["copies"] // 7)             # a block that is copied is copied a few times
        data = [_filled(case["blocks"], nkv, hd, bits, g, scale) for _ in range(case["layers"])]
        return dict(case=case, data=data, whole=[d.view(torch.float16 if bits == 16 else torch.uint8) for d in data], to=where[:n].int(), source=where[n:][torch.arange(n, device=dev) % min(few, case["blocks"] - n)].int())
    groups, lens = _batch(case)
    nq, M = case["nq"], case["q"]
    runs = [min(M, n) if n else 1 for n in lens]                        # an unused slot has one token and no keys
    first, rows, starts, at, s = [], [], [0], 0, 0
    width = max((n + 15) // 16 for n in lens)
    count = sum(sh // 16 for sh, _ in groups) + sum((lens[i] + 15) // 16 for i in range(len(lens))) + 3
    order = torch.randperm(count, generator=g, device=dev).tolist()     # (more blocks than the tables name)
    for sh, size in groups:
        first, at = order[at:at + sh // 16], at + sh // 16
        for _ in range(size):
            more = (lens[s] + 15) // 16 - len(first)
            rows.append(first + order[at:at + more] + [0] * (width - len(first) - more))
            at, s = at + more, s + 1
        starts.append(s)
    rows += [[0] * width for _ in range(case["pad"])]
    cu = [0]
    for n in runs:
        cu.append(cu[-1] + n)
    return dict(case=case, q=(rand(cu[-1], nq, hd) / math.sqrt(hd)).half(), data=_filled(count, nkv, hd, bits, g, scale), blocks=count, tables=whole(rows), lens=whole(lens), cu=whole(cu),
                starts=whole(starts), shared=whole([sh for sh, _ in groups]), out=torch.zeros(cu[-1], nq, hd, dtype=torch.float16, device=dev))


# ---- one pass ---------------------------------------------------------------------------------------------------------------

def _copy(st):
    case = st["case"]
    blocks, nkv, hd, bits, to, source = case["blocks"], case["nkv"], case["hd"], case["bits"], st["to"].long(), st["source"].long()
    layers = [d.view(torch.int32).view(2 if bits == 16 else 1, blocks, -1) for d in st["data"]]
    [d.index_copy_(1, to, d[:, source]) for d in layers]
    if bits == 16:
        return st["whole"]
    tokens = (to[:, None] * 16 + torch.arange(16, device=to.device)).flatten()
    return [x.half() for d in st["data"] for x in _get(d, blocks, nkv, hd, bits, tokens // 16, tokens % 16)]


def _attend(st):
    case = st["case"]
    nq, nkv, hd, M = (case[n] for n in ("nq", "nkv", "hd", "q"))
    lens, cu = st["lens"].long(), st["cu"].long()
    S, L, G = lens.numel(), st["tables"].shape[1] * 16, nq // nkv
    at = torch.arange(L, device=lens.device)
    k, v = _get(st["data"], st["blocks"], nkv, hd, case["bits"], st["tables"].long()[:, at // 16], (at % 16).expand(S, -1))    # [S, keys, nkv, hd]
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.transpose(1, 2).contiguous()
    i = torch.arange(M, device=lens.device)
    run_ = cu[1:] - cu[:-1]
    mine = i < run_[:, None]
    row = torch.where(mine, cu[:-1, None] + i, 0)
    pos = lens[:, None] - run_[:, None] + i
    q = st["q"].float()[row].view(S, M, nkv, G, hd).permute(0, 2, 1, 3, 4).reshape(S, nkv, M * G, hd)
    s = torch.matmul(q, k).view(S, nkv, M, G, L)
    s = torch.where((at <= pos[:, :, None])[:, None, :, None, :], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(S, nkv, M * G, L), v).view(S, nkv, M, G, hd)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(S, M, nq, hd)
    st["out"][row[mine]] = o[mine].clamp(-65504, 65504).half()
    return st["out"]


def _logprobs(st):
    case = st["case"]
    x, tokens = st["logits"].float(), st["tokens"].long()
    V = x.shape[1]
    there = (tokens >= 0) & (tokens < V)
    top = x.amax(-1, keepdim=True)
    d = x - top
    if st["inverse"] is not None:
        d = d * st["inverse"][:, None]
    e = torch.exp(d)
    total = e.sum(-1, keepdim=True)
    entropy = (torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(-1, keepdim=True) / total)[:, 0]
    out = dict(entropy=entropy)
    if case["given"]:
        safe = torch.where(there, tokens, 0)
        at = x.gather(1, safe)
        i = torch.arange(V, device=x.device)
        above = [((x > at[:, j:j + 1]) | ((x == at[:, j:j + 1]) & (i < safe[:, j:j + 1]))).sum(-1) for j in range(case["given"])]
        out["logprobs"] = torch.where(there, d.gather(1, safe) - torch.log(total), 0.0)
        out["ranks"] = torch.where(there, torch.stack(above, 1), -1).int()
    if case["k"]:
        # one whole number a token, larger for a larger logit, then for a lower id
        b = (x + 0.0).view(torch.int32).long()
        key = torch.where(b < 0, -(b & 0x7FFFFFFF), b) * (1 << 31) - torch.arange(V, device=x.device)
        ids = torch.topk(key, case["k"], dim=-1).indices
        out["top_ids"], out["top_logprobs"] = ids.int(), d.gather(1, ids) - torch.log(total)
    return out


def run(state):
    case = state["case"]
    if not own:
        return {"copy": _copy, "attend": _attend, "logprobs": _logprobs}[case["op"]](state)
    import paper_2604_07609_amd as B
    # what a serving program keeps from call to call: the caches' descriptions, workspaces and outputs
    new = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")      # noqa: E731
    if case["op"] == "logprobs":
        R, V, G, k = case["rows"], case["vocab"], case["given"], case["k"]
        if "workspace" not in state:
            state["workspace"] = torch.zeros(B.token_logprobs_workspace_bytes(R, V, n_given=G, k=k), dtype=torch.uint8, device="cuda")
            state["results"] = dict(entropy=new(R), **(dict(logprobs=new(R, G), ranks=new(R, G, t=torch.int32)) if G else {}),
                                    **(dict(top_ids=new(R, k, t=torch.int32), top_logprobs=new(R, k)) if k else {}))
        B.token_logprobs(state["logits"], state["workspace"], tokens=state["tokens"] if G else None, inverse_temperature=state["inverse"], **state["results"])
        return state["results"]
    if "caches" not in state:
        state["caches"] = [B.KVCache(d, state["blocks"] if "blocks" in state else case["blocks"], case["nkv"], case["hd"], bits=case["bits"])
                           for d in (state["data"] if case["op"] == "copy" else [state["data"]])]
    caches = state["caches"]
    if case["op"] == "copy":
        B.kv_cache_copy(caches, state["source"], state["to"])
        if case["bits"] == 16:
            return state["whole"]
        if "read" not in state:
            state["read"] = [new(case["copies"] * 16, case["nkv"], case["hd"], t=torch.float16) for _ in range(2 * case["layers"])]
            state["slots"] = (state["to"][:, None] * 16 + torch.arange(16, device="cuda", dtype=torch.int32)).flatten()
        for n, c in enumerate(caches):
            B.kv_cache_read(c, state["slots"], state["read"][2 * n], state["read"][2 * n + 1])
        return state["read"]
    if "workspace" not in state:
        n = B.shared_attention_workspace_bytes(case["nq"], caches[0], state["lens"].numel(), state["shared"].numel(), state["q"].shape[0], max_q=case["q"])
        state["workspace"] = torch.zeros(n, dtype=torch.uint8, device="cuda")
    B.shared_attention(state["q"], caches[0], state["tables"], state["lens"], state["cu"], state["starts"], state["shared"], state["out"], state["workspace"], max_q=case["q"])
    return state["out"]


# ---- what a pass cannot do without --------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "logprobs":
        R, V, G, k = case["rows"], case["vocab"], case["given"], case["k"]
        return dict(bytes=R * V * TYPES[case["dtype"]].itemsize + R * (4 + 12 * G + 8 * k + 4 * case["temperature"]), flops=R * V * 6)
    nkv, hd, bits = case["nkv"], case["hd"], case["bits"]
    per_key = nkv * (4 * hd if bits == 16 else 17 * hd // 16)            # bytes of a token's key and value
    if case["op"] == "copy":
        n = case["copies"] * case["layers"] * 16
        few = min(max(1, case["copies"] // 7), case["blocks"] - case["copies"]) * case["layers"] * 16       # each source once
        return dict(bytes=(n + few) * per_key + (n * nkv * hd * 4 if bits == 4 else 0) + 8 * case["copies"], flops=0)
    groups, lens = _batch(case)
    nq, M, tokens, pairs = case["nq"], case["q"], 0, 0
    keys, s = sum(sh // 16 * 16 for sh, _ in groups), 0
    for n in lens:
        m = min(M, n) if n else 1
        tokens += m
        pairs += sum(range(n - m + 1, n + 1)) if n else 0
    for sh, size in groups:
        keys += sum(n - sh // 16 * 16 for n in lens[s:s + size])
        s += size
    return dict(bytes=tokens * nq * hd * 4 + keys * per_key + 4 * len(lens) + keys // 4, flops=4 * hd * nq * pairs)


# ---- from the definitions, in 64 bits -------------------------------------------------------------------------------------------

def _exact_tokens(data, blocks, nkv, hd, bits, ids):
    """Keys and values [16 len(ids)][kv head][hd] of whole blocks."""
    if bits == 16:
        pool = data.view(torch.float16).view(2, blocks, nkv, 16 * hd)[:, ids].double()
        return pool[0].view(-1, nkv, 16, hd).permute(0, 2, 1, 3).reshape(-1, nkv, hd), pool[1].view(-1, nkv, hd, 16).permute(0, 3, 1, 2).reshape(-1, nkv, hd)
    rec = data.view(blocks, nkv, 17 * hd)[ids].long()
    two = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float64, device=data.device)
    kv = []
    for part in (0, 1):
        c = rec[..., 8 * hd * part:8 * hd * (part + 1)]
        if part:
            c = c.reshape(-1, nkv, 4, 16, 4, hd // 32).permute(0, 1, 2, 4, 3, 5)
        c = c.reshape(-1, nkv, 16, hd // 2)
        x = torch.stack((two[c % 16], two[c // 16]), -1).reshape(-1, nkv, 16, hd)
        e = rec[..., 16 * hd + hd // 2 * part:16 * hd + hd // 2 * (part + 1)].reshape(-1, nkv, hd // 32, 16).transpose(2, 3)
        kv.append((x * (2.0 ** (e.double() - 127)).repeat_interleave(32, -1)).permute(0, 2, 1, 3).reshape(-1, nkv, hd))
    return kv


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "copy":
        to, source = st["to"].long(), st["source"].long()
        out = []
        for d in st["data"]:
            if case["bits"] == 16:
                pool = d.view(torch.float16).double().view(2, case["blocks"], -1)
                pool[0, to], pool[1, to] = pool[0, source], pool[1, source]
                out.append(pool.flatten())
            else:
                out += _exact_tokens(d, case["blocks"], case["nkv"], case["hd"], 4, source)
        return out
    if case["op"] == "logprobs":
        got = dict(entropy=[], logprobs=[], ranks=None, top_ids=None, top_logprobs=[])
        for r in range(0, case["rows"], 64):
            x = st["logits"][r:r + 64].double()
            if st["inverse"] is not None:
                x = x * st["inverse"][r:r + 64, None].double()
            z = x - torch.logsumexp(x, -1, keepdim=True)
            got["entropy"].append(-torch.where(z > -math.inf, torch.exp(z) * z, 0.0).sum(-1))
            t = st["tokens"][r:r + 64].long()
            got["logprobs"].append(torch.where(t < 0, 0.0, z.gather(1, t.clamp_min(0))))
            got["top_logprobs"].append(torch.sort(z, -1, descending=True).values[:, :case["k"]])
        given, k = case["given"] > 0, case["k"] > 0
        return {n: v if v is None else torch.cat(v) for n, v in got.items() if (given or n not in ("logprobs", "ranks")) and (k or n not in ("top_ids", "top_logprobs"))}
    # every sequence by itself
    nq, nkv, hd, G = case["nq"], case["nkv"], case["hd"], case["nq"] // case["nkv"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=st["out"].device)
    cu = st["cu"].tolist()
    for s, n in enumerate(st["lens"].tolist()):
        if not n:
            continue
        k, v = (x[:n] for x in _exact_tokens(st["data"], st["blocks"], nkv, hd, case["bits"], st["tables"][s].long()[:(n + 15) // 16]))
        k, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
        m = cu[s + 1] - cu[s]
        q = st["q"][cu[s]:cu[s + 1]].double().view(m, nkv, G, hd).permute(1, 0, 2, 3).reshape(nkv, m * G, hd)
        a = torch.matmul(q, k).view(nkv, m, G, n)
        hidden = torch.arange(n, device=out.device) > torch.arange(n - m, n, device=out.device)[:, None]
        a = torch.softmax(a.masked_fill(hidden[None, :, None, :], -math.inf), -1)
        out[cu[s]:cu[s + 1]] = torch.matmul(a.view(nkv, m * G, n), v).view(nkv, m, G, hd).permute(1, 0, 2, 3).reshape(m, nq, hd)
    return out
