"""The key-value cache in 4 bits, as measurable cases: writing it, reading it back, and attention over it.

What is held: for each token, head and group of `group` neighbouring elements of a key or a value, sixteen steps between the
group's least and greatest element,

    m = f16(min x),   s = f16(max((max x - min x) / 15, 2^-24)),   c = clamp(round((x - m) / s), 0, 15),   x^ = m + s c

with differences and quotients in binary32, f16 the nearest binary16 number and round() to the nearest even whole number.  The cache is a pool of pages of `page`
tokens; a table names the pages of every sequence in their order.

A case is a dict of plain values:
  op        "write"   the newest tokens of every sequence into the cache, and what now stands there as values
            "read"    the newest tokens of every sequence as values
            "attend"  softmax attention of the newest tokens' queries over everything their sequence holds, the query at
                      position p over the positions up to p (window w > 0: the last w of them)
  batch     sequences; heads (of the queries), kv_heads, dim, group, page; act: "bf16" or "f32" (queries, keys, values, results)
  new, past the newest tokens of a sequence and the tokens before them; ragged: each at most that, by `lengths`
  window    0 for none;  lse: also return the logarithm of the softmax's sums
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(op, batch, new, past, *, kv_heads, dim, group, heads=0, page=64, act="bf16", ragged=False, window=0, lse=False):
    return {"op": op, "batch": batch, "new": new, "past": past, "heads": heads or kv_heads, "kv_heads": kv_heads, "dim": dim, "group": group,
            "page": page, "act": act, "ragged": ragged, "window": window, "lse": lse}


def listed():
    named = {
        # one decoding step of one sequence, 32 heads as in the 4096-wide block: nothing but latency
        "write_32x128_1tok": _case("write", 1, 1, 514, kv_heads=32, dim=128, group=128),
        # a step of sixteen sequences with grouped queries (8 heads of keys and values, the 8192-wide block)
        "write_8x128_g64_16seq": _case("write", 16, 1, 4096, heads=64, kv_heads=8, dim=128, group=64, ragged=True),
        # three prompts of odd lengths in fp32, the finest groups, the 5120-wide block
        "write_40x128_g32_f32": _case("write", 3, 515, 70, kv_heads=40, dim=128, group=32, page=32, act="f32", ragged=True),
        # the largest prompt batch: 8192 tokens of the 4096-wide block
        "write_32x128_8192tok": _case("write", 1, 8192, 0, kv_heads=32, dim=128, group=128, page=256),
        # one sequence taken out of the cache
        "read_8x128_g64_515tok": _case("read", 1, 515, 0, kv_heads=8, dim=128, group=64),
        # sequences of different lengths, heads of 64, to fp32
        "read_32x64_g32_f32": _case("read", 6, 4096, 33, kv_heads=32, dim=64, group=32, page=128, act="f32", ragged=True),
        # one token of one sequence that is 515 long: the smallest attention
        "attend_32x128_1tok_515": _case("attend", 1, 1, 514, kv_heads=32, dim=128, group=128),
        # sixteen sequences of up to 4096 tokens decode together, eight query heads to a head of the cache
        "attend_64to8x128_g64_16seq": _case("attend", 16, 1, 4095, heads=64, kv_heads=8, dim=128, group=64, ragged=True, lse=True),
        # a few tokens a sequence at once, fp32, five query heads to a head of the cache, a window
        "attend_40to8x64_g32_f32_3tok": _case("attend", 8, 3, 1000, heads=40, kv_heads=8, dim=64, group=32, page=32, act="f32", ragged=True,
                                              window=333),
        # the largest cache: 32 sequences of up to 32768 tokens decode together
        "attend_64to8x128_32seq_32768": _case("attend", 32, 1, 32767, heads=64, kv_heads=8, dim=128, group=128, page=256, ragged=True),
        # a prompt of 333 tokens right after it was written
        "attend_32x128_333tok": _case("attend", 1, 333, 0, kv_heads=32, dim=128, group=128),
        # the largest prompt: 8192 tokens
        "attend_64to8x128_8192tok": _case("attend", 1, 8192, 0, heads=64, kv_heads=8, dim=128, group=128, page=128),
    }
    return [dict(c, name=n) for n, c in named.items()]


# ---- drawn cases -----------------------------------------------------------------------------------------------------------
MOST_HELD = 16 * 32768 * 8 * 128            # elements of the keys in a cache that a drawn case attends over
MOST_MOVED = 8192 * 32 * 128                # ... or writes or reads
MOST_FLOPS = 2 * 64 * 128 * 8192 * 8192     # of a drawn attention, its mask apart from the causal one left out


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    op = rng.choices(["write", "read", "attend"], [25, 15, 60])[0]
    dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    c = _case(op, _log(rng, 1, 32), 1, 0, kv_heads=kv_heads, dim=dim, group=rng.choice([g for g in (32, 64, 128) if g <= dim]),
              page=rng.choice([32, 64, 128, 256]), act=rng.choice(["bf16", "bf16", "bf16", "f32"]), ragged=rng.random() < 0.6)
    if op == "attend":
        c["heads"] = kv_heads * rng.choice([1, 2, 4, 5, 7, 8] if kv_heads <= 8 else [1, 2])
        c["new"] = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 17, 8192)])
        c["past"] = _log(rng, 1, 32768)
        c["window"] = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
        c["lse"] = c["new"] == 1 and rng.random() < 0.4          # wanted where attention over parts of a long sequence is joined
        while c["batch"] * (c["new"] + c["past"]) * kv_heads * dim > MOST_HELD or work(dict(c, window=0, ragged=False))["flops"] > MOST_FLOPS:
            biggest = max(("batch", "new", "past"), key=lambda k: math.log(c[k] + 1) / math.log({"batch": 32, "new": 8192, "past": 32768}[k]))
            c[biggest] = max(1, c[biggest] // 2)
    else:
        c["heads"] = kv_heads * rng.choice([1, 1, 4, 8])
        c["new"], c["past"] = rng.choice([1, _log(rng, 1, 8192)]), _log(rng, 1, 4096)
        while c["batch"] * c["new"] * kv_heads * dim > MOST_MOVED:
            biggest = "new" if c["new"] > c["batch"] else "batch"
            c[biggest] //= 2
    return c


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def lengths(case):
    """[(newest tokens, tokens before them)] of the sequences; ragged batches of four and more have one with nothing new."""
    if not case["ragged"]:
        return [(case["new"], case["past"])] * case["batch"]
    rng = random.Random(f"{case['batch']} {case['new']} {case['past']}")
    return [(case["new"], case["past"])] + [(0 if i == 3 else rng.randint((case["new"] + 2) // 3, case["new"]), rng.randint(case["past"] // 3, case["past"]))
                                            for i in range(1, case["batch"])]


def _rows(gen, tokens, heads, dim, dtype, key=False):
    """Keys have elements that differ in scale and stand off zero, as trained projections give them; values and queries are even."""
    x = torch.empty((tokens, heads, dim), dtype=torch.float32, device="cuda").normal_(generator=gen)
    if key:
        scale = torch.empty((heads, dim), dtype=torch.float32, device="cuda").normal_(0.0, 0.5, generator=gen).exp_()
        x.mul_(scale).add_(torch.empty((heads, dim), dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=gen))
    return x.to(dtype)


def _starts(counts):
    return [sum(counts[:i]) for i in range(len(counts) + 1)]


def _inputs(case, seed):
    """What any implementation starts from: the keys and values of all sequences one after the other (a write's new ones; else all that stand in
    the cache), the queries, the pages of the sequences in a pool that is one page larger."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    H, Hq, D, P, dt = case["kv_heads"], case["heads"], case["dim"], case["page"], DTYPE[case["act"]]
    seqs = lengths(case)
    held = [n if case["op"] == "write" else n + past for n, past in seqs]
    n_pages = [-(-(n + past) // P) for n, past in seqs]
    order = random.Random(seed).sample(range(sum(n_pages) + 1), sum(n_pages))
    first = _starts(n_pages)
    return {"seqs": seqs, "held": held, "k": _rows(gen, sum(held), H, D, dt, key=True), "v": _rows(gen, sum(held), H, D, dt),
            "q": _rows(gen, sum(n for n, _ in seqs), Hq, D, dt) if case["op"] == "attend" else None,
            "pages": [order[first[i]:first[i + 1]] for i in range(len(seqs))], "pool": sum(n_pages) + 1}


def prepare(case, seed):
    x = _inputs(case, seed)
    H, Hq, D, g, P, dt = case["kv_heads"], case["heads"], case["dim"], case["group"], case["page"], DTYPE[case["act"]]
    new, kv_len = [n for n, _ in x["seqs"]], [n + past for n, past in x["seqs"]]
    T, width = sum(new), max(len(p) for p in x["pages"])
    table = torch.tensor([p + [0] * (width - len(p)) for p in x["pages"]], dtype=torch.int32, device="cuda")
    lens = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
    st = {"case": dict(case), "own": own, "q": x["q"]}
    if case["op"] == "write":             # as the stacked q|k|v projection leaves them: slices of its rows
        qkv = torch.zeros((T, (Hq + 2 * H) * D), dtype=dt, device="cuda")
        st["k"], st["v"] = qkv[:, Hq * D:(Hq + H) * D].view(T, H, D), qkv[:, (Hq + H) * D:].view(T, H, D)
        st["k"].copy_(x["k"])
        st["v"].copy_(x["v"])
    if own:                               # the framework's cache, which lays its pages out in its own way
        import paper_2407_11062_amd as eq

        def batch(counts):
            return eq.KvBatch(table, lens, torch.tensor(_starts(counts), dtype=torch.int32, device="cuda"), tokens=sum(counts), max_new=max(counts),
                              max_len=max(kv_len))

        st["cache"], st["batch"] = eq.KvCache(H, D, g, P, x["pool"], dtype=dt), batch(new)
        if case["op"] != "write":
            eq.eqat_kv_write(st["cache"], batch(x["held"]), x["k"], x["v"])
        if case["op"] == "attend":
            st["ws"], st["out"] = eq.kv_workspace(st["cache"], st["batch"], Hq), torch.empty_like(x["q"])
            st["lse"] = torch.empty((T, Hq), dtype=torch.float32, device="cuda") if case["lse"] else None
        else:
            st["ko"], st["vo"] = (torch.empty((T, H, D), dtype=dt, device="cuda") for _ in "kv")
        return st
    st.update(table=table.long(), lens=lens.long(), new=torch.tensor(new, device="cuda"), max_len=max(kv_len), max_new=max(new), tokens=T)
    for name in "kv":
        st[name + "_codes"] = torch.zeros((x["pool"], P, H, D // 2), dtype=torch.uint8, device="cuda")
        st[name + "_steps"] = torch.zeros((x["pool"], P, H, D // g, 2), dtype=torch.float16, device="cuda")
        if case["op"] != "write":
            _put(st, name, _newest(st, torch.tensor(x["held"], device="cuda"), sum(x["held"])), x[name])
    return st


# ---- the plain form --------------------------------------------------------------------------------------------------------
def _newest(st, counts, total):
    """sequences and positions of their newest `counts` tokens, one after the other"""
    seq = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), counts, output_size=total)
    return seq, torch.arange(total, device="cuda") + (st["lens"] - counts.cumsum(0))[seq]


def _where(st, at):
    """pages, and places in them, of positions of sequences"""
    seq, pos = at
    return st["table"][seq, pos // st["case"]["page"]], pos % st["case"]["page"]


def _put(st, name, at, x):
    g = st["case"]["group"]
    T, H, D = x.shape
    x = x.float().view(T, H, D // g, g)
    least, greatest = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    fifteen = torch.full((), 15.0, device="cuda")             # (a Python number would be a product with its reciprocal, which rounds otherwise)
    m, s = least.half(), ((greatest - least) / fifteen).clamp_min(2.0 ** -24).half()
    c = ((x - m.float()) / s.float()).round().clamp(0, 15).to(torch.uint8).view(T, H, D)
    at = _where(st, at)
    st[name + "_codes"][at] = c[..., 0::2] | (c[..., 1::2] << 4)
    st[name + "_steps"][at] = torch.cat((s, m), -1)


def _get(st, name, at):
    at = _where(st, at)
    two = st[name + "_codes"][at]
    c = torch.stack((two & 15, two >> 4), -1).flatten(-2).float().unflatten(-1, (-1, st["case"]["group"]))
    steps = st[name + "_steps"][at].float()
    return (steps[..., 1:] + steps[..., :1] * c).flatten(-2)


def _attend(st):
    """All sequences at once, each as long as the longest: keys past a sequence's end and queries past its newest tokens are masked."""
    case, B, N, L = st["case"], len(st["lens"]), st["max_new"], st["max_len"]
    H, D, R = case["kv_heads"], case["dim"], case["heads"] // case["kv_heads"]
    at = torch.arange(B, device="cuda")[:, None], torch.minimum(torch.arange(L, device="cuda"), (st["lens"] - 1).clamp_min(0)[:, None])
    k = _get(st, "k", at).permute(0, 2, 3, 1).contiguous()                        # [B, H, D, L]
    v = _get(st, "v", at).permute(0, 2, 1, 3).contiguous()                        # [B, H, L, D]
    token, pos = _newest(st, st["new"], st["tokens"])
    row = pos - (st["lens"] - st["new"])[token]                                   # which of its sequence's new tokens
    q = torch.zeros((B, N, H, R, D), device="cuda")
    q[token, row] = st["q"].float().view(-1, H, R, D) / math.sqrt(D)
    S = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(B, H, N * R, D), k).view(B, H, N, R, L)
    last = (st["lens"] - st["new"])[:, None, None] + torch.arange(N, device="cuda")[:, None]
    key = torch.arange(L, device="cuda")
    hidden = (key > last) | (key >= st["lens"][:, None, None])                    # [B, N, L]
    if case["window"]:
        hidden |= key <= last - case["window"]
    S.masked_fill_(hidden[:, None, :, None], -math.inf)
    top = S.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    S.sub_(top).exp_()
    total = S.sum(-1, keepdim=True)
    out = torch.matmul(S.view(B, H, N * R, L), v).view(B, H, N, R, D) / total
    pick = lambda t: t.permute(0, 2, 1, 3, 4)[token, row].flatten(1, 2)           # [tokens, heads, ...]
    return pick(out), pick(top + total.log()).squeeze(-1)


def _plain(st):
    case, dt = st["case"], DTYPE[st["case"]["act"]]
    if case["op"] == "attend":
        out, lse = _attend(st)
        return (out.to(dt), lse) if case["lse"] else out.to(dt)
    at = _newest(st, st["new"], st["tokens"])
    if case["op"] == "write":
        _put(st, "k", at, st["k"])
        _put(st, "v", at, st["v"])
    return _get(st, "k", at).to(dt), _get(st, "v", at).to(dt)


def run(st):
    if not st["own"]:
        return _plain(st)
    import paper_2407_11062_amd as eq
    case, cache, batch = st["case"], st["cache"], st["batch"]
    if case["op"] == "attend":
        eq.eqat_kv_attention(cache, batch, st["q"], window=case["window"], out=st["out"], lse=st["lse"], ws=st["ws"])
        return (st["out"], st["lse"]) if case["lse"] else st["out"]
    if case["op"] == "write":
        eq.eqat_kv_write(cache, batch, st["k"], st["v"])
    eq.eqat_kv_read(cache, batch, k=st["ko"], v=st["vo"])
    return st["ko"], st["vo"]


# ---- the definition, in 64 bits --------------------------------------------------------------------------------------------
def _stands_for(x, g):
    """the values that a cache holds for x [tokens, heads, dim], in 64 bits; the codes by the definition's binary32 quotient"""
    y = x.double().reshape(x.shape[0], x.shape[1], -1, g)
    lo, hi = y.min(dim=3).values, y.max(dim=3).values
    m = lo.half().double().unsqueeze(3)
    s = torch.maximum(((hi - lo).float().double() / torch.full((), 15.0, dtype=torch.float64, device=x.device)).float(), torch.tensor(2.0 ** -24, device=x.device)).half().double().unsqueeze(3)
    c = ((y - m).float().double() / s).float().double().round().clamp(0.0, 15.0)
    return (m + s * c).reshape(x.shape)


def exact(case, seed):
    x = _inputs(case, seed)
    g, R = case["group"], case["heads"] // case["kv_heads"]
    first = _starts(x["held"])
    if case["op"] != "attend":
        newest = [torch.arange(first[b + 1] - n, first[b + 1], device="cuda") for b, (n, _) in enumerate(x["seqs"])]
        return tuple(_stands_for(x[name][torch.cat(newest)], g) for name in "kv")
    out = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(x["q"].shape[:2], dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, past) in enumerate(x["seqs"]):
        L = n + past
        step = max(1, (1 << 26) // L) if n else 1
        for h in range(case["kv_heads"] if n else 0):
            K, V = (_stands_for(x[name][first[b]:first[b + 1], h:h + 1], g)[:, 0].contiguous() for name in "kv")
            K = K.t().contiguous()
            for i in range(0, n, step):
                j = torch.arange(L, device="cuda").unsqueeze(0)
                last = torch.arange(past + i, past + min(n, i + step), device="cuda").unsqueeze(1)
                seen = (j <= last) & (j > last - case["window"]) if case["window"] else j <= last
                rows = slice(at + i, at + i + len(last))
                for r in range(h * R, (h + 1) * R):
                    logit = (x["q"][rows, r].double() @ K / case["dim"] ** 0.5).where(seen, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
                    lse[rows, r] = torch.logsumexp(logit, 1)
                    out[rows, r] = torch.exp(logit - lse[rows, r].unsqueeze(1)) @ V
        at += n
    return (out, lse) if case["lse"] else out


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------
def work(case):
    H, Hq, D, a = case["kv_heads"], case["heads"], case["dim"], 2 if case["act"] == "bf16" else 4
    held = D + 8 * (D // case["group"])                              # bytes of a token and head in the cache, key and value
    seqs = lengths(case)
    T = sum(n for n, _ in seqs)
    if case["op"] != "attend":
        # a written element: a difference, a quotient, a rounding; a read one: a product and a sum
        moved = 2 * T * H * D
        return {"bytes": moved * a + T * H * held + (moved * a if case["op"] == "write" else 0), "flops": moved * (5 if case["op"] == "write" else 2)}
    w, pairs, seen = case["window"], 0, 0
    for n, past in seqs:
        if n == 0:
            continue
        if w:
            pairs += sum(min(w, past + i + 1) for i in range(n))
            seen += min(n + past, w + n - 1)
        else:
            pairs += n * past + n * (n + 1) // 2
            seen += n + past
    return {"bytes": seen * H * held + 2 * T * Hq * D * a + (4 * T * Hq if case["lse"] else 0), "flops": 4 * Hq * D * pairs}
