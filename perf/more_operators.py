"""Operators of a server's step over a paged cache: requests of different size planned, written, attended and verified.

A case is a dict of plain values; `kind` names the operator:

  plan    block tables and slot maps from the requests' lengths, and the blocks given back (hgca.kv_plan, hgca.kv_release)
  write   rows of packed tokens written to a tier by slot (hgca.kv_write)
  chunk   attention of packed new tokens, any number per sequence, over a tier whose last tokens they are: causal or not, with a
          window, a prefix that all see, documents, scores capped by a tanh, a bias by distance (hgca.chunk_attn)
  verify  drafted tokens accepted or refused by the target's probabilities and given random numbers, with the token that
          follows (hgca.verify_drafts)

With `own` false, run() computes the same in elementary torch operations, in 32 bits (probabilities' sums in 64).  exact() computes
it in 64 bits.  Shapes are those of the repository's workloads (heads of 64 and 128, groups of 1 to 8 query heads per KV head, up to
64 K tokens, contiguous or in blocks, fp32 and bf16) and sizes between them.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"


def _case(kind, name=None, *, dtype="bf16", batch, n=1, spread="same", q_heads=32, kv_heads=8, head_dim=128, length=0, block=16, pad=0,
          out="", cap=0.0, window=0, bias=False, prefix=0, docs=False, causal=True, vocab=0, tree=False, sure=False, scarce=False):
    c = dict(kind=kind, dtype=dtype, batch=batch, n=n, spread=spread, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
             length=length, block=block, pad=pad, out=out or dtype, cap=cap, window=window, bias=bias, prefix=prefix, docs=docs,
             causal=causal, vocab=vocab, tree=tree, sure=sure, scarce=scarce)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the smallest: one token for each of 64 conversations, a few of which begin a new block
        _case("plan", "plan_step", batch=64, n=1, length=4096),
        # a server takes up the prompts of 512 requests, some conversations' further ones among them
        _case("plan", "plan_prompts", batch=512, n=512, spread="ragged", length=8192),
        # the step's 64 tokens enter the blocks that were planned
        _case("write", "write_step", batch=64, n=1, length=1024),
        # prompts of 16 requests enter, as parts of a fused projection's rows, with padding behind them
        _case("write", "write_prompts", batch=16, n=1500, spread="ragged", length=4096, pad=37),
        # four drafted tokens of 8 conversations behind the last one, a small vocabulary
        _case("verify", "verify_chain", dtype="f32", batch=8, n=5, vocab=32000),
        # trees of 16 tokens of 32 conversations over a large one
        _case("verify", "verify_tree", dtype="f32", batch=32, n=16, vocab=128000, tree=True),
        # one fp32 sequence of a tiny model: five tokens, scores biased by distance
        _case("chunk", "chunk_tiny_f32", dtype="f32", batch=1, n=5, q_heads=4, kv_heads=4, head_dim=64, length=260, block=0, bias=True),
        # one token of 8 conversations of an 8B-class layer with capped scores over everything
        _case("chunk", "chunk_step_8b", batch=8, n=1, length=28672, cap=50.0),
        # a step of a busy server: most requests have one token, a few a part of their prompt, in a layer with a window and capped scores
        _case("chunk", "chunk_mixed_8b", batch=32, n=1024, spread="mixed", length=16384, cap=30.0, window=4096),
        # two prompts of 4096 tokens of a 70B-class layer, whose first 600 (an instruction, a picture) see each other both ways
        _case("chunk", "chunk_prompt_70b", batch=2, n=4096, q_heads=64, length=4096, prefix=600),
        # documents packed into one row of 16 K tokens, each for itself, scores biased by distance
        _case("chunk", "chunk_docs_8b", batch=1, n=16384, length=16384, block=0, bias=True, docs=True),
        # an exact layer's prompts of different length
        _case("chunk", "chunk_prompts_f32", dtype="f32", batch=4, n=1024, spread="ragged", length=2048),
    ]


# ---- sizes ----------------------------------------------------------------------------------------------------------

def _numbers(seed, salt):
    return torch.Generator().manual_seed(int(seed) * 131 + salt)


def _tokens(case):
    """New tokens of every sequence (Python ints), the case's own: they set the outputs' sizes."""
    B, n, g = case["batch"], case["n"], _numbers(case["batch"] + case["n"], 3)
    if case["spread"] == "same":
        return [n] * B
    u = torch.rand(B, generator=g, dtype=torch.float64).tolist()
    some = [min(n, max(1, int(round(math.exp(x * math.log(n)))))) for x in u]
    if case["spread"] == "ragged":
        return some
    few = torch.rand(B, generator=g, dtype=torch.float64).tolist()              # mixed: one in four has more than one, one has all
    got = [m if f < 0.25 else 1 for m, f in zip(some, few)]
    got[B // 2] = n
    return got


def _lens(case, seed, counts):
    """Tokens of every sequence, the new ones among them."""
    T, g = case["length"], _numbers(seed, 5)
    u = torch.rand(case["batch"], generator=g, dtype=torch.float64).tolist()
    if case["spread"] == "same" and case["kind"] == "chunk":
        return [max(T, m) for m in counts]
    return [max(m, T - int(x * T / 2)) for m, x in zip(counts, u)]


def _bounds(case, seed, counts, lens):
    """The first token that each new token may see, by documents (None without)."""
    if not case["docs"]:
        return None
    g, got = _numbers(seed, 7), []
    for m, length in zip(counts, lens):
        starts, at = [], 0
        while at < length:                       # documents of 64 to 4096 tokens
            u = float(torch.rand((), generator=g, dtype=torch.float64))
            run = min(int(64 * 64 ** u), length - at)
            starts += [at] * run
            at += run
        got += starts[length - m:]
    return got


def _pairs(case, seed):
    """Pairs of a new token and a token that it sees, and tokens that any of a sequence's new ones sees."""
    counts = _tokens(case)
    lens = _lens(case, seed, counts)
    first, at, pairs, seen = _bounds(case, seed, counts, lens), 0, 0, 0
    for m, length in zip(counts, lens):
        p = torch.arange(length - m, length)
        lo = torch.zeros_like(p) if first is None else torch.tensor(first[at: at + m], dtype=torch.int64)
        at += m
        if case["window"]:
            lo = torch.maximum(lo, p - case["window"] + 1)
        hi = p + 1 if case["causal"] else torch.full_like(p, length)
        pre = min(case["prefix"], length)
        extra = lo.clamp(max=pre) + (pre - hi).clamp(min=0)
        pairs += int((hi - lo).clamp(min=0).sum() + extra.sum())
        seen += length - max(int(lo.min()) - pre, 0) if m else 0
    return sum(counts), pairs, seen


def work(case):
    kind, B, Hq, Hkv, d = (case[k] for k in ("kind", "batch", "q_heads", "kv_heads", "head_dim"))
    e = 4 if case["dtype"] == "f32" else 2
    if kind == "verify":                         # the rows of the node where the walk ends
        return {"bytes": float(B * case["vocab"] * e * (1 if case["sure"] else 2)), "flops": float(4 * B * case["vocab"])}
    counts = _tokens(case)
    if kind == "plan":
        return {"bytes": float(20 * B + 8 * (sum(counts) + case["pad"]) + 12 * sum(counts) / case["block"]), "flops": float(4 * sum(counts))}
    if kind == "write":
        return {"bytes": float(4 * sum(counts) * Hkv * d * e + 4 * sum(counts)), "flops": 0.0}
    tokens, pairs, seen = _pairs(case, 1)
    o = 4 if case["out"] == "f32" else 2
    return {"bytes": float(2 * seen * Hkv * d * e + tokens * Hq * (d * (e + o) + 4)), "flops": float(4 * pairs * Hq * d)}


def _cost(case):
    w = work(case)
    return 2e-6 + w["bytes"] / 5e12 + w["flops"] / (1e14 if case["dtype"] == "f32" else 1e15)


def _room(case):
    """Bytes that a state holds."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "verify":
        return case["batch"] * case["n"] * case["vocab"] * e * 2
    if case["kind"] == "plan":
        return case["batch"] * case["length"]
    return (case["batch"] * case["kv_heads"] * case["length"] * 2 + case["batch"] * case["n"] * case["q_heads"] * 2) * case["head_dim"] * e


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["plan", "write", "verify", "verify", "chunk", "chunk", "chunk", "chunk"])
    like = [c for c in listed() if c["kind"] == kind]
    most, room = max(_cost(c) for c in like), max(_room(c) for c in like)
    while True:
        heads, kv = rng.choice([(4, 4), (32, 8), (32, 8), (40, 40), (64, 8), (16, 8)])
        c = dict(dtype="f32" if rng.random() < 0.25 else "bf16", q_heads=heads, kv_heads=kv, head_dim=rng.choice([64, 128, 128]),
                 block=rng.choice([16, 16, 32, 48, 64]), pad=rng.choice([0, 0, 1, 29]), spread=rng.choice(["same", "ragged", "mixed"]))
        if kind == "plan":
            c.update(batch=span(1, 1024), n=span(1, 512), length=span(512, 8192), scarce=rng.random() < 0.3)
        elif kind == "write":
            c.update(batch=span(1, 64), n=span(1, 2048), block=rng.choice([0, c["block"]]))
            c["length"] = c["n"] + span(16, 2048)
        elif kind == "verify":
            c.update(batch=span(1, 64), n=span(1, 64), vocab=span(1000, 160000), tree=rng.random() < 0.5, sure=rng.random() < 0.3)
        else:
            c.update(batch=span(1, 32), n=rng.choice([1, span(1, 64), span(1, 4096)]), block=rng.choice([0, c["block"], c["block"]]),
                     out="f32" if rng.random() < 0.2 else c["dtype"], cap=rng.choice([0.0, 0.0, 20.0, 30.0, 50.0]),
                     window=rng.choice([0, 0, span(16, 4096)]), bias=rng.random() < 0.3, prefix=rng.choice([0, 0, span(1, 2000)]),
                     docs=rng.random() < 0.25, causal=rng.random() < 0.85)
            c["length"] = c["n"] + span(1, 32768)
        case = _case(kind, **c)
        if _room(case) <= room and _cost(case) <= most:
            return case


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _randn(g, dt, *shape):
    return torch.randn(*shape, generator=g, dtype=dt, device=DEV)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _cu(counts):
    return _i32([0] + torch.tensor(counts, dtype=torch.int64).cumsum(0).tolist())


def _prepare_plan(case, seed, g):
    B, bs, counts = case["batch"], case["block"], _tokens(case)
    lens = [m // 2 for m in _lens(case, seed, [1] * B)]
    lens = [0 if i % 5 == 4 else m for i, m in enumerate(lens)]                 # some requests are new
    row = -(-(case["length"] + case["n"]) // bs)
    held = [-(-m // bs) for m in lens]
    need = sum(-(-(m + x) // bs) - h for m, x, h in zip(lens, counts, held))
    blocks = B * row                             # of which the stack has enough, or two thirds of that
    spare = need * 2 // 3 if case["scarce"] else blocks - sum(held)
    order = torch.randperm(blocks, generator=g, device=DEV).to(torch.int32)
    table = torch.full((B, row), -1, dtype=torch.int32, device=DEV)
    at = torch.arange(row, device=DEV) < _i32(held)[:, None]
    table[at] = order[: sum(held)]
    free = torch.full((blocks,), -1, dtype=torch.int32, device=DEV)
    free[:spare] = order[sum(held): sum(held) + spare]
    return {"table": table, "held": _i32(held), "lens": _i32(lens), "free": free, "count": _i32([spare]), "n_new": _i32(counts),
            "most": sum(counts) + case["pad"], "row": row}


def _prepare_verify(case, seed, g):
    B, n, V, dt = case["batch"], case["n"], case["vocab"], _dtype(case["dtype"])
    # a draft model that is near the target: their logits have most in common; some mass on few tokens, as with real ones
    logits = 2.5 * _randn(g, torch.float32, B, n, V)
    target = torch.softmax(logits + 0.7 * _randn(g, torch.float32, B, n, V), -1).to(dt)
    draft = torch.softmax(logits, -1).to(dt)
    i = torch.arange(n, device=DEV)
    if case["tree"]:                             # a node's parent is one of the few before it
        back = (torch.rand(B, n, generator=g, device=DEV) * torch.minimum(i, torch.tensor(4, device=DEV))).long() + 1
        parent = (i - back).clamp(min=0)
    else:
        parent = (i - 1).clamp(min=0).expand(B, n).contiguous()
    # a child's token is drawn from its parent's distribution by the draft model (the likeliest one where it is sure of itself)
    tokens = torch.zeros(B, n, dtype=torch.int32, device=DEV)
    b = torch.arange(B, device=DEV)
    for j in range(1, n):
        rows = draft[b, parent[:, j]].float()
        if not case["sure"]:
            rows = rows.log() - torch.log(-torch.log(torch.rand(B, V, generator=g, device=DEV).clamp(1e-20, 1 - 1e-7)))
        else:
            rows = rows * (1 + 0.5 * torch.rand(B, V, generator=g, device=DEV))
        tokens[:, j] = rows.argmax(-1).to(torch.int32)
    live = torch.randint(max(1, n - 2), n + 1, (B, 1), generator=g, device=DEV)
    tokens = torch.where(i < live, tokens, torch.full_like(tokens, -1))         # some sequences have fewer drafts
    return {"target": target, "draft": None if case["sure"] else draft, "tokens": tokens,
            "parents": parent.to(torch.int32) if case["tree"] else None,
            "u": torch.rand(B, n, generator=g, device=DEV), "u_next": torch.rand(B, generator=g, device=DEV)}


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind, B, Hq, Hkv, d, bs = (case[k] for k in ("kind", "batch", "q_heads", "kv_heads", "head_dim", "block"))
    dt = _dtype(case["dtype"])
    if kind == "plan":
        return {"case": case, **_prepare_plan(case, seed, g)}
    if kind == "verify":
        return {"case": case, **_prepare_verify(case, seed, g)}
    counts = _tokens(case)
    lens = _lens(case, seed, counts)
    T, most = sum(counts) + case["pad"], max(case["length"], case["n"])
    s = {"case": case, "scale": 1.0 / math.sqrt(d), "counts": counts, "length": lens, "lens": _i32(lens), "cu": _cu(counts), "most": most}
    row = -(-most // bs) if bs else 0
    nb, cap = (B * row, bs) if bs else (B, most)
    s["table"] = torch.randperm(nb, generator=g, device=DEV).to(torch.int32).view(B, row) if bs else None
    s["k"], s["v"] = _randn(g, dt, nb, Hkv, cap, d), _randn(g, dt, nb, Hkv, cap, d)
    if kind == "write":
        # K and V are parts of the rows of one product, as a fused projection leaves them
        rows = _randn(g, dt, T, (Hq + 2 * Hkv) * d)
        s["k_in"] = rows[:, Hq * d: (Hq + Hkv) * d].unflatten(-1, (Hkv, d))
        s["v_in"] = rows[:, (Hq + Hkv) * d:].unflatten(-1, (Hkv, d))
        where = []
        for b, (m, length) in enumerate(zip(counts, lens)):
            p = torch.arange(length - m, length, device=DEV)
            where.append((s["table"][b].long()[p // bs] * bs + p % bs) if bs else b * cap + p)
        where.append(torch.full((case["pad"],), -1, dtype=torch.int64, device=DEV))
        s["slots"] = torch.cat(where).to(torch.int32)
        return s
    s["q"] = _randn(g, dt, T, Hq, d) * (3 if case["cap"] else 1)
    s["o"] = torch.zeros(T, Hq, d, dtype=_dtype(case["out"]), device=DEV)
    s["lse"] = torch.zeros(T, Hq, dtype=torch.float32, device=DEV)
    s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq)).float() if case["bias"] else None
    s["prefix"] = None
    if case["prefix"]:
        s["prefix"] = torch.randint(case["prefix"] // 2, case["prefix"] + 1, (B,), generator=g, device=DEV).to(torch.int32)
        s["prefix"][0] = case["prefix"]
    first = _bounds(case, seed, counts, lens)
    s["first"] = None if first is None else _i32(first + [0] * case["pad"])
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _line(s, x, b, length):
    """Rows [Hkv, length, d] of a sequence, blocks put in order."""
    if s["table"] is None:
        return x[b, :, :length]
    return x[s["table"][b].long()].transpose(0, 1).flatten(1, 2)[:, :length]


def _plain_plan(s):
    case, bs, most = s["case"], s["case"]["block"], s["most"]
    B, row = s["table"].shape
    lens, held, new, count = s["lens"].long(), s["held"].long(), s["n_new"].long().clamp(min=0), s["count"].long()
    need = ((lens + new + bs - 1) // bs - held).clamp(min=0)
    fits = lens + new <= row * bs                # a row of the table too short: the sequence takes no part
    need, new = need * fits, new * fits
    got = ((need == 0) | (need.cumsum(0) <= count)) & ((new == 0) | (new.cumsum(0) <= most))
    need, new = need * got, new * got
    cu = torch.cat((torch.zeros(1, dtype=torch.int64, device=DEV), new.cumsum(0)))
    before = need.cumsum(0) - need
    # granted blocks come off the top of the stack
    j = torch.arange(row, device=DEV) - held[:, None]
    mine = (j >= 0) & (j < need[:, None])
    k = (count - 1 - (before[:, None] + j)).clamp(min=0)
    table = torch.where(mine, s["free"].long()[k.clamp(max=s["free"].numel() - 1)], s["table"].long())
    t = torch.arange(most, device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True)
    real = b < B
    b = b.clamp(max=B - 1)
    pos = torch.where(real, lens[b] + t - cu[b], torch.zeros_like(t))
    slot = torch.where(real, table[b, (pos // bs).clamp(max=row - 1)] * bs + pos % bs, torch.full_like(t, -1))
    # the tokens are taken back: lengths, blocks held and the stack are what they were, the rows keep their entries
    s["table"].copy_(table.to(torch.int32))
    back = (count + torch.zeros_like(need) - before - need)                     # where a sequence's blocks lie on the stack
    free = s["free"].long()
    place = (back[:, None] + need[:, None] - 1 - j)[mine]
    free = free.index_put((place,), table[mine])
    s["free"].copy_(free.to(torch.int32))
    i = torch.int32
    return {"cu": cu.to(i), "pos": pos.to(i), "slots": slot.to(i), "table": s["table"], "lens": s["lens"], "held": s["held"],
            "free": s["free"], "count": s["count"]}


def _plain_write(s):
    bs, real = s["case"]["block"] or s["most"], s["slots"] >= 0
    at = s["slots"].long()[real]
    for x in "kv":
        s[x][at // bs, :, at % bs] = s[x + "_in"][real]
    return {"k": s["k"], "v": s["v"]}


def _plain_chunk(s):
    case = s["case"]
    Hq, Hkv, d = (case[x] for x in ("q_heads", "kv_heads", "head_dim"))
    G, at = Hq // Hkv, 0
    slopes = None if s["slopes"] is None else s["slopes"].view(Hkv, G, 1, 1)
    for b, (m, length) in enumerate(zip(s["counts"], s["length"])):
        K, V = _line(s, s["k"], b, length).float(), _line(s, s["v"], b, length).float()
        j = torch.arange(length, device=DEV)
        pre = 0 if s["prefix"] is None else s["prefix"][b]
        for i0 in range(0, m, 1024):
            i1 = min(i0 + 1024, m)
            p = torch.arange(length - m + i0, length - m + i1, device=DEV)[:, None]
            sees = torch.ones(i1 - i0, length, dtype=torch.bool, device=DEV)
            if case["causal"]:
                sees &= j <= p
            if case["window"]:
                sees &= p - j < case["window"]
            if s["first"] is not None:
                sees &= j >= s["first"][at + i0: at + i1, None]
            sees |= j < pre
            q = s["q"][at + i0: at + i1].float().view(i1 - i0, Hkv, G, d).permute(1, 2, 0, 3).reshape(Hkv, -1, d)
            x = torch.matmul(q, K.transpose(-1, -2)).mul_(s["scale"]).view(Hkv, G, i1 - i0, length)
            if case["cap"]:
                x = x.div_(case["cap"]).tanh_().mul_(case["cap"])
            if slopes is not None:
                x = x - slopes * (p - j).abs().float()
            x = x.masked_fill_(~sees, -math.inf)
            top = x.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            w = x.sub_(top).exp_()
            total = w.sum(-1, keepdim=True)
            o = torch.matmul(w.view(Hkv, -1, length), V).view(Hkv, G, i1 - i0, d) / torch.where(total == 0, torch.ones_like(total), total)
            s["o"][at + i0: at + i1] = o.permute(2, 0, 1, 3).reshape(i1 - i0, Hq, d).to(s["o"].dtype)
            s["lse"][at + i0: at + i1] = (top + total.log()).squeeze(-1).permute(2, 0, 1).reshape(i1 - i0, Hq)
        at += m
    return {"o": s["o"], "lse": s["lse"]}


def _plain_verify(s):
    target, draft, tokens = s["target"], s["draft"], s["tokens"].long()
    B, n, V = target.shape
    b, f64 = torch.arange(B, device=DEV), torch.float64
    parents = torch.arange(-1, n - 1, device=DEV).expand(B, n) if s["parents"] is None else s["parents"].long()
    cur, cnt = torch.zeros(B, dtype=torch.int64, device=DEV), torch.ones(B, dtype=torch.int64, device=DEV)
    path = torch.full((B, n), -1, dtype=torch.int64, device=DEV)
    path[:, 0] = 0
    p = target[b, cur].to(f64).clamp(min=0)      # the node's target, what is left of it, and the draft model's row
    q = None if draft is None else draft[b, cur].to(f64).clamp(min=0)
    c, mass, rest = torch.zeros(B, dtype=f64, device=DEV), torch.ones(B, dtype=f64, device=DEV), p
    for j in range(1, n):
        x = tokens[:, j]
        test = (parents[:, j] == cur) & (x >= 0) & (x < V)
        x = x.clamp(0, V - 1)
        qx = torch.ones_like(mass) if q is None else q[b, x]
        good = test & (s["u"][:, j].to(f64) * qx * mass < rest[b, x])
        bad = test & ~good
        # refused: the draft's share leaves the target
        c = torch.where(bad, c + mass, c)
        if q is None:
            gone = torch.zeros_like(rest).scatter_(1, x[:, None], 1.0) * bad[:, None]
            rest = rest * (1 - gone)
        else:
            rest = torch.where(bad[:, None], (p - c[:, None] * q).clamp(min=0), rest)
        mass = torch.where(bad, rest.sum(-1), mass)
        # accepted: on to its own children
        cur = torch.where(good, torch.full_like(cur, j), cur)
        path.scatter_(1, cnt[:, None].clamp(max=n - 1), torch.where(good, torch.full_like(cur, j), path.gather(1, cnt[:, None].clamp(max=n - 1))[:, 0])[:, None])
        cnt = cnt + good
        p = torch.where(good[:, None], target[b, cur].to(f64).clamp(min=0), p)
        if q is not None:
            q = torch.where(good[:, None], draft[b, cur].to(f64).clamp(min=0), q)
        c, mass, rest = torch.where(good, torch.zeros_like(c), c), torch.where(good, torch.ones_like(mass), mass), torch.where(good[:, None], p, rest)
    rest = torch.where(rest.sum(-1, keepdim=True) > 0, rest, p)
    run = rest.cumsum(-1)
    total = run[:, -1]
    # the first token whose running sum passes the threshold
    after = run > (s["u_next"].to(f64) * total)[:, None]
    token = torch.where(total > 0, torch.where(after.any(-1), after.to(torch.int32).argmax(-1), (rest > 0).cumsum(-1).argmax(-1)),
                        torch.full_like(cur, -1))
    i = torch.int32
    return {"path": path.to(i), "cnt": cnt.to(i), "next": token.to(i)}


_PLAIN = {"plan": _plain_plan, "write": _plain_write, "chunk": _plain_chunk, "verify": _plain_verify}


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _handles(s):
    """What a program makes once and keeps: shape, views, states, output buffers, workspace."""
    from paper_2507_03153_amd import hgca

    case = s["case"]
    kind, B, Hq, Hkv, d, bs = (case[k] for k in ("kind", "batch", "q_heads", "kv_heads", "head_dim", "block"))
    i32 = dict(dtype=torch.int32, device=DEV)
    if kind == "plan":
        return {"state": hgca.BlockState(s["table"], s["held"], s["lens"], s["free"], s["count"], bs), "kept": s["lens"].clone(),
                "cu": torch.empty(B + 1, **i32), "pos": torch.empty(s["most"], **i32), "slots": torch.empty(s["most"], **i32)}
    if kind == "verify":
        n = case["n"]
        return {"path": torch.empty(B, n, **i32), "cnt": torch.empty(B, **i32), "next": torch.empty(B, **i32),
                "ws": hgca.verify_workspace(B, case["vocab"], DEV)}
    shape = hgca.Shape(hgca.F32 if case["dtype"] == "f32" else hgca.BF16, B, Hq, Hkv, d, s["scale"])
    h = {"shape": shape, "tier": hgca.Tier(s["k"], s["v"], s["most"], s["lens"], s["table"], bs)}
    if kind == "chunk":
        h["ws"] = hgca.chunk_workspace(shape, s["q"].shape[0], s["most"], DEV)
    return h


def _own(s):
    from paper_2507_03153_amd import hgca

    case = s["case"]
    kind = case["kind"]
    h = s.get("handles")
    if h is None:
        h = s["handles"] = _handles(s)
    if kind == "plan":
        hgca.kv_plan(h["state"], s["n_new"], h["cu"], h["pos"], h["slots"])
        hgca.kv_release(h["state"], h["kept"])
        return {"cu": h["cu"], "pos": h["pos"], "slots": h["slots"], "table": s["table"], "lens": s["lens"], "held": s["held"],
                "free": s["free"], "count": s["count"]}
    if kind == "write":
        hgca.kv_write(h["shape"], h["tier"], s["slots"], s["k_in"], s["v_in"])
        return {"k": s["k"], "v": s["v"]}
    if kind == "verify":
        hgca.verify_drafts(s["target"], s["draft"], s["tokens"], s["u"], s["u_next"], h["path"], h["cnt"], h["next"], h["ws"],
                           parents=s["parents"])
        return {"path": h["path"], "cnt": h["cnt"], "next": h["next"]}
    hgca.chunk_attn(h["shape"], s["q"], s["cu"], h["tier"], s["o"], s["lse"], h["ws"], causal=case["causal"], window=case["window"],
                    cap=case["cap"], slopes=s["slopes"], prefix_lens=s["prefix"], first=s["first"])
    return {"o": s["o"], "lse": s["lse"]}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ---- in 64 bits -----------------------------------------------------------------------------------------------------

def _exact_chunk(case, s):
    Hq, Hkv, d = (case[x] for x in ("q_heads", "kv_heads", "head_dim"))
    f64 = torch.float64
    o, lse, at = s["o"].to(f64), s["lse"].to(f64), 0
    for b, (m, length) in enumerate(zip(s["counts"], s["length"])):
        pos, tok = torch.arange(length - m, length, device=DEV).view(-1, 1), torch.arange(length, device=DEV).view(1, -1)
        hidden = torch.zeros(m, length, dtype=torch.bool, device=DEV)
        if case["causal"]:
            hidden = hidden | (tok > pos)
        if case["window"] > 0:
            hidden = hidden | (tok <= pos - case["window"])
        if s["first"] is not None:
            hidden = hidden | (tok < s["first"][at: at + m].view(-1, 1))
        if s["prefix"] is not None:
            hidden = hidden & (tok >= int(s["prefix"][b]))
        if s["table"] is None:
            K, V = s["k"][b], s["v"][b]
        else:
            K, V = (torch.cat([s[x][i] for i in s["table"][b].tolist()], 1) for x in "kv")
        for h in range(Hq):
            k, v = K[h * Hkv // Hq, :length].to(f64), V[h * Hkv // Hq, :length].to(f64)
            for i in range(0, m, 4096):
                e = min(i + 4096, m)
                z = (s["q"][at + i: at + e, h].to(f64) @ k.t()) * s["scale"]
                if case["cap"] > 0:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][h].to(f64) * (pos[i: e] - tok).abs().to(f64)
                z[hidden[i: e]] = -math.inf
                w = torch.logsumexp(z, -1)
                lse[at + i: at + e, h] = w
                w = torch.where(w == -math.inf, torch.zeros_like(w), w)
                o[at + i: at + e, h] = torch.exp(z - w[:, None]) @ v
        at += m
    return {"o": o, "lse": lse}


def _exact_verify(case, s):
    paths, counts, following = [], [], []
    V, n = case["vocab"], case["n"]
    tokens, u, last = s["tokens"].tolist(), s["u"].double().tolist(), s["u_next"].double().tolist()
    for b in range(case["batch"]):
        up = list(range(-1, n - 1)) if s["parents"] is None else s["parents"][b].tolist()
        node, path = 0, [0]
        while True:
            full = s["target"][b, node].double()
            dist, step = full, None              # dist is a distribution from the first refusal on
            q = None if s["draft"] is None else s["draft"][b, node].double()
            for j in range(node + 1, n):
                x = tokens[b][j]
                if up[j] != node or not 0 <= x < V:
                    continue
                if u[b][j] * (1.0 if q is None else float(q[x])) < float(dist[x]):
                    step = j
                    break
                if q is None:
                    left = dist.clone()
                    left[x] = 0.0
                else:
                    left = torch.clamp(dist - q, min=0.0)
                total = float(left.sum())
                dist = left / total if total > 0 else left
            if step is None:
                break
            node = step
            path.append(node)
        if float(dist.sum()) == 0.0:
            dist = full
        at = torch.cumsum(dist, 0)
        over = (at > last[b] * at[-1]).nonzero()
        counts.append(len(path))
        paths.append(path + [-1] * (n - len(path)))
        following.append((int(over[0]) if len(over) else int(dist.nonzero()[-1])) if float(at[-1]) > 0 else -1)
    return {"path": _i32(paths), "cnt": _i32(counts), "next": _i32(following)}


def _exact_plan(case, s):
    bs, most, row = case["block"], s["most"], s["row"]
    lens, held, new = s["lens"].tolist(), s["held"].tolist(), s["n_new"].tolist()
    table, free, left = s["table"].tolist(), s["free"].tolist(), int(s["count"])
    asked = tokens = top = 0
    cu, pos, slots = [0], [], []
    for b, (m, x) in enumerate(zip(lens, new)):
        need = -(-(m + x) // bs) - held[b]
        good = m + x <= row * bs
        if good:
            asked += need
            tokens += x
            good = (need == 0 or asked <= left) and (x == 0 or tokens <= most)
        if good:
            for i in range(need):
                table[b][held[b] + i] = free[left - 1 - top]
                top += 1
            pos += range(m, m + x)
            slots += [table[b][p // bs] * bs + p % bs for p in range(m, m + x)]
        cu.append(len(pos))
    pad = most - len(pos)
    return {"cu": _i32(cu), "pos": _i32(pos + [0] * pad), "slots": _i32(slots + [-1] * pad), "table": _i32(table), "lens": s["lens"],
            "held": s["held"], "free": s["free"], "count": s["count"]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return _exact_plan(case, s)
    if case["kind"] == "verify":
        return _exact_verify(case, s)
    if case["kind"] == "chunk":
        return _exact_chunk(case, s)
    width, slots = case["block"] or s["most"], s["slots"].tolist()
    for x in "kv":
        flat = s[x].transpose(1, 2).reshape(-1, case["kv_heads"], case["head_dim"]).double()
        keep = [i for i, slot in enumerate(slots) if slot >= 0]
        flat[s["slots"][keep].long()] = s[x + "_in"][keep].double()
        s[x] = flat.unflatten(0, (-1, width)).transpose(1, 2).contiguous()
    return {"k": s["k"], "v": s["v"]}
