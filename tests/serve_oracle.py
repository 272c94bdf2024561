"""Plain 64-bit forms (numpy, on the CPU) of token plans, packed writes, attention of packed chunks and verification of drafts; the tests
of those operators share them."""
import numpy as np


def plan(block_size, table, held, lens, free, n_new, max_tokens):
    """free: list, top last.  Returns cu, positions, slots (lists) and the status bits; table, held, lens, free are updated."""
    B, row = len(lens), table.shape[1] if len(table) else 0
    asked = tokens = 0
    grants, bits, count = [], 0, len(free)
    for b in range(B):
        n = max(int(n_new[b]), 0)
        if lens[b] + n > row * block_size:
            bits |= 2
            grants.append((0, 0))
            continue
        need = max(-(-(lens[b] + n) // block_size) - held[b], 0)
        asked, tokens = asked + need, tokens + n
        if need and asked > count:
            bits |= 8
        if n and tokens > max_tokens:
            bits |= 16
        grants.append((0, 0) if (need and asked > count) or (n and tokens > max_tokens) else (n, need))
    cu, pos, slots = [0], [], []
    for b, (n, need) in enumerate(grants):
        for i in range(need):
            table[b, held[b] + i] = free.pop()
        for p in range(lens[b], lens[b] + n):
            pos.append(p)
            slots.append(int(table[b, p // block_size]) * block_size + p % block_size)
        held[b] += need
        lens[b] += n
        cu.append(len(pos))
    return cu, pos, slots, bits


def release(block_size, table, held, lens, free, new_lens):
    for b in reversed(range(len(lens))):
        lens[b] = min(max(int(new_lens[b]), 0), lens[b])
        keep = min(-(-lens[b] // block_size), held[b])
        for j in reversed(range(keep, held[b])):
            free.append(int(table[b, j]))
        held[b] = keep


def sees(n, length, causal=True, window=0, prefix=0, first=None):
    """[n, length]: what the last n tokens of a sequence see."""
    p, j = np.arange(length - n, length)[:, None], np.arange(length)[None, :]
    m = np.ones((n, length), bool)
    if causal:
        m &= j <= p
    if window:
        m &= p - j < window
    if first is not None:
        m &= j >= np.asarray(first).reshape(-1, 1)
    return m | (j < prefix)


def chunk(q, cu, K, V, lens, scale, causal=True, window=0, cap=0.0, slopes=None, prefix=None, first=None):
    """q [T,Hq,d], K, V [B,Hkv,cap,d] -> O, lse for the rows up to cu[-1].  A row that a query does not see is not looked at."""
    T, Hq, d = q.shape
    G = Hq // K.shape[1]
    O, lse = np.zeros(q.shape), np.full((T, Hq), -np.inf)
    for b, L in enumerate(lens):
        r0, r1 = cu[b], cu[b + 1]
        n, L = r1 - r0, int(L)
        if n == 0 or L == 0:
            continue
        m = sees(n, L, causal, window, 0 if prefix is None else int(prefix[b]), None if first is None else first[r0:r1])
        dist = np.abs(np.arange(L - n, L)[:, None] - np.arange(L)[None, :]).astype(np.float64)
        used = m.any(0)
        for h in range(Hq):
            k, v = K[b, h // G, :L], V[b, h // G, :L]
            s = np.full((n, L), -np.inf)
            s[:, used] = scale * (q[r0:r1, h].astype(np.float64) @ np.where(used[:, None], k, 0)[used].astype(np.float64).T)
            if cap:
                s = cap * np.tanh(s / cap)
            if slopes is not None:
                s = s - float(slopes[h]) * dist
            s = np.where(m, s, -np.inf)
            top = s.max(1, keepdims=True)
            w = np.where(m, np.exp(s - np.where(np.isneginf(top), 0, top)), 0)
            total = w.sum(1)
            some = total > 0
            O[r0:r1, h][some] = (w @ np.where(used[:, None], v, 0).astype(np.float64))[some] / total[some, None]
            lse[r0:r1, h][some] = top[some, 0] + np.log(total[some])
    return O, lse


def verify(target, draft, tokens, u, u_next, parents=None):
    """target, draft [B,n,V] (draft None), tokens [B,n] -> path, cnt, next, and the least margin by which any decision was taken."""
    B, n, V = target.shape
    sane = lambda x: np.where(np.isfinite(x) & (x > 0), x, 0).astype(np.float64)
    path, cnt, nxt, margin = np.full((B, n), -1, np.int64), np.zeros(B, np.int64), np.zeros(B, np.int64), 1.0
    for b in range(B):
        up = list(range(-1, n - 1)) if parents is None else [int(x) for x in parents[b]]
        node, got = 0, [0]
        while True:
            full = sane(target[b, node])
            dist, q = full.copy(), None if draft is None else sane(draft[b, node])
            step = None
            for j in range(node + 1, n):
                x = int(tokens[b, j])
                if up[j] != node or not 0 <= x < V:
                    continue
                left, right = float(u[b, j]) * (1.0 if q is None else q[x]), dist[x]
                if left != right:
                    margin = min(margin, abs(left - right) / max(left, right))
                if left < right:
                    step = j
                    break
                if q is None:
                    dist[x] = 0
                else:
                    dist = np.maximum(dist - q, 0)
                total = dist.sum()
                dist = dist / total if total > 0 else dist
            if step is None:
                break
            node = step
            got.append(node)
        if dist.sum() == 0:
            dist = full
        run = np.cumsum(dist)
        t = float(u_next[b]) * run[-1]
        if run[-1] > 0:
            over = np.nonzero((run > t) & (dist > 0))[0]
            nxt[b] = over[0] if len(over) else np.nonzero(dist)[0][-1]
            if t > 0:
                margin = min(margin, float(np.abs(run[dist > 0] - t).min()) / run[-1])
        else:
            nxt[b] = -1
        path[b, :len(got)], cnt[b] = got, len(got)
    return path, cnt, nxt, margin
