"""Plain 64-bit forms (numpy, on the CPU) of norm with rotation, tree attention and the 8-bit rows, and builders of their
inputs; the tests of those operators share them."""
import numpy as np

from paper_2507_03153_amd import workloads as wl


def to_bf16(x):
    """fp64/fp32 array rounded once to bf16, as fp32 values."""
    return wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(np.ascontiguousarray(x, np.float32)))


def ancestors(rng, n):
    """A random tree over n drafted tokens as bit masks: parent of i is an earlier token or none."""
    m = []
    for i in range(n):
        p = int(rng.integers(-1, i)) if i else -1
        m.append((m[p] if p >= 0 else 0) | 1 << i)
    return m


def as_int64(masks):
    """Masks [B][n] (Python ints of up to 64 bits) as an int64 array of the same bits."""
    return np.array([[x - (1 << 64) if x >> 63 else x for x in row] for row in masks], np.int64)


def rows_attention(q, K, V, lens, scale, masks=None):
    """q [B,n,Hq,d], K, V [B,Hkv,T,d], lens [B], masks[b][i] or None -> O, lse.  A row that a query does not see is not looked at."""
    B, n, Hq, d = q.shape
    G = Hq // K.shape[1]
    O, lse = np.zeros(q.shape), np.full((B, n, Hq), -np.inf)
    for b in range(B):
        L = int(lens[b])
        for i in range(n):
            sees = np.ones(L, bool)
            if masks is not None:
                for t in range(max(L - n, 0), L):
                    sees[t] = bool(masks[b][i] >> (t - (L - n)) & 1)
            if not sees.any():
                continue
            for h in range(Hq):
                s = scale * (K[b, h // G, :L][sees] @ q[b, i, h])
                m = s.max()
                w = np.exp(s - m)
                O[b, i, h] = (w[:, None] * V[b, h // G, :L][sees]).sum(0) / w.sum()
                lse[b, i, h] = m + np.log(w.sum())
    return O, lse


def encode(x):
    """Rows [..., d] -> E4M3 codes and E8M0 codes (uint8), from the definition."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = np.where(np.isfinite(b), np.abs(b), 0).max(-1)
    e = np.full(top.shape, -110)
    for c in range(-110, 121):                   # the least exponent at which the block fits
        e = np.where(top > 448.0 * 2.0 ** c, c + 1, e)
    with np.errstate(invalid="ignore"):
        y = b / 2.0 ** e[..., None].astype(np.float64)
    a = np.abs(np.where(np.isfinite(y), y, 0))
    _, up = np.frexp(a)
    step = 2.0 ** (np.maximum(up - 1, -6) - 3).astype(np.float64)
    r = np.rint(a / step) * step                 # ties to even: a / step is exact
    r = np.where(r * 2.0 ** e[..., None].astype(np.float64) >= 2.0 ** 128, 240.0, r)      # nothing finite becomes an infinity
    m, up = np.frexp(r)
    small = r < 2.0 ** -6
    code = np.where(small, np.rint(r * 2.0 ** 9), ((up - 1 + 7) << 3) + np.rint((m * 2 - 1) * 8)).astype(np.int64)
    code = np.where(np.isfinite(b), code, 0x7f) | (np.signbit(b).astype(np.int64) << 7)
    return code.reshape(x.shape).astype(np.uint8), (e + 127).astype(np.uint8)


def decode(codes, scales):
    """What the bytes stand for, fp64; NaN codes are NaN."""
    c = codes.astype(np.int64)
    e, f = c >> 3 & 15, (c & 7).astype(np.float64)
    x = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10).astype(np.float64))
    x = np.where((c & 0x7f) == 0x7f, np.nan, x) * np.where(c >> 7, -1.0, 1.0)
    return x * np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, -1)


def norm_rope(x, w, eps, pos, freq, interleaved):
    """x [B,n,H,d], w [d] or None, pos [B,n], freq [rot/2] -> fp64."""
    x = np.asarray(x, np.float64)
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)
    half = len(freq)
    t = pos.astype(np.longdouble)[..., None] * freq.astype(np.longdouble)
    c, s = np.cos(t).astype(np.float64)[:, :, None], np.sin(t).astype(np.float64)[:, :, None]
    j = np.arange(half)
    i, k = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
    y = x.copy()
    y[..., i], y[..., k] = x[..., i] * c - x[..., k] * s, x[..., i] * s + x[..., k] * c
    return y


def paged(rng, x, block, first, extra=0):
    """Rows [B,H,T,d] in shuffled blocks: blocks [n,H,block,d], table [B,row] whose row b starts at entry first[b].  Slots behind
    T keep what was in the block: NaN (float) or 0xff (bytes)."""
    B, H, T, d = x.shape
    nb = -(-T // block)
    row = nb + int(max(first)) + extra
    perm = rng.permutation(B * row).astype(np.int32).reshape(B, row)
    out = np.full((B * row, H, block, d), np.nan if x.dtype.kind == "f" else 0xff, x.dtype)
    for b in range(B):
        for j in range(nb):
            n = min(block, T - j * block)
            out[perm[b, first[b] + j], :, :n] = x[b, :, j * block:j * block + n]
    return out, perm
