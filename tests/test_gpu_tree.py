"""Attention of drafted tokens over a tier that ends in them (hgca_tree_attn) and the commit of accepted ones against 64 bits.

Tolerances.  A score is a sum of d products in fp32: off by at most d * 2^-23 * scale * sum |q_i k_i| (the order of the sum is
free), relative to the weight the same, and 4 roundings of 2^-24 |s| for scale, shift and exponent; O is off by twice that (weights and
their sum) times max |v|, plus the sums over tokens, at most T / 32 + 64 additions of 2^-23 in a chain.  Over a whole output these
errors are random: their 2-norm is held to 2e-6 of the output's (weights that were rounded to 16 bits would be 2.4e-6 off).  bf16 O adds
half a step, 2^-8 relative."""
import sys

import numpy as np
import pytest

import draft_oracle as do
from paper_2507_03153_amd import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2507_03153_amd import hgca
    hgca.lib()
    return torch, hgca


def put(torch, a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV)
    return t.to(torch.float32 if dtype == "f32" else torch.bfloat16)


def i32(torch, a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def inputs(seed, dtype, B, n, Hq, Hkv, d, T):
    rng = np.random.default_rng(seed)
    r = (lambda *s: rng.standard_normal(s).astype(np.float32)) if dtype == "f32" else (lambda *s: do.to_bf16(rng.standard_normal(s)))
    return rng, r(B, n, Hq, d), r(B, Hkv, T, d), r(B, Hkv, T, d)


def tier_of(gpu, rng, dtype, K, V, lens, block):
    torch, hgca = gpu
    B, T = K.shape[0], K.shape[2]
    if not block:
        return hgca.Tier(put(torch, K, dtype), put(torch, V, dtype), T, i32(torch, lens))
    first = rng.integers(0, 3, B)
    state = rng.bit_generator.state
    kb, table = do.paged(rng, K, block, first)
    rng.bit_generator.state = state
    vb, _ = do.paged(rng, V, block, first)
    return hgca.Tier(put(torch, kb, dtype), put(torch, vb, dtype), T, i32(torch, lens), i32(torch, table), block, i32(torch, first))


def call(gpu, shape, q, tier, mask, out, ws_fill=0xff):
    torch, hgca = gpu
    B, n, Hq, d = q.shape
    o = torch.full(q.shape, float("nan"), dtype=torch.float32 if out == "f32" else torch.bfloat16, device=DEV)
    lse = torch.full((B, n, Hq), float("nan"), device=DEV)
    ws = hgca.tree_workspace(shape, n, tier.cap, DEV)
    ws.fill_(ws_fill)
    hgca.tree_attn(shape, q, tier, mask, o, lse, ws)
    torch.cuda.synchronize()
    return o, lse


def bounds(q, K, V, lens, scale, T):
    """(tolerance of O, of lse) from the docstring's sums."""
    d = q.shape[-1]
    amp = max(float(np.abs(q[b]).max() * np.abs(K[b, :, :L]).sum(-1).max()) if L else 0.0 for b, L in enumerate(lens)) * scale
    s = scale * max(float(np.linalg.norm(q[b], axis=-1).max() * np.linalg.norm(K[b, :, :L], axis=-1).max()) if L else 0.0
                    for b, L in enumerate(lens))
    e = d * 2.0 ** -23 * amp + 4 * 2.0 ** -24 * s
    vmax = max(float(np.abs(V[b, :, :L]).max()) if L else 0.0 for b, L in enumerate(lens))
    return (2 * e + (T / 32 + 64) * 2.0 ** -23) * vmax, e + (T / 32 + 64) * 2.0 ** -23 + 4 * 2.0 ** -24 * (s + np.log(T + 1.0))


def check(o, lse, O, L, tol_o, tol_l, out):
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = np.isneginf(L)
    assert np.array_equal(np.isneginf(lse), empty), "rows that see nothing differ"
    assert np.isfinite(o).all() and (o[empty] == 0).all()
    err, err_l = np.abs(o - O), np.abs(lse - L)[~empty]
    rel = np.linalg.norm(o - O) / max(np.linalg.norm(O), 1e-30)
    print(f"    max|dO|={err.max(initial=0):.2e} (of {tol_o:.2e}) rel={rel:.2e} max|dlse|={err_l.max(initial=0):.2e} (of {tol_l:.2e})", flush=True)
    assert (err <= tol_o + (2.0 ** -8 * np.abs(O) if out == "bf16" else 0)).all()
    assert err_l.max(initial=0) <= tol_l
    assert rel <= (2e-6 if out == "f32" else 2.0 ** -8)


CASES = [
    # dtype, d, Hq, Hkv, n, block, out, lens
    ("bf16", 128, 8, 2, 5, 0, "f32", [200, 5, 129]),
    ("bf16", 128, 8, 1, 1, 16, "f32", [1, 17, 0, 300]),
    ("bf16", 128, 4, 4, 33, 48, "f32", [33, 10, 200]),
    ("bf16", 128, 16, 2, 64, 16, "f32", [700, 64, 65]),
    ("bf16", 128, 16, 2, 64, 0, "bf16", [63, 64, 0, 515]),
    ("bf16", 64, 8, 4, 17, 16, "f32", [97, 128, 1000]),
    ("bf16", 64, 8, 8, 2, 0, "bf16", [2, 31, 32]),
    ("bf16", 64, 16, 2, 16, 32, "f32", [160, 161]),
    ("bf16", 128, 16, 2, 8, 16, "f32", [700, 8, 90, 1900]),
    ("bf16", 64, 4, 4, 64, 0, "bf16", [300, 64]),
    ("f32", 128, 8, 2, 5, 0, "f32", [200, 5, 129]),
    ("f32", 128, 8, 1, 9, 16, "f32", [9, 3, 400]),
    ("f32", 128, 4, 4, 64, 48, "bf16", [65, 260]),
    ("f32", 64, 4, 4, 4, 0, "f32", [260, 0, 4]),
    ("f32", 64, 16, 2, 33, 16, "f32", [33, 48, 111]),
    ("f32", 64, 2, 1, 1, 16, "f32", [1, 15, 16, 17]),
]


@pytest.mark.parametrize("masks", ["tree", "sparse", "none"])
@pytest.mark.parametrize("dtype,d,Hq,Hkv,n,block,out,lens", CASES)
def test_against_64_bits(gpu, dtype, d, Hq, Hkv, n, block, out, lens, masks):
    torch, hgca = gpu
    B, T = len(lens), max(lens) + 3
    print(f"\n[case] {dtype} d={d} {Hq}/{Hkv} n={n} block={block} out={out} lens={lens} {masks}", flush=True)
    rng, q, K, V = inputs(n * 1000 + d + Hq, dtype, B, n, Hq, Hkv, d, T)
    if masks == "tree":
        m = [do.ancestors(rng, n) for _ in range(B)]
    elif masks == "sparse":                      # any bits, many rows with none
        m = [[int(rng.integers(0, 2) * rng.integers(0, 1 << 62)) & ((1 << n) - 1) for _ in range(n)] for _ in range(B)]
    else:
        m = None
    for b, L in enumerate(lens):                 # behind the last token lies anything
        K[b, :, L:], V[b, :, L:] = np.nan, np.inf
    scale = 1.0 / np.sqrt(d)
    tier = tier_of(gpu, rng, dtype, K, V, lens, block)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, scale)
    scale = float(np.float32(scale))
    # bits of drafts that do not exist are set: they are ignored
    sent = None if m is None else torch.from_numpy(do.as_int64([[x | (((1 << 64) - 1) ^ ((1 << n) - 1)) for x in r] for r in m])).to(DEV)
    o, lse = call(gpu, shape, put(torch, q, dtype), tier, sent, out)
    O, L = do.rows_attention(q.astype(np.float64), K.astype(np.float64), V.astype(np.float64), lens, scale, m)
    check(o, lse, O, L, *bounds(q, K, V, lens, scale, T), out)


@pytest.mark.parametrize("B,T,n,block,out", [(64, 1024, 6, 16, "f32"), (64, 1008, 6, 0, "f32"), (64, 1024, 5, 0, "bf16"), (1, 65541, 8, 48, "f32")])
def test_17_to_32_rows_over_many_tokens(gpu, B, T, n, block, out):
    """Both sides of 2^17 tokens of all sequences and KV heads, where heads of 128 change kernels; lengths from none to all."""
    torch, hgca = gpu
    Hq, Hkv, d = 8, 2, 128
    rng, q, K, V = inputs(B + T + n, "bf16", B, n, Hq, Hkv, d, T)
    lens = [T] + [int(x) for x in rng.integers(0, T + 1, B - 1)]
    lens[1:4] = [0, 1, n + 1][:B - 1]
    m = [do.ancestors(rng, n) for _ in range(B)]
    for b, L in enumerate(lens):
        K[b, :, L:], V[b, :, L:] = np.nan, np.inf
    scale = float(np.float32(d ** -0.5))
    tier = tier_of(gpu, rng, "bf16", K, V, lens, block)
    o, lse = call(gpu, hgca.Shape(hgca.BF16, B, Hq, Hkv, d, scale), put(torch, q, "bf16"), tier, torch.from_numpy(do.as_int64(m)).to(DEV), out)
    O, L = do.rows_attention(q.astype(np.float64), K.astype(np.float64), V.astype(np.float64), lens, scale, m)
    check(o, lse, O, L, *bounds(q, K, V, lens, scale, T), out)


def test_empty_prefix_and_empty_rows(gpu):
    """Nothing but drafted tokens, a query without any bit."""
    torch, hgca = gpu
    for dtype in ("bf16", "f32"):
        rng, q, K, V = inputs(5, dtype, 1, 4, 2, 1, 64, 4)
        shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 1, 2, 1, 64, 0.125)
        m = [[0, 2, 1, 15]]
        tier = tier_of(gpu, rng, dtype, K, V, [4], 0)
        o, lse = call(gpu, shape, put(torch, q, dtype), tier, torch.from_numpy(do.as_int64(m)).to(DEV), "f32")
        O, L = do.rows_attention(q, K, V, [4], 0.125, m)
        check(o, lse, O, L, *bounds(q, K, V, [4], 0.125, 4), "f32")
        assert np.isneginf(lse[0, 0].cpu().numpy()).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("rows", [1, 40])
def test_rows_that_are_not_seen_may_hold_anything(gpu, dtype, d, rows):
    """Drafted rows with infinities and NaN: queries that do not see them are as without them, those that do see an infinity of
    its sign, or NaN."""
    torch, hgca = gpu
    n, Hq, T = max(rows // 2, 5), 2, 75
    rng, q, K, V = inputs(77 + rows, dtype, 1, n, Hq, 1, d, T)
    tail = T - n
    m = [[(1 << i) | 16 if i % 2 else 1 << i for i in range(n)]]
    m[0][4] = 1 << 3
    bad = V.copy()
    bad[0, 0, tail + 4, 0], bad[0, 0, tail + 4, d - 1], bad[0, 0, tail + 4, 7] = np.inf, -np.inf, np.nan
    badk = K.copy()
    badk[0, 0, tail + 2] = np.nan                # seen by query 2 alone
    m[0][2] = 0 if n < 3 else 1 << 2
    scale = float(np.float32(d ** -0.5))
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 1, Hq, 1, d, scale)
    mask = torch.from_numpy(do.as_int64(m)).to(DEV)
    good, lse0 = call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, K, V, [T], 0), mask, "f32")
    o, lse = call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, badk, bad, [T], 0), mask, "f32")
    sees = np.array([x >> 4 & 1 for x in m[0]], bool)
    nan_k = np.arange(n) == 2
    o, good, lse, lse0 = (x[0].cpu().numpy() for x in (o, good, lse, lse0))
    assert np.array_equal(o[~sees & ~nan_k], good[~sees & ~nan_k]) and np.array_equal(lse[~nan_k], lse0[~nan_k])
    assert np.isnan(o[nan_k]).all() and np.isnan(lse[nan_k]).all()
    at = sees & ~nan_k
    assert (o[at][..., 0] == np.inf).all() and (o[at][..., d - 1] == -np.inf).all() and np.isnan(o[at][..., 7]).all()
    rest = [c for c in range(d) if c not in (0, 7, d - 1)]
    assert np.array_equal(o[at][..., rest], good[at][..., rest])


@pytest.mark.parametrize("T", [1, 33, 129, 1217])
@pytest.mark.parametrize("dtype,d,n,Hq", [("bf16", 128, 3, 2), ("bf16", 64, 9, 2), ("bf16", 128, 20, 2), ("bf16", 64, 64, 2), ("f32", 64, 3, 2), ("f32", 128, 20, 2)])
def test_nan_scores_reach_the_result(gpu, dtype, d, n, Hq, T):
    """A query of NaN, and a key of NaN where it is the only token of a wave or of a split: the rows concerned are NaN, the others
    as without it."""
    torch, hgca = gpu
    rng, q, K, V = inputs(5, dtype, 2, n, Hq, 1, d, T)
    bad_q, bad_k = q.copy(), K.copy()
    bad_q[0, 0, 1] = np.nan                      # one head of one query
    bad_k[1, 0, T - 1] = np.nan                  # the last draft, which even queries see
    m = [[1 << max(n - T, 0) | (1 << (n - 1) if i % 2 == 0 else 0) for i in range(n)] for _ in range(2)]
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 2, Hq, 1, d, 0.1)
    mask = torch.from_numpy(do.as_int64(m)).to(DEV)
    run = lambda q, K: call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, K, V, [T, T], 0), mask, "f32")
    good, lse0 = (x.cpu().numpy() for x in run(q, K))
    o, lse = (x.cpu().numpy() for x in run(bad_q, bad_k))
    hit = np.zeros((2, n, Hq), bool)
    hit[0, 0, 1] = True
    hit[1, [i for i in range(n) if m[1][i] >> (n - 1) & 1]] = True
    assert np.isfinite(good).all() and np.isfinite(lse0).all()
    assert np.isnan(o[hit]).all() and np.isnan(lse[hit]).all()
    assert np.array_equal(o[~hit], good[~hit]) and np.array_equal(lse[~hit], lse0[~hit])


def test_large_scores(gpu):
    """Scores of +-2000: the maximum of a row lies anywhere, and far below it weights are 0."""
    torch, hgca = gpu
    rng, q, K, V = inputs(9, "f32", 2, 8, 4, 2, 64, 333)
    q *= 60.0
    shape = hgca.Shape(hgca.F32, 2, 4, 2, 64, 1.0)
    m = [do.ancestors(rng, 8) for _ in range(2)]
    o, lse = call(gpu, shape, put(torch, q, "f32"), tier_of(gpu, rng, "f32", K, V, [333, 50], 0), torch.from_numpy(do.as_int64(m)).to(DEV), "f32")
    O, L = do.rows_attention(q.astype(np.float64), K.astype(np.float64), V.astype(np.float64), [333, 50], 1.0, m)
    tol_o, tol_l = bounds(q, K, V, [333, 50], 1.0, 333)
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.abs(o - O).max() <= tol_o and np.abs(lse - L).max() <= tol_l


def test_a_long_sequence_among_short_ones(gpu):
    """More tokens per workgroup than one table of block rows covers (8192), lengths from 0 on; only the drafted tokens' and some
    other rows matter: the rest weighs nothing."""
    torch, hgca = gpu
    B, n, d, T, bs = 600, 3, 64, 8500, 16
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 40, B).astype(np.int32)
    lens[17], lens[599] = T, 8193
    n_blk = [-(-int(x) // bs) for x in lens]
    total = sum(n_blk)
    table = np.zeros((B, -(-T // bs)), np.int32)
    perm, at = rng.permutation(total).astype(np.int32), 0
    for b, x in enumerate(n_blk):
        table[b, :x] = perm[at:at + x]
        at += x
    kb, vb = (do.to_bf16(rng.standard_normal((total, 2, bs, d))) for _ in range(2))
    q = do.to_bf16(rng.standard_normal((B, n, 4, d)))
    m = [do.ancestors(rng, n) for _ in range(B)]
    tier = hgca.Tier(put(torch, kb, "bf16"), put(torch, vb, "bf16"), T, i32(torch, lens), i32(torch, table), bs)
    shape = hgca.Shape(hgca.BF16, B, 4, 2, d, 0.125)
    o, lse = call(gpu, shape, put(torch, q, "bf16"), tier, torch.from_numpy(do.as_int64(m)).to(DEV), "f32")
    for b in (0, 16, 17, 18, 300, 599):
        L = int(lens[b])
        K = np.concatenate([kb[i] for i in table[b, :n_blk[b]]] or [np.zeros((2, 0, d))], 1)[None, :, :max(L, 1)]
        V = np.concatenate([vb[i] for i in table[b, :n_blk[b]]] or [np.zeros((2, 0, d))], 1)[None, :, :max(L, 1)]
        O, Ls = do.rows_attention(q[b:b + 1], K, V, [L], 0.125, m[b:b + 1])
        check(o[b:b + 1], lse[b:b + 1], O, Ls, *bounds(q[b:b + 1], K, V, [L], 0.125, max(L, 1)), "f32")


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("n,Hq,d", [(4, 8, 128), (5, 8, 128), (12, 8, 128), (20, 8, 64), (40, 16, 128)])
def test_several_tables_per_workgroup(gpu, n, Hq, d, kv8):
    """Sequences that are one workgroup's work per KV head and longer than the tables of two passes (8192 tokens each), for every number of
    rows per workgroup."""
    torch, hgca = gpu
    B, T, bs = 150, 17000, 16
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 40, B).astype(np.int32)
    lens[17], lens[3], lens[149] = T, 2 * 8192, 8193
    n_blk = [-(-int(x) // bs) for x in lens]
    total = sum(n_blk)
    table = np.zeros((B, -(-T // bs)), np.int32)
    perm, at = rng.permutation(total).astype(np.int32), 0
    for b, x in enumerate(n_blk):
        table[b, :x] = perm[at:at + x]
        at += x
    kb, vb = (do.to_bf16(rng.standard_normal((total, 2, bs, d))) for _ in range(2))
    q = do.to_bf16(rng.standard_normal((B, n, Hq, d)))
    shape = hgca.Shape(hgca.BF16, B, Hq, 2, d, 0.125)
    rest = (T, i32(torch, lens), i32(torch, table), bs)
    if kv8:
        (kc, ks), (vc, vs) = do.encode(kb), do.encode(vb)
        kb, vb, m = do.decode(kc, ks), do.decode(vc, vs), None
        o, lse = torch.empty(B, n, Hq, d, device=DEV), torch.empty(B, n, Hq, device=DEV)
        hgca.kv8_attn(shape, put(torch, q, "bf16"), hgca.Kv8Tier(*(torch.from_numpy(x).to(DEV) for x in (kc, vc, ks, vs)), *rest), o, lse,
                      hgca.kv8_workspace(shape, n, T, DEV))
    else:
        m = [do.ancestors(rng, n) for _ in range(B)]
        o, lse = call(gpu, shape, put(torch, q, "bf16"), hgca.Tier(put(torch, kb, "bf16"), put(torch, vb, "bf16"), *rest),
                      torch.from_numpy(do.as_int64(m)).to(DEV), "f32")
    for b in (3, 17, 18, 149):
        L = int(lens[b])
        K, V = (np.concatenate([x[i] for i in table[b, :n_blk[b]]] or [np.zeros((2, 0, d))], 1)[None, :, :L] for x in (kb, vb))
        O, Ls = do.rows_attention(q[b:b + 1].astype(np.float64), K.astype(np.float64), V.astype(np.float64), [L], 0.125, None if m is None else m[b:b + 1])
        check(o[b:b + 1], lse[b:b + 1], O, Ls, *bounds(q[b:b + 1], K, V, [L], 0.125, max(L, 1)), "f32")


@pytest.mark.parametrize("dtype,B,n,Hq,Hkv,lens", [
    ("bf16", 130, 2, 4, 1, "ragged"),            # a lane has several sequences
    ("f32", 70, 3, 2, 1, "ragged"),
    ("bf16", 40, 40, 4, 1, "one long"),          # 160 rows: two blocks of 128
    ("bf16", 5, 20, 8, 2, "one long"),
    ("bf16", 512, 1, 1, 1, "equal"),
    ("bf16", 300, 1, 2, 1, "empty"),
    ("f32", 3, 1, 8, 8, "empty"),
])
def test_batches_share_the_splits_by_their_lengths(gpu, dtype, B, n, Hq, Hkv, lens):
    """Sequences of very different length, all of one length, and of none: each row is folded from its own sequence's splits."""
    torch, hgca = gpu
    d, bs, T = 64, 16, 2000
    rng = np.random.default_rng(B + n)
    L = {"ragged": lambda: (T * rng.random(B) ** 4).astype(np.int32), "one long": lambda: np.r_[np.full(B - 1, n), T].astype(np.int32),
         "equal": lambda: np.full(B, 700, np.int32), "empty": lambda: np.zeros(B, np.int32)}[lens]()
    print(f"\n[case] {dtype} B={B} n={n} {Hq}/{Hkv} {lens}", flush=True)
    n_blk = [-(-int(x) // bs) for x in L]
    table, at = np.zeros((B, T // bs), np.int32), 0
    perm = rng.permutation(max(sum(n_blk), 1)).astype(np.int32)
    for b, x in enumerate(n_blk):
        table[b, :x] = perm[at:at + x]
        at += x
    r = (lambda *s: rng.standard_normal(s).astype(np.float32)) if dtype == "f32" else (lambda *s: do.to_bf16(rng.standard_normal(s)))
    kb, vb, q = r(len(perm), Hkv, bs, d), r(len(perm), Hkv, bs, d), r(B, n, Hq, d)
    m = [do.ancestors(rng, n) for _ in range(B)]
    tier = hgca.Tier(put(torch, kb, dtype), put(torch, vb, dtype), T, i32(torch, L), i32(torch, table), bs)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, 0.125)
    o, lse = call(gpu, shape, put(torch, q, dtype), tier, torch.from_numpy(do.as_int64(m)).to(DEV), "f32")
    for b in sorted({0, 1, B // 2, B - 2, B - 1, int(np.argmax(L)), int(np.argmin(L))}):
        K, V = (np.concatenate([x[i] for i in table[b, :n_blk[b]]] or [np.zeros((Hkv, 1, d))], 1)[None] for x in (kb, vb))
        O, Ls = do.rows_attention(q[b:b + 1].astype(np.float64), K.astype(np.float64), V.astype(np.float64), L[b:b + 1], 0.125, m[b:b + 1])
        check(o[b:b + 1], lse[b:b + 1], O, Ls, *bounds(q[b:b + 1], K, V, L[b:b + 1], 0.125, T), "f32")


def test_same_result_again_and_in_a_graph(gpu):
    """Two runs agree bit for bit; a captured call follows its inputs, beside eager calls with a workspace of their own."""
    torch, hgca = gpu
    B, n, T = 3, 12, 700
    rng, q, K, V = inputs(31, "bf16", B, n, 8, 2, 128, T)
    shape = hgca.Shape(hgca.BF16, B, 8, 2, 128, 0.09)
    tier = tier_of(gpu, rng, "bf16", K, V, [700, 12, 333], 16)
    mask = torch.from_numpy(do.as_int64([do.ancestors(rng, n) for _ in range(B)])).to(DEV)
    qd = put(torch, q, "bf16")
    o1, l1 = call(gpu, shape, qd, tier, mask, "f32", 0x00)
    o2, l2 = call(gpu, shape, qd, tier, mask, "f32", 0xff)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)
    o, lse, ws = torch.empty_like(o1), torch.empty_like(l1), hgca.tree_workspace(shape, n, T, DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        hgca.tree_attn(shape, qd, tier, mask, o, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hgca.tree_attn(shape, qd, tier, mask, o, lse, ws)
    for i in range(4):
        qd.copy_(put(torch, q * (i + 1), "bf16"))
        o.fill_(7.0)
        graph.replay()
        want, want_l = call(gpu, shape, qd, tier, mask, "f32")
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(lse, want_l)


def test_two_streams(gpu):
    torch, hgca = gpu
    rng, q, K, V = inputs(32, "bf16", 2, 9, 8, 2, 128, 900)
    shape = hgca.Shape(hgca.BF16, 2, 8, 2, 128, 0.09)
    tier = tier_of(gpu, rng, "bf16", K, V, [900, 450], 0)
    qd = put(torch, q, "bf16")
    want, want_l = call(gpu, shape, qd, tier, None, "f32")
    outs = []
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        s.wait_stream(torch.cuda.current_stream())
        o, lse, ws = torch.empty_like(want), torch.empty_like(want_l), hgca.tree_workspace(shape, 9, 900, DEV)
        for _ in range(5):
            hgca.tree_attn(shape, qd, tier, None, o, lse, ws, stream=s)
        outs.append((o, lse, ws))
    torch.cuda.synchronize()
    for o, lse, _ in outs:
        assert torch.equal(o, want) and torch.equal(lse, want_l)


# ---- commit of accepted tokens ----

@pytest.mark.parametrize("dtype,block,given", [("bf16", 16, True), ("f32", 0, True), ("bf16", 48, False)])
def test_commit(gpu, dtype, block, given):
    torch, hgca = gpu
    B, n, Hkv, d, T = 4, 7, 3, 64, 100
    rng, _, K, V = inputs(41, dtype, B, 1, Hkv, Hkv, d, T)
    tier = tier_of(gpu, rng, dtype, K, V, [T] * B, block)
    lens = np.array([0, 37, 93, 97], np.int32)   # the last has room for three
    kin, vin = (put(torch, rng.standard_normal((B, n, Hkv, d)), dtype) for _ in range(2))
    path = np.sort(rng.permuted(np.tile(np.arange(n), (B, 1)), axis=1)[:, :n], 1)
    path[1], path[2] = [1, 3, 6, 9, -5, 0, 0], [2, 2, 5, 6, 6, 6, 6]
    cnt = np.array([0, 5, 7, 6], np.int32) if given else np.full(B, n, np.int32)
    eff = path if given else np.tile(np.arange(n), (B, 1))
    status, out = torch.zeros(1, dtype=torch.int32, device=DEV), torch.full((B,), -1, dtype=torch.int32, device=DEV)
    before = [t.clone() for t in (tier.k, tier.v)]
    hgca.kv_commit(hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hkv, Hkv, d, 1.0), tier, i32(torch, lens), kin, vin, out,
                   path=i32(torch, path) if given else None, cnt=i32(torch, cnt) if given else None, status=status)
    torch.cuda.synchronize()
    took = np.minimum(cnt, T - lens)
    if block:                                    # blocks of a table row: 112 or 144 slots, the capacity is 100 all the same
        assert tier.cap == T
    for t, src, old in ((tier.k, kin, before[0]), (tier.v, vin, before[1])):
        want = old.clone()
        for b in range(B):
            for i in range(took[b]):
                p, s = int(lens[b]) + i, min(max(int(eff[b, i]), 0), n - 1)
                if block:
                    blk = int(tier.block_table[b, int(tier.first_block[b]) + p // block])
                    want[blk, :, p % block] = src[b, s]
                else:
                    want[b, :, p] = src[b, s]
        assert torch.equal(t.view(torch.int32 if dtype == "f32" else torch.int16), want.view(torch.int32 if dtype == "f32" else torch.int16))
    assert out.cpu().tolist() == (lens + took).tolist()
    assert status.item() == hgca.CACHE_CONTEXT_FULL


def test_commit_into_its_own_lengths_and_defaults(gpu):
    """lens_out may be the tier's lengths; without first, path and cnt all rows go to the start."""
    torch, hgca = gpu
    B, n, Hkv, d = 2, 5, 2, 128
    tier = hgca.Tier(*(torch.zeros(B, Hkv, 8, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)), 8, torch.full((B,), 3, dtype=torch.int32, device=DEV))
    kin, vin = (torch.randn(B, n, Hkv, d, device=DEV).bfloat16() for _ in range(2))
    hgca.kv_commit(hgca.Shape(hgca.BF16, B, Hkv, Hkv, d, 1.0), tier, None, kin, vin, tier.seq_lens)
    torch.cuda.synchronize()
    assert tier.seq_lens.tolist() == [5, 5]
    assert torch.equal(tier.k[:, :, :5].transpose(1, 2), kin) and torch.equal(tier.v[:, :, :5].transpose(1, 2), vin)
    assert not tier.k[:, :, 5:].any()
