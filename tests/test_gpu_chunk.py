"""Attention of packed new tokens over one tier (hgca_chunk_attn) against 64 bits.

Tolerances.  A score is a sum of d products in fp32: off by at most d * 2^-23 * scale * sum |q_i k_i| (the order of the sum is free),
relative to the weight the same, and 4 roundings of 2^-24 |s| for scale, shift and exponent.  A cap's tanh is off by 3.5e-7 of itself (bf16 O: the fit, at most
0.7 cap there) or by 4 roundings and two approximate instructions (2^-22 of the cap), and does not enlarge what its argument is
off by; a bias is rounded, its product and its sum, 3 * 2^-24 of the largest slope * distance that a row sees.  O is off by twice
all that (weights and their sum) times max |v|, plus the sums over tokens, at most T / 32 + 64 additions of 2^-23 in a chain.  These errors are
random over an output: for fp32 O its 2-norm is held to 2e-6 of the output's plus twice what cap and bias may add.  bf16 O adds half a
step, 2^-8 relative, and for bf16 inputs weights that are rounded to bf16, at most 2^-8 each, so 2^-8 max |v| of the sum; as 2-norms, independent
of each other, sqrt(2) * 2^-8."""
import numpy as np
import pytest

import draft_oracle as do
import serve_oracle as so

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


def f32(torch, a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV)


def inputs(seed, dtype, counts, Hq, Hkv, d, T, sharp=1.0):
    rng = np.random.default_rng(seed)
    r = (lambda *s: rng.standard_normal(s).astype(np.float32)) if dtype == "f32" else (lambda *s: do.to_bf16(rng.standard_normal(s)))
    q = r(sum(counts), Hq, d)
    return rng, q if sharp == 1 else do.to_bf16(q * sharp) if dtype == "bf16" else q * np.float32(sharp), r(len(counts), Hkv, T, d), r(len(counts), Hkv, T, d)


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


def call(gpu, shape, q, cu, tier, out, pad=0, wide=0, ws=None, **opt):
    """pad: rows behind the last sequence; wide: columns between the rows of q."""
    torch, hgca = gpu
    T, Hq, d = q.shape
    big = torch.full((T + pad, Hq * d + wide), float("nan"), dtype=q.dtype, device=DEV)
    big[:T, :Hq * d] = q.reshape(T, Hq * d)
    qq = big[:, :Hq * d].unflatten(-1, (Hq, d))
    o = torch.full((T + pad, Hq, d), 77.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device=DEV)
    lse = torch.full((T + pad, Hq), 55.0, device=DEV)
    if ws is None:
        ws = hgca.chunk_workspace(shape, T + pad, tier.cap, DEV)
    ws.fill_(0xff)
    for k, t in (("slopes", f32), ("prefix_lens", i32), ("first", i32)):
        if opt.get(k) is not None:
            a = np.asarray(opt[k])
            opt[k] = t(torch, np.concatenate([a, np.zeros(pad, a.dtype)]) if k == "first" else a)
    hgca.chunk_attn(shape, qq, i32(torch, cu), tier, o, lse, ws, **opt)
    torch.cuda.synchronize()
    assert (o[T:] == 77).all() and (lse[T:] == 55).all(), "rows behind the last sequence"
    return o[:T], lse[:T]


def bounds(dtype, out, q, K, V, lens, scale, cap=0.0, slopes=None, T=1):
    """(tolerance of O, of lse, what cap and bias add) from the docstring's sums."""
    d, one = q.shape[-1], [(K[b, :, :L], V[b, :, :L]) for b, L in enumerate(lens) if L]
    if not one or not len(q):
        return 1.0, 1.0, 0.0
    amp = float(np.abs(q).max()) * max(float(np.abs(k[np.isfinite(k).all(-1)]).sum(-1).max(initial=0)) for k, _ in one) * scale
    s = scale * float(np.linalg.norm(q, axis=-1).max()) * max(float(np.linalg.norm(k[np.isfinite(k).all(-1)], axis=-1).max(initial=0)) for k, _ in one)
    more = cap * (0.7 * 3.5e-7 + 2.0 ** -22) + (0.0 if slopes is None else 3 * 2.0 ** -24 * float(np.abs(slopes).max()) * T)
    e = d * 2.0 ** -23 * amp + 4 * 2.0 ** -24 * s + more
    vmax = max(float(np.abs(v[np.isfinite(v)]).max(initial=0)) for _, v in one)
    tol = (2 * e + (T / 32 + 64) * 2.0 ** -23) * vmax
    if out == "bf16" and dtype == "bf16":
        tol += 2.0 ** -8 * vmax
    return tol, e + (T / 32 + 64) * 2.0 ** -23 + 4 * 2.0 ** -24 * (s + np.log(T + 1.0)), more


def check(o, lse, O, L, tol_o, tol_l, more, out, dtype="bf16"):
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = np.isneginf(L)
    assert np.array_equal(np.isneginf(lse), empty), "rows that see nothing differ"
    assert np.isfinite(o).all() and (o[empty] == 0).all()
    err, err_l = np.abs(o - O), np.abs(lse - L)[~empty]
    rel = np.linalg.norm(o - O) / max(np.linalg.norm(O), 1e-30)
    print(f"    max|dO|={err.max(initial=0):.2e} (of {tol_o:.2e}) rel={rel:.2e} max|dlse|={err_l.max(initial=0):.2e} (of {tol_l:.2e})", flush=True)
    assert (err <= tol_o + (2.0 ** -8 * np.abs(O) if out == "bf16" else 0)).all()
    assert err_l.max(initial=0) <= tol_l
    assert rel <= (2e-6 + 2 * more if out == "f32" else 2.0 ** -8 * (2 ** 0.5 if dtype == "bf16" else 1))


def slopes_of(Hq):
    return (2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq)).astype(np.float32)


SHAPES = [
    # dtype, d, Hq, Hkv, block, out, counts, lens
    ("bf16", 128, 8, 2, 16, "bf16", [1, 40, 0, 7, 129], [200, 40, 33, 5, 300]),
    ("bf16", 128, 8, 1, 0, "f32", [17, 1, 1], [17, 1, 515]),
    ("bf16", 128, 4, 4, 48, "bf16", [130, 64, 1], [260, 64, 0]),
    ("bf16", 64, 16, 2, 16, "bf16", [33, 16, 200], [97, 128, 700]),
    ("bf16", 64, 4, 2, 32, "f32", [65, 3], [65, 2]),
    ("bf16", 128, 16, 2, 64, "bf16", [1, 1, 2, 1], [1900, 64, 65, 1030]),
    ("f32", 128, 8, 2, 16, "f32", [1, 40, 0, 7, 129], [200, 40, 33, 5, 300]),
    ("f32", 64, 8, 1, 0, "f32", [17, 1, 1], [17, 1, 515]),
    ("f32", 128, 4, 4, 48, "bf16", [33, 1], [65, 100]),
    ("f32", 64, 16, 2, 16, "f32", [9, 100], [333, 400]),
]
MASKS = ["causal", "all", "window", "prefix", "docs", "everything"]
SCORES = ["plain", "cap", "bias", "cap+bias"]


def options(rng, masks, scores, counts, lens, Hq):
    opt, T = dict(causal=masks not in ("all", "docs")), sum(counts)
    if masks in ("window", "everything"):
        opt["window"] = 37
    if masks in ("prefix", "everything"):
        opt["prefix_lens"] = np.array([int(rng.integers(-2, L + 5)) for L in lens])
    if masks in ("docs", "everything"):          # any first token, behind the row's own position too: rows that see nothing
        opt["first"] = np.concatenate([rng.integers(-3, L + 2, n) for n, L in zip(counts, lens)] + [np.zeros(0, np.int64)])
    if "cap" in scores:
        opt["cap"] = 5.0 if masks == "causal" else 30.0
    if "bias" in scores:
        opt["slopes"] = slopes_of(Hq)
    return opt


@pytest.mark.parametrize("masks", MASKS)
@pytest.mark.parametrize("scores", SCORES)
@pytest.mark.parametrize("dtype,d,Hq,Hkv,block,out,counts,lens", SHAPES)
def test_against_64_bits(gpu, dtype, d, Hq, Hkv, block, out, counts, lens, masks, scores):
    torch, hgca = gpu
    B, T = len(lens), max(lens) + 3
    print(f"\n[case] {dtype} d={d} {Hq}/{Hkv} block={block} out={out} counts={counts} lens={lens} {masks} {scores}", flush=True)
    rng, q, K, V = inputs(sum(counts) * 100 + d + Hq, dtype, counts, Hq, Hkv, d, T, sharp=3.0 if "cap" in scores else 1.0)
    opt = options(rng, masks, scores, counts, lens, Hq)
    for b, L in enumerate(lens):                 # behind the last token lies anything
        K[b, :, L:], V[b, :, L:] = np.nan, np.inf
    scale = float(np.float32(1.0 / np.sqrt(d)))
    tier = tier_of(gpu, rng, dtype, K, V, lens, block)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, scale)
    cu = np.concatenate([[0], np.cumsum(counts)])
    o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, out, pad=5, wide=d, **dict(opt))
    kw = dict(opt)
    prefix = None if "prefix_lens" not in kw else np.clip(kw.pop("prefix_lens"), 0, None)
    O, L = so.chunk(q, cu, K, V, lens, scale, prefix=prefix, **kw)
    check(o, lse, O, L, *bounds(dtype, out, q, K, V, lens, scale, opt.get("cap", 0.0), opt.get("slopes"), T), out, dtype)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("counts,lens,block", [([1], [20011], 16), ([5, 1, 300, 1], [9000, 17, 2400, 4097], 0), ([1] * 70, None, 16),
                                               ([2, 0, 1, 40] * 40, None, 16)])
def test_shares_of_long_tiers(gpu, dtype, out, counts, lens, block):
    """Sequences cut into shares, one long one among short ones, more sequences than a wave has lanes; two calls give the same bits, and so does a workspace
    of another size."""
    torch, hgca = gpu
    Hq, Hkv, d, B = 8, 2, 64 if len(counts) > 8 else 128, len(counts)
    rng = np.random.default_rng(B)
    if lens is None:
        lens = [int(x) for x in np.maximum(rng.integers(0, 1500, B), counts)]
        lens[3], lens[B - 2] = 6000, 0
    T = max(lens)
    rng, q, K, V = inputs(B + T, dtype, counts, Hq, Hkv, d, T)
    scale = float(np.float32(d ** -0.5))
    tier = tier_of(gpu, rng, dtype, K, V, lens, block)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, scale)
    cu = np.concatenate([[0], np.cumsum(counts)])
    print(f"\n[case] {dtype}->{out} B={B} T={T}", flush=True)
    for opt in (dict(), dict(window=1000, cap=20.0, prefix_lens=np.full(B, 70))):
        o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, out, **dict(opt))
        big = hgca.chunk_workspace(shape, 4 * len(q) + 300, tier.cap + 5000, DEV)
        o2, lse2 = call(gpu, shape, put(torch, q, dtype), cu, tier, out, ws=big, **dict(opt))
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        kw = dict(opt)
        prefix = kw.pop("prefix_lens", None)
        O, L = so.chunk(q, cu, K, V, lens, scale, prefix=prefix, **kw)
        check(o, lse, O, L, *bounds(dtype, out, q, K, V, lens, scale, opt.get("cap", 0.0), None, T), out, dtype)


@pytest.mark.parametrize("dtype,d,block", [("bf16", 128, 16), ("bf16", 64, 0), ("f32", 128, 0), ("f32", 64, 16)])
@pytest.mark.parametrize("length", [300, 5000])
def test_rows_that_are_not_seen_may_hold_anything(gpu, dtype, d, block, length):
    """Infinities and NaN in V, and in K where no row sees them: rows that do not see them are as without them, those that do see an infinity of its
    sign, or NaN for a NaN or infinities of both signs, whatever they weigh."""
    torch, hgca = gpu
    Hq, Hkv, counts, lens = 4, 2, [90, 3], [length, 200]
    rng, q, K, V = inputs(length + d, dtype, counts, Hq, Hkv, d, length)
    scale = float(np.float32(d ** -0.5))
    cu = np.array([0, 90, 93])
    K[0, :, 40], V[0, :, 40] = np.nan, np.nan    # seen by nobody: before all windows and behind the prefix
    marks = [(length - 60, 1, np.inf), (length - 59, 1, -np.inf), (length - 50, 3, np.inf), (length - 30, 5, np.nan), (length - 1, 7, -np.inf), (10, 9, np.inf)]
    clean = V.copy()
    clean[0, :, 40] = 0
    for t, col, x in marks:
        V[0, 1, t, col] = x
        clean[0, 1, t, col] = 0
    opt = dict(window=100, prefix_lens=np.array([20, 0]))
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 2, Hq, Hkv, d, scale)
    tier = tier_of(gpu, rng, dtype, K, V, lens, block)
    out = "f32"
    o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, out, **dict(opt))
    K[0, :, 40] = 0
    O, L = so.chunk(q, cu, K, clean, lens, scale, window=100, prefix=[20, 0])
    o = o.double().cpu().numpy()
    m = so.sees(90, length, True, 100, 20)
    for h in (2, 3):                             # the heads of KV head 1
        for i in range(90):
            for col in {c for _, c, _ in marks}:
                seen = [x for t, c, x in marks if c == col and m[i, t]]
                if not seen:
                    continue
                want = sum(seen)                 # inf - inf and NaN are NaN
                assert np.array_equal(o[i, h, col], want, equal_nan=True), (i, h, col, o[i, h, col], want)
                o[i, h, col] = O[i, h, col]
    clean[0, 1, 10, 9] = 0
    check(torch.from_numpy(o), lse, O, L, *bounds(dtype, out, q, K, clean, lens, scale, T=length), out, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_odd_scores(gpu, dtype):
    """A NaN score of a row makes it NaN; scores of -inf weigh nothing, capped infinities are the cap; very large scores keep their weights."""
    torch, hgca = gpu
    d, L = 64, 150
    rng, q, K, V = inputs(4, dtype, [3], 2, 2, d, L)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 1, 2, 2, d, 0.125)
    cu = np.array([0, 3])
    q[:, :, 0] = np.abs(q[:, :, 0]) + 1
    q = do.to_bf16(q) if dtype == "bf16" else q                  # what `put` makes of it
    K[0, 0, 20, 0] = np.nan
    K[0, 1, 30, 0] = -np.inf
    tier = tier_of(gpu, rng, dtype, K, V, [L], 0)
    o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, "f32")
    assert torch.isnan(o[:, 0]).all() and torch.isnan(lse[:, 0]).all()
    K[0, 0, 20, 0] = 0
    K2 = K.copy()
    K2[0, 1, 30, 0] = -1e4                       # weight 0 all the same
    O, Ls = so.chunk(q, cu, K2, V, [L], 0.125)
    K[0, 1, 30] = K2[0, 1, 30]
    assert np.isfinite(o[:, 1].double().cpu().numpy()).all()
    assert np.abs(o[:, 1].double().cpu().numpy() - O[:, 1]).max() < 1e-5
    K[0, 1, 30, 0] = np.inf                      # capped: the cap itself
    tier = tier_of(gpu, rng, dtype, K, V, [L], 0)
    o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, "f32", cap=4.0)
    with np.errstate(invalid="ignore", over="ignore"):
        K2[0, 1, 30, 0] = 1e30
        O, Ls = so.chunk(q, cu, K2, V, [L], 0.125, cap=4.0)
    assert np.abs(o[:, 1].double().cpu().numpy() - O[:, 1]).max() < 2e-5
    # scaled scores beyond 2^30: two that differ in their last bits keep the ratio of their weights or are far apart
    K[:] = 0
    K[0, :, :3, 0] = 2.0 ** 40
    tier = tier_of(gpu, rng, dtype, K, V, [L], 0)
    q[:] = 0
    q[:, :, 0] = 1
    o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, "f32")
    assert np.abs(o[0, 0].double().cpu().numpy() - V[0, 0, :3].mean(0)).max() < 1e-5
    assert abs(float(lse[0, 0]) / 2.0 ** 37 - 1) < 1e-6


def test_any_slopes_and_far_distances(gpu):
    """Negative and zero slopes, distances in both directions."""
    torch, hgca = gpu
    d, L = 64, 900
    rng, q, K, V = inputs(6, "f32", [60], 4, 2, d, L)
    shape = hgca.Shape(hgca.F32, 1, 4, 2, d, 0.125)
    slopes = np.array([-0.01, 0.0, 0.5, 3.0], np.float32)
    tier = tier_of(gpu, rng, "f32", K, V, [L], 16)
    o, lse = call(gpu, shape, put(torch, q, "f32"), [0, 60], tier, "f32", causal=False, slopes=slopes)
    O, Ls = so.chunk(q, [0, 60], K, V, [L], 0.125, causal=False, slopes=slopes)
    check(o, lse, O, Ls, *bounds("f32", "f32", q, K, V, [L], 0.125, 0.0, slopes, L), "f32", "f32")


def test_row_counts_that_do_not_fit(gpu):
    """Beginnings that do not ascend or lie behind the rows give some result and touch nothing else."""
    torch, hgca = gpu
    rng, q, K, V = inputs(9, "bf16", [20, 20], 4, 2, 64, 300)
    shape = hgca.Shape(hgca.BF16, 2, 4, 2, 64, 0.125)
    tier = tier_of(gpu, rng, "bf16", K, V, [300, 300], 16)
    for cu in ([0, 30, 10], [5, 100000, 7], [-3, -1, 2 ** 30]):
        call(gpu, shape, put(torch, q, "bf16"), cu, tier, "bf16", pad=0)


def test_beyond_4_gib_of_a_tier(gpu):
    """Blocks whose rows lie beyond 4 GiB."""
    torch, hgca = gpu
    for dtype, dt in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        nb, Hkv, bs, d = (20000 if dtype == "bf16" else 10000), 8, 64, 128
        k, v = (torch.zeros(nb, Hkv, bs, d, dtype=dt, device=DEV) for _ in "kv")
        far = [nb - 1, nb - 7, 3, nb - 300]
        rng, q, K, V = inputs(3, dtype, [5], 16, Hkv, d, 256)
        for j, blk in enumerate(far):
            k[blk], v[blk] = put(torch, K[0, :, 64 * j:64 * j + 64], dtype), put(torch, V[0, :, 64 * j:64 * j + 64], dtype)
        tier = hgca.Tier(k, v, 256, i32(torch, [250]), i32(torch, [far]), bs)
        shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 1, 16, Hkv, d, 0.125)
        print(f"\n[case] far {dtype}", flush=True)
        o, lse = call(gpu, shape, put(torch, q, dtype), [0, 5], tier, "f32")
        O, Ls = so.chunk(q, [0, 5], K, V, [250], 0.125)
        check(o, lse, O, Ls, *bounds(dtype, "f32", q, K, V, [250], 0.125, T=256), "f32", dtype)
        del k, v, tier


def test_no_lengths_and_no_tokens(gpu):
    """A tier without lengths holds `cap` tokens of every sequence; one of capacity 0 holds none."""
    torch, hgca = gpu
    for dtype in ("bf16", "f32"):
        rng, q, K, V = inputs(12, dtype, [30, 2], 4, 2, 64, 77)
        shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 2, 4, 2, 64, 0.125)
        tier = hgca.Tier(put(torch, K, dtype), put(torch, V, dtype), 77)
        cu = [0, 30, 32]
        o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, "f32")
        O, L = so.chunk(q, cu, K, V, [77, 77], 0.125)
        check(o, lse, O, L, *bounds(dtype, "f32", q, K, V, [77, 77], 0.125, T=77), "f32", dtype)
        tier = hgca.Tier(put(torch, K[:, :, :0], dtype), put(torch, V[:, :, :0], dtype), 0)
        o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, "f32")
        assert (o == 0).all() and torch.isneginf(lse).all()


def test_captured_with_many_sequences(gpu):
    """More sequences than a wave has lanes (a launch of its own works out the shares), captured and replayed with other lengths, counts and rows."""
    torch, hgca = gpu
    B, Hq, Hkv, d, T = 70, 4, 2, 64, 900
    rng = np.random.default_rng(1)
    shape = hgca.Shape(hgca.BF16, B, Hq, Hkv, d, 0.125)
    K, V = (do.to_bf16(rng.standard_normal((B, Hkv, T, d))) for _ in "kv")
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    cu = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    tier = hgca.Tier(put(torch, K, "bf16"), put(torch, V, "bf16"), T, lens)
    q = torch.zeros(400, Hq, d, dtype=torch.bfloat16, device=DEV)
    outs = [(torch.zeros(400, Hq, d, device=DEV), torch.zeros(400, Hq, device=DEV), hgca.chunk_workspace(shape, 400, T, DEV)) for _ in range(2)]
    run = lambda i: hgca.chunk_attn(shape, q, cu, tier, *outs[i], window=500)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for turn in range(5):
        counts = np.minimum(rng.integers(0, 9, B), 400)
        counts[turn] = 30
        n = rng.integers(0, T + 1, B)
        Q = do.to_bf16(rng.standard_normal((400, Hq, d)))
        q.copy_(torch.from_numpy(Q))
        lens.copy_(i32(torch, n))
        cu.copy_(i32(torch, np.concatenate([[0], np.cumsum(counts)])))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            if turn == 0:
                run(0)
            else:
                if turn == 1:
                    with torch.cuda.graph(graph, stream=side):
                        run(0)
                graph.replay()
        torch.cuda.synchronize()
        run(1)
        torch.cuda.synchronize()
        at = int(counts.sum())
        assert torch.equal(outs[0][0][:at], outs[1][0][:at]) and torch.equal(outs[0][1][:at], outs[1][1][:at])
        O, L = so.chunk(Q[:at], cu.tolist(), K, V, n, 0.125, window=500)
        check(outs[0][0][:at], outs[0][1][:at], O, L, *bounds("bf16", "f32", Q[:at], K, V, n, 0.125, T=T), "f32")


@pytest.mark.parametrize("seed", range(40))
def test_calls_at_random(gpu, seed):
    """Types, heads, blocks, counts, lengths, masks and scores as they come; single tokens and whole prompts in one call, up to 100 sequences, tiers that are cut and
    that are not; in half of them values of V that are infinite or NaN, which are in the columns of the rows that see them and nowhere else."""
    torch, hgca = gpu
    rng = np.random.default_rng(seed)
    pick = lambda *x: x[int(rng.integers(len(x)))]
    dtype, d, Hkv, group, B = pick("f32", "bf16"), pick(64, 128), pick(1, 2, 8), pick(1, 4, 8), pick(1, 3, 9, 66, 100)
    out, block, Hq = "f32" if dtype == "f32" else pick("f32", "bf16"), pick(0, 16, 48, 128), Hkv * group
    T = pick(64, 300, 700, 1500) if B < 20 else pick(64, 200, 700)
    counts = [int(x) for x in rng.integers(0, pick(1, 4, 20, 150) + 1 if B < 20 else 5, B)]
    counts[0] = pick(1, 30, min(600, T, 16384 // Hq))
    lens = [min(T, max(int(x), c)) if rng.random() < 0.8 else int(x) for x, c in zip(rng.integers(0, T + 1, B), counts)]
    opt = dict(causal=rng.random() < 0.8)
    if rng.random() < 0.4:
        opt["window"] = pick(1, 17, 64, 300, 5000)
    if rng.random() < 0.4:
        opt["cap"] = pick(5.0, 30.0, 50.0)
    if rng.random() < 0.4:
        opt["slopes"] = slopes_of(Hq)
    if rng.random() < 0.4:
        opt["prefix_lens"] = rng.integers(0, T, B)
    if rng.random() < 0.4:
        opt["first"] = np.concatenate([np.sort(rng.integers(-3, L + 2, n)) for n, L in zip(counts, lens)])
    r, q, K, V = inputs(seed, dtype, counts, Hq, Hkv, d, T, pick(1.0, 3.0))
    clean = V.copy()
    odd = [(int(rng.integers(B)), int(rng.integers(Hkv)), int(rng.integers(T)), int(rng.integers(d)), pick(np.inf, -np.inf, np.nan)) for _ in range(5)] if seed % 2 else []
    for b, h, t, c, x in odd:
        V[b, h, t, c], clean[b, h, t, c] = x, 0
    print(f"\n[case] {dtype} {out} d={d} {Hq}/{Hkv} B={B} T={T} block={block} tokens={sum(counts)} {sorted(opt)} odd={len(odd)}", flush=True)
    scale = float(np.float32(d ** -0.5))
    cu = np.concatenate([[0], np.cumsum(counts)])
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, scale)
    o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier_of(gpu, r, dtype, K, V, lens, block), out, pad=3, wide=pick(0, d), **dict(opt))
    kw = dict(opt)
    prefix = kw.pop("prefix_lens", None)
    O, L = so.chunk(q, cu, K, clean, lens, scale, prefix=prefix, **kw)
    kinds = np.zeros(O.shape, int)
    for b, h, t, c, _ in odd:
        if t >= lens[b]:
            continue
        rows = slice(cu[b], cu[b + 1])
        seen = so.sees(counts[b], lens[b], opt["causal"], opt.get("window", 0), 0 if prefix is None else int(prefix[b]),
                       None if "first" not in opt else opt["first"][rows])[:, t]
        x = V[b, h, t, c]                        # (a place may have been drawn twice)
        kinds[rows, h * group:(h + 1) * group, c] |= np.where(seen, 1 if x == np.inf else 2 if x == -np.inf else 4, 0)[:, None]
    got = o.double().cpu().numpy()
    assert np.array_equal(got == np.inf, kinds == 1) and np.array_equal(got == -np.inf, kinds == 2) and np.array_equal(np.isnan(got), kinds > 2)
    o = torch.where(torch.from_numpy(kinds > 0).to(DEV), torch.zeros_like(o), o)
    check(o, lse, np.where(kinds > 0, 0, O), L, *bounds(dtype, out, q, K, clean, lens, scale, opt.get("cap", 0.0), opt.get("slopes"), T), out, dtype)
