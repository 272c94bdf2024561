"""8-bit tiers: the bytes that are written, equal to the definition's; what is read back, exact; attention over them against 64 bits
(tolerances as derived in test_gpu_tree.py: the values that the bytes stand for are exact, so nothing is added)."""
import numpy as np
import pytest

import draft_oracle as do
from test_gpu_tree import DEV, bounds, check, gpu, i32, put  # noqa: F401

pytestmark = pytest.mark.gpu


def tier8(gpu, rng, rows, lens, block=0, T=None):
    """(Kv8Tier, codes and scales of K and V in token order) for values of K, V rows [B,Hkv,T,d]."""
    torch, hgca = gpu
    K, V = rows
    B, T = K.shape[0], K.shape[2]
    enc = [do.encode(x) for x in (K, V)]
    first, table, out = rng.integers(0, 3, B), None, []
    for arr in (enc[0][0], enc[1][0], enc[0][1], enc[1][1]):
        if block:
            state = rng.bit_generator.state
            arr, table = do.paged(rng, arr, block, first)
            rng.bit_generator.state = state
        out.append(torch.from_numpy(arr).to(DEV))
    t = hgca.Kv8Tier(out[0], out[1], out[2], out[3], T, i32(torch, lens), i32(torch, table), block, i32(torch, first) if block else None)
    return t, enc


def values(rng, *shape):
    """Rows whose blocks of 32 have magnitudes of very different size."""
    x = rng.standard_normal(shape)
    return x * 2.0 ** rng.integers(-20, 20, (*shape[:-1], shape[-1] // 32)).repeat(32, -1)


@pytest.mark.parametrize("dtype,d,block,Hkv,n", [("bf16", 128, 0, 3, 5), ("bf16", 64, 16, 2, 33), ("f32", 128, 48, 2, 17),
                                                 ("f32", 64, 0, 1, 1), ("bf16", 128, 16, 8, 1)])
def test_written_bytes_and_rows_read_back(gpu, dtype, d, block, Hkv, n):
    torch, hgca = gpu
    B, T = 3, 60
    rng = np.random.default_rng(n + d)
    K, V = (np.zeros((B, Hkv, T, d)) for _ in range(2))
    tier, _ = tier8(gpu, rng, (K, V), [T] * B, block)
    for x in (tier.k, tier.v, tier.k_scale, tier.v_scale):
        x.fill_(0xa5)
    first = np.array([0, 7, T - n], np.int32)
    rows = [values(rng, B, n, Hkv, d) for _ in range(2)]
    rows = [x.astype(np.float32) if dtype == "f32" else do.to_bf16(x) for x in rows]
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, 2 * Hkv, Hkv, d, 1.0)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    hgca.kv8_write_tokens(shape, tier, i32(torch, first), put(torch, rows[0], dtype), put(torch, rows[1], dtype), status=status)
    ko, vo = (torch.full((B, n, Hkv, d), 5.0, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device=DEV) for _ in range(2))
    hgca.kv8_read(shape, tier, i32(torch, first), ko, vo)
    torch.cuda.synchronize()
    assert status.item() == 0
    where = np.zeros((B, T), bool)
    for b in range(B):
        where[b, first[b]:first[b] + n] = True

    def line(t):                                 # a tier's bytes in token order [B,T,Hkv,w]
        t = t.cpu().numpy()
        if not block:
            return t.transpose(0, 2, 1, 3)
        tab, f = tier.block_table.cpu().numpy(), tier.first_block.cpu().numpy()
        return np.stack([np.concatenate([t[tab[b, f[b] + j]] for j in range(-(-T // block))], 1)[:, :T].transpose(1, 0, 2) for b in range(B)])
    for x, codes, scales, back in ((rows[0], tier.k, tier.k_scale, ko), (rows[1], tier.v, tier.v_scale, vo)):
        c, s = do.encode(x)
        gc, gs = line(codes), line(scales)
        assert np.array_equal(gc[where], c.reshape(-1, Hkv, d)) and np.array_equal(gs[where], s.reshape(-1, Hkv, d // 32))
        assert (gc[~where] == 0xa5).all() and (gs[~where] == 0xa5).all()
        assert np.array_equal(back.double().cpu().numpy(), do.decode(c, s))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_kind_of_value(gpu, dtype):
    """All bf16 values, in blocks of neighbours and in blocks with a fixed largest value; ties, zeros of both signs, subnormals,
    the ends of the range, infinities and NaN."""
    torch, hgca = gpu
    bits = np.arange(65536, dtype=np.uint16)
    x = (bits.astype(np.uint32) << 16).view(np.float32)
    a = x.reshape(-1, 32)
    top = x.copy().reshape(-1, 32)
    with np.errstate(invalid="ignore", over="ignore"):
        top[:, 0] = np.where(np.abs(a[:, 1]) < 1e30, np.abs(a[:, 1]) * 300, 1.0)          # small against their block's largest
    rng = np.random.default_rng(4)
    ties = (rng.integers(0, 449 * 16, (512, 32)) / 16.0).astype(np.float32)               # halves of steps of every binade
    ties[:, 5] = 448
    rows = np.concatenate([a, top, ties, -ties, np.zeros((4, 32), np.float32), np.full((4, 32), np.nan, np.float32),
                           np.full((4, 32), -np.inf, np.float32)])
    if dtype == "f32":
        odd = (rng.integers(0, 1 << 32, (4096, 32), dtype=np.uint64).astype(np.uint32)).view(np.float32)
        near = np.float32(464) * (1 + np.float32(2 ** -23) * rng.integers(-2, 3, (64, 32))).astype(np.float32)
        rows = np.concatenate([rows, odd, near, near / 2 ** 12])
    rows = rows[: len(rows) // 4 * 4].reshape(1, -1, 1, 128)
    n = rows.shape[1]
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 1, 1, 1, 128, 1.0)
    z = lambda w: torch.zeros(1, 1, n, w, dtype=torch.uint8, device=DEV)
    tier = hgca.Kv8Tier(z(128), z(128), z(4), z(4), n)
    t = torch.from_numpy(rows.copy()).to(DEV)
    t = t if dtype == "f32" else (t.view(torch.int32) >> 16).to(torch.int16).view(torch.bfloat16)
    hgca.kv8_write_tokens(shape, tier, None, t, t)
    ko, vo = torch.empty_like(t), torch.empty_like(t)
    hgca.kv8_read(shape, tier, None, ko, vo)
    torch.cuda.synchronize()
    ref = t.float().cpu().numpy().astype(np.float64)
    with np.errstate(all="ignore"):
        c, s = do.encode(ref)
    gc, gs = tier.k.cpu().numpy().transpose(0, 2, 1, 3), tier.k_scale.cpu().numpy().transpose(0, 2, 1, 3)
    assert np.array_equal(gs, s)
    nan = ~np.isfinite(ref)
    assert np.array_equal(gc[~nan], c[~nan]) and ((gc[nan] & 0x7f) == 0x7f).all()
    assert torch.equal(tier.k, tier.v)
    back = ko.double().cpu().numpy()
    assert np.isnan(back[nan]).all() and np.array_equal(back[~nan], do.decode(c, s)[~nan])


def test_from_a_tier_and_what_does_not_fit(gpu):
    """Only tokens from `first` to the source's length, at most max_tokens; a full tier takes what it has room for."""
    torch, hgca = gpu
    B, Hkv, d, T = 4, 2, 64, 50
    rng = np.random.default_rng(8)
    K, V = (do.to_bf16(values(rng, B, Hkv, T, d)) for _ in range(2))
    lens, first = [50, 20, 5, 50], np.array([3, 4, 9, 41], np.int32)
    src = hgca.Tier(put(torch, K, "bf16"), put(torch, V, "bf16"), T, i32(torch, lens))
    shape = hgca.Shape(hgca.BF16, B, Hkv, Hkv, d, 1.0)
    z = lambda w: torch.full((B, Hkv, 45, w), 0xa5, dtype=torch.uint8, device=DEV)
    tier = hgca.Kv8Tier(z(d), z(d), z(d // 32), z(d // 32), 45)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    hgca.kv8_write_tier(shape, tier, i32(torch, first), src, 16, status=status)
    torch.cuda.synchronize()
    assert status.item() == hgca.CACHE_CONTEXT_FULL
    for x, codes, scales in ((K, tier.k, tier.k_scale), (V, tier.v, tier.v_scale)):
        c, s = do.encode(x)
        want_c, want_s = np.full((B, Hkv, 45, d), 0xa5, np.uint8), np.full((B, Hkv, 45, d // 32), 0xa5, np.uint8)
        for b in range(B):
            e = min(first[b] + 16, lens[b], 45)
            if e > first[b]:
                want_c[b, :, first[b]:e], want_s[b, :, first[b]:e] = c[b, :, first[b]:e], s[b, :, first[b]:e]
        assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    # rows beyond the length are left as they are when read back
    tier.seq_lens = i32(torch, [45, 20, 5, 43])
    ko, vo = (torch.full((B, 6, Hkv, d), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    hgca.kv8_read(shape, tier, i32(torch, [10, 17, 9, 41]), ko, vo)
    torch.cuda.synchronize()
    got = ko.float().cpu().numpy()
    c, s = do.encode(K)
    y = do.decode(c, s)
    for b, (f, e) in enumerate(((10, 16), (17, 20), (9, 9), (41, 43))):
        assert np.array_equal(got[b, :e - f], y[b, :, f:e].transpose(1, 0, 2)) and (got[b, e - f:] == 9.0).all()


CASES = [
    # dtype of q, d, Hq, Hkv, n, block, out, lens
    ("bf16", 128, 8, 2, 1, 0, "f32", [300, 1, 0, 129]),
    ("bf16", 128, 16, 2, 5, 16, "f32", [17, 640]),
    ("bf16", 128, 4, 4, 70, 48, "f32", [200, 33]),
    ("bf16", 128, 16, 2, 16, 16, "bf16", [515, 16]),
    ("bf16", 64, 8, 1, 1, 16, "f32", [1000, 31]),
    ("bf16", 128, 16, 2, 8, 16, "f32", [515, 33, 0, 1500]),
    ("bf16", 64, 8, 8, 50, 0, "bf16", [97, 1]),
    ("bf16", 64, 8, 4, 40, 0, "bf16", [97, 15]),
    ("f32", 128, 8, 2, 5, 0, "f32", [300, 1]),
    ("f32", 128, 8, 1, 9, 16, "bf16", [333, 47]),
    ("f32", 64, 4, 4, 1, 32, "f32", [260, 0]),
    ("f32", 64, 8, 1, 33, 0, "f32", [111, 128]),
]


@pytest.mark.parametrize("dtype,d,Hq,Hkv,n,block,out,lens", CASES)
def test_attention(gpu, dtype, d, Hq, Hkv, n, block, out, lens):
    torch, hgca = gpu
    print(f"\n[case] kv8 q={dtype} d={d} {Hq}/{Hkv} n={n} block={block} out={out} lens={lens}", flush=True)
    B, T = len(lens), max(lens) + 5
    rng = np.random.default_rng(n + Hq)
    K, V = rng.standard_normal((B, Hkv, T, d)), rng.standard_normal((B, Hkv, T, d))
    K *= 2.0 ** rng.integers(-2, 2, (1, 1, 1, d // 32)).repeat(32, -1)
    for b, L in enumerate(lens):
        K[b, :, L:], V[b, :, L:] = np.nan, np.nan
    q = rng.standard_normal((B, n, Hq, d)).astype(np.float32)
    q = q if dtype == "f32" else do.to_bf16(q)
    with np.errstate(all="ignore"):
        tier, enc = tier8(gpu, rng, (K, V), lens, block)
    Kq, Vq = (do.decode(*e) for e in enc)
    scale = float(np.float32(d ** -0.5))
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, scale)
    o = torch.full(q.shape, float("nan"), dtype=torch.float32 if out == "f32" else torch.bfloat16, device=DEV)
    lse = torch.full((B, n, Hq), float("nan"), device=DEV)
    ws = hgca.kv8_workspace(shape, n, T, DEV).fill_(0xff)
    hgca.kv8_attn(shape, put(torch, q, dtype), tier, o, lse, ws)
    torch.cuda.synchronize()
    O, L = do.rows_attention(q.astype(np.float64), Kq, Vq, lens, scale)
    check(o, lse, O, L, *bounds(q, Kq, Vq, lens, scale, T), out)


def test_fp32_queries_at_the_ends_of_the_range(gpu):
    """Queries of 1e30 over keys of 1e-30 and the other way round: the parts of a query lose nothing."""
    torch, hgca = gpu
    rng = np.random.default_rng(2)
    for amp in (1e30, 1e-25, 3.3e38):
        q = (rng.standard_normal((1, 3, 2, 64)).clip(-1, 1) * amp).astype(np.float32)
        K, V = rng.standard_normal((1, 1, 40, 64)) / amp, rng.standard_normal((1, 1, 40, 64))
        tier, enc = tier8(gpu, rng, (K, V), [40])
        Kq, Vq = (do.decode(*e) for e in enc)
        shape = hgca.Shape(hgca.F32, 1, 2, 1, 64, 1.0)
        o, lse = torch.empty(1, 3, 2, 64, device=DEV), torch.empty(1, 3, 2, device=DEV)
        hgca.kv8_attn(shape, put(torch, q, "f32"), tier, o, lse, hgca.kv8_workspace(shape, 3, 40, DEV))
        torch.cuda.synchronize()
        O, L = do.rows_attention(q.astype(np.float64), Kq, Vq, [40], 1.0)
        check(o, lse, O, L, *bounds(q.astype(np.float64), Kq, Vq, [40], 1.0, 40), "f32")


@pytest.mark.parametrize("T", [1, 129, 1217])
@pytest.mark.parametrize("dtype,d,n,Hq", [("bf16", 128, 1, 4), ("bf16", 64, 12, 2), ("bf16", 128, 20, 2), ("bf16", 64, 70, 2), ("f32", 64, 3, 2)])
def test_nan_scores_reach_the_result(gpu, dtype, d, n, Hq, T):
    """A query of NaN, and a key of NaN codes behind a whole number of steps: the rows concerned are NaN, the others as without."""
    torch, hgca = gpu
    rng = np.random.default_rng(8)
    K, V, q = rng.standard_normal((2, 1, T, d)), rng.standard_normal((2, 1, T, d)), rng.standard_normal((2, n, Hq, d))
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 2, Hq, 1, d, 0.1)

    def run(q, K):
        tier, _ = tier8(gpu, rng, (K, V), [T, T])
        o, lse = torch.empty(2, n, Hq, d, device=DEV), torch.empty(2, n, Hq, device=DEV)
        hgca.kv8_attn(shape, put(torch, q, dtype), tier, o, lse, hgca.kv8_workspace(shape, n, T, DEV))
        return o.cpu().numpy(), lse.cpu().numpy()
    good, lse0 = run(q, K)
    bad_q, bad_k = q.copy(), K.copy()
    bad_q[0, 0, 1], bad_k[1, 0, T - 1] = np.nan, np.nan
    with np.errstate(all="ignore"):
        o, lse = run(bad_q, bad_k)
    hit = np.zeros((2, n, Hq), bool)
    hit[0, 0, 1], hit[1] = True, True
    assert np.isfinite(good).all() and np.isnan(o[hit]).all() and np.isnan(lse[hit]).all()
    assert np.array_equal(o[~hit], good[~hit]) and np.array_equal(lse[~hit], lse0[~hit])


def test_captured_write_and_attention(gpu):
    """A token enters the tier and is attended to in one captured graph, replayed with new tokens and positions."""
    torch, hgca = gpu
    B, Hq, Hkv, d, T = 2, 8, 2, 128, 64
    shape = hgca.Shape(hgca.BF16, B, Hq, Hkv, d, 0.1)
    z = lambda w: torch.zeros(B, Hkv, T, w, dtype=torch.uint8, device=DEV)
    tier = hgca.Kv8Tier(z(d), z(d), z(d // 32), z(d // 32), T, torch.zeros(B, dtype=torch.int32, device=DEV))
    at = torch.zeros(B, dtype=torch.int32, device=DEV)
    k, v, q = (torch.empty(B, 1, h, d, dtype=torch.bfloat16, device=DEV) for h in (Hkv, Hkv, Hq))
    o, lse, ws = torch.empty(B, 1, Hq, d, device=DEV), torch.empty(B, 1, Hq, device=DEV), hgca.kv8_workspace(shape, 1, T, DEV)

    def step():
        hgca.kv8_write_tokens(shape, tier, at, k, v)
        tier.seq_lens.copy_(at + 1)
        hgca.kv8_attn(shape, q, tier, o, lse, ws)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rng = np.random.default_rng(6)
    ks, vs = [], []
    for i in range(5):
        new = [do.to_bf16(rng.standard_normal(t.shape)) for t in (k, v, q)]
        for t, x in zip((k, v, q), new):
            t.copy_(put(torch, x, "bf16"))
        at.fill_(i)
        o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        ks.append(new[0][:, 0]), vs.append(new[1][:, 0])
        Kq, Vq = (do.decode(*do.encode(np.stack(x, 2))) for x in (ks, vs))
        O, L = do.rows_attention(new[2].astype(np.float64), Kq, Vq, [i + 1] * B, float(np.float32(0.1)))
        check(o, lse, O, L, *bounds(new[2], Kq, Vq, [i + 1] * B, 0.1, T), "f32")
