"""Infinities and NaN in V rows that queries see, anywhere in a tier: a column in which a query sees infinities of one sign is that
infinity, of both signs or a NaN it is NaN, whatever the rows weigh; the other columns and the other queries are as without them, bit
for bit.  (Weights enter a matrix product in parts, some of them negative or 0: an infinity times those is no sum.)"""
import numpy as np
import pytest

import draft_oracle as do
from test_gpu_kv8 import tier8
from test_gpu_tree import DEV, call, gpu, i32, inputs, put, tier_of  # noqa: F401

pytestmark = pytest.mark.gpu

KINDS = [                                        # dtype, d, Hq, n: 4 to 16 rows per KV head, 17 to 32, 33 to 64, more
    ("bf16", 128, 4, 1), ("bf16", 64, 2, 7), ("bf16", 128, 4, 6), ("bf16", 64, 4, 8), ("bf16", 128, 4, 12), ("bf16", 64, 1, 64), ("bf16", 128, 8, 20),
    ("f32", 64, 4, 3), ("f32", 128, 2, 5), ("f32", 128, 4, 8),
]


def expected(good, V, sees):
    """What O is by V's odd values alone: `good` where a query sees none in a column."""
    with np.errstate(invalid="ignore"):
        up, down, nan = ((V == np.inf), (V == -np.inf), np.isnan(V))
    want = good.copy()
    for i in range(good.shape[0]):
        u, m, x = (k[sees[i]].any(0) for k in (up, down, nan))
        x = x | (u & m)
        want[i][:, u], want[i][:, m] = np.inf, -np.inf
        want[i][:, x] = np.nan
    return want


@pytest.mark.parametrize("T,block", [(75, 0), (333, 16), (2100, 0), (9000, 48)])
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("dtype,d,Hq,n", KINDS)
def test_seen_at_any_place(gpu, dtype, d, Hq, n, masked, T, block):
    torch, hgca = gpu
    print(f"\n[case] {dtype} d={d} Hq={Hq} n={n} T={T} block={block} masked={masked}", flush=True)
    rng, q, K, V = inputs(T + n, dtype, 1, n, Hq, 1, d, T)
    m = [do.ancestors(rng, n)] if masked else None
    sent = None if m is None else torch.from_numpy(do.as_int64(m)).to(DEV)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 1, Hq, 1, d, float(np.float32(d ** -0.5)))
    tail = T - n
    bad = V.copy()
    # columns 0 .. : an infinity in the first token, the last before the drafts, the middle, any; both signs far apart; NaN; a draft
    bad[0, 0, 0, 0], bad[0, 0, tail - 1, 1], bad[0, 0, tail // 2, 2] = np.inf, -np.inf, np.inf
    bad[0, 0, rng.integers(0, tail, 3), 3] = -np.inf
    bad[0, 0, 1, 4], bad[0, 0, tail - 2, 4] = np.inf, -np.inf
    bad[0, 0, int(rng.integers(0, tail)), 5] = np.nan
    bad[0, 0, tail + n // 2, d - 1] = np.inf
    bad[0, 0, tail + n // 2, d - 2], bad[0, 0, tail // 3, d - 2] = -np.inf, np.inf
    state = rng.bit_generator.state
    good, lse0 = call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, K, V, [T], block), sent, "f32")
    rng.bit_generator.state = state
    o, lse = call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, K, bad, [T], block), sent, "f32")
    sees = np.ones((n, T), bool)
    if masked:
        sees[:, tail:] = [[m[0][i] >> j & 1 for j in range(n)] for i in range(n)]
    want = expected(good[0].cpu().numpy(), bad[0, 0], sees)
    assert np.array_equal(o[0].cpu().numpy(), want, equal_nan=True)
    assert torch.equal(lse, lse0)


@pytest.mark.parametrize("dtype,d,Hq,n", KINDS)
def test_whatever_the_row_weighs(gpu, dtype, d, Hq, n):
    """Two rows with infinities whose weights are 0 in fp32, in the first and in the last of several splits."""
    torch, hgca = gpu
    T = 3000
    rng, q, K, V = inputs(n, dtype, 1, n, Hq, 1, d, T)
    q = np.abs(q) + 0.5
    far = [0, T - n - 3]
    K[0, 0] = np.abs(K[0, 0])
    K[0, 0, far] = -np.abs(K[0, 0, far]) - 64.0  # scores hundreds below the others'
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 1, Hq, 1, d, 1.0)
    bad = V.copy()
    bad[0, 0, far[0], 0], bad[0, 0, far[1], 1], bad[0, 0, far, 2] = np.inf, -np.inf, np.inf
    good, lse0 = call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, K, V, [T], 0), None, "f32")
    o, lse = call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, K, bad, [T], 0), None, "f32")
    want = expected(good[0].cpu().numpy(), bad[0, 0], np.ones((n, T), bool))
    assert np.array_equal(o[0].cpu().numpy(), want, equal_nan=True) and torch.equal(lse, lse0)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n", [4, 40])
def test_a_batch_of_which_one_sequence_has_them(gpu, dtype, out, n):
    """bf16 results too; the other sequences, empty ones among them, and the other KV heads are as without; a NaN score is still NaN."""
    torch, hgca = gpu
    B, Hq, Hkv, d, T = 4, 4, 2, 64, 700
    lens = [700, n, 0, 650]
    rng, q, K, V = inputs(3, dtype, B, n, Hq, Hkv, d, T)
    m = [do.ancestors(rng, n) for _ in range(B)]
    sent = torch.from_numpy(do.as_int64(m)).to(DEV)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, 0.125)
    bad = V.copy()
    bad[0, 1, 5, 3], bad[0, 1, 600, 4] = np.inf, np.nan
    bad_q = q.copy()
    bad_q[0, 0, Hq - 1] = np.nan
    run = lambda q, V: call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, K, V, lens, 0), sent, out)
    good, lse0 = run(q, V)
    o, lse = run(bad_q, bad)
    good, o, lse, lse0 = (x.float().cpu().numpy() for x in (good, o, lse, lse0))
    want, want_l = good.copy(), lse0.copy()
    want[0, :, 2:, 3], want[0, :, 2:, 4] = np.inf, np.nan
    want[0, 0, Hq - 1], want_l[0, 0, Hq - 1] = np.nan, np.nan
    assert np.array_equal(o, want, equal_nan=True) and np.array_equal(lse, want_l, equal_nan=True)


@pytest.mark.parametrize("d,Hq,n", [(128, 4, 1), (64, 4, 6), (64, 1, 64), (128, 8, 20)])
def test_nan_codes_of_an_8_bit_tier(gpu, d, Hq, n):
    torch, hgca = gpu
    T = 2100
    rng = np.random.default_rng(n)
    q, K, V = do.to_bf16(rng.standard_normal((1, n, Hq, d))), rng.standard_normal((1, 1, T, d)), rng.standard_normal((1, 1, T, d))
    V[0, 0, 7, 3] = V[0, 0, T - 1, 4] = 0.125    # (so that blocks keep their scales)
    bad = V.copy()
    bad[0, 0, 7, 3], bad[0, 0, T - 1, 4] = np.inf, np.nan
    shape, outs = hgca.Shape(hgca.BF16, 1, Hq, 1, d, 0.1), []
    for x in (V, bad):
        with np.errstate(all="ignore"):
            tier, _ = tier8(gpu, rng, (K, x), [T])
        o, lse = torch.empty(1, n, Hq, d, device=DEV), torch.empty(1, n, Hq, device=DEV)
        hgca.kv8_attn(shape, put(torch, q, "bf16"), tier, o, lse, hgca.kv8_workspace(shape, n, T, DEV))
        outs.append((o[0].cpu().numpy(), lse.cpu().numpy()))
    want = outs[0][0].copy()
    want[..., 3] = want[..., 4] = np.nan
    assert np.array_equal(outs[1][0], want, equal_nan=True) and np.array_equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("dtype,d,Hq,n", [("bf16", 128, 4, 3), ("bf16", 128, 4, 6), ("bf16", 64, 4, 12), ("bf16", 64, 8, 20), ("f32", 64, 4, 3)])
def test_behind_the_first_table_of_block_rows(gpu, dtype, d, Hq, n):
    """A sequence that is one workgroup's work and longer than two tables (8192 tokens each), among 299 short ones: values in each of its
    three passes, the drafts in the last."""
    torch, hgca = gpu
    B, T, bs, at = 300, 17000, 16, 211
    rng = np.random.default_rng(n)
    lens = rng.integers(1, 40, B).astype(np.int32)
    lens[at] = T - 5
    n_blk = [-(-int(x) // bs) for x in lens]
    table, perm, start = np.zeros((B, -(-T // bs)), np.int32), rng.permutation(sum(n_blk)).astype(np.int32), 0
    for b, x in enumerate(n_blk):
        table[b, :x] = perm[start:start + x]
        start += x
    r = (lambda *s: rng.standard_normal(s).astype(np.float32)) if dtype == "f32" else (lambda *s: do.to_bf16(rng.standard_normal(s)))
    kb, vb, q = r(len(perm), 1, bs, d), r(len(perm), 1, bs, d), r(B, n, Hq, d)
    m = [do.ancestors(rng, n) for _ in range(B)]
    bad, L = vb.copy(), T - 5
    put_at = lambda tok, col, x: bad.__setitem__((table[at, tok // bs], 0, tok % bs, col), x)
    for tok, col, x in ((3, 0, np.inf), (8191, 1, -np.inf), (8192, 2, np.inf), (9000, 3, np.nan), (16384, 4, np.inf), (L - n - 1, 5, -np.inf),
                        (2, 6, np.inf), (12000, 6, -np.inf), (L - n, 7, np.inf), (L - 1, 8, -np.inf)):
        put_at(tok, col, x)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, 1, d, 0.125)
    sent, outs = torch.from_numpy(do.as_int64(m)).to(DEV), []
    for v in (vb, bad):
        tier = hgca.Tier(put(torch, kb, dtype), put(torch, v, dtype), T, i32(torch, lens), i32(torch, table), bs)
        outs.append([x.cpu().numpy() for x in call(gpu, shape, put(torch, q, dtype), tier, sent, "f32")])
    (good, lse0), (o, lse) = outs
    V = np.concatenate([bad[i, 0] for i in table[at, :n_blk[at]]])[:L]
    sees = np.ones((n, L), bool)
    sees[:, L - n:] = [[m[at][i] >> j & 1 for j in range(n)] for i in range(n)]
    want = good.copy()
    want[at] = expected(good[at], V, sees)
    assert np.isfinite(good).all() and np.array_equal(o, want, equal_nan=True) and np.array_equal(lse, lse0)
