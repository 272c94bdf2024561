"""Tiers whose rows lie beyond 4 GiB: drafted tokens committed, attended to, written in 8 bits and read back at the far end of the second
of two sequences.  All other rows are zeros, whose scores are 0 against scores near 40 of the last rows, so that the result is that of the
last rows (2^25 e^-40 of the sum is 1e-10).  Tolerances: a score of 43 from 128 fp32 additions is off by at most 128 * 2^-23 * 43 = 6.6e-4,
so is lse (2e-3 asked), and O by twice that of max |v| < 5 (1e-2 asked)."""
import numpy as np
import pytest

import draft_oracle as do
from test_gpu_tree import DEV, gpu, i32, put  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,n,Hq", [("bf16", 128, 3, 2), ("bf16", 128, 24, 4), ("f32", 128, 3, 2)])
def test_commit_and_attention(gpu, dtype, d, n, Hq):
    torch, hgca = gpu
    e = 4 if dtype == "f32" else 2
    cap = (1 << 32) // (d * e) + 64              # a sequence's rows are more than 4 GiB
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    k, v = (torch.zeros(2, 1, cap, d, dtype=td, device=DEV) for _ in range(2))
    rng = np.random.default_rng(d + n)
    rows = [rng.standard_normal((2, n, 1, d)).astype(np.float32) for _ in range(2)]
    q = np.tile(rows[0].mean(1, keepdims=True), (1, n, Hq, 1)) * 2
    rows[0] = np.sign(q[:, :1, :1].repeat(n, 1)) * (1 + np.abs(rows[0]) / 8)
    rows, q = [do.to_bf16(x) for x in rows], do.to_bf16(q)
    scale = float(np.float32(40 / np.einsum("bnd,bnd->bn", q[:, :, 0], rows[0][:, :, 0]).min()))
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 2, Hq, 1, d, scale)
    lens = torch.tensor([5, cap - n], dtype=torch.int32, device=DEV)
    tier = hgca.Tier(k, v, cap, lens)
    hgca.kv_commit(shape, tier, lens.clone(), put(torch, rows[0], dtype), put(torch, rows[1], dtype), lens)
    masks = [[(1 << n) - 1 if i % 2 else 1 << i for i in range(n)] for _ in range(2)]
    o, lse = torch.empty(2, n, Hq, d, device=DEV), torch.empty(2, n, Hq, device=DEV)
    hgca.tree_attn(shape, put(torch, q, dtype), tier, torch.from_numpy(do.as_int64(masks)).to(DEV), o, lse, hgca.tree_workspace(shape, n, cap, DEV))
    torch.cuda.synchronize()
    assert lens.tolist() == [5 + n, cap]
    back = k[1, 0, cap - n:].float().cpu().numpy(), v[1, 0, cap - n:].float().cpu().numpy()
    assert np.array_equal(back[0], rows[0][1, :, 0]) and np.array_equal(back[1], rows[1][1, :, 0])
    assert not k[0, 0, 5 + n:5 + n + 4096].any() and not v[1, 0, :4096].any()          # where offsets cut to 32 bits would lie
    K, V = (np.stack([x[b].swapaxes(0, 1) for b in range(2)]).astype(np.float64) for x in rows)
    O, L = do.rows_attention(q.astype(np.float64), K, V, [n, n], scale, masks)
    assert np.abs(V).max() < 5 and np.abs(o.double().cpu().numpy() - O).max() <= 1e-2 and np.abs(lse.double().cpu().numpy() - L).max() <= 2e-3


@pytest.mark.parametrize("n,Hq", [(3, 2), (24, 4)])
def test_8_bits(gpu, n, Hq):
    torch, hgca = gpu
    d, cap = 128, (1 << 25) + 64
    z = lambda w: torch.zeros(2, 1, cap, w, dtype=torch.uint8, device=DEV)
    lens = torch.tensor([n, cap], dtype=torch.int32, device=DEV)
    tier = hgca.Kv8Tier(z(d), z(d), z(d // 32), z(d // 32), cap, lens)
    rng = np.random.default_rng(n)
    rows = [rng.standard_normal((2, n, 1, d)) for _ in range(2)]
    q = np.tile(rows[0].mean(1, keepdims=True), (1, n, Hq, 1)) * 2
    rows[0] = np.sign(q[:, :1, :1].repeat(n, 1)) * (1 + np.abs(rows[0]) / 8)
    rows, q = [do.to_bf16(x) for x in rows], do.to_bf16(q)
    dec = [do.decode(*do.encode(x)) for x in rows]
    scale = float(np.float32(40 / np.einsum("bnd,bnd->bn", q[:, :, 0], dec[0][:, :, 0]).min()))
    shape = hgca.Shape(hgca.BF16, 2, Hq, 1, d, scale)
    first = lens - n
    hgca.kv8_write_tokens(shape, tier, first, put(torch, rows[0], "bf16"), put(torch, rows[1], "bf16"))
    ko, vo = (torch.empty(2, n, 1, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    hgca.kv8_read(shape, tier, first, ko, vo)
    o, lse = torch.empty(2, n, Hq, d, device=DEV), torch.empty(2, n, Hq, device=DEV)
    hgca.kv8_attn(shape, put(torch, q, "bf16"), tier, o, lse, hgca.kv8_workspace(shape, n, cap, DEV))
    torch.cuda.synchronize()
    assert np.array_equal(ko.double().cpu().numpy(), dec[0]) and np.array_equal(vo.double().cpu().numpy(), dec[1])
    assert not tier.k[0, 0, n:n + 4096].any() and not tier.k[1, 0, :4096].any() and not tier.v_scale[1, 0, :4096].any()
    K, V = (np.stack([x[b].swapaxes(0, 1) for b in range(2)]) for x in dec)
    O, L = do.rows_attention(q.astype(np.float64), K, V, [n, n], scale)
    assert np.abs(V).max() < 5 and np.abs(o.double().cpu().numpy() - O).max() <= 1e-2 and np.abs(lse.double().cpu().numpy() - L).max() <= 2e-3


def test_shares_of_a_hundred_million_tokens(gpu):
    """160 000 100 tokens are 500 shares of 2500 steps of 128 tokens and a step: the quotient is so close above 500 that fp32 does not tell.
    The rows that matter are in the last step."""
    torch, hgca = gpu
    d, n, Hq, L = 64, 1, 2, 500 * 2500 * 128 + 100
    z = lambda w: torch.zeros(2, 1, L, w, dtype=torch.uint8, device=DEV)
    lens = torch.tensor([L, 24106 * 128], dtype=torch.int32, device=DEV)
    tier = hgca.Kv8Tier(z(d), z(d), z(d // 32), z(d // 32), L, lens)
    rng = np.random.default_rng(1)
    k, v = np.ones((2, 1, 1, d)), do.to_bf16(rng.standard_normal((2, 1, 1, d)))
    shape = hgca.Shape(hgca.BF16, 2, Hq, 1, d, 40 / d)
    hgca.kv8_write_tokens(shape, tier, lens - 1, put(torch, k, "bf16"), put(torch, v, "bf16"))
    o, lse = torch.empty(2, n, Hq, d, device=DEV), torch.empty(2, n, Hq, device=DEV)
    hgca.kv8_attn(shape, put(torch, np.ones((2, n, Hq, d)), "bf16"), tier, o, lse, hgca.kv8_workspace(shape, n, L, DEV))
    torch.cuda.synchronize()
    V = do.decode(*do.encode(v))
    assert np.abs(o.double().cpu().numpy() - V).max() <= 1e-2 and np.abs(lse.cpu().numpy() - 40).max() <= 2e-3
