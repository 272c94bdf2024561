"""Scores whose exponents have no digits left in fp32: the largest one takes all of the weight, whatever its size.

The inputs' largest score of every row stands more than 1e-3 of it above the row's next one, hundreds of times what 128 fp32 additions
can be off by (2^-16) and, from 1e9 on, a million units: in 64 bits the other weights are 0.  O is then a row of V, off by the few
roundings of 2^-24 of its weight's parts, their sum and the quotient: 2^-20 relative; lse is the score, off by what `bounds` allows."""
import numpy as np
import pytest

import draft_oracle as do
from test_gpu_kv8 import tier8
from test_gpu_tree import DEV, bounds, call, gpu, inputs, put, tier_of  # noqa: F401

pytestmark = pytest.mark.gpu

KINDS = [("bf16", 128, 4, 1), ("bf16", 64, 4, 7), ("bf16", 128, 4, 6), ("bf16", 64, 1, 40), ("bf16", 128, 8, 20), ("f32", 64, 4, 3), ("f32", 128, 4, 8)]


def spread(rng, q, K, size):
    """Queries of one size, keys along them with random lengths: scores of both signs up to `size` with gaps between them."""
    d = q.shape[-1]
    q[:] = np.sign(q[:, :1, :1])                 # all rows of a sequence ask in one direction
    T = K.shape[2]
    steps = np.stack([rng.permutation(np.linspace(-1.0, 1.0, T)) for _ in range(K.shape[0])])
    steps[:, int(rng.integers(0, T))] = 1.01     # (the next one is at 1)
    K[:] = q[:, 0, 0][:, None, None, :] * steps[:, None, :, None] * (size / d)
    return q, K


@pytest.mark.parametrize("size", [1e9, 3e10, 1e20, 1e37])
@pytest.mark.parametrize("T", [60, 3000])
@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("dtype,d,Hq,n", KINDS)
def test_the_largest_takes_all(gpu, dtype, d, Hq, n, kv8, T, size):
    torch, hgca = gpu
    print(f"\n[case] {dtype} d={d} Hq={Hq} n={n} kv8={kv8} T={T} size={size}", flush=True)
    rng, q, K, V = inputs(n + T, dtype, 2, n, Hq, 1, d, T)
    q, K = spread(rng, q, K, size)
    K = K.astype(np.float32) if dtype == "f32" and not kv8 else do.to_bf16(K)
    lens, shape = [T, T - 7], hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 2, Hq, 1, d, 1.0)
    if kv8:
        with np.errstate(all="ignore"):
            tier, enc = tier8(gpu, rng, (K, V), lens)
        K, V = (do.decode(*e) for e in enc)
        o, lse = torch.empty(2, n, Hq, d, device=DEV), torch.empty(2, n, Hq, device=DEV)
        hgca.kv8_attn(shape, put(torch, q, dtype), tier, o, lse, hgca.kv8_workspace(shape, n, T, DEV))
        m = None
    else:
        m = [do.ancestors(rng, n) for _ in range(2)]
        o, lse = call(gpu, shape, put(torch, q, dtype), tier_of(gpu, rng, dtype, K, V, lens, 0), torch.from_numpy(do.as_int64(m)).to(DEV), "f32")
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    q, K, V = (x.astype(np.float64) for x in (q, K, V))
    tol_l = bounds(q, K, V, lens, 1.0, T)[1]
    for b, L in enumerate(lens):
        sees = np.ones((n, L), bool)
        if m is not None:
            sees[:, L - n:] = [[m[b][i] >> j & 1 for j in range(n)] for i in range(n)]
        s = np.where(sees, (K[b, 0, :L] @ q[b, 0, 0])[None], -np.inf)
        for i in range(n):
            top = s[i].max()
            at = np.flatnonzero(s[i] >= top * (1 - 1e-3))              # rounded keys may be equal: their rows in equal parts
            if (s[i][at] < top).any():
                continue
            want = V[b, 0, at].mean(0)
            assert np.abs(o[b, i] - want).max() <= 2.0 ** -20 * np.abs(V[b, 0, at]).max(), (b, i)
            assert np.abs(lse[b, i] - (top + np.log(len(at)))).max() <= tol_l
