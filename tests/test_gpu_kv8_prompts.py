"""Attention of whole prompts over an 8-bit tier, up to the most queries that a call takes, against 64 bits (tolerances of test_gpu_tree.py);
one query more is refused, and so are more blocks of rows than a grid has."""
import ctypes

import numpy as np
import pytest

import draft_oracle as do
from test_gpu_kv8 import tier8
from test_gpu_tree import DEV, bounds, check, gpu, put  # noqa: F401


def attention(q, K, V, lens, scale):
    """As do.rows_attention without masks, a head's queries at once."""
    B, n, Hq, d = q.shape
    G = Hq // K.shape[1]
    O, lse = np.zeros(q.shape), np.full((B, n, Hq), -np.inf)
    for b, L in enumerate(lens):
        for h in range(Hq if L else 0):
            s = scale * (q[b, :, h] @ K[b, h // G, :L].T)
            m = s.max(-1, keepdims=True)
            w = np.exp(s - m)
            O[b, :, h] = w @ V[b, h // G, :L] / w.sum(-1, keepdims=True)
            lse[b, :, h] = (m + np.log(w.sum(-1, keepdims=True)))[:, 0]
    return O, lse


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,Hq,Hkv,n,block,out,lens", [
    ("bf16", 128, 8, 2, 300, 0, "f32", [130, 1, 700]),
    ("bf16", 64, 2, 1, 4096, 16, "bf16", [97, 0]),
    ("bf16", 128, 4, 4, 129, 48, "f32", [2500, 33]),
    ("f32", 64, 4, 1, 1001, 0, "f32", [300, 129]),
    ("f32", 128, 2, 2, 77, 16, "f32", [1200]),
])
def test_against_64_bits(gpu, dtype, d, Hq, Hkv, n, block, out, lens):
    torch, hgca = gpu
    print(f"\n[case] kv8 q={dtype} d={d} {Hq}/{Hkv} n={n} block={block} out={out} lens={lens}", flush=True)
    B, T = len(lens), max(lens) + 5
    rng = np.random.default_rng(n)
    K, V, q = rng.standard_normal((B, Hkv, T, d)), rng.standard_normal((B, Hkv, T, d)), rng.standard_normal((B, n, Hq, d)).astype(np.float32)
    q = q if dtype == "f32" else do.to_bf16(q)
    tier, enc = tier8(gpu, rng, (K, V), lens, block)
    K, V = (do.decode(*e) for e in enc)
    scale = float(np.float32(d ** -0.5))
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, scale)
    o = torch.full(q.shape, float("nan"), dtype=torch.float32 if out == "f32" else torch.bfloat16, device=DEV)
    lse = torch.full((B, n, Hq), float("nan"), device=DEV)
    hgca.kv8_attn(shape, put(torch, q, dtype), tier, o, lse, hgca.kv8_workspace(shape, n, T, DEV))
    torch.cuda.synchronize()
    O, L = attention(q.astype(np.float64), K, V, lens, scale)
    check(o, lse, O, L, *bounds(q, K, V, lens, scale, T), out)


def test_refused():
    from paper_2507_03153_amd import build, hgca
    build.build(force=False)
    view, at = hgca.Kv8View(*[0x100000] * 4, None, None, 64, 0, 0, None), 0x100000
    call = lambda B, n, dtype=hgca.F32: hgca.lib().hgca_kv8_attn(ctypes.byref(hgca.Shape(dtype, B, 8, 1, 128, 0.1)), at, n, ctypes.byref(view), at, 0, at,
                                                                 at, 1 << 50, None)
    assert call(1, 4097) == call(1, 4097, hgca.BF16) == hgca.ERR_UNSUPPORTED
    assert call(65535, 4096) == call(65535, 4096, hgca.BF16) == hgca.ERR_UNSUPPORTED       # 2048 and 256 blocks of rows each
