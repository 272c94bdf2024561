"""Queries and keys normed per head and rotated, against 64 bits (angles in 80).

Tolerance: the norm's sum of d squares, reciprocal root and two products are at most 24 roundings of 2^-24, sine and cosine 2^-23 of
their own plus the angle's conversion to a fraction of a turn (2 pi * 2^-25) and, for positions up to 2^31, its product in fp64
(2 pi * 2^-23 at the very most); the two products and their sum 3 more: 64 * 2^-24 of |a| + |b|.  bf16 adds half a step."""
import numpy as np
import pytest

import draft_oracle as do
from test_gpu_tree import DEV, gpu, i32, put  # noqa: F401

pytestmark = pytest.mark.gpu


def freqs(rot, base=1e4):
    return (base ** (-np.arange(rot // 2) * 2.0 / rot)).astype(np.float32)


def run(gpu, dtype, B, n, Hq, Hkv, d, rot, interleaved, weights, how, pos=None, first=None, seed=0, amp=1.0):
    torch, hgca = gpu
    print(f"\n[case] {dtype} B={B} n={n} {Hq}/{Hkv} d={d} rot={rot} interleaved={interleaved} weights={weights} {how}", flush=True)
    rng = np.random.default_rng(seed)
    r = (lambda *s: (amp * rng.standard_normal(s)).astype(np.float32)) if dtype == "f32" else (lambda *s: do.to_bf16(amp * rng.standard_normal(s)))
    q, k = r(B, n, Hq, d), r(B, n, Hkv, d)
    qw, kw = (do.to_bf16(1 + rng.standard_normal(d) * 0.3) if w else None for w in weights)
    freq, td = freqs(rot), torch.float32 if dtype == "f32" else torch.bfloat16
    if how == "fused":                           # parts of wider rows
        wide = torch.full((B, n, (Hq + 2 * Hkv) * d), float("nan"), dtype=td, device=DEV)
        qd, kd = wide[..., :Hq * d].unflatten(-1, (Hq, d)), wide[..., Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d))
        qd.copy_(put(torch, q, dtype)), kd.copy_(put(torch, k, dtype))
    else:
        qd, kd = put(torch, q, dtype), put(torch, k, dtype)
    qo, ko = (qd, kd) if how == "in place" else (torch.full((B, n, h, d), float("nan"), dtype=td, device=DEV) for h in (Hq, Hkv))
    g = lambda w: None if w is None else put(torch, w, dtype)
    hgca.qk_norm_rope(hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, 1.0), qd, kd, qo, ko,
                      torch.from_numpy(freq).to(DEV), q_weight=g(qw), k_weight=g(kw), eps=1e-5, positions=i32(torch, pos),
                      first_pos=i32(torch, first), interleaved=interleaved)
    torch.cuda.synchronize()
    p = pos if pos is not None else (np.zeros(B, np.int64) if first is None else np.asarray(first, np.int64))[:, None] + np.arange(n)
    for name, x, w, got in (("q", q, qw, qo), ("k", k, kw, ko)):
        want = do.norm_rope(x, w, 1e-5, np.asarray(p), freq, interleaved)
        size = np.abs(do.norm_rope(x, w, 1e-5, np.zeros((B, n)), freq, interleaved))
        half = rot // 2
        j = np.arange(half)
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        size[..., a] = size[..., b] = size[..., a] + size[..., b]
        err = np.abs(got.double().cpu().numpy() - want)
        tol = 64 * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0) + 1e-30
        print(f"    {name}: worst {np.max(err / tol):.3f} of the tolerance", flush=True)
        assert (err <= tol).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,B,n,Hq,Hkv,d,rot,weights,how", [
    ("bf16", 2, 3, 8, 2, 128, 128, (1, 1), "fused"),
    ("bf16", 1, 1, 32, 8, 128, 128, (1, 1), "dense"),
    ("bf16", 3, 5, 4, 4, 64, 64, (0, 1), "in place"),
    ("bf16", 2, 700, 4, 1, 64, 32, (1, 1), "dense"),
    ("bf16", 2, 2, 40, 40, 128, 64, (1, 0), "fused"),
    ("f32", 2, 3, 8, 2, 128, 128, (1, 1), "fused"),
    ("f32", 1, 7, 4, 4, 64, 64, (0, 0), "in place"),
    ("f32", 1, 1100, 5, 5, 64, 16, (1, 1), "dense"),
    ("f32", 4, 1, 3, 1, 128, 112, (1, 0), "dense"),
])
def test_against_64_bits(gpu, dtype, B, n, Hq, Hkv, d, rot, weights, how, interleaved):
    rng = np.random.default_rng(n)
    pos = rng.integers(0, 5000, (B, n)).astype(np.int32)
    Hkv_ok = Hq // Hkv in (1, 2, 4, 8)
    if not Hkv_ok:
        Hq = 4 * Hkv
    run(gpu, dtype, B, n, Hq, Hkv, d, rot, interleaved, weights, how, pos=pos, seed=n)


def test_far_and_negative_positions(gpu):
    pos = np.array([[0, 1, 1 << 20, (1 << 31) - 1, -1, -(1 << 31), 999983, 16777217]], np.int32)
    run(gpu, "f32", 1, 8, 2, 1, 128, 128, False, (1, 1), "dense", pos=pos)
    run(gpu, "f32", 1, 8, 2, 1, 64, 64, True, (0, 0), "dense", pos=pos)


def test_positions_from_the_first(gpu):
    run(gpu, "f32", 3, 6, 4, 2, 64, 64, False, (1, 1), "dense", first=np.array([0, 1000003, 2147483645], np.int32))
    run(gpu, "bf16", 2, 4, 4, 2, 128, 128, True, (1, 1), "dense")


def test_tiny_and_large_values(gpu):
    """eps carries a row of almost nothing, and squares of 1e15 still have a sum."""
    for amp in (1e-12, 1e15):
        run(gpu, "f32", 1, 2, 2, 2, 128, 128, False, (1, 1), "dense", first=np.array([7], np.int32), amp=amp)


def test_captured_in_place(gpu):
    torch, hgca = gpu
    B, n, Hq, Hkv, d = 2, 2, 8, 2, 128
    shape = hgca.Shape(hgca.BF16, B, Hq, Hkv, d, 1.0)
    q, k = torch.randn(B, n, Hq, d, device=DEV).bfloat16(), torch.randn(B, n, Hkv, d, device=DEV).bfloat16()
    f, first = torch.from_numpy(freqs(d)).to(DEV), torch.tensor([5, 9], dtype=torch.int32, device=DEV)
    a, b = torch.empty_like(q), torch.empty_like(k)
    qo, ko = torch.empty_like(q), torch.empty_like(k)

    def step():
        a.copy_(q), b.copy_(k)
        hgca.qk_norm_rope(shape, a, b, a, b, f, first_pos=first)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        first.add_(i)
        graph.replay()
        hgca.qk_norm_rope(shape, q, k, qo, ko, f, first_pos=first)
        torch.cuda.synchronize()
        assert torch.equal(a, qo) and torch.equal(b, ko)
