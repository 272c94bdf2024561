"""Capped scores of packed chunks (hgca_chunk_attn) with caps of every size, against 64 bits.

Tolerances.  What a cap adds is relative to the capped score, not to the cap.  |s| up to 0.7 cap: the fit (2.7e-8), the rounding of the
factors, of the polynomial's last step and of the product, 4 * 2^-24 in all.  Beyond, 1 - 2 / (1 + e^2x): the exponential's argument and result, sum and
quotient make 1.4 * 2^-23 of 1 at x = 0.7 (less behind it), 4.5 * 2^-24 of tanh x; roundings of x, of the difference and of the factor as much again: 9 * 2^-24.  The 2-norm
of an fp32 output sees them as what they are, of either sign: half of that and 2e-6 as without a cap."""
import numpy as np
import pytest

import serve_oracle as so
from test_gpu_chunk import bounds, call, gpu, inputs, put, tier_of  # noqa: F401

pytestmark = pytest.mark.gpu
# cap, sm_scale * sqrt(d), factor of q (a power of two)
CAPS = [(20.0, 1, 1.0), (30.0, 1, 4.0), (30.0, 1, 16.0), (5.0, 1, 4.0), (250.0, 1, 2.0), (270.0, 1, 2.0), (890.0, 1, 2.0), (1e3, 1, 1.0), (1e4, 1, 2.0), (1e5, 1, 1.0), (1e6, 1, 1.0),
        (1e9, 1, 2.0), (1e20, 1, 1.0), (2e38, 1, 1.0), (79.0, 2.0 ** -4, 16.0), (1e5, 2.0 ** -10, 1024.0),
        # scores within tiny caps, and far beyond them
        (2.2e-5, 1, 2.0 ** -18), (1.7e-5, 1, 2.0 ** -19), (1e-5, 1, 2.0 ** -20), (1e-8, 1, 2.0 ** -30), (1e-5, 1, 1.0),
        # a large or small sm_scale, and with it a cap far from 1 for the products
        (5.0, 2.0 ** 20, 2.0 ** -20), (1e4, 2.0 ** 20, 2.0 ** -20), (1e9, 2.0 ** 40, 2.0 ** -40), (40.0, 2.0 ** 60, 2.0 ** -60), (30.0, 2.0 ** -60, 2.0 ** 60)]
# dtype, out, d, counts, lens: few rows straight from memory, 17 to 32 of them, whole units
SHAPES = [("bf16", "bf16", 128, [3, 60], [150, 260]), ("bf16", "f32", 128, [60, 1], [130, 700]), ("bf16", "f32", 64, [2, 5], [100, 333]),
          ("f32", "f32", 64, [2, 8, 40], [70, 300, 120]), ("f32", "f32", 128, [1, 6, 50], [500, 90, 64])]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype,out,d,counts,lens", SHAPES)
@pytest.mark.parametrize("cap,times,sharp", CAPS)
def test_caps_of_every_size(gpu, cap, times, sharp, dtype, out, d, counts, lens, bias):  # noqa: F811
    torch, hgca = gpu
    Hq, Hkv, B = 8, 2, len(lens)
    rng, q, K, V = inputs(d + len(counts), dtype, counts, Hq, Hkv, d, max(lens))
    q *= np.float32(sharp)
    scale, cap = float(np.float32(times / np.sqrt(d))), float(np.float32(cap))
    slopes = (2.0 ** -np.arange(1, Hq + 1)).astype(np.float32) if bias else None
    cu = np.concatenate([[0], np.cumsum(counts)])
    tier = tier_of(gpu, rng, dtype, K, V, lens, 16)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, scale)
    o, lse = call(gpu, shape, put(torch, q, dtype), cu, tier, out, cap=cap, slopes=slopes)
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    O, L = so.chunk(q, cu, K, V, lens, scale, cap=cap, slopes=slopes)
    s = max(np.abs(np.einsum("nhd,htd->nht", q[cu[b]:cu[b + 1]].astype(np.float64), np.repeat(K[b, :, :n], Hq // Hkv, 0).astype(np.float64))).max()
            for b, n in enumerate(lens)) * scale
    S = cap * np.tanh(s / cap)
    more = S * (4 if s < 0.69 * cap else 9) * 2.0 ** -24
    tol_o, tol_l, biased = bounds(dtype, out, q, K, V, lens, scale, 0.0, slopes, max(lens))      # (a cap enlarges no error of its argument)
    vmax = float(np.abs(V).max())
    err, err_l, rel = np.abs(o - O), np.abs(lse - L), np.linalg.norm(o - O) / np.linalg.norm(O)
    print(f"\n[case] {dtype}->{out} d={d} cap={cap:g} scale={scale:.3g} |s|={s:.3g} bias={bias}: max|dO|={err.max():.2e} (of {tol_o + 2 * more * vmax:.2e}) "
          f"rel={rel:.2e} (of {2e-6 + more / 2 + 2 * biased:.2e}) max|dlse|={err_l.max():.2e} (of {tol_l + more:.2e})", flush=True)
    assert np.isfinite(o).all() and np.isfinite(lse).all()
    assert (err <= tol_o + 2 * more * vmax + (2.0 ** -8 * np.abs(O) if out == "bf16" else 0)).all()
    assert err_l.max() <= tol_l + more
    assert rel <= (2e-6 + more / 2 + 2 * biased if out == "f32" else 2.0 ** -8 * 2 ** 0.5)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("cap", [30.0, 1e4])
def test_scores_that_are_not_seen_change_no_bit(gpu, dtype, out, cap):  # noqa: F811
    """Scores far beyond the cap that only later rows see: the earlier rows of the same waves are what they are without them."""
    torch, hgca = gpu
    d, counts, lens = 128, [50, 3], [90, 40]
    rng, q, K, V = inputs(7, dtype, counts, 4, 2, d, 90)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 2, 4, 2, d, float(np.float32(d ** -0.5)))
    got = []
    for factor in (1, 2.0 ** 14):
        K[0, :, 70:] *= np.float32(factor)       # seen from row 30 on
        K[1, :, 39:] *= np.float32(factor)       # from row 2 on
        tier = tier_of(gpu, np.random.default_rng(1), dtype, K, V, lens, 16)
        got.append(call(gpu, shape, put(torch, q, dtype), [0, 50, 53], tier, out, cap=cap))
    for x, y in zip(*got):
        for r0, r1 in ((0, 30), (50, 52)):
            assert torch.equal(x[r0:r1], y[r0:r1])
        assert not torch.equal(x[30:50], y[30:50])
