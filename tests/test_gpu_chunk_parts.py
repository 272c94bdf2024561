"""The digits that the weights of packed chunks (hgca_chunk_attn) enter the second product with: 16 bits for bf16 O, 8 for callers that ask for
one part.

Tolerances.  Two bf16 parts leave 2^-9 * 2^-9 of a weight, sums as for fp32 O 2e-6 in the 2-norm: before its one rounding O is off by
e = 6e-6 of its root mean square at most.  It is then another bf16 number than the nearest to 64 bits where those e reach a border between two, which are 2^-8 |x|
apart or more: for a normal distribution a share of 2 * 256 e (1 + ln(1 / (512 e))) 0.8 = 1.7 %; 2 % are allowed, one step each.  With one part a
weight is off by at most 2^-9 of itself, so O by 2^-9 max |v| besides."""
import numpy as np
import pytest

import draft_oracle as do
import serve_oracle as so
from test_gpu_chunk import call, gpu, inputs, put, slopes_of, tier_of  # noqa: F401

pytestmark = pytest.mark.gpu
CASES = [
    # d, Hq, Hkv, block, counts, lens
    (128, 32, 8, 16, [300, 40], [900, 700]),     # whole units
    (64, 16, 2, 0, [200, 129], [200, 2100]),
    (128, 32, 4, 16, [1] * 24, [1500 + 7 * i for i in range(24)]),             # few rows, straight from memory
    (64, 8, 8, 48, [2] * 40, [77 + 31 * i for i in range(40)]),
    (128, 8, 1, 0, [5], [9000]),                 # shares
]
SCORES = [dict(), dict(cap=30.0), dict(slopes=True), dict(cap=5.0, slopes=True, window=300)]


def case(gpu, d, Hq, Hkv, block, counts, lens, opt, dtype="bf16"):  # noqa: F811
    torch, hgca = gpu
    rng, q, K, V = inputs(d + Hq + len(counts), dtype, counts, Hq, Hkv, d, max(lens), sharp=2.0)
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = slopes_of(Hq)
    scale = float(np.float32(d ** -0.5))
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, len(lens), Hq, Hkv, d, scale)
    cu = np.concatenate([[0], np.cumsum(counts)])
    tier = tier_of(gpu, rng, dtype, K, V, lens, block)
    run = lambda out, **more: call(gpu, shape, put(torch, q, dtype), cu, tier, out, **opt, **more)
    return run, lambda: so.chunk(q, cu, K, V, lens, scale, **opt), float(np.abs(V).max())


@pytest.mark.parametrize("opt", SCORES)
@pytest.mark.parametrize("d,Hq,Hkv,block,counts,lens", CASES)
def test_bf16_outputs_are_the_nearest(gpu, d, Hq, Hkv, block, counts, lens, opt):  # noqa: F811
    run, exact, vmax = case(gpu, d, Hq, Hkv, block, counts, lens, opt)
    (o, lse), (O, L) = run("bf16"), exact()
    o = o.float().cpu().numpy()
    nearest = do.to_bf16(O).reshape(o.shape)
    off = o != nearest
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(nearest), 1e-30))) - 7)
    print(f"\n[case] d={d} {Hq}/{Hkv} {len(counts)} x {counts[0]} {list(opt)}: {off.mean():.2%} are not the nearest, worst "
          f"{(np.abs(o - nearest) / step).max():.2f} steps", flush=True)
    assert off.mean() <= 0.02
    assert (np.abs(o - O) <= 1.01 * step / 2 + 2e-4 * vmax).all()


@pytest.mark.parametrize("opt", SCORES)
@pytest.mark.parametrize("d,Hq,Hkv,block,counts,lens", CASES)
def test_one_part(gpu, d, Hq, Hkv, block, counts, lens, opt):  # noqa: F811
    """As before its rounding, but for 2^-9 of each weight; lse has no part in it."""
    torch, _ = gpu
    run, exact, vmax = case(gpu, d, Hq, Hkv, block, counts, lens, opt)
    (o, lse), (o2, lse2), (O, L) = run("bf16", one_part_p=True), run("bf16"), exact()
    assert "cap" in opt or torch.equal(lse, lse2)
    assert not torch.equal(o, o2)
    err = np.abs(o.double().cpu().numpy() - O)
    assert (err <= 2.0 ** -8 * np.abs(O) + (2.0 ** -9 + 2e-4) * vmax).all()
    assert np.linalg.norm(err) <= 2.0 ** -8 * 2 ** 0.5 * np.linalg.norm(O)


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_one_part_is_for_bf16_outputs_of_bf16(gpu, dtype, out):  # noqa: F811
    torch, _ = gpu
    run, _, _ = case(gpu, 128, 8, 2, 16, [40, 1], [300, 100], dict(cap=30.0), dtype)
    for x, y in zip(run(out, one_part_p=True), run(out)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("one_part", [False, True])
@pytest.mark.parametrize("d,counts,lens", [(128, [150, 3], [400, 300]), (64, [90, 40], [90, 2000]), (128, [1, 2], [6000, 77])])
def test_infinities_and_nan_of_v(gpu, d, counts, lens, one_part):  # noqa: F811
    """A further part of a weight may be negative or 0: an infinity or NaN of V is in the columns of the rows that see it, and nowhere else."""
    torch, hgca = gpu
    rng, q, K, V = inputs(d + lens[0], "bf16", counts, 4, 2, d, max(lens))
    clean = V.copy()
    odd = [(b, h, int(rng.integers(n)), int(rng.integers(d)), x) for b, n in enumerate(lens) for h in range(2) for x in (np.inf, -np.inf, np.nan)]
    for b, h, t, c, x in odd:
        V[b, h, t, c], clean[b, h, t, c] = x, 0
    cu, scale = np.concatenate([[0], np.cumsum(counts)]), float(np.float32(d ** -0.5))
    shape = hgca.Shape(hgca.BF16, 2, 4, 2, d, scale)
    tier = tier_of(gpu, rng, "bf16", K, V, lens, 16)
    o, _ = call(gpu, shape, put(torch, q, "bf16"), cu, tier, "bf16", window=200, one_part_p=one_part)
    O, _ = so.chunk(q, cu, K, clean, lens, scale, window=200)
    kinds = np.zeros(O.shape, int)
    for b, h, t, c, _ in odd:
        rows, x = slice(cu[b], cu[b + 1]), V[b, h, t, c]
        seen = so.sees(counts[b], lens[b], True, 200)[:, t]
        kinds[rows, 2 * h:2 * h + 2, c] |= np.where(seen, 1 if x == np.inf else 2 if x == -np.inf else 4, 0)[:, None]
    got = o.double().cpu().numpy()
    assert np.array_equal(got == np.inf, kinds == 1) and np.array_equal(got == -np.inf, kinds == 2) and np.array_equal(np.isnan(got), kinds > 2)
    err = np.abs(np.where(kinds > 0, 0, got) - np.where(kinds > 0, 0, O))
    assert (err <= 2.0 ** -8 * np.abs(O) + ((2.0 ** -9 if one_part else 0) + 2e-4) * np.abs(clean).max()).all()
