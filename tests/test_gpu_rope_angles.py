"""Sines and cosines of the rotation are as exact as fp32 holds them: the fraction of a turn is not rounded before they are formed.

A pair (1, 0) without a norm becomes (cos t, sin t).  Held here, in [1/2, 1), where a unit in the last place is 2^-24: a function
good to one unit and one rounding behind it are off by at most 1.5 units; two roundings, each evenly spread over half a unit to either
side, have a root of the mean square of sqrt(2 / 3) of 2^-25, and 2^-25 is asked for.  (An angle in (-pi, pi] rounded to fp32 alone is
off by up to pi / 4 units more, and by more than that in what it does to a sine near 0.)"""
import numpy as np
import pytest

from test_gpu_tree import DEV, gpu, i32  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_cosines_and_sines(gpu, d):
    torch, hgca = gpu
    n = 4096
    rng = np.random.default_rng(d)
    freq = (1e4 ** (-np.arange(d // 2) * 2.0 / d)).astype(np.float32)
    pos = rng.integers(-(1 << 20), 1 << 20, (1, n)).astype(np.int32)
    q = torch.zeros(1, n, 1, d, device=DEV)
    q[..., :d // 2] = 1.0
    o, ko = torch.empty_like(q), torch.empty_like(q)
    hgca.qk_norm_rope(hgca.Shape(hgca.F32, 1, 1, 1, d, 1.0), q, q.clone(), o, ko, torch.from_numpy(freq).to(DEV), positions=i32(torch, pos))
    torch.cuda.synchronize()
    t = pos[0].astype(np.longdouble)[:, None] * freq.astype(np.longdouble)
    want = np.concatenate([np.cos(t), np.sin(t)], -1)
    err = (o[0, :, 0].cpu().numpy().astype(np.longdouble) - want).astype(np.float64)
    print(f"\n    d={d}: worst {np.abs(err).max() * 2 ** 24:.3f} of 2^-24, root of mean square {np.sqrt((err ** 2).mean()) * 2 ** 25:.3f} of 2^-25", flush=True)
    assert torch.equal(o, ko)
    assert np.abs(err).max() <= 1.5 * 2.0 ** -24 and np.sqrt((err ** 2).mean()) <= 2.0 ** -25
