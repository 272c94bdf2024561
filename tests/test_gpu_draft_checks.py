"""A draft step that the host refuses has changed nothing: the drafts join the window only once all arguments are in order."""
import numpy as np
import pytest

import draft_oracle as do
from test_gpu_tree import DEV, gpu, i32, put  # noqa: F401

pytestmark = pytest.mark.gpu
B, Hq, Hkv, d, BS = 2, 4, 2, 64, 16


def make(torch, pool8, max_blocks=4):
    from paper_2507_03153_amd.cache import LayerCache
    return LayerCache(torch.bfloat16, B, Hq, Hkv, d, BS, 2, max_blocks, 16, 0.125, DEV, win_cap_blocks=4, pool8=pool8)


def drafts(torch, rng, n):
    q, k, v = (put(torch, rng.standard_normal((B, n, h, d)), "bf16") for h in (Hq, Hkv, Hkv))
    masks = [do.ancestors(rng, n) for _ in range(B)]
    return q, k, v, masks, torch.from_numpy(do.as_int64(masks)).to(DEV), i32(torch, np.tile(np.arange(n), (B, 1)))


def test_a_refused_call_leaves_the_window_alone(gpu):
    torch, hgca = gpu
    rng = np.random.default_rng(6)
    C = make(torch, False)
    q, k, v, _, mask, path = drafts(torch, rng, 3)
    C.draft_step(q, k, v, mask)
    C.commit(k, v, path, i32(torch, [3, 1]), beta=1.0)
    state = lambda: [x.clone() for x in (C.win_lens, C.pool_lens, C.k_blocks, C.v_blocks, C.draft_first)]
    torch.cuda.synchronize()
    before = state()
    for bad in (dict(q=q.float()), dict(q=q[..., :32]), dict(q=q[:, :, :2]), dict(mask=mask.int()), dict(mask=mask[:1]), dict(k=k[:, :2]),
                dict(v=v.float()), dict(k=k.transpose(1, 2)), dict(v=v.cpu())):
        with pytest.raises(ValueError):
            C.draft_step(bad.get("q", q), bad.get("k", k), bad.get("v", v), bad.get("mask", mask))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(state(), before))
    C.draft_step(q, k, v, mask)
    for cnt in (torch.tensor([1, 1], device=DEV), torch.ones(3, dtype=torch.int32, device=DEV)):
        with pytest.raises(ValueError, match="cnt"):
            C.commit(k, v, path, cnt, beta=1.0)
