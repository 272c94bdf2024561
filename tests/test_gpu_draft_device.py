"""Draft steps and commits with another GPU as the current one are refused: part of their calls would go to that one's stream."""
import pytest

from test_gpu_draft_checks import drafts, make
from test_gpu_tree import gpu, i32  # noqa: F401

pytestmark = pytest.mark.gpu


def test_another_current_device(gpu, monkeypatch):
    import numpy as np
    torch, hgca = gpu
    C = make(torch, False)
    q, k, v, _, mask, path = drafts(torch, np.random.default_rng(1), 3)
    with monkeypatch.context() as m:             # (there is one GPU here; nothing is launched)
        m.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="cuda:0, the current device is cuda:1"):
            C.draft_step(q, k, v, mask)
    C.draft_step(q, k, v, mask)
    torch.cuda.synchronize()
    assert C.win_lens.tolist() == [3, 3]
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="the current device is cuda:1"):
            C.commit(k, v, path, i32(torch, [1, 2]), beta=1.0)
    C.commit(k, v, path, i32(torch, [1, 2]), beta=1.0)
    torch.cuda.synchronize()
    assert C.win_lens.tolist() == [1, 2]
