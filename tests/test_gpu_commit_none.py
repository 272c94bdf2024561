"""Commits of nothing: no drafted tokens at all is no call, drafted tokens of which none is accepted give the lengths of before."""
import pytest

from test_gpu_tree import DEV, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def test_no_tokens_and_none_accepted(gpu):
    torch, hgca = gpu
    B, Hkv, d = 3, 2, 64
    shape = hgca.Shape(hgca.BF16, B, Hkv, Hkv, d, 1.0)
    k, v = (torch.randn(B, Hkv, 40, d, device=DEV).bfloat16() for _ in range(2))
    tier = hgca.Tier(k.clone(), v.clone(), 40)
    first = torch.tensor([0, 7, 40], dtype=torch.int32, device=DEV)
    lens = torch.full((B,), -5, dtype=torch.int32, device=DEV)
    new = lambda n: torch.randn(B, n, Hkv, d, device=DEV).bfloat16()
    hgca.kv_commit(shape, tier, first, new(0), new(0), lens)
    torch.cuda.synchronize()
    assert lens.tolist() == [-5] * B
    hgca.kv_commit(shape, tier, first, new(4), new(4), lens, cnt=torch.zeros(B, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert lens.tolist() == first.tolist()
    assert torch.equal(tier.k, k) and torch.equal(tier.v, v)
