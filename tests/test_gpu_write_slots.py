"""Rows of packed tokens entered by slot (hgca_kv_write) where the tier's slots are not whole blocks: every token whose slot is below n_slots is written, no
other.  (A block of a contiguous tier is a sequence's whole capacity.)"""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n_slots", [1, 40, 63, 64, 65, 100, 127, 128])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_any_number_of_slots(dtype, paged, n_slots):
    import torch
    from paper_2507_03153_amd import hgca
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    Hkv, d, bs = 2, 64, 16 if paged else 64
    k, v = (torch.full((128 // bs, Hkv, bs, d), 7.0, dtype=dt, device=DEV) for _ in "kv")
    rng = np.random.default_rng(n_slots)
    slots = torch.from_numpy(rng.permutation(128)[:120].astype(np.int32)).to(DEV)
    k_in, v_in = (torch.from_numpy(rng.standard_normal((120, Hkv, d)).astype(np.float32)).to(DEV).to(dt) for _ in "kv")
    table = torch.arange(8, dtype=torch.int32, device=DEV).reshape(2, 4)
    view = hgca.KvView(k.data_ptr(), v.data_ptr(), None, table.data_ptr() if paged else None, 64, 16 if paged else 0, 4 if paged else 0, None)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, 2, 4, Hkv, d, 0.1)
    torch.cuda.synchronize()
    rc = hgca.lib().hgca_kv_write(ctypes.byref(shape), ctypes.byref(view), n_slots, slots.data_ptr(), k_in.data_ptr(), 0, v_in.data_ptr(), 0, 120,
                                  torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == hgca.OK
    for tier, rows in ((k, k_in), (v, v_in)):
        want = torch.full_like(tier, 7.0)
        for t, s in enumerate(slots.tolist()):
            if s < n_slots:
                want[s // bs, :, s % bs] = rows[t]
        assert torch.equal(tier, want)
