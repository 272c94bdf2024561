"""Beginnings of sequences that do not ascend, repeat or lie behind the rows (hgca_chunk_attn): some result, and nothing else is touched: not what lies
around o, lse and the workspace, and no row that is in no sequence."""
import numpy as np
import pytest

from test_gpu_chunk import gpu, i32  # noqa: F401

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def guarded(torch, shape, dtype, fill, pad=4096):
    """A tensor in the middle of a larger one, and a check of what lies around it."""
    n = int(np.prod(shape))
    big = torch.full((n + 2 * pad,), fill, dtype=dtype, device=DEV)
    return big[pad:pad + n].view(*shape), lambda: bool((big[:pad] == fill).all() and (big[pad + n:] == fill).all())


def check(gpu, cu, T, length, Hq, Hkv, d, out="bf16", dtype="bf16", **opt):  # noqa: F811
    """A paged tier in which all sequences have the same blocks."""
    torch, hgca = gpu
    B, bs = len(cu) - 1, 16
    blocks = (length + bs - 1) // bs
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(B)
    k, v, q = (torch.randn(*s, dtype=dt, device=DEV, generator=g) for s in ((blocks, Hkv, bs, d), (blocks, Hkv, bs, d), (T, Hq, d)))
    table = torch.arange(blocks, dtype=torch.int32, device=DEV).repeat(B, 1)
    tier = hgca.Tier(k, v, blocks * bs, torch.full((B,), length, dtype=torch.int32, device=DEV), table, bs)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hq, Hkv, d, 0.125)
    size = hgca.chunk_workspace(shape, T, tier.cap, DEV).numel()
    o, o_ok = guarded(torch, (T, Hq, d), torch.bfloat16 if out == "bf16" else torch.float32, 77.0)
    lse, lse_ok = guarded(torch, (T, Hq), torch.float32, 55.0)
    ws, ws_ok = guarded(torch, (size,), torch.uint8, 0xff)
    print(f"\n[case] B={B} T={T} length={length} {Hq}/{Hkv} d={d} {dtype}->{out} {opt}", flush=True)
    torch.cuda.synchronize()
    hgca.chunk_attn(shape, q, i32(torch, cu), tier, o, lse, ws, **opt)
    torch.cuda.synchronize()
    assert o_ok() and lse_ok() and ws_ok()
    used = np.zeros(T + 1, np.int64)             # sequences of a row, as differences
    n0 = np.clip(cu[:-1], 0, T)
    n1 = np.clip(np.maximum(cu[1:], n0), 0, T)
    np.add.at(used, n0, 1)
    np.add.at(used, n1, -1)
    free = torch.from_numpy(np.cumsum(used)[:T] == 0).to(DEV)
    assert (o[free] == 77).all() and (lse[free] == 55).all()
    return o, lse, free


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("length", [300, 5000])
@pytest.mark.parametrize("cu", [[0, 30, 10], [5, 100000, 7], [-3, -1, 2 ** 30], [40, 40, 40], [60, 20, 0], [-2 ** 31, 2 ** 31 - 1, -2 ** 31]])
def test_two_sequences(gpu, cu, length, dtype, out):  # noqa: F811
    check(gpu, np.array(cu), 40, length, 4, 2, 64, out, dtype)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("opt", [dict(), dict(cap=20.0, window=700)])
def test_many_sequences_of_the_same_rows(gpu, dtype, out, opt):  # noqa: F811
    """Many times the shares and partials that there is room for, with up to 64 sequences and more."""
    rng = np.random.default_rng(5)
    for B in (64, 65, 100, 1500):
        repeated = np.tile([0, 40], B)[:B + 1]
        check(gpu, repeated, 40, 9000, 8, 2, 64, out, dtype, **opt)
        check(gpu, repeated * 3, 130, 4000, 8, 2, 128, out, dtype, **opt)
        check(gpu, rng.integers(-50, 300, B + 1), 200, 2500, 8, 1, 64, out, dtype, **opt)


def test_sums_beyond_32_bits(gpu):  # noqa: F811
    """65 534 sequences, every second of which has all of 2^21 rows times 8 heads: 2^32 units are asked for."""
    B, T = 65534, 1 << 21
    _, _, free = check(gpu, np.tile([0, T], B)[:B + 1], T, 64, 8, 1, 64)
    assert not free.any()


def test_sequences_with_rows_between_them(gpu):  # noqa: F811
    """Beginnings that ascend, but not from 0: rows before the first are left alone, the others as they are with the rows before left out."""
    torch, hgca = gpu
    cu = np.array([13, 20, 20, 57])
    o, lse, free = check(gpu, cu, 64, 200, 4, 2, 64)
    assert int(free.sum()) == 20 and torch.isfinite(o[13:57].float()).all() and not (o[13:57] == 77).any()
