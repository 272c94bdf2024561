"""Refusals of the calls around drafted tokens and 8-bit tiers, without a GPU: nothing reaches a launch.  The oracle's own
pins are here too."""
import ctypes

import numpy as np
import pytest

import draft_oracle as do

FAKE, ODD = 0x100000, 0x100004
BIG = 1 << 40


@pytest.fixture(scope="module")
def hg():
    from paper_2507_03153_amd import build, hgca
    build.build(force=False)
    hgca.lib()
    return hgca


def shape(hg, dtype=None, B=2, Hq=8, Hkv=2, d=128, scale=0.1):
    return hg.Shape(hg.BF16 if dtype is None else dtype, B, Hq, Hkv, d, scale)


def view(hg, cap=64, k=FAKE, v=FAKE, table=None, bs=0, mb=0):
    return hg.KvView(k, v, None, table, cap, bs, mb, None)


def view8(hg, cap=64, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, table=None, bs=0, mb=0):
    return hg.Kv8View(k, v, ks, vs, None, table, cap, bs, mb, None)


def tree(hg, sh=None, kv=None, q=FAKE, n=4, mask=FAKE, o=FAKE, o_dtype=0, lse=FAKE, ws=FAKE, ws_bytes=BIG):
    return hg.lib().hgca_tree_attn(ctypes.byref(sh or shape(hg)), q, n, ctypes.byref(kv or view(hg)), mask, o, o_dtype, lse, ws,
                                   ws_bytes, None)


def attn8(hg, sh=None, kv=None, q=FAKE, n=4, o=FAKE, o_dtype=0, lse=FAKE, ws=FAKE, ws_bytes=BIG):
    return hg.lib().hgca_kv8_attn(ctypes.byref(sh or shape(hg)), q, n, ctypes.byref(kv or view8(hg)), o, o_dtype, lse, ws, ws_bytes,
                                  None)


def test_tree_refusals(hg):
    I, U, W = hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED, hg.ERR_WORKSPACE
    assert tree(hg, q=None) == tree(hg, q=ODD) == tree(hg, o=None) == tree(hg, o=ODD) == tree(hg, lse=None) == I
    assert tree(hg, mask=FAKE + 4) == I
    assert tree(hg, n=0) == tree(hg, n=-1) == I
    assert tree(hg, n=65) == U
    assert tree(hg, o_dtype=2) == U
    assert tree(hg, ws=None) == tree(hg, ws_bytes=0) == tree(hg, ws=ODD) == W
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert tree(hg, sh=shape(hg, scale=scale)) == I
    assert tree(hg, sh=shape(hg, d=96)) == U
    assert tree(hg, sh=shape(hg, Hq=6, Hkv=2)) == U
    assert tree(hg, kv=view(hg, v=None)) == tree(hg, kv=view(hg, k=ODD)) == I
    assert tree(hg, kv=view(hg, table=FAKE, bs=24, mb=9)) == U
    assert tree(hg, kv=view(hg, table=FAKE, bs=16, mb=3)) == I                 # 48 tokens for a capacity of 64
    assert tree(hg, sh=shape(hg, B=1, Hkv=1, Hq=1), kv=view(hg, cap=(1 << 30) + 1)) == U
    assert tree(hg, sh=shape(hg, B=0), q=None, ws=None) == hg.OK
    sh = shape(hg)
    need = hg.lib().hgca_tree_workspace_bytes(ctypes.byref(sh), 4, 4096)
    assert tree(hg, kv=view(hg, cap=4096), ws_bytes=need - 1) == W
    assert hg.lib().hgca_tree_workspace_bytes(ctypes.byref(sh), 65, 4096) == 0
    assert hg.lib().hgca_tree_workspace_bytes(ctypes.byref(sh), 0, 4096) == 0
    assert hg.lib().hgca_tree_workspace_bytes(ctypes.byref(sh), 4, -1) == 0


def test_workspace_serves_smaller_capacities(hg):
    L = hg.lib()
    for B, Hq, Hkv in ((1, 4, 4), (3, 32, 8), (64, 64, 8)):
        for n in (1, 3, 5, 8, 16, 64):
            sh = shape(hg, B=B, Hq=Hq, Hkv=Hkv)
            for f in (L.hgca_tree_workspace_bytes, L.hgca_kv8_workspace_bytes):
                sizes = [f(ctypes.byref(sh), n, c) for c in (0, 1, 127, 128, 129, 1000, 4096, 100000)]
                assert sizes == sorted(sizes) and sizes[0] > 0


def test_kv8_attn_refusals(hg):
    I, U, W = hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED, hg.ERR_WORKSPACE
    assert attn8(hg, q=None) == attn8(hg, o=ODD) == attn8(hg, lse=None) == attn8(hg, n=0) == I
    assert attn8(hg, n=4097) == attn8(hg, o_dtype=7) == U
    assert attn8(hg, ws=None) == attn8(hg, ws_bytes=16) == W
    for bad in (dict(k=None), dict(v=ODD), dict(ks=None), dict(vs=None), dict(ks=FAKE + 2)):
        assert attn8(hg, kv=view8(hg, **bad)) == I
    assert attn8(hg, kv=view8(hg, table=FAKE, bs=8, mb=9)) == U
    assert attn8(hg, sh=shape(hg, scale=0.0)) == I
    assert attn8(hg, sh=shape(hg, B=0), q=None, ws=None) == hg.OK


def test_kv8_rows_refusals(hg):
    L, I, U, OK = hg.lib(), hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED, hg.OK

    def write(sh=None, kv=None, k=FAKE, v=FAKE, n=3):
        return L.hgca_kv8_write_tokens(ctypes.byref(sh or shape(hg)), ctypes.byref(kv or view8(hg)), None, k, v, n, None, None)

    def read(kv=None, k=FAKE, v=FAKE, n=3):
        return L.hgca_kv8_read(ctypes.byref(shape(hg)), ctypes.byref(kv or view8(hg)), None, n, k, v, None)

    def from_tier(kv=None, src=None, n=3):
        return L.hgca_kv8_write_tier(ctypes.byref(shape(hg)), ctypes.byref(kv or view8(hg)), None, ctypes.byref(src or view(hg)), n,
                                     None, None)
    for call in (write, read):
        assert call(k=None) == call(v=ODD) == call(n=-1) == I
        assert call(n=0, k=None) == OK
    for call in (write, read, from_tier):
        assert call(kv=view8(hg, ks=None)) == call(kv=view8(hg, vs=FAKE + 1)) == call(kv=view8(hg, k=ODD)) == I
        assert call(kv=view8(hg, table=FAKE, bs=20, mb=9)) == U
    assert from_tier(src=view(hg, v=None)) == from_tier(n=-1) == I
    assert from_tier(n=0) == OK and write(sh=shape(hg, B=0), k=None) == OK


def test_commit_refusals(hg):
    L, I, OK = hg.lib(), hg.ERR_INVALID_ARG, hg.OK

    def commit(sh=None, kv=None, first=FAKE, k=FAKE, v=FAKE, n=3, lens=FAKE + 64):
        return L.hgca_kv_commit(ctypes.byref(sh or shape(hg)), ctypes.byref(kv or view(hg)), first, k, v, n, None, None, lens, None, None)
    assert commit(k=None) == commit(v=ODD) == commit(n=-1) == commit(lens=None) == commit(lens=FAKE) == I
    assert commit(kv=view(hg, k=None)) == commit(kv=view(hg, cap=-1)) == I
    assert commit(n=0) == OK and commit(sh=shape(hg, B=0), lens=None) == OK
    # the drafts are rows of the tier itself: 2 x 2 heads of 64 rows of 256 bytes from FAKE and from `far` on
    far, rows = FAKE + (1 << 20), 4 * 64 * 256
    for inside in (FAKE, FAKE + rows - 16, far, far + rows - 16, far - 16):
        assert commit(kv=view(hg, v=far), k=inside, v=FAKE + (1 << 19)) == commit(kv=view(hg, v=far), k=FAKE + (1 << 19), v=inside) == I
    assert commit(n=1 << 31 - 1, sh=shape(hg, B=65535), kv=view(hg, cap=0, k=None, v=None)) == hg.ERR_UNSUPPORTED


def test_rope_refusals(hg):
    L, I, U, OK = hg.lib(), hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED, hg.OK
    Q, K, QO, KO = (0x1000000 * i for i in (1, 2, 3, 4))

    def rope(sh=None, q=Q, qs=0, k=K, ks=0, n=5, qw=FAKE, kw=FAKE, eps=1e-6, freq=FAKE, rot=128, pos=None, flags=0, qo=QO, ko=KO):
        return L.hgca_qk_norm_rope(ctypes.byref(sh or shape(hg)), q, qs, k, ks, n, qw, kw, eps, freq, rot, pos, None, flags, qo, ko, None)
    assert rope(q=None) == rope(k=ODD) == rope(qo=None) == rope(ko=ODD) == rope(freq=None) == rope(qw=ODD) == I
    assert rope(n=-1) == rope(flags=2) == rope(eps=-1.0) == rope(eps=float("nan")) == I
    assert rope(rot=0) == rope(rot=144) == I and rope(rot=24) == U
    assert rope(qs=8 * 128 - 8) == rope(ks=2 * 128 + 4) == I                   # rows that overlap, rows off 16 bytes
    assert rope(qs=1 << 50) == U
    assert rope(qo=Q + 16) == rope(ko=K + 16) == rope(qo=K) == rope(ko=Q) == rope(ko=QO) == I      # overlaps
    assert rope(qs=2048, qo=Q) == I                                            # in place only where rows are dense
    assert rope(n=0, q=None) == OK and rope(sh=shape(hg, B=0), q=None) == OK


def test_python_checks(hg):
    """Types and sizes are checked before the library is asked; tensors on the CPU are refused."""
    import torch
    B, n, Hq, Hkv, d = 2, 3, 8, 2, 128
    sh = shape(hg, B=B)
    bf = dict(dtype=torch.bfloat16)
    q, o, lse = torch.zeros(B, n, Hq, d, **bf), torch.zeros(B, n, Hq, d), torch.zeros(B, n, Hq)
    kv = torch.zeros(B, Hkv, 64, d, **bf)
    ws, mask = torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(B, n, dtype=torch.int64)
    tier = hg.Tier(kv, kv.clone(), 64)
    with pytest.raises(ValueError, match="GPU"):
        hg.tree_attn(sh, q, tier, mask, o, lse, ws)
    with pytest.raises(ValueError, match="GPU"):
        hg.kv8_attn(sh, q, tier, o, lse, ws)
    with pytest.raises(ValueError, match="GPU"):
        hg.qk_norm_rope(sh, q, q, q, q, o)
    with pytest.raises(ValueError, match="GPU"):
        hg.kv_commit(sh, tier, None, q, q, lse)
    # as one GPU's tensors are checked (device -1 stands for it)
    hg._need("mask", mask, torch.int64, (B, n), -1)
    with pytest.raises(ValueError, match="mask must be"):
        hg._need("mask", mask.int(), torch.int64, (B, n), -1)
    with pytest.raises(ValueError, match="lse_out must be"):
        hg._need("lse_out", lse[:, :2], torch.float32, (B, n, Hq), -1)
    with pytest.raises(ValueError, match="contiguous"):
        hg._need("lse_out", lse.transpose(0, 1), torch.float32, (n, B, Hq), -1)
    with pytest.raises(ValueError, match="other tensors on cuda:1"):
        hg._need("mask", mask, torch.int64, (B, n), 1)
    with pytest.raises(ValueError, match="tier.k must be"):
        hg._tier_view(hg.Tier(kv, kv, 65), B, Hkv, d, torch.bfloat16, -1)
    with pytest.raises(ValueError, match="seq_lens"):
        hg._tier_view(hg.Tier(kv, kv, 64, torch.zeros(B)), B, Hkv, d, torch.bfloat16, -1)
    with pytest.raises(ValueError, match="block_table"):
        hg._tier_view(hg.Tier(kv, kv, 64, None, torch.zeros(B + 1, 4, dtype=torch.int32), 64), B, Hkv, d, torch.bfloat16, -1)
    z = lambda w: torch.zeros(B, Hkv, 64, w, dtype=torch.uint8)
    with pytest.raises(ValueError, match="k_scale"):
        hg._tier_view(hg.Kv8Tier(z(d), z(d), z(2), z(4), 64), B, Hkv, d, torch.uint8, -1)
    wide = torch.zeros(B, n, (Hq + 2 * Hkv) * d, **bf)
    qv, kv_ = wide[..., :Hq * d].unflatten(-1, (Hq, d)), wide[..., Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d))
    assert hg._token_stride("q", qv) == hg._token_stride("k", kv_) == (Hq + 2 * Hkv) * d
    assert hg._token_stride("q", qv[:1, :1]) == Hq * d
    with pytest.raises(ValueError, match="side by side"):
        hg._token_stride("q", wide.unflatten(-1, (-1, d)).transpose(1, 2))


# ---- the oracle ----

def test_oracle_codes():
    import torch
    rng = np.random.default_rng(0)
    x = rng.standard_normal((64, 128)) * 2.0 ** rng.integers(-60, 60, (64, 4)).repeat(32, 1)
    x = x.astype(np.float32)
    codes, scales = do.encode(x)
    y = do.decode(codes, scales)
    step = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, -1)
    assert np.all(np.abs(y - x) <= np.maximum(np.abs(x) * 2.0 ** -4, step * 2.0 ** -10))
    # the library that reads these bytes elsewhere agrees on what they stand for
    ref = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mine = do.decode(np.arange(256, dtype=np.uint8).reshape(8, 32), np.full((8, 1), 127, np.uint8)).reshape(-1)
    assert np.array_equal(ref, mine, equal_nan=True)
    tops = np.zeros((4, 32)); tops[:, 0] = [448, 449, 464, 0]
    c, s = do.encode(tops)
    assert s[:, 0].tolist() == [127, 128, 128, 17] and c[0, 0] == 0x7e and c[3, 0] == 0


def test_oracle_tree():
    """A mask of all earlier drafts is causal attention; no mask sees everything; an empty row is empty."""
    rng = np.random.default_rng(1)
    q, K, V = rng.standard_normal((1, 3, 2, 8)), rng.standard_normal((1, 1, 5, 8)), rng.standard_normal((1, 1, 5, 8))
    O, lse = do.rows_attention(q, K, V, [5], 0.5, [[1, 3, 7]])
    for i in range(3):
        s = 0.5 * (K[0, 0, :3 + i] @ q[0, i, 1])
        assert np.allclose(lse[0, i, 1], np.log(np.exp(s).sum()))
        assert np.allclose(O[0, i, 1], np.exp(s) / np.exp(s).sum() @ V[0, 0, :3 + i])
    O, lse = do.rows_attention(q, K, V, [3], 0.5, [[0, 1, 5]])
    assert np.isneginf(lse[0, 0]).all() and (O[0, 0] == 0).all() and np.isfinite(lse[0, 1:]).all()
    O2, _ = do.rows_attention(q, K, V, [5], 0.5)
    O1, _ = do.rows_attention(q, K, V, [5], 0.5, [[7, 7, 7]])
    assert np.allclose(O1, O2)
