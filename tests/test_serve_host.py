"""Refusals of the calls of a server's step (plans, packed rows, packed chunks, verification), without a GPU: nothing reaches a launch.  The
oracle's own pins are here too."""
import ctypes

import numpy as np
import pytest

import serve_oracle as so

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


def at(i):
    return 0x10000000 * (i + 1)


def blocks(hg, **kw):
    f = dict(block_table=at(0), held=at(1), lens=at(2), free_blocks=at(3), free_count=at(4), status=None, scratch=at(5), batch=4, block_size=16,
             max_blocks=8, n_blocks=100)
    f.update(kw)
    return hg.BlockStateView(*f.values())


def plan(hg, st=None, n_new=at(6), most=50, cu=at(7), pos=at(8), slots=at(9)):
    return hg.lib().hgca_kv_plan(ctypes.byref(st or blocks(hg)), n_new, most, cu, pos, slots, None)


def test_plan_refusals(hg):
    I, U = hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED
    assert hg.lib().hgca_kv_plan(None, at(6), 5, at(7), at(8), at(9), None) == I
    assert plan(hg, n_new=None) == plan(hg, cu=None) == plan(hg, pos=None) == plan(hg, slots=None) == plan(hg, most=-1) == I
    assert plan(hg, most=(1 << 30) + 1) == U
    for bad in (dict(batch=-1), dict(block_size=0), dict(max_blocks=-1), dict(n_blocks=-1), dict(held=None), dict(lens=None), dict(free_count=None),
                dict(scratch=None), dict(block_table=None), dict(free_blocks=None)):
        assert plan(hg, blocks(hg, **bad)) == I
    assert plan(hg, blocks(hg, batch=65536)) == U
    assert plan(hg, blocks(hg, max_blocks=1 << 28)) == U
    assert plan(hg, blocks(hg, n_blocks=1 << 27)) == U                        # 2^31 slots
    # outputs over what is read
    for i in range(7):
        assert plan(hg, cu=at(i)) == plan(hg, pos=at(i)) == plan(hg, slots=at(i)) == I
    assert plan(hg, pos=at(9)) == plan(hg, cu=at(8) + 4 * 49) == I
    assert plan(hg, n_new=at(1)) == plan(hg, n_new=at(2) + 4) == plan(hg, n_new=at(5) + 48) == I
    assert plan(hg, blocks(hg, status=at(7))) == I
    assert plan(hg, blocks(hg, batch=0), n_new=None, cu=None, pos=None, slots=None) == hg.OK


def test_release_refusals(hg):
    I = hg.ERR_INVALID_ARG
    f = lambda st=None, lens=at(6): hg.lib().hgca_kv_release(ctypes.byref(st or blocks(hg)), lens, None)
    assert f(lens=None) == I
    assert f(lens=at(1)) == f(lens=at(2) + 4) == f(lens=at(3) + 396) == f(lens=at(4)) == I
    assert f(blocks(hg, lens=None)) == I
    assert f(blocks(hg, batch=0), lens=None) == hg.OK


def write(hg, sh=None, kv=None, n_slots=128, slots=at(0), k=at(1), ks=0, v=at(2), vs=0, n=4):
    return hg.lib().hgca_kv_write(ctypes.byref(sh or shape(hg)), ctypes.byref(kv or view(hg, k=at(3), v=at(4))), n_slots, slots, k, ks, v, vs, n, None)


def test_write_refusals(hg):
    I, U = hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED
    assert write(hg, slots=None) == write(hg, k=None) == write(hg, v=None) == write(hg, k=at(1) + 8) == write(hg, n=-1) == write(hg, n_slots=-1) == I
    assert write(hg, ks=255) == write(hg, vs=128) == write(hg, ks=257) == write(hg, vs=260) == I        # rows overlap, rows not aligned
    assert write(hg, n_slots=129) == I                                        # a contiguous tier of 2 x 64
    assert write(hg, kv=view(hg, k=at(3), v=at(4), table=FAKE, bs=16, mb=4), n_slots=1 << 31) == U
    assert write(hg, kv=view(hg, k=at(3), v=at(4), table=FAKE, bs=24, mb=4)) == U
    assert write(hg, n=(1 << 23) + 1) == U
    assert write(hg, ks=1 << 41) == U
    # inputs over the tier's rows
    assert write(hg, k=at(3)) == write(hg, v=at(3) + 512 * 127) == write(hg, k=at(4) - 512 * 3) == write(hg, slots=at(4) + 16) == I
    assert write(hg, n=0, k=None) == write(hg, sh=shape(hg, B=0), k=None, n_slots=0) == hg.OK


def chunk(hg, sh=None, kv=None, q=FAKE, qs=0, cu=FAKE, T=10, flags=1, window=0, cap=0.0, slopes=None, prefix=None, first=None, o=FAKE, od=1, lse=FAKE,
          ws=FAKE, ws_bytes=BIG):
    return hg.lib().hgca_chunk_attn(ctypes.byref(sh or shape(hg)), q, qs, cu, T, ctypes.byref(kv or view(hg)), flags, window, cap, slopes, prefix, first, o,
                                    od, lse, ws, ws_bytes, None)


def test_chunk_refusals(hg):
    I, U, W = hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED, hg.ERR_WORKSPACE
    assert chunk(hg, q=None) == chunk(hg, q=ODD) == chunk(hg, cu=None) == chunk(hg, o=None) == chunk(hg, o=ODD) == chunk(hg, lse=None) == I
    assert chunk(hg, T=-1) == chunk(hg, flags=2) == chunk(hg, window=-1) == chunk(hg, qs=1020) == chunk(hg, qs=1025) == I
    for cap in (-1.0, float("nan"), float("inf"), 1e-40):
        assert chunk(hg, cap=cap) == I
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert chunk(hg, sh=shape(hg, scale=scale)) == I
    assert chunk(hg, od=2) == chunk(hg, sh=shape(hg, d=96)) == chunk(hg, sh=shape(hg, Hq=6, Hkv=2)) == U
    assert chunk(hg, kv=view(hg, v=None)) == chunk(hg, kv=view(hg, k=ODD)) == I
    assert chunk(hg, kv=view(hg, table=FAKE, bs=16, mb=3)) == I
    assert chunk(hg, kv=view(hg, table=FAKE, bs=24, mb=9)) == U
    assert chunk(hg, sh=shape(hg, B=1, Hkv=1, Hq=1), kv=view(hg, cap=(1 << 30) + 1)) == U
    assert chunk(hg, T=1 << 30) == U and chunk(hg, qs=1 << 40) == U
    assert chunk(hg, ws=None) == chunk(hg, ws_bytes=0) == chunk(hg, ws=ODD) == W
    sh = shape(hg)
    need = hg.lib().hgca_chunk_workspace_bytes(ctypes.byref(sh), 10, 4096)
    assert chunk(hg, kv=view(hg, cap=4096), ws_bytes=need - 1) == W
    assert hg.lib().hgca_chunk_workspace_bytes(ctypes.byref(sh), -1, 64) == hg.lib().hgca_chunk_workspace_bytes(ctypes.byref(sh), 1, -1) == 0
    assert chunk(hg, sh=shape(hg, B=0), q=None, ws=None) == chunk(hg, T=0, q=None, ws=None) == hg.OK


def test_chunk_workspace_serves_smaller_calls(hg):
    L = hg.lib()
    for B, Hq, Hkv, d in ((1, 4, 4, 64), (3, 32, 8, 128), (64, 64, 8, 128), (3000, 16, 2, 64)):
        sh = shape(hg, B=B, Hq=Hq, Hkv=Hkv, d=d)
        caps, tokens = (0, 1, 255, 256, 257, 1000, 100000), (0, 1, 3, 64, 1000, 70000)
        size = [[L.hgca_chunk_workspace_bytes(ctypes.byref(sh), t, c) for c in caps] for t in tokens]
        assert size[0][0] > 0
        assert all(r == sorted(r) for r in size) and all(list(c) == sorted(c) for c in zip(*size))


def verify(hg, B=2, n=4, V=100, dt=0, t=at(0), tr=0, ts=0, q=at(1), qr=0, qs=0, tok=at(2), par=None, u=at(3), un=at(4), path=at(5), cnt=at(6),
           nxt=at(7), ws=at(8), ws_bytes=BIG):
    return hg.lib().hgca_verify_drafts(B, n, V, dt, t, tr, ts, q, qr, qs, tok, par, u, un, path, cnt, nxt, ws, ws_bytes, None)


def test_verify_refusals(hg):
    I, U, W = hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED, hg.ERR_WORKSPACE
    for bad in (dict(t=None), dict(tok=None), dict(u=None), dict(un=None), dict(path=None), dict(cnt=None), dict(nxt=None), dict(B=-1), dict(n=0),
                dict(V=0), dict(t=at(0) + 2), dict(q=at(1) + 1), dict(tr=99), dict(qr=50), dict(ts=-1), dict(qs=-5)):
        assert verify(hg, **bad) == I, bad
    assert verify(hg, n=65) == verify(hg, dt=2) == verify(hg, V=(1 << 30) + 1) == verify(hg, B=65536) == verify(hg, tr=1 << 36) == U
    need = hg.lib().hgca_verify_workspace_bytes(2, 5000)
    assert verify(hg, ws=None) == verify(hg, ws=at(8) + 4) == verify(hg, V=5000, ws_bytes=need - 1) == W
    assert hg.lib().hgca_verify_workspace_bytes(-1, 5) == hg.lib().hgca_verify_workspace_bytes(5, 0) == 0
    assert verify(hg, B=0, t=None) == hg.OK


def test_overlaps(hg):
    """Arrays that a call writes while it reads others; a byte behind the other's end is no overlap."""
    I, W = hg.ERR_INVALID_ARG, hg.ERR_WORKSPACE
    assert verify(hg, path=at(2)) == verify(hg, cnt=at(2) + 28) == verify(hg, nxt=at(4)) == verify(hg, path=at(3) - 4) == verify(hg, cnt=at(6), nxt=at(6) + 4) == I
    assert verify(hg, par=at(9), cnt=at(9)) == verify(hg, path=at(5), nxt=at(5) + 28) == I
    assert verify(hg, cnt=at(2) + 32, ws=None) == verify(hg, nxt=at(6) + 8, ws=None) == W          # (checked before the overlaps)
    q, o, lse = 1 << 30, 1 << 31, 1 << 32        # 10 tokens of 8 x 128 bf16: 20 480 bytes; fp32 O 40 960, lse 320
    args = dict(T=10, sh=shape(hg, B=1, Hq=8, Hkv=2, d=128), od=0)
    for bad in (dict(q=q, o=q, lse=lse), dict(q=q, o=q + 20464, lse=lse), dict(q=q, o=o, lse=o + 40956), dict(q=q, o=o, lse=q + 16), dict(q=q, o=q - 40944, lse=lse)):
        assert chunk(hg, **args, **bad) == I, bad
    sh, k = shape(hg, B=1, Hq=2, Hkv=2, d=64), 1 << 30               # 100 slots of 2 x 64 bf16: 25 600 bytes
    two = lambda v: hg.lib().hgca_kv_write(ctypes.byref(sh), ctypes.byref(view(hg, k=k, v=v, cap=100)), 100, 1 << 33, 1 << 34, 0, 1 << 35, 0, 1, None)
    assert two(k) == two(k + 25584) == two(k - 25584) == I


# ---- the oracle's pins ----

def test_plan_pin():
    table = np.array([[4, 9, -1, -1], [7, -1, -1, -1], [-1, -1, -1, -1]])
    held, lens, free = [2, 1, 0], [20, 16, 0], [0, 2, 3]
    cu, pos, slots, bits = so.plan(16, table, held, lens, free, [13, 1, 17], 100)
    assert cu == [0, 13, 14, 14] and bits == 8                                 # blocks 3, 2 are granted; the third needs two more than one
    assert pos == list(range(20, 33)) + [16]
    assert slots == [9 * 16 + i for i in range(4, 16)] + [48, 32]
    assert free == [0] and held == [3, 2, 0] and lens == [33, 17, 0]
    so.release(16, table, held, lens, free, [20, 16, 0])
    assert free == [0, 2, 3] and held == [2, 1, 0]


def test_sees_pin():
    assert so.sees(2, 4).astype(int).tolist() == [[1, 1, 1, 0], [1, 1, 1, 1]]
    assert so.sees(2, 4, window=2).astype(int).tolist() == [[0, 1, 1, 0], [0, 0, 1, 1]]
    assert so.sees(2, 4, window=1, prefix=1).astype(int).tolist() == [[1, 0, 1, 0], [1, 0, 0, 1]]
    assert so.sees(2, 4, causal=False, first=[1, 3]).astype(int).tolist() == [[0, 1, 1, 1], [0, 0, 0, 1]]
    assert so.sees(3, 2).astype(int).tolist() == [[0, 0], [1, 0], [1, 1]]      # a tier with fewer tokens holds the last ones


def test_chunk_pin():
    """One query over two tokens, by hand: scores 1 and 3, capped at 2, less 0.5 a token of distance."""
    q, K, V = np.array([[[1.0]]]), np.array([[[[1.0], [3.0]]]]), np.array([[[[10.0], [20.0]]]])
    O, lse = so.chunk(q, [0, 1], K, V, [2], 1.0, cap=2.0, slopes=[0.5])
    a, b = 2 * np.tanh(0.5) - 0.5, 2 * np.tanh(1.5)
    assert abs(O[0, 0, 0] - (10 * np.exp(a) + 20 * np.exp(b)) / (np.exp(a) + np.exp(b))) < 1e-12
    assert abs(lse[0, 0] - np.log(np.exp(a) + np.exp(b))) < 1e-12


def test_verify_pin():
    """Three tokens, p = .5 .3 .2, q = .2 .7 .1: token 1 is accepted below 3/7; after its refusal max(p - q, 0) = .3 0 .1, of which token 0 has
    three quarters."""
    p, q = np.array([[[.5, .3, .2]] * 2]), np.array([[[.2, .7, .1]] * 2])
    for u, un, want in ((.42, .9, ([0, 1], 2, 2)), (.43, .74, ([0, -1], 1, 0)), (.43, .76, ([0, -1], 1, 2))):
        path, cnt, nxt, _ = so.verify(p, q, np.array([[0, 1]]), np.array([[0, u]]), [un])
        assert (path[0].tolist(), cnt[0], nxt[0]) == want
    path, cnt, nxt, _ = so.verify(p, None, np.array([[0, 1]]), np.array([[0, .31]]), [.72])        # without q: .5 and .2 are left
    assert (cnt[0], nxt[0]) == (1, 2)
