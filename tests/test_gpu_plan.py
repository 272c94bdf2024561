"""Block tables and slot maps from the requests' lengths (hgca_kv_plan, hgca_kv_release) and rows of packed tokens written by slot
(hgca_kv_write), against a plain Python form: whole numbers and bytes, equal."""
import numpy as np
import pytest

import serve_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2507_03153_amd import hgca
    hgca.lib()
    return torch, hgca


def i32(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


class Both:
    """A state on both sides."""

    def __init__(self, gpu, rng, B, bs, row, n_blocks, lens, ahead=0):
        torch, hgca = gpu
        self.torch, self.hgca, self.bs, self.B = torch, hgca, bs, B
        order = [int(x) for x in rng.permutation(n_blocks)]
        self.lens = [int(x) for x in lens]
        self.held = [min(-(-x // bs) + (ahead if i % 3 == 0 else 0), row) for i, x in enumerate(self.lens)]
        self.table = np.full((B, row), -7, np.int64)
        for b in range(B):
            for j in range(self.held[b]):
                self.table[b, j] = order.pop()
        self.free = order
        stack = np.full(n_blocks, -3, np.int64)
        stack[:len(order)] = order
        self.state = hgca.BlockState(i32(torch, self.table), i32(torch, self.held), i32(torch, self.lens), i32(torch, stack),
                                     i32(torch, [len(order)]), bs, status=torch.zeros(1, dtype=torch.int32, device=DEV))
        self.state.scratch.fill_(-1)
        self.bits = 0

    def plan(self, n_new, most):
        torch = self.torch
        cu, pos, slots = (torch.full((k,), -99, dtype=torch.int32, device=DEV) for k in (self.B + 1, most, most))
        self.hgca.kv_plan(self.state, i32(torch, n_new), cu, pos, slots)
        want = so.plan(self.bs, self.table, self.held, self.lens, self.free, n_new, most)
        self.bits |= want[3]
        torch.cuda.synchronize()
        assert cu.tolist() == want[0]
        pad = most - len(want[1])
        assert pos.tolist() == want[1] + [0] * pad
        assert slots.tolist() == want[2] + [-1] * pad
        self.same()
        return cu, pos, slots

    def release(self, new_lens):
        self.hgca.kv_release(self.state, self.state.lens if new_lens is None else i32(self.torch, new_lens))
        so.release(self.bs, self.table, self.held, self.lens, self.free, self.lens if new_lens is None else new_lens)
        self.torch.cuda.synchronize()
        self.same()

    def same(self):
        s = self.state
        assert s.lens.tolist() == self.lens and s.held.tolist() == self.held
        assert int(s.free_count) == len(self.free)
        assert s.free_blocks[:len(self.free)].tolist() == self.free
        assert s.block_table.tolist() == self.table.tolist()
        assert int(s.status) == self.bits


@pytest.mark.parametrize("B,bs,row,most", [(1, 16, 4, 64), (5, 16, 9, 300), (64, 16, 20, 3000), (3, 1, 40, 100), (7, 48, 5, 1200),
                                           (1025, 16, 3, 4096), (1025, 16, 3, 4097), (2100, 32, 4, 30000), (130, 16, 300, 200000)])
def test_many_rounds(gpu, B, bs, row, most):
    """Plans and releases in turn, from none to all of a sequence; rows too short, blocks and tokens that run out among them."""
    rng = np.random.default_rng(B * 7 + bs + most)
    lens = rng.integers(0, row * bs // 2 + 1, B)
    S = Both(gpu, rng, B, bs, row, int(sum(-(-x // bs) for x in lens)) + B + max(B * row // 3, 1), lens, ahead=1)
    top = max(2 * most // B, 2)
    for turn in range(5):
        print(f"\n[turn] {turn} of B={B} bs={bs} row={row} most={most}", flush=True)
        S.plan(rng.integers(-1, top, B) * (rng.random(B) < 0.8), most)
        new = [int(x) for x in S.lens]
        for b in range(B):
            if rng.random() < 0.5:
                new[b] = int(rng.integers(-1, S.lens[b] + 3))
        S.release(new)
    S.release([0] * B)
    assert sum(S.held) == 0 and len(S.free) == S.state.free_blocks.numel()


def test_release_undoes_a_plan(gpu):
    rng = np.random.default_rng(2)
    S = Both(gpu, rng, 40, 16, 30, 1500, rng.integers(0, 200, 40))
    lens, free = list(S.lens), list(S.free)
    S.plan(rng.integers(0, 200, 40), 9000)
    S.release(lens)
    assert S.free == free and S.state.free_blocks[:len(free)].tolist() == free


def test_first_come_first_served(gpu):
    """A sequence without blocks keeps later ones from theirs, but not those that need none."""
    rng = np.random.default_rng(3)
    S = Both(gpu, rng, 5, 16, 8, 5 + 3, [16, 16, 16, 10, 16])        # five in use, three free
    S.plan([16, 48, 16, 6, 1], 100)
    assert S.lens == [32, 16, 16, 16, 16] and S.bits == 8
    S = Both(gpu, rng, 3, 16, 2, 12, [30, 4, 0])
    S.plan([3, 4, 5], 8)                                             # the first one's row ends, the third's tokens are too many
    assert S.lens == [30, 8, 0] and S.bits == 2 | 16


def test_no_tokens_and_no_sequences(gpu):
    torch, hgca = gpu
    rng = np.random.default_rng(4)
    S = Both(gpu, rng, 3, 16, 4, 10, [5, 0, 16])
    S.plan([0, 0, 0], 0)
    S.plan([0, -5, 0], 7)
    S.release(None)
    z = torch.zeros(0, dtype=torch.int32, device=DEV)
    empty = hgca.BlockState(z.view(0, 4), z, z.clone(), z.clone(), torch.zeros(1, dtype=torch.int32, device=DEV), 16)
    hgca.kv_plan(empty, z.clone(), torch.full((1,), 9, dtype=torch.int32, device=DEV), z.clone(), z.clone())


def test_lens_set_by_a_commit_are_released(gpu):
    """After lens has been set to fewer tokens elsewhere, a release to lens itself gives the blocks back."""
    torch, hgca = gpu
    rng = np.random.default_rng(5)
    S = Both(gpu, rng, 4, 16, 8, 40, [20, 3, 0, 64])
    S.plan([20, 40, 17, 0], 100)
    S.lens = [21, 3, 16, 64]
    S.state.lens.copy_(i32(torch, S.lens))
    S.release(None)
    assert S.held == [2, 1, 1, 4]


@pytest.mark.parametrize("dtype,d,Hkv,block,T", [("bf16", 128, 8, 16, 33), ("bf16", 64, 1, 48, 5), ("f32", 128, 3, 16, 200), ("f32", 64, 40, 0, 77),
                                                 ("bf16", 128, 40, 32, 1), ("bf16", 64, 2, 0, 1000)])
def test_write(gpu, dtype, d, Hkv, block, T):
    """Rows go where their slots say, all else stays; K and V as parts of wider rows and dense."""
    torch, hgca = gpu
    rng = np.random.default_rng(T)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    B, cap = 3, 700
    nb, width = (60, block) if block else (B, cap)
    g = torch.Generator(device=DEV).manual_seed(T)
    k, v = (torch.randn(nb, Hkv, width, d, generator=g, device=DEV, dtype=dt) for _ in "kv")
    n_slots = nb * width
    slots = rng.permutation(n_slots)[:T]
    slots[rng.random(T) < 0.2] = -1
    slots[0], slots[T // 2] = n_slots, slots[T // 2]                 # behind the last one: left out
    if T > 4:
        slots[3], slots[4] = -2 ** 31, 2 ** 31 - 1
    wide = torch.randn(T, (2 * Hkv + 3) * d, generator=g, device=DEV, dtype=dt)
    shape = hgca.Shape(hgca.F32 if dtype == "f32" else hgca.BF16, B, Hkv, Hkv, d, 1.0)
    table = torch.zeros(B, 60, dtype=torch.int32, device=DEV) if block else None
    for dense in (False, True):
        ki, vi = wide[:, d:(Hkv + 1) * d].unflatten(-1, (Hkv, d)), wide[:, (Hkv + 2) * d:(2 * Hkv + 2) * d].unflatten(-1, (Hkv, d))
        if dense:
            ki, vi = vi.contiguous(), ki.contiguous()
        want = [x.clone() for x in (k, v)]
        for t, s in enumerate(slots.tolist()):
            if 0 <= s < n_slots:
                want[0][s // width, :, s % width], want[1][s // width, :, s % width] = ki[t], vi[t]
        tier = hgca.Tier(k, v, 60 * block if block else cap, None, table, block)
        hgca.kv_write(shape, tier, i32(torch, slots), ki, vi)
        torch.cuda.synchronize()
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_write_beyond_4_gib(gpu):
    """Slots whose rows lie beyond 4 GiB of a tier."""
    torch, hgca = gpu
    nb, Hkv, bs, d = 9000, 8, 64, 512 // 4
    k = torch.empty(nb, Hkv, bs, d, dtype=torch.float32, device=DEV)
    v = torch.empty_like(k)
    slots = [nb * bs - 1, nb * bs - 70, 1, 8300 * bs]
    ki, vi = torch.randn(4, Hkv, d, device=DEV), torch.randn(4, Hkv, d, device=DEV)
    table = torch.zeros(1, nb, dtype=torch.int32, device=DEV)
    hgca.kv_write(hgca.Shape(hgca.F32, 1, Hkv, Hkv, d, 1.0), hgca.Tier(k, v, 64, None, table, bs), i32(torch, slots), ki, vi)
    torch.cuda.synchronize()
    for t, s in enumerate(slots):
        assert torch.equal(k[s // bs, :, s % bs], ki[t]) and torch.equal(v[s // bs, :, s % bs], vi[t])
