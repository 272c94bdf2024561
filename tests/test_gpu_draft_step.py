"""The calls around drafted tokens as a decoder layer uses them together, over a managed cache: queries and keys are normed and
rotated, the drafts join the window, are attended to under their tree mask beside the whole pool (in the cache's type or in
8 bits), the accepted path is committed, full windows evict and what left them is stored in 8 bits.  Everything that the device
decides is mirrored in plain Python; outputs are compared with 64 bits, with the tolerances of test_gpu_tree.py (a merge of two
parts adds 8 roundings of 2^-24 of max |v|: within the 64 additions counted there)."""
import numpy as np
import pytest

import draft_oracle as do
from test_gpu_tree import DEV, bounds, gpu, i32, put  # noqa: F401

pytestmark = pytest.mark.gpu


def run(gpu, dtype, pool8, rounds=10, seed=0):
    torch, hgca = gpu
    from paper_2507_03153_amd.cache import LayerCache
    B, Hq, Hkv, d, n, bs, wb = 3, 8, 2, 64, 9, 16, 3
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    rng = np.random.default_rng(seed)
    scale = float(np.float32(d ** -0.5))
    C = LayerCache(td, B, Hq, Hkv, d, bs, wb, 24, 64, scale, DEV, win_cap_blocks=wb + 2, pool8=pool8)
    l_max = wb * bs
    rows = [[] for _ in range(B)]                # (K, V) rows [Hkv,d] of every token that stayed, oldest first
    pool = [0] * B
    freq = torch.from_numpy((1e4 ** (-np.arange(d // 2) * 2.0 / d)).astype(np.float32)).to(DEV)
    w = put(torch, 1 + 0.1 * rng.standard_normal(d), dtype)
    qr, kr = (torch.empty(B, n, h, d, dtype=td, device=DEV) for h in (Hq, Hkv))
    host = lambda t: t.float().cpu().numpy().astype(np.float64)
    for r in range(rounds):
        parent = np.array([[int(rng.integers(max(-1, i - 3), i)) if i else -1 for i in range(n)] for _ in range(B)])
        depth, masks = np.zeros((B, n), int), [[0] * n for _ in range(B)]
        for b in range(B):
            for i in range(n):
                p = parent[b, i]
                depth[b, i] = 0 if p < 0 else depth[b, p] + 1
                masks[b][i] = (masks[b][p] if p >= 0 else 0) | 1 << i
        # q and k are parts of one projection's rows; a draft's position is its depth behind the conversation
        wide = put(torch, rng.standard_normal((B, n, (Hq + 2 * Hkv) * d)), dtype)
        q, k = wide[..., :Hq * d].unflatten(-1, (Hq, d)), wide[..., Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d))
        v = wide[..., (Hq + Hkv) * d:].unflatten(-1, (Hkv, d)).contiguous()
        pos = i32(torch, depth + np.array([[len(x)] for x in rows]))
        hgca.qk_norm_rope(C.shape, q, k, qr, kr, freq, q_weight=w, k_weight=w, positions=pos)
        kd = kr.clone()
        C.draft_step(qr, kd, v, torch.from_numpy(do.as_int64(masks)).to(DEV))
        # the accepted path: from a random draft up to its root, for one sequence now and then none
        path, cnt = np.zeros((B, n), np.int32), np.zeros(B, np.int32)
        for b in range(B):
            at, up = int(rng.integers(0, n)), []
            while at >= 0:
                up.append(at)
                at = parent[b, at]
            if rng.random() < 0.15:
                up = []
            path[b, :len(up)], cnt[b] = up[::-1], len(up)
        o, lse = C.o_draft.double().cpu().numpy(), C.lse_draft.double().cpu().numpy()
        qh, kh, vh = host(qr), host(kd), host(v)
        if r == 0:
            want = do.norm_rope(host(k), host(w), 1e-6, pos.cpu().numpy(), freq.cpu().numpy(), False)
            assert np.abs(kh - want).max() <= (2.0 ** -8 + 64 * 2.0 ** -23) * np.abs(want).max()
        for b in range(B):
            K, V = (np.stack([x[j] for x in rows[b]] + [y[b, i] for i in range(n)], 1)[None] for j, y in ((0, kh), (1, vh)))
            if pool8 and pool[b]:
                for x in (K, V):
                    x[:, :, :pool[b]] = do.decode(*do.encode(x[:, :, :pool[b]]))
            T = K.shape[2]
            O, L = do.rows_attention(qh[b:b + 1], K, V, [T], scale, masks[b:b + 1])
            tol_o, tol_l = bounds(qh[b:b + 1], K, V, [T], scale, T)
            eo, el = np.abs(o[b:b + 1] - O).max(), np.abs(lse[b:b + 1] - L).max()
            if dtype == "bf16" and not pool8:    # the append stage's weights have two parts: 2^-17 each
                tol_o += 2.0 ** -16 * np.abs(V).max()
            assert eo <= tol_o and el <= tol_l, f"round {r} sequence {b}: dO={eo} of {tol_o}, dlse={el} of {tol_l}"
        C.commit(kd, v, i32(torch, path), i32(torch, cnt), beta=1.0)
        torch.cuda.synchronize()
        for b in range(B):
            rows[b] += [(kh[b, i], vh[b, i]) for i in path[b, :cnt[b]]]
            win = len(rows[b]) - pool[b]
            if win >= l_max:
                pool[b] += -(-(win - l_max + 1) // bs) * bs
        assert C.pool_lens.tolist() == pool
        assert C.win_lens.tolist() == [len(x) - p for x, p in zip(rows, pool)]
        assert C.status.item() == 0
    assert max(pool) >= 2 * bs, "no eviction was met"
    return C


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pool8", [True, False])
def test_draft_steps_over_a_managed_cache(gpu, dtype, pool8):
    run(gpu, dtype, pool8, rounds=36, seed=3 + pool8)


def test_too_many_drafts_for_the_window(gpu):
    torch, hgca = gpu
    from paper_2507_03153_amd.cache import LayerCache
    C = LayerCache(torch.bfloat16, 1, 2, 1, 64, 16, 2, 8, 16, 0.1, DEV)
    z = lambda h: torch.zeros(1, 2, h, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError, match="win_cap_blocks"):
        C.draft_step(z(2), z(1), z(1))
    with pytest.raises(hgca.HgcaError):          # more than HGCA_MAX_DRAFTS
        hgca.tree_workspace(C.shape, 65, 64, DEV)


def test_decode_steps_and_draft_steps_take_turns(gpu):
    """A managed decode step after committed drafts sees what they left (lengths, rows), and its evictions reach the 8-bit pool."""
    torch, hgca = gpu
    C = run(gpu, "bf16", True, rounds=36, seed=9)
    B, Hq, Hkv, d = C.B, C.Hq, C.Hkv, C.d
    g = torch.Generator(device=DEV).manual_seed(1)
    bf = dict(dtype=torch.bfloat16, device=DEV, generator=g)
    before = C.pool_lens.clone()
    for _ in range(40):
        C.decode_step(torch.randn(B, Hq, d, **bf), torch.randn(B, Hkv, d, **bf), torch.randn(B, Hkv, d, **bf), 0.3, 1.0, one_call=True)
        C.sync_pool8()
    torch.cuda.synchronize()
    assert (C.pool_lens > before).all() and C.status.item() == 0
    L = int(C.pool_lens.min())
    first = torch.zeros(B, dtype=torch.int32, device=DEV)
    ko, vo = (torch.zeros(B, L, Hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    hgca.kv8_read(C.shape, C.pool8, first, ko, vo)
    torch.cuda.synchronize()
    for back, blocks in ((ko, C.k_blocks), (vo, C.v_blocks)):
        x = blocks[C.block_table[:, :L // 16].long()].permute(0, 1, 3, 2, 4).reshape(B, L, Hkv, d).float().cpu().numpy()
        assert np.array_equal(back.double().cpu().numpy(), do.decode(*do.encode(x)))


def test_captured_draft_steps(gpu):
    """Two graphs, of draft steps and commits with 3 and with 5 tokens, replayed in turn with eager steps between: each as the same
    steps on a cache without graphs.  A first step inside a capture is refused."""
    torch, hgca = gpu
    from paper_2507_03153_amd.cache import LayerCache
    B, Hq, Hkv, d = 2, 4, 2, 64
    make = lambda: LayerCache(torch.bfloat16, B, Hq, Hkv, d, 16, 2, 16, 16, 0.125, DEV, win_cap_blocks=3, pool8=True)
    G, E = make(), make()
    bf = dict(dtype=torch.bfloat16, device=DEV)
    ins = {n: [torch.zeros(B, n, h, d, **bf) for h in (Hq, Hkv, Hkv)] for n in (3, 5)}
    mask = {n: torch.tensor([[(2 << i) - 1 for i in range(n)]] * B, dtype=torch.int64, device=DEV) for n in ins}
    path = {n: torch.arange(n, dtype=torch.int32, device=DEV).expand(B, n).contiguous() for n in ins}
    cnt = torch.tensor([2, 3], dtype=torch.int32, device=DEV)

    def step(C, n):
        q, k, v = ins[n]
        C.draft_step(q, k, v, mask[n])
        C.commit(k, v, path[n], cnt, 1.0)
    fresh = make()
    with pytest.raises(RuntimeError, match="before the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            step(fresh, 3)
    torch.cuda.synchronize()
    graphs, outs = {}, {}
    for n in ins:
        step(G, n)
        step(E, n)
    torch.cuda.synchronize()
    for n in ins:
        graphs[n] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[n]):
            step(G, n)
        outs[n] = G.o_draft
    gen = torch.Generator(device=DEV).manual_seed(3)
    for r in range(24):
        n = (3, 5)[r % 2]
        for t in ins[n]:
            t.copy_(torch.randn(t.shape, generator=gen, **bf))
        if r % 5 == 4:
            step(G, n)
        else:
            graphs[n].replay()
        step(E, n)
        torch.cuda.synchronize()
        assert torch.equal(outs[n], E.o_draft) and torch.equal(G.lse_draft if r % 5 == 4 else G._drafts[n].lse[0], E.lse_draft)
        assert torch.equal(G.win_lens, E.win_lens) and torch.equal(G.pool_lens, E.pool_lens) and G.status.item() == 0
    assert G.pool_lens.max() > 0
