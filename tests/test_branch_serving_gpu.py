"""The operators of requests that branch as a server runs them, turn after turn: plan, rotary append, tree attention,
verification, compaction; then a request forked in two, its last page copied, one of them ended and the pages
collected.  The oracle is each request's whole history in 64 bits, token by token."""
import numpy as np
import pytest

import branch_ref
import paged_ref
from gpu_helpers import host, log, workspace

pytestmark = pytest.mark.gpu
H, HKV, DH, PS, PAIRS, POOL, WIDTH, T, V, RR = 6, 2, 128, 16, [32], 40, 12, 96, 200, 4


@pytest.mark.parametrize("fp8,graph", [(False, False), (False, True), (True, False)])
def test_turns_of_trees_and_a_fork(fp8, graph):
    import torch
    import paper_2602_15922_amd as w
    log(f"branch serving fp8={fp8} graph={graph}")
    g, rng = torch.Generator().manual_seed(5), np.random.default_rng(5)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    put = lambda t, x: t.copy_(torch.as_tensor(np.asarray(x)))  # noqa: E731
    layers = []
    for _ in range(2):
        k, v = (torch.full((POOL, PS, HKV, DH), 0x7F, dtype=torch.uint8, device="cuda") if fp8 else
                torch.full((POOL, PS, HKV, DH), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ex = i32(POOL, PS, HKV) if fp8 else None
        layers.append((k, v, ex, w.make_paged_cache(k, v, k_exp=ex, v_scale=6.0 / 448)))
    cache_len, new_len, held, held2, kv_len, n_path, nxt = (i32(RR) for _ in range(7))
    n_free, n_free2, q_start, slots, status, st2 = i32(1), i32(1), i32(RR + 1), i32(T), i32(4), i32(2)
    table, free = i32(RR, WIDTH) - 1, torch.randperm(POOL, generator=g).int().cuda()
    n_free.fill_(POOL)
    qkv, pos = torch.zeros(2, T, (H + 2 * HKV) * DH, dtype=torch.bfloat16, device="cuda"), i32(T, 1)
    q, o = (torch.zeros(2, T, H, DH, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mask, tokens, parent, path = i32(T, 1), i32(T), i32(T), i32(T)
    probs, drafts = (torch.zeros(T, V, device="cuda") for _ in range(2))
    u, u_next = torch.zeros(T, device="cuda"), torch.zeros(RR, device="cuda")
    ws = workspace(w.wam_attn_tree_workspace_bytes(layers[0][3], R=RR, T=T, Hq=H, max_kv=WIDTH * PS))
    ws2 = workspace(w.wam_verify_tree_workspace_bytes(RR, T, V, True))

    def turn():
        w.wam_page_plan(cache_len, new_len, held, n_free, table, free, held2, n_free2, q_start, kv_len, slots, status, page_size=PS)
        for i, (_, _, _, cache) in enumerate(layers):
            w.wam_rope_qkv_paged(cache, qkv[i], pos, slots, q[i], pairs=PAIRS)
            w.wam_attn_tree(cache, q[i], table, q_start, kv_len, mask, o[i], ws)
        w.wam_verify_tree(probs, drafts, tokens, parent, u, u_next, q_start, path, n_path, nxt, ws2, kv_len=kv_len, cache_len=cache_len)
        for _, _, _, cache in layers:
            w.wam_cache_compact(cache, table, q_start, kv_len, path, n_path)
        held.copy_(held2)
        n_free.copy_(n_free2)

    def stored(i, r, m):
        """Layer i's first m keys and values of request r, as the cache holds them."""
        k, v, ex, _ = layers[i]
        ids = table[r, :-(-m // PS)].long()
        if not fp8:
            return [host(x[ids]).reshape(-1, HKV, DH)[:m] for x in (k, v)]
        kk, vv = (paged_ref.E4M3[x[ids].cpu().numpy()].reshape(-1, HKV, DH)[:m] for x in (k, v))
        e = (ex[ids].cpu().numpy().reshape(-1, HKV)[:m].astype(np.int64)[..., None] >> (8 * np.arange(4))) & 255
        return [kk * np.repeat(2.0 ** (e - 127.0), 32, -1), vv * float(np.float32(6.0 / 448))]

    cg = None
    # what the cache must hold: for each layer and request the rows appended and kept, as they were read back then
    kept = [[[np.zeros((0, HKV, DH)) for _ in range(2)] for _ in range(RR)] for _ in range(2)]

    def step(sizes):
        nonlocal cg
        lens = [len(kept[0][r][0]) for r in range(RR)]
        starts = np.concatenate([[0], np.cumsum(sizes)])
        n = int(starts[-1])
        put(new_len, sizes)
        qkv.copy_(torch.randn(qkv.shape, generator=g).bfloat16())
        par, depth, bits = np.full(T, -1), np.zeros(T, int), np.zeros((T, 1), np.int32)
        z = rng.normal(size=(T, V)) * 2
        p = np.exp(z) / np.exp(z).sum(-1, keepdims=True)
        d = np.exp(z + rng.normal(size=z.shape))
        d /= d.sum(-1, keepdims=True)
        tok = np.zeros(T, int)
        for r, (a, m) in enumerate(zip(starts, sizes)):
            for i in range(1, m):
                par[a + i] = rng.integers(max(0, i - 3), i)
                tok[a + i] = rng.choice(V, p=d[a + par[a + i]])
            for i in range(m):
                depth[a + i] = lens[r] + (depth[a + par[a + i]] - lens[r] + 1 if i else 0)
            if m:
                bits[a:a + m] = w.wam_tree_mask([int(x) for x in par[a:a + m]], 1).numpy()
        for t, x in ((pos, depth[:, None]), (mask, bits), (tokens, tok), (parent, par), (u, rng.random(T)), (u_next, rng.random(RR))):
            put(t, x)
        put(probs, p.astype(np.float32)), put(drafts, d.astype(np.float32))
        q.fill_(3.0), o.fill_(3.0), path.fill_(-9)
        if graph and cg is None:
            before = [x.clone() for x in (cache_len, held, n_free, table, free)]
            turn()  # (the kernels are loaded)
            torch.cuda.synchronize()
            for x, y in zip((cache_len, held, n_free, table, free), before):
                x.copy_(y)
            q.fill_(3.0), o.fill_(3.0), path.fill_(-9)
            cg = torch.cuda.CUDAGraph()
            with torch.cuda.graph(cg):
                turn()
        cg.replay() if graph else turn()
        torch.cuda.synchronize()
        assert status.tolist() == [0, 0, 0, 0] and q_start.tolist() == starts.tolist()
        rows = host(qkv).reshape(2, T, -1, DH)
        for r, (a, m) in enumerate(zip(starts, sizes)):
            nodes, token = branch_ref.verify(host(probs)[a:a + m], host(drafts)[a:a + m], tok[a:a + m], par[a:a + m], host(u)[a:a + m],
                                             host(u_next)[r])
            assert n_path[r] == len(nodes) and path[a:a + len(nodes)].tolist() == nodes and nxt[r] == token
            assert cache_len[r] == lens[r] + len(nodes)
            seen = branch_ref.tree_seen(bits, a, m, lens[r] + m, 1 << 30)
            for i in range(2):
                y = paged_ref.rotate(rows[i, a:a + m, :H + HKV], paged_ref.angles(depth[a:a + m, None], PAIRS, 10000.0), False)
                new_k, new_v = y[:, H:], rows[i, a:a + m, H + HKV:]
                kk, vv = stored(i, r, lens[r] + len(nodes))
                # the history untouched bit by bit, then the path's rows as the append writes them
                assert np.array_equal(kk[:lens[r]], kept[i][r][0]) and np.array_equal(vv[:lens[r]], kept[i][r][1])
                near = 2.0 ** -4 if fp8 else 2.0 ** -8
                assert np.all(np.abs(kk[lens[r]:] - new_k[nodes]) <= near * np.abs(new_k[nodes]) + (0.02 if fp8 else 1e-4))
                assert np.all(np.abs(vv[lens[r]:] - new_v[nodes]) <= near * np.abs(new_v[nodes]) + (0.01 if fp8 else 0))
                if not fp8:  # the attention saw all new rows, the ones not kept among them: their values are known exactly here
                    bf = lambda x: torch.from_numpy(x).bfloat16().double().numpy()  # noqa: E731
                    ak, av = np.concatenate([kept[i][r][0], bf(new_k)]), np.concatenate([kept[i][r][1], bf(new_v)])
                    for h in range(H):
                        ref, wt = paged_ref.attend(host(q[i])[a:a + m, h], ak[:, h // 3], av[:, h // 3], seen, DH ** -0.5)
                        # (a rotated key may round to bf16 one step off what the formula in 64 bits rounds to: 2^-8 of a score of
                        # at most 60, as a part of 2^-2 of the weights, in rare dims: within twice the tolerance)
                        assert np.all(np.abs(host(o[i])[a:a + m, h] - ref) <= 2 * paged_ref.attention_tolerance(wt) + 1e-3)
                kept[i][r] = [kk, vv]
        assert (q[:, n:] == 3.0).all() and (o[:, n:] == 3.0).all()

    def pages_add_up():
        used = {p for r in range(RR) for p in table[r, :int(held[r])].tolist()}
        assert used | set(free[:int(n_free)].tolist()) == set(range(POOL)) and len(used) + int(n_free) == POOL

    step([20, 9, 0, 0])
    step([12, 1, 0, 0])
    step([5, 32, 0, 0])
    pages_add_up()
    # request 0 goes on as two more, whole and without its first page
    n0 = len(kept[0][0][0])
    first = min(1, n0 // PS)
    copies, one = i32(2, 3), lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    # (the last turn's surplus pages first, so that the fork finds them)
    collected, some = i32(1), i32(RR)
    w.wam_page_collect(cache_len, held, table, free, some, collected, st2, page_size=PS)
    held.copy_(some), n_free.copy_(collected)
    w.wam_page_fork(one(0, 0), one(2, 3), one(0, first), one(n0, n0 - first * PS), held, n_free, table, free, held2, n_free2, copies, st2,
                    page_size=PS)
    for _, _, _, cache in layers:
        w.wam_page_copy(cache, copies)
    held.copy_(held2), n_free.copy_(n_free2)
    put(cache_len, [n0, len(kept[0][1][0]), n0, n0 - first * PS])
    torch.cuda.synchronize()
    assert st2.tolist() == [0, 0]
    for i in range(2):
        for r, skip in ((2, 0), (3, first * PS)):
            kept[i][r] = [x[skip:] for x in kept[i][0]]
            assert all(np.array_equal(x, y) for x, y in zip(stored(i, r, n0 - skip), kept[i][r]))
    pages_add_up()
    # each grows on its own; what they share stays as it was
    step([6, 2, 11, 4])
    # request 0 ends: the pages that 2 and 3 share with it stay, the rest is free; then the plan has nothing to take back
    cache_len[0] = 0
    for i in range(2):
        kept[i][0] = [x[:0] for x in kept[i][0]]
    w.wam_page_collect(cache_len, held, table, free, some, collected, st2, page_size=PS)
    held.copy_(some), n_free.copy_(collected)
    torch.cuda.synchronize()
    assert st2.tolist() == [0, 0] and held[0] == 0
    pages_add_up()
    step([0, 3, 9, 9])
    pages_add_up()
