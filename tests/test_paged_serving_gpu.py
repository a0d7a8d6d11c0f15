"""The paged operators as a server runs them: three robots' requests over several turns, each turn the page plan, the
rotary append of the new tokens, the attention over the pages and the cross-attention to instructions of their own
lengths; requests end and new ones take their pages.  The oracle is each request's whole history in 64 bits."""
import numpy as np
import pytest

import paged_ref
from gpu_helpers import host, log, workspace

pytestmark = pytest.mark.gpu
H, HKV, DH, PS, PAIRS, POOL, WIDTH, T = 6, 2, 128, 16, [22, 21, 21], 24, 12, 160


@pytest.mark.parametrize("fp8,graph", [(False, False), (False, True), (True, False)])
def test_turns_of_three_requests(fp8, graph):
    import torch
    import paper_2602_15922_amd as w
    log(f"serving fp8={fp8} graph={graph}")
    g = torch.Generator().manual_seed(5)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    kind = torch.uint8 if fp8 else torch.bfloat16
    k, v = (torch.full((POOL, PS, HKV, DH), 0x7F, dtype=torch.uint8, device="cuda") if fp8 else
            torch.full((POOL, PS, HKV, DH), float("nan"), dtype=kind, device="cuda") for _ in range(2))
    ex = i32(POOL, PS, HKV) if fp8 else None
    v_scale = 6.0 / 448
    cache = w.make_paged_cache(k, v, k_exp=ex, v_scale=v_scale)
    cache_len, new_len, held, held2, kv_len = (i32(3) for _ in range(5))
    n_free, n_free2, q_start, slots, status = i32(1), i32(1), i32(4), i32(T), i32(4)
    table, free = i32(3, WIDTH) - 1, torch.randperm(POOL, generator=g).int().cuda()
    n_free.fill_(POOL)
    qkv, pos = torch.zeros(T, (H + 2 * HKV) * DH, dtype=torch.bfloat16, device="cuda"), i32(T, 3)
    q = torch.zeros(T, H, DH, dtype=torch.bfloat16, device="cuda")
    o, x = torch.zeros_like(q), torch.zeros_like(q)
    text_len = [9, 0, 40]
    text = torch.randn(3, 40, 2, HKV, DH, generator=g).bfloat16()
    dtext = text.cuda().flatten(0, 1)
    k_start, k_len = torch.tensor([0, 40, 80], dtype=torch.int32).cuda(), torch.tensor(text_len, dtype=torch.int32).cuda()
    ws = workspace(w.wam_attn_paged_workspace_bytes(cache, R=3, T=T, Hq=H, max_kv=WIDTH * PS))
    ws2 = workspace(w.wam_attn_cross_workspace_bytes(R=3, T=T, Hq=H, Hkv=HKV, Dh=DH, max_k=40))

    def turn():
        w.wam_page_plan(cache_len, new_len, held, n_free, table, free, held2, n_free2, q_start, kv_len, slots, status,
                        page_size=PS)
        w.wam_rope_qkv_paged(cache, qkv, pos, slots, q, pairs=PAIRS)
        w.wam_attn_paged(cache, q, table, q_start, kv_len, o, ws, chunk=0)
        w.wam_attn_cross(o, dtext[:, 0], dtext[:, 1], q_start, k_start, x, ws2, max_k=40, k_len=k_len)
        held.copy_(held2)
        n_free.copy_(n_free2)

    cg = None
    history = [np.zeros((0, H + 2 * HKV, DH)) for _ in range(3)]
    hpos = [np.zeros((0, 3)) for _ in range(3)]
    for step, (kept, new) in enumerate([([0, 0, 0], [40, 1, 33]), ([40, 1, 33], [40, 1, 5]), ([0, 2, 38], [90, 1, 0]),
                                        ([90, 3, 0], [1, 100, 0]), ([91, 3, 0], [1, 60, 70])]):
        cache_len.copy_(torch.tensor(kept)), new_len.copy_(torch.tensor(new))
        n = sum(new)
        qkv.copy_(torch.randn(T, qkv.shape[1], generator=g).bfloat16())
        pos.copy_(torch.randint(0, 500, (T, 3), generator=g).int())
        q.fill_(3.0), o.fill_(3.0), x.fill_(3.0)
        if graph and cg is None:
            cg = torch.cuda.CUDAGraph()
            with torch.cuda.graph(cg):
                turn()
        cg.replay() if graph else turn()
        torch.cuda.synchronize()
        assert status.tolist() == [0, 0, 0, 0]
        want_pages = [-(-(a + b) // PS) for a, b in zip(kept, new)]
        assert held.tolist() == want_pages and n_free.item() == POOL - sum(want_pages)
        mine = [p for r in range(3) for p in table[r, :want_pages[r]].tolist()]
        assert sorted(mine + free[:n_free.item()].tolist()) == list(range(POOL))  # no page lost or given twice
        rows, at = host(qkv).reshape(T, -1, DH), 0
        for r in range(3):
            now = slice(at, at + new[r])
            history[r] = np.concatenate([history[r][:kept[r]], rows[now]])
            hpos[r] = np.concatenate([hpos[r][:kept[r]], pos.cpu().numpy()[now]])
            y = paged_ref.rotate(history[r][:, :H + HKV], paged_ref.angles(hpos[r], PAIRS, 10000.0), False)
            m = len(y)
            for h in range(H):
                # the operands as they are stored: q and K rounded once (bf16; the FP8 cache's codes, read back)
                qq = host(q)[now, h]
                ids = table[r, :want_pages[r]].long()
                if fp8:
                    code = lambda t: paged_ref.E4M3[t[ids].cpu().numpy()].reshape(-1, HKV, DH)[:m, h // 3]  # noqa: E731
                    e = (ex[ids].cpu().numpy().reshape(-1, HKV)[:m, h // 3].astype(np.int64)[:, None] >> (8 * np.arange(4))) & 255
                    kk, vv = code(k) * np.repeat(2.0 ** (e - 127.0), 32, 1), code(v) * float(np.float32(v_scale))
                    assert np.all(np.abs(kk - y[:, H + h // 3]) <= 2.0 ** -4 * np.abs(kk) + 2.0 ** -10 * 2.0 ** (np.repeat(e, 32, 1) - 127.0) + 1e-4)
                else:
                    kk, vv = (host(t[ids]).reshape(-1, HKV, DH)[:m, h // 3] for t in (k, v))
                    assert np.all(np.abs(kk - y[:, H + h // 3]) <= 2.0 ** -8 * np.abs(kk) + 1e-4)
                    assert np.array_equal(vv, history[r][:, H + HKV + h // 3])
                ref, a = paged_ref.attend(qq, kk, vv, np.ones((new[r], m), bool), DH ** -0.5)
                assert np.all(np.abs(host(o)[now, h] - ref) <= paged_ref.attention_tolerance(a)), (step, r, h)
                tk, tv = (text[r, :text_len[r], i, h // 3].double().numpy() for i in (0, 1))
                ref, a = paged_ref.attend(host(o)[now, h], tk, tv, np.ones((new[r], text_len[r]), bool), DH ** -0.5)
                assert np.all(np.abs(host(x)[now, h] - ref) <= paged_ref.attention_tolerance(a)), (step, r, h)
            at += new[r]
        for t in (q, o, x):
            assert (t[n:] == 3.0).all()
