"""Forks whose last, partly filled page is absent in their source: absent in the fork too, so that it sees what its source sees."""
import numpy as np
import pytest

import branch_ref
from gpu_helpers import host, log, workspace
from paged_ref import Batch
from test_page_branch_gpu import fork_case, i32, run_fork, same

pytestmark = pytest.mark.gpu


def fork(src, dst, first, length, held, n_free, table, free_list, ps, n_pages):
    """branch_ref.fork, with the entries of absent last pages shared like those of whole ones: no page is taken for them."""
    short, shared = np.array(length), []
    R, width = table.shape
    for i, (s, d, n) in enumerate(zip(src, dst, length)):
        f = int(first[i]) if first is not None else 0
        if 0 <= s < R and f >= 0 and n > 0 and n % ps and f * ps + n <= min(max(held[s], 0), width) * ps:
            page = int(table[s, f + n // ps])
            if not 0 <= page < n_pages:
                short[i] -= n % ps
                shared.append((i, int(d), n // ps, page))
    out = branch_ref.fork(src, dst, first, short, held, n_free, table, free_list, ps, n_pages)
    named = [int(d) for d in dst]
    for i, d, w, page in shared:
        if 0 <= d < R and named.index(d) == i and held[d] == 0:
            out["table"][d, w] = page
            out["held_out"][d] += 1
    return out


@pytest.mark.parametrize("R,forks,ps,width,spare,wrong", [
    (1, 1, 16, 4, 3, 0), (3, 12, 48, 9, 0, 0), (5, 40, 16, 20, 10, 0.3), (40, 300, 32, 3, 60, 0.2), (90, 1200, 16, 6, 500, 0.1)])
def test_holes_in_the_sources(R, forks, ps, width, spare, wrong):
    for seed, share in ((1, 0.3), (2, 1.0), (3, 0.0)):
        src, dst, first, length, held, n_free, table, free, ps, n_pages = fork_case(seed, R, forks, ps, width, spare, wrong)
        g = np.random.default_rng(seed)
        holes = g.random(table.shape) < share
        table[holes] = g.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31], holes.sum())
        log(f"fork of holes R={R} forks={forks} ps={ps} width={width} wrong={wrong} share={share}")
        same(run_fork(src, dst, first, length, held, n_free, table, free, ps),
             fork(src, dst, first, length, held, n_free, table, free, ps, n_pages))


@pytest.mark.parametrize("fp8", [False, True])
def test_a_fork_sees_what_its_source_sees(fp8):
    """History and hole, the fork, its copies and the attention over both: the same bits (the pool's free pages hold NaN)."""
    import torch
    import paper_2602_15922_amd as w
    b = Batch([(1, 100), (1, 48)], 4, 2, 128, 16, seed=5, fp8=fp8, spare=4)
    n, width = 40, b.width  # tokens of the forks: two whole pages and half of the third
    table = np.full((4, width), -1, np.int32)
    table[:2] = b.table
    table[0, 2] = -1
    left = [p for p in range(b.n_pages) if p not in b.table]
    free = np.full(b.n_pages, -1, np.int32)
    free[:len(left)] = left
    c, t = b.cache(), i32(table)
    held_out, n_out, copies, status = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((4,), (1,), (2, 3), (2,)))
    log(f"fork and attention over a hole fp8={fp8}")
    w.wam_page_fork(i32([0, 1]), i32([2, 3]), None, i32([n, n]), i32([7, 3, 0, 0]), i32([len(left)]), t, i32(free), held_out, n_out, copies,
                    status, page_size=16)
    w.wam_page_copy(c, copies)
    q = b.q[:1].repeat(4, 1, 1).cuda()
    o = torch.zeros_like(q)
    ws = workspace(w.wam_attn_paged_workspace_bytes(c, R=4, T=4, Hq=4, max_kv=width * 16))
    w.wam_attn_paged(c, q, t, i32(np.arange(5)), i32([n] * 4), o, ws)
    torch.cuda.synchronize()
    got = host(o)
    assert np.isfinite(got).all() and np.array_equal(got[:2], got[2:])
    assert copies.tolist() == [[-1, -1, 0], [int(table[1, 2]), left[-1], 8]]
    assert held_out.tolist() == [7, 3, 3, 3] and n_out.tolist() == [len(left) - 1] and status.tolist() == [0, 0]
