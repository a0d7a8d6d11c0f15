"""The operators of requests that branch allocate nothing: neither the device's free memory nor torch's allocator moves."""
import pytest

from gpu_helpers import log, workspace
from paged_ref import Batch

pytestmark = pytest.mark.gpu


def test_the_operators_allocate_nothing():
    import torch
    import paper_2602_15922_amd as w
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    zeros = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    b = Batch([(1, 1500), (40, 900), (2, 300)], 8, 2, 128, 16, seed=3, junk=0.0)
    c, q, o = b.cache(), b.q.cuda(), torch.zeros(b.T, 8, 128, dtype=torch.bfloat16, device="cuda")
    table, starts, kv, mask = i32(b.table), i32(b.q_start), i32(b.kv_len), zeros(b.T, 2)
    ws = workspace(w.wam_attn_tree_workspace_bytes(c, R=3, T=b.T, Hq=8, max_kv=b.width * 16))
    p, q2 = torch.rand(b.T, 5000, device="cuda"), torch.rand(b.T, 5000, device="cuda")
    u, u_next, tokens, parent = torch.rand(b.T, device="cuda"), torch.rand(3, device="cuda"), zeros(b.T), zeros(b.T)
    ws2 = workspace(w.wam_verify_tree_workspace_bytes(3, b.T, 5000, True))
    path, n_path, nxt = zeros(b.T), zeros(3), zeros(3)
    held, held_out, n_free, n_out, free, copies, status = i32([3, 0, 0]), zeros(3), i32([5]), zeros(1), zeros(b.n_pages), zeros(1, 3), zeros(2)
    src, dst, length, lens, fork_table = i32([0]), i32([1]), i32([20]), i32([40, 0, 0]), zeros(3, 8)
    log("branch operators, no allocation")

    def calls():
        w.wam_page_fork(src, dst, None, length, held, n_free, fork_table, free, held_out, n_out, copies, status, page_size=16)
        w.wam_page_copy(c, copies)
        w.wam_attn_tree(c, q, table, starts, kv, mask, o, ws)
        w.wam_verify_tree(p, q2, tokens, parent, u, u_next, starts, path, n_path, nxt, ws2)
        w.wam_cache_compact(c, table, starts, kv, path, n_path)
        w.wam_page_collect(lens, held, fork_table, free, held_out, n_out, status, page_size=16)

    calls()  # the kernels are loaded
    torch.cuda.synchronize()
    now, made = torch.cuda.mem_get_info()[0], torch.cuda.memory_stats()["allocation.all.allocated"]
    for _ in range(50):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == now
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == made
