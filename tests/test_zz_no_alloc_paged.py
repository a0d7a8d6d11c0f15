"""The paged operators allocate nothing: neither the device's free memory nor torch's allocator moves over many calls, the
split and joined forms among them."""
import pytest

from gpu_helpers import log, workspace
from paged_ref import Batch

pytestmark = pytest.mark.gpu


def test_the_paged_operators_allocate_nothing():
    import torch
    import paper_2602_15922_amd as w
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    b = Batch([(1, 1500), (40, 900), (2, 300)], 8, 2, 128, 16, seed=3)
    c, q, o = b.cache(), b.q.cuda(), torch.zeros(b.T, 8, 128, dtype=torch.bfloat16, device="cuda")
    table, starts, kv = i32(b.table), i32(b.q_start), i32(b.kv_len)
    ws = workspace(w.wam_attn_paged_workspace_bytes(c, R=3, T=b.T, Hq=8, max_kv=b.width * 16))
    states = torch.zeros(2000, 2, 128, dtype=torch.bfloat16, device="cuda")
    k_start, k_len = i32([0, 5, 9]), i32([1900, 0, 77])
    ws2 = workspace(w.wam_attn_cross_workspace_bytes(R=3, T=b.T, Hq=8, Hkv=2, Dh=128, max_k=2000))
    qkv, pos, slots = torch.zeros(b.T, 12 * 128, dtype=torch.bfloat16, device="cuda"), i32([[7, 8]] * b.T), i32([-1] * b.T)
    zeros = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    plan = dict(cache_len=zeros(3), new_len=i32([5, 0, 9]), held=zeros(3), n_free=i32([b.n_pages]), block_table=zeros(3, b.width),
                free_list=torch.arange(b.n_pages, dtype=torch.int32, device="cuda"), held_out=zeros(3), n_free_out=zeros(1),
                q_start=zeros(4), kv_len=zeros(3), slots=zeros(b.T), status=zeros(4))
    log("paged operators, no allocation")

    def calls():
        w.wam_page_plan(**plan, page_size=16)
        w.wam_rope_qkv_paged(c, qkv, pos, slots, o, pairs=[32, 32])
        w.wam_attn_paged(c, q, table, starts, kv, o, ws, chunk=1)
        w.wam_attn_cross(q, states, states, starts, k_start, o, ws2, k_len=k_len)

    calls()  # the kernels are loaded
    torch.cuda.synchronize()
    free, made = torch.cuda.mem_get_info()[0], torch.cuda.memory_stats()["allocation.all.allocated"]
    for _ in range(50):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == made
