"""wam_page_plan with buffers side by side: all of them in one allocation, some between the table's rows, two inputs in one."""
import numpy as np
import pytest

import paged_ref
from gpu_helpers import log
from test_page_plan_gpu import NAMES, case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,gap", [(1, 0), (9, 40), (40, 3)])
def test_neighbouring_buffers(R, gap):
    import torch
    import paper_2602_15922_amd as w
    cache, new, held, stack, n_free, table, ps, n_pages, T = case(R, 16, 90 + R, hi=120, new_hi=9)
    width = table.shape[1]
    log(f"plan neighbours R={R} gap={gap}")
    sizes = dict(cache=R, new=R, held=R, n_free=1, free_list=n_pages, held_out=R, n_free_out=1, q_start=R + 1, kv_len=R,
                 slots=T, token_pos=T, status=4)
    big = torch.full((R * (width + gap) + sum(sizes.values()),), -9, dtype=torch.int32, device="cuda")
    wide = big[:R * (width + gap)].view(R, width + gap)
    d, at = {"table": wide[:, :width]}, R * (width + gap)
    for n, k in sizes.items():
        if gap >= R and n in ("held_out", "held", "kv_len"):  # behind the first rows of the table
            row = ("held_out", "held", "kv_len").index(n)
            d[n] = wide[row, width:width + k]
        else:
            d[n], at = big[at:at + k], at + k
    for n, x in (("cache", cache), ("new", new), ("held", held), ("n_free", [n_free]), ("free_list", stack), ("table", table)):
        d[n].copy_(torch.tensor(np.asarray(x), dtype=torch.int32))
    w.wam_page_plan(d["cache"], d["new"], d["held"], d["n_free"], d["table"], d["free_list"], d["held_out"], d["n_free_out"],
                    d["q_start"], d["kv_len"], d["slots"], d["status"], page_size=ps, token_pos=d["token_pos"])
    torch.cuda.synchronize()
    check({n: d[n].cpu().numpy() for n in NAMES}, paged_ref.plan(cache, new, held, stack, n_free, table, ps, n_pages, T))
    assert d["cache"].tolist() == list(cache) and d["new"].tolist() == list(new) and d["held"].tolist() == list(held)


def test_two_inputs_in_one_buffer():
    """As many new tokens as there are kept ones."""
    import torch
    import paper_2602_15922_amd as w
    R, ps, n_pages, T = 6, 16, 40, 200
    n = np.array([0, 3, 17, 33, 1, 40])
    held = -(-n // ps)
    table = np.full((R, 8), -1, np.int32)
    ids = iter(range(n_pages))
    for r in range(R):
        table[r, :held[r]] = [next(ids) for _ in range(held[r])]
    free = list(ids)
    stack = np.full(n_pages, -3, np.int32)
    stack[:len(free)] = free
    log("plan cache_len is new_len")
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    d = dict(table=i32(table), free_list=i32(stack), held_out=i32([0] * R), n_free_out=i32([0]), q_start=i32([0] * (R + 1)),
             kv_len=i32([0] * R), slots=i32([0] * T), token_pos=i32([0] * T), status=i32([0] * 4))
    lens = i32(n)
    w.wam_page_plan(lens, lens, i32(held), i32([len(free)]), d["table"], d["free_list"], d["held_out"], d["n_free_out"],
                    d["q_start"], d["kv_len"], d["slots"], d["status"], page_size=ps, token_pos=d["token_pos"])
    torch.cuda.synchronize()
    check({k: d[k].cpu().numpy() for k in NAMES}, paged_ref.plan(n, n, held, stack, len(free), table, ps, n_pages, T))
