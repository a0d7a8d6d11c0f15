"""wam_page_plan against the plan made step by step with a Python list as the stack (equal, entry for entry)."""
import numpy as np
import pytest

import paged_ref
from gpu_helpers import log

pytestmark = pytest.mark.gpu
NAMES = ("table", "free_list", "held_out", "n_free_out", "q_start", "kv_len", "slots", "token_pos", "status")


def run(cache, new, held, free, n_free, table, ps, n_pages, T, outs=None, stride=None, stream=None):
    import torch
    import paper_2602_15922_amd as w
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    R, width = table.shape
    d = dict(cache=i32(cache), new=i32(new), held=i32(held), n_free=i32([n_free]), free_list=i32(free),
             held_out=i32([-7] * R), n_free_out=i32([-7]), q_start=i32([-7] * (R + 1)), kv_len=i32([-7] * R),
             slots=i32([-7] * T), token_pos=i32([-7] * T), status=i32([-7] * 4))
    wide = torch.full((R, stride or width), -9, dtype=torch.int32, device="cuda")
    d["table"] = wide[:, :width]
    d["table"].copy_(i32(table))

    def call():
        w.wam_page_plan(d["cache"], d["new"], d["held"], d["n_free"], d["table"], d["free_list"], d["held_out"],
                        d["n_free_out"], d["q_start"], d["kv_len"], d["slots"], d["status"], page_size=ps,
                        token_pos=d["token_pos"])
    call()
    torch.cuda.synchronize()
    if stride:
        assert (wide[:, width:] == -9).all()
    return {n: d[n].cpu().numpy() for n in NAMES}, d, call


def check(got, ref):
    for n in NAMES:
        assert np.array_equal(got[n], np.asarray(ref[n])), n


def case(R, ps, seed, lo=0, hi=400, new_hi=60, ends=0.2, spare=5, width=None):
    g = np.random.default_rng(seed)
    cache, new = g.integers(lo, hi + 1, R), g.integers(0, new_hi + 1, R)
    held = -(-cache // ps) + g.integers(0, 2, R) * (g.random(R) < 0.3)
    over = g.random(R) < ends
    cache[over], new[over] = 0, 0
    need = -(-(cache + new) // ps)
    width = width or max(1, int(max(need.max(initial=0), held.max(initial=0))))
    held = np.minimum(held, width)
    free = max(0, int((need - held).sum())) + spare
    n_pages = int(held.sum()) + free
    ids = g.permutation(n_pages)
    table = np.full((R, width), -1, np.int32)
    for r in range(R):
        table[r, :held[r]], ids = ids[:held[r]], ids[held[r]:]
    stack = np.full(n_pages, -3, np.int32)
    stack[:free] = ids
    return cache, new, held, stack, free, table, ps, n_pages, int(new.sum()) + 9


@pytest.mark.parametrize("R,ps,kw", [
    (1, 16, {}), (3, 64, {}), (64, 16, {}), (65, 48, dict(ends=0.6)), (1000, 16, {}), (1025, 112, dict(new_hi=3)),
    (2500, 16, dict(hi=40, new_hi=1)), (4096, 16, dict(hi=30, new_hi=9)), (7, 16, dict(hi=9000, new_hi=9000, lo=1)),
    (20, 16, dict(ends=1.0)), (20, 1024, dict(hi=0, new_hi=5000))])
def test_plan(R, ps, kw):
    import torch
    for seed in range(3):
        log(f"plan R={R} ps={ps} {kw} seed={seed}")
        c = case(R, ps, seed, **kw)
        got, d, call = run(*c, stride=c[5].shape[1] + 3)
        ref = paged_ref.plan(*c)
        check(got, ref)
        call()  # the same inputs again: the same result
        torch.cuda.synchronize()
        check({n: d[n].cpu().numpy() for n in NAMES}, ref)


def test_short_stack_narrow_table_and_too_many_rows():
    for seed in range(4):
        log(f"plan short seed={seed}")
        cache, new, held, stack, free, table, ps, n_pages, T = case(40, 16, 50 + seed, ends=0.05 * seed)
        for n in (0, 1, free // 3):
            c = (cache, new, held, stack, n, table, ps, n_pages, T)
            ref = paged_ref.plan(*c)
            check(run(*c)[0], ref)
        c = (cache, new, held, stack, free, table, ps, n_pages, T // 2)
        check(run(*c)[0], paged_ref.plan(*c))
    c = case(30, 16, 77, hi=300, width=12)
    assert paged_ref.plan(*c)["status"][1] > 0
    check(run(*c)[0], paged_ref.plan(*c))


def test_invalid_device_values_are_cut_to_their_ranges():
    log("plan invalid values")
    cache, new, held, stack, free, table, ps, n_pages, T = case(12, 16, 5)
    cache, new, held = cache.copy(), new.copy(), held.copy()
    cache[1], new[2], held[3], held[4] = -5, -2147483648, -1, 1 << 30
    c = (cache, new, held, stack, n_pages + 9, table, ps, n_pages, T)
    ref = paged_ref.plan(*c)
    assert ref["status"][3] == 5
    check(run(*c)[0], ref)
    # entries of the table that are no pages: their tokens have no slot
    cache, new, held, stack, free, table, ps, n_pages, T = case(12, 16, 6, ends=0.0)
    table = table.copy()
    table[0, 0], table[5, : held[5]] = n_pages, -17
    c = (cache, new, held, stack, free, table, ps, n_pages, T)
    check(run(*c)[0], paged_ref.plan(*c))
    # lengths at the end of their type
    big = np.array([2147483647, 0, 2147483647]), np.array([2147483647, 3, 0])
    c = (*big, np.array([1, 0, 0]), np.arange(8, dtype=np.int32), 7, np.array([[7, -1], [-1, -1], [-1, -1]], np.int32), 16, 8, 10)
    ref = paged_ref.plan(*c)
    got = run(*c)[0]
    for n in ("table", "held_out", "n_free_out", "q_start", "slots", "free_list"):
        assert np.array_equal(got[n], np.asarray(ref[n])), n
    assert got["kv_len"].tolist() == [min(x, 2147483647) for x in ref["kv_len"]]


def test_no_requests_and_no_rows():
    import torch
    import paper_2602_15922_amd as w
    log("plan R=0")
    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    free, n_free, q_start, slots, status, n_out = i32(4), torch.zeros(1, dtype=torch.int32, device="cuda"), i32(1), i32(5), i32(4), i32(1)
    w.wam_page_plan(i32(0), i32(0), i32(0), n_free, i32(0, 0), free, i32(0), n_out, q_start, i32(0), slots, status, page_size=16)
    torch.cuda.synchronize()
    assert q_start.tolist() == [0] and slots.tolist() == [-1] * 5 and status.tolist() == [0] * 4 and n_out.tolist() == [0]
    c = list(case(9, 16, 3))
    c[8] = 0
    log("plan T=0")
    check(run(*c)[0], paged_ref.plan(*c))


def test_replayed_from_a_graph_with_other_lengths():
    import torch
    log("plan graph")
    a = case(33, 16, 11)
    got, d, call = run(*a)
    table0, list0 = torch.tensor(a[5], device="cuda"), torch.tensor(a[3], dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            call()
    for k in range(3):
        new = np.maximum(a[1] - k, 0)
        d["new"].copy_(torch.tensor(new, dtype=torch.int32))
        d["table"].copy_(table0)
        d["free_list"].copy_(list0)
        g.replay()
        torch.cuda.synchronize()
        c = (a[0], new, *a[2:])
        check({n: d[n].cpu().numpy() for n in NAMES}, paged_ref.plan(*c))
