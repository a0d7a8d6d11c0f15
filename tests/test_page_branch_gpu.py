"""Forks, copies, collections and compactions of a paged cache against their plain definitions, bit for bit."""
import numpy as np
import pytest

import branch_ref
import paged_ref
from gpu_helpers import log
from paged_ref import Batch

pytestmark = pytest.mark.gpu
OLD = 77


def i32(x):
    import torch
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def wide_table(table, gap):
    """The table on the device with `gap` entries between its rows."""
    import torch
    R, width = table.shape
    big = torch.full((R, width + gap), OLD, dtype=torch.int32, device="cuda")
    big[:, :width] = i32(table)
    return big, big[:, :width]


# ---- fork ----
def run_fork(src, dst, first, length, held, n_free, table, free_list, ps, gap=3):
    import torch
    import paper_2602_15922_amd as w
    R, N = len(held), len(src)
    old = lambda *s: torch.full(s, OLD, dtype=torch.int32, device="cuda")  # noqa: E731
    big, t = wide_table(table, gap)
    held_out, n_out, copies, status, stack = old(R + 1), old(2), old(N + 1, 3), old(3), i32(free_list)
    for _ in range(2):  # (again on the same inputs: the same)
        w.wam_page_fork(i32(src), i32(dst), i32(first), i32(length), i32(held), i32([n_free]), t, stack, held_out[:R], n_out[:1], copies[:N],
                        status[:2], page_size=ps)
    torch.cuda.synchronize()
    for x in (held_out[R:], n_out[1:], copies[N:], status[2:], big[:, table.shape[1]:]):
        assert (x == OLD).all()
    assert np.array_equal(stack.cpu().numpy(), free_list)
    return dict(table=t.cpu().numpy(), held_out=held_out[:R].tolist(), n_free_out=n_out[:1].tolist(), copies=copies[:N].cpu().numpy(),
                status=status[:2].tolist())


def same(got, want):
    for name, x in want.items():
        assert np.array_equal(got[name], x), (name, got[name], x)


def fork_case(seed, R, forks, ps, width, spare, wrong=0.0):
    """R requests with histories and `forks` empty rows; some of the forks are wrong in one way or another."""
    g = np.random.default_rng(seed)
    held = np.concatenate([g.integers(0, width + 1, R), np.zeros(forks, int)])
    n_pages = int(held.sum()) + spare
    ids = g.permutation(n_pages)
    table, at = np.full((R + forks, width), -1, np.int32), 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    free = np.full(n_pages, -1, np.int32)
    free[:n_pages - at] = ids[at:]
    src, dst = g.integers(0, R, forks), R + g.permutation(forks)
    first = np.array([g.integers(0, held[s] + 1) for s in src])
    length = np.array([g.integers(0, (held[s] - f) * ps + 1) for s, f in zip(src, first)])
    for i in range(forks):
        if g.random() < wrong:
            kind = g.integers(0, 7)
            if kind == 0:
                src[i] = g.choice([-1, R + forks, 2 ** 31 - 1, -2 ** 31])
            elif kind == 1:
                dst[i] = g.choice([-1, R + forks, -2 ** 31])
            elif kind == 2:
                dst[i] = dst[g.integers(0, forks)]
            elif kind == 3:
                length[i] = (held[src[i]] - first[i]) * ps + 1
            elif kind == 4:
                first[i] = g.choice([-1, width, 2 ** 31 - 1])
            elif kind == 5:
                length[i] = g.choice([-1, 2 ** 31 - 1])
            else:
                dst[i] = g.integers(0, R)
    return src, dst, first, length, held, n_pages - at, table, free, ps, n_pages


@pytest.mark.parametrize("R,forks,ps,width,spare,wrong", [
    (1, 1, 16, 4, 3, 0), (1, 8, 64, 300, 20, 0), (3, 7, 48, 9, 0, 0), (5, 40, 16, 20, 10, 0.4), (40, 300, 32, 3, 500, 0.2),
    (90, 1200, 16, 6, 900, 0.1), (20, 4076, 16, 2, 1000, 0.3)])
def test_fork(R, forks, ps, width, spare, wrong):
    for seed in (1, 2):
        case = fork_case(seed, R, forks, ps, width, spare, wrong)
        log(f"fork R={R} forks={forks} ps={ps} width={width} spare={spare} wrong={wrong}")
        same(run_fork(*case[:-1]), branch_ref.fork(*case))


def test_fork_without_first_and_without_forks():
    src, dst, first, length, held, n_free, table, free, ps, n_pages = fork_case(5, 4, 6, 16, 8, 9)
    length = np.array([held[s] * ps for s in src]) - np.array([0, 1, 0, 5, 15, 16])
    length = np.maximum(length, 0)
    log("fork without first")
    case = (src, dst, None, length, held, n_free, table, free, ps)
    same(run_fork(*case), branch_ref.fork(*case, n_pages))
    log("fork of nothing")
    case = (src[:0], dst[:0], None, length[:0], held, n_free, table, free, ps)
    same(run_fork(*case), branch_ref.fork(*case, n_pages))


def test_fork_counts_out_of_range():
    src, dst, first, length, held, n_free, table, free, ps, n_pages = fork_case(6, 4, 6, 16, 8, 9)
    for n, h0 in ((-5, 3), (10 ** 9, 3), (n_free, -7), (n_free, 2 ** 31 - 1), (2, 10 ** 6)):
        held = held.copy()
        held[0] = h0
        log(f"fork n_free={n} held={h0}")
        case = (src, dst, first, np.minimum(length, 16), held, n, table, free, ps)
        same(run_fork(*case), branch_ref.fork(*case, n_pages))


def test_a_request_is_source_and_target_of_nothing():
    """A row without pages may be forked (no tokens) while another fork fills it."""
    table = np.array([[3, 4, 5], [-1, -1, -1], [-1, -1, -1]], np.int32)
    case = ([0, 1], [1, 2], [1, 0], [20, 0], [3, 0, 0], 2, table, np.array([7, 8, 0, 0, 0, 0, 0, 0, 0], np.int32), 16)
    log("fork chain")
    same(run_fork(*case), branch_ref.fork(*case, 9))


# ---- copy ----
@pytest.mark.parametrize("Hkv,Dh,ps,layout,fp8", [(1, 64, 16, "nhd", False), (3, 128, 48, "hnd", False), (40, 128, 64, "kv", False),
                                                  (5, 64, 1024, "nhd", False), (1, 128, 16, "kv", True), (7, 128, 32, "hnd", True), (16, 128, 64, "nhd", True)])
def test_copy(Hkv, Dh, ps, layout, fp8):
    import torch
    import paper_2602_15922_amd as w
    b = Batch([(1, 5 * ps), (1, 3 * ps)], Hkv, Hkv, Dh, ps, seed=Hkv + ps, junk=1.5, fp8=fp8, layout=layout, spare=3)
    p = [int(x) for x in b.table.flatten() if x >= 0]
    left = [x for x in range(b.n_pages) if x not in p]
    copies = [(p[0], left[0], ps), (p[1], left[1], 1), (p[2], left[2], ps - 3), (p[0], p[3], 7), (p[0], p[4], 0), (-1, p[5], 5), (p[0], b.n_pages, 5),
              (b.n_pages, p[5], 5), (p[0], -1, 2), (p[5], p[6], 10 ** 9), (p[5], p[7], -4), (2 ** 31 - 1, -2 ** 31, ps)]
    log(f"copy Hkv={Hkv} Dh={Dh} ps={ps} {layout} fp8={fp8}")
    c = b.cache()
    w.wam_page_copy(c, i32(copies))
    torch.cuda.synchronize()
    for host, dev in ((b.k, b.dk), (b.v, b.dv), (b.k_exp, b.dex)):
        if host is None:
            continue
        want = host.clone() if host.dim() == 4 and host is not b.k_exp else host.view(torch.int32).squeeze(-1).clone()
        for s, d, n in copies:
            if 0 <= s < b.n_pages and 0 <= d < b.n_pages and n > 0:
                want[d, :min(n, ps)] = want[s, :min(n, ps)]
        assert torch.equal(dev.cpu().contiguous().view(torch.uint8), want.contiguous().view(torch.uint8))


# ---- collect ----
def run_collect(cache_len, held, table, n_pages, ps, gap=3):
    import torch
    import paper_2602_15922_amd as w
    R = len(held)
    old = lambda n: torch.full((n,), OLD, dtype=torch.int32, device="cuda")  # noqa: E731
    big, t = wide_table(table, gap)
    free, held_out, n_out, status = old(n_pages + 1), old(R + 1), old(2), old(3)
    w.wam_page_collect(i32(cache_len), i32(held), t, free[:n_pages], held_out[:R], n_out[:1], status[:2], page_size=ps)
    torch.cuda.synchronize()
    for x in (free[n_pages:], held_out[R:], n_out[1:], status[2:], big[:, table.shape[1]:]):
        assert (x == OLD).all()
    return dict(free_list=free[:n_pages].cpu().numpy(), held_out=held_out[:R].tolist(), n_free_out=n_out[:1].tolist(), status=status[:2].tolist())


@pytest.mark.parametrize("R,width,ps,n_pages", [
    (0, 4, 16, 50), (1, 1, 16, 1), (3, 5, 64, 20), (3, 5, 64, 0), (7, 40, 16, 31), (7, 40, 16, 32), (7, 40, 16, 33), (50, 300, 48, 9000), (16, 64, 16, 32767),
    (16, 64, 16, 32769), (1030, 20, 16, 40000), (4096, 3, 32, 20000), (5, 2000, 16, 155648), (90, 2000, 16, 155649), (5, 2000, 16, 300001),
    (3, 4, 16, 1 << 20), (40, 3001, 16, 700007)])
def test_collect(R, width, ps, n_pages):
    g = np.random.default_rng(R + width)
    held = g.integers(0, width + 1, R)
    table = g.integers(0, max(n_pages, 1), (R, width)).astype(np.int32)  # pages shared at random
    cache_len = np.where(g.random(R) < 0.2, 0, g.integers(0, width * ps + 200, R))
    free = np.full(n_pages, OLD, np.int32)
    for wrong in (False, True):
        if wrong and R:
            table[g.random(table.shape) < 0.1] = -1
            table[0, 0], table[-1, -1] = n_pages, -2 ** 31
            held[0], held[-1] = -3, 10 ** 9
            cache_len[R // 2] = -1
        log(f"collect R={R} width={width} ps={ps} n_pages={n_pages} wrong={wrong}")
        same(run_collect(cache_len, held, table, n_pages, ps), branch_ref.collect(cache_len, held, table, free, ps, n_pages))


# ---- compact ----
def run_compact(b, keep, n_keep, q_len=None, q_start=None, kv_len=None, table=None, T=None):
    import torch
    import paper_2602_15922_amd as w
    c = b.cache()
    w.wam_cache_compact(c, i32(b.table if table is None else table), i32(b.q_start if q_start is None else q_start),
                        i32(b.kv_len if kv_len is None else kv_len), i32(keep), i32(n_keep), q_len=i32(q_len))
    torch.cuda.synchronize()


def check_compact(b, keep, n_keep, q_len=None, q_start=None, kv_len=None, table=None):
    import torch
    run_compact(b, keep, n_keep, q_len, q_start, kv_len, table)
    pick = lambda x, y: y if x is None else x  # noqa: E731
    for host, dev in ((b.k, b.dk), (b.v, b.dv), (b.k_exp, b.dex)):
        if host is None:
            continue
        x = host.view(torch.int32).squeeze(-1) if host is b.k_exp else host
        want = branch_ref.compact(x, pick(table, b.table), pick(q_start, b.q_start), q_len, pick(kv_len, b.kv_len), keep, n_keep, b.ps)
        assert torch.equal(dev.cpu().contiguous().view(torch.uint8), want.contiguous().view(torch.uint8))


def keeps(b, g, share):
    keep, n_keep = np.full(b.T, 10 ** 9, np.int64), []
    for at, (n, _) in zip(b.q_start, b.lens):
        m = int(g.integers(0, n + 1)) if share is None else min(n, max(0, int(round(n * share))))
        keep[at:at + m] = np.sort(g.permutation(n)[:m])
        n_keep.append(m)
    return keep, np.array(n_keep)


@pytest.mark.parametrize("Hkv,Dh,ps,layout,fp8", [(1, 64, 16, "nhd", False), (3, 128, 48, "hnd", False), (5, 128, 16, "kv", False), (2, 64, 64, "kv", False),
                                                  (2, 128, 16, "nhd", True), (3, 128, 32, "hnd", True), (1, 128, 48, "kv", True)])
def test_compact(Hkv, Dh, ps, layout, fp8):
    lens = [(1, 1), (7, 40), (0, 30), (16, 16), (17, 60), (33, 200), (130, 131), (300, 420), (64, 65)]
    g = np.random.default_rng(ps)
    for share in (None, 0.0, 1.0, 0.9, 0.1):
        b = Batch(lens, Hkv, Hkv, Dh, ps, seed=Hkv + Dh, junk=2.5, fp8=fp8, layout=layout)
        log(f"compact Hkv={Hkv} Dh={Dh} ps={ps} {layout} fp8={fp8} share={share}")
        check_compact(b, *keeps(b, g, share))


@pytest.mark.parametrize("n,m,fp8", [(3000, 1500, False), (2000, 1999, True), (1000, 1, False)])
def test_compact_long_lists(n, m, fp8):
    """More rows than a workgroup holds at once: each group's targets are the next ones' sources."""
    g = np.random.default_rng(n)
    b = Batch([(n, n + 37)], 2, 2, 128, 16, seed=n, junk=0.5, fp8=fp8)
    keep = np.zeros(b.T, int)
    keep[:m] = np.sort(g.permutation(n)[:m])
    log(f"compact long {n} {m} fp8={fp8}")
    check_compact(b, keep, [m])
    keep[:m] = n - m + np.arange(m)  # the last m: a plain shift
    check_compact(b, keep, [m])


def test_compact_padded_absent_and_out_of_range():
    g = np.random.default_rng(3)
    lens = [(9, 30), (0, 9), (40, 200), (5, 3), (20, 20)]
    b = Batch(lens, 2, 2, 64, 16, seed=4, junk=1.0, gap=4)
    keep, n_keep = keeps(b, g, 0.6)
    log("compact padded")
    check_compact(b, keep, n_keep, q_len=b.q_len)
    table = b.table.copy()
    table[2, 11], table[2, 5], table[4, 1] = -1, b.n_pages, 2 ** 31 - 1
    log("compact absent pages")
    check_compact(b, keep, n_keep, q_len=b.q_len, table=table)
    keep[2::7] = [-1, 10 ** 9, -2 ** 31, 2 ** 31 - 1, 41, 50, 60, 70, 80, 90, 5, 7, 9, 11][:len(keep[2::7])]
    log("compact numbers out of range")
    run_compact(b, np.clip(keep, -2 ** 31, 2 ** 31 - 1), n_keep, q_len=b.q_len)
    for n in ([10 ** 9] * 5, [-3] * 5):
        log(f"compact n_keep {n}")
        run_compact(b, np.arange(b.T), n, q_len=b.q_len)
    for starts in ([0, 9, 9, 40, 10 ** 9, 10 ** 9], [-100, 5, 5, 45, 46, 50], [90, 80, 70, 60, 50, 40]):
        for kv in (b.kv_len, [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
            log(f"compact starts {starts} kv {kv}")
            run_compact(b, np.arange(b.T)[::-1].copy(), [3, 50, 50, 50, 50], q_start=starts, kv_len=kv)


@pytest.mark.parametrize("n", [9, 700, 3000])
def test_compact_of_any_list(n):
    """Numbers in any order, again and again the same, out of range: those past their place move, as all rows were before."""
    g = np.random.default_rng(n)
    b = Batch([(n, n + 100)], 2, 2, 128, 16, seed=7, junk=1.0)
    keep = g.integers(-5, n + 5, b.T)
    log(f"compact any list {n}")
    check_compact(b, keep, [n])
    keep[:] = n - 1
    check_compact(b, keep, [n])


def test_offsets_past_32_bits():
    """Pages whose rows lie more than 4 GiB apart."""
    import torch
    import paper_2602_15922_amd as w
    b = Batch([(33, 50)], 1, 1, 128, 16, seed=14, junk=1.0, spare=3)
    n, span = b.n_pages, 400_000_000
    log("copy and compact far pages")
    big = torch.empty(n * span, dtype=torch.bfloat16, device="cuda")
    k = torch.as_strided(big, (n, 16, 1, 128), (span, 128, 128, 1))
    v = torch.as_strided(big, (n, 16, 1, 128), (span, 128, 128, 1), storage_offset=16 * 128)
    k.copy_(b.k), v.copy_(b.v)
    c = w.make_paged_cache(k, v)
    keep = [1, 5, 20, 30, 32] + [0] * 31
    src, dst = int(b.table[0, 0]), [x for x in range(n) if x not in b.table[0]][-1]
    copies = [(src, dst, 13)]
    w.wam_cache_compact(c, i32(b.table), i32(b.q_start), i32(b.kv_len), i32(keep), i32([5]))
    w.wam_page_copy(c, i32(copies))
    torch.cuda.synchronize()
    for host, dev in ((b.k, k), (b.v, v)):
        want = branch_ref.compact(host, b.table, b.q_start, None, b.kv_len, keep, [5], 16)
        want[dst, :13] = want[src, :13]
        assert torch.equal(dev.cpu(), want)
    del big, k, v
    torch.cuda.empty_cache()
