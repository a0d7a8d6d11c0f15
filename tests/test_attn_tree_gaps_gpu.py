"""wam_attn_tree with long masks and long parts of the key axis: stretches that no row of a tile sees in the middle of a part are
left out, also by the wavefronts without rows, with pages missing and values that are not finite in them and behind them.  The
definition in 64 bits, on the GPU in plain products of matrices."""
import numpy as np
import pytest

import branch_ref
import paged_ref
from gpu_helpers import log
from paged_ref import Batch
from test_attn_tree_gpu import OLD, bits_of, run_tree
from test_tree_plan import tree

pytestmark = pytest.mark.gpu
ROWS, TILE, WINDOW = 128, 64, 16  # rows of a workgroup, keys of a tile, tiles of a window


def gaps(b, sees, plan):
    """(row tiles and parts with a gap in mid-part, those of them with a whole wavefront without rows, those whose part ends in the
    gap), from the plan and the masks alone."""
    count = idle = past_end = 0
    G = b.Hq // b.Hkv
    for (n, m), seen in zip(b.lens, sees):
        hist = m - n
        for m0 in range(0, n * G, ROWS):
            rows = seen[m0 // G:(min(m0 + ROWS, n * G) - 1) // G + 1]
            new = np.flatnonzero(rows.any(0))
            if not len(new):
                continue
            first, end = hist + int(new[0]), min(m, hist + int(new[-1]) + 1)
            for start in range(0, plan["splits"] * plan["keys"], plan["keys"]):
                t0, nt = start // TILE, -(-min(end, start + plan["keys"]) // TILE)
                after = hist // TILE + 1
                gap = t0 if after <= t0 else t0 + -(-(after - t0) // WINDOW) * WINDOW
                if t0 < gap < nt and first // TILE >= gap + WINDOW:
                    count += 1
                    idle += n * G - m0 <= 96
                    past_end += gap + (first // TILE - gap) // WINDOW * WINDOW >= nt
    return count, idle, past_end


def expected(b, sees):
    """(o, weighted |v| mean) [T][Hq][Dh] on the GPU; a value that is not finite and is seen makes NaN."""
    import torch
    o, a = torch.full((b.T, b.Hq, b.Dh), OLD, dtype=torch.float64, device="cuda"), torch.zeros(b.T, b.Hq, b.Dh, dtype=torch.float64, device="cuda")
    q, G = b.q.cuda().double(), b.Hq // b.Hkv
    for r, (n, m) in enumerate(b.lens):
        at = int(b.q_start[r])
        k, v, there = b.kv64(r)
        seen = np.concatenate([np.ones((n, m - n), bool), sees[r]], 1) & there
        k, v, seen = (torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (k, v, seen))
        odd = ~v.isfinite()
        v = v.masked_fill(odd, 0.0)
        none = ~seen.any(1, keepdim=True)
        for h in range(b.Hq):
            s = torch.matmul(q[at:at + n, h], k[:, h // G].T.contiguous()) * b.Dh ** -0.5
            s = s.masked_fill(~seen, -np.inf).masked_fill(none, 0.0)
            w = torch.softmax(s, 1) * seen
            o[at:at + n, h] = torch.matmul(w, v[:, h // G].contiguous())
            a[at:at + n, h] = torch.matmul(w, v[:, h // G].abs().contiguous())
            if bool(odd.any()):
                o[at:at + n, h] += torch.where(torch.matmul(seen.double(), odd[:, h // G].double().contiguous()) > 0, float("nan"), 0.0)
    return o, a


def check(b, sees, what):
    import torch
    mask = np.zeros((b.T, -(-max(n for n, _ in b.lens) // 32)), np.int32)
    for at, s in zip(b.q_start, sees):
        rows = bits_of(s)
        mask[at:at + len(rows), :rows.shape[1]] = rows
    assert all(np.array_equal(branch_ref.tree_seen(mask, int(at), 3, m - n + 3, m)[:, m - n:], s[:3, :3])
               for at, s, (n, m) in zip(b.q_start, sees, b.lens))
    got = torch.from_numpy(run_tree(b, mask)).cuda()
    o, a = expected(b, sees)
    assert torch.equal(got.isnan(), o.isnan()), what
    tol = paged_ref.attention_tolerance(a)
    worst = torch.where(o.isnan(), -1.0, (got - o).abs() - tol)
    assert float(worst.max()) <= 0, (what, float(worst.max()), np.unravel_index(int(worst.argmax()), tuple(worst.shape)))


def kinds(n):
    i, j = np.arange(n)[:, None], np.arange(n)
    return {"late": (j >= n - 300) & (j < n - 20) & ((i + j) % 5 > 0), "late, all": (j >= n - 250) & (j < n - 30) & (i >= 0),
            "quarters": i * 4 // n == j * 4 // n, "near": (j <= i) & (j > i - 50), "last rows late": np.where(i >= n - 140, j >= n - 200, j < 100)}


@pytest.mark.parametrize("lens,Hq,Hkv,Dh,ps,fp8,ends", [
    ([(2700, 2800)], 12, 12, 128, 64, False, False), ([(2740, 2777)], 16, 16, 128, 16, True, False), ([(2700, 2700)], 24, 24, 64, 16, False, False),
    ([(2700, 2830), (2500, 2500)], 8, 8, 128, 48, False, False), ([(2380, 3100)], 16, 8, 128, 16, False, False),
    ([(2700, 2800)], 12, 12, 64, 16, False, True)])
def test_unseen_stretches_in_mid_part(lens, Hq, Hkv, Dh, ps, fp8, ends):
    """ends: parts that end inside the stretch."""
    b = Batch(lens, Hq, Hkv, Dh, ps, seed=29, fp8=fp8)
    plan = tree(len(lens), b.T, Hq, Hkv, Dh, b.width * ps)
    assert plan["hull"] and plan["groups"] == 1 and plan["rows"] == ROWS
    reached, idle = 0, 0
    nan = 0x7F if fp8 else float("nan")
    for name in kinds(2):
        sees = [kinds(n)[name] for n, _ in lens]
        count, without_rows, past_end = gaps(b, sees, plan)
        reached, idle = reached + count, idle + without_rows
        assert past_end > 0 or not ends or name not in ("late", "late, all")
        log(f"tree gaps {lens} Hq={Hq} Dh={Dh} fp8={fp8} {name}: {count} gaps, {without_rows} with idle wavefronts, {past_end} to the part's end")
        check(b, sees, name)
    assert reached >= 3 and idle >= 1, (reached, idle)
    # pages missing before, in and behind the stretch; then values that are not finite there (of tokens that few or none see)
    sees, table = [kinds(n)["late"] for n, _ in lens], b.table.copy()
    for r, (n, m) in enumerate(lens):
        for j in (m - n, m - n + n // 2, m - n + n // 2 + 3 * ps, m - 280, m - 100):
            b.table[r, j // ps] = -1
    check(b, sees, "absent pages")
    b.table = table
    for r, (n, m) in enumerate(lens):
        for j in (m - n + 5, m - n + n // 2, m - 290, m - 60, m - 3):
            b.v[b.table[r, j // ps], j % ps] = nan
    for name in ("late", "near", "quarters"):
        check(b, [kinds(n)[name] for n, _ in lens], f"not finite, {name}")
