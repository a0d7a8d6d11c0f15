"""Where the ragged attentions write: rows before the output's first and past its last stay as they were, whatever the
starts say, and rows whose starts still say something hold their results."""
import numpy as np
import pytest

import paged_ref
from gpu_helpers import host, log, workspace
from paged_ref import Batch

pytestmark = pytest.mark.gpu
OLD, GUARD = 5.0, 40


def run_guarded(b, chunk, q_len):
    """The call with o as rows GUARD .. GUARD + T of a larger buffer; returns those rows."""
    import torch
    import paper_2602_15922_amd as w
    c = b.cache()
    i32 = lambda x: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    big = torch.full((b.T + 2 * GUARD, b.Hq + 1, b.Dh), OLD, dtype=torch.bfloat16, device="cuda")
    o = big[GUARD:GUARD + b.T, :b.Hq]
    ws = workspace(w.wam_attn_paged_workspace_bytes(c, R=len(b.lens), T=b.T, Hq=b.Hq, max_kv=b.width * b.ps)).fill_(0xFF)
    w.wam_attn_paged(c, b.q.cuda(), i32(b.table), i32(b.q_start), i32(b.kv_len), o, ws, chunk=chunk, q_len=i32(q_len))
    torch.cuda.synchronize()
    assert (big[:GUARD] == OLD).all() and (big[GUARD + b.T:] == OLD).all() and (big[:, b.Hq:] == OLD).all()
    return host(o)


@pytest.mark.parametrize("lens,Hq,Hkv,Dh", [([(5, 30), (0, 9), (40, 200), (1, 1)], 6, 3, 64), ([(5, 1300), (0, 9), (40, 2000), (1, 1)], 4, 4, 128)])
def test_starts_out_of_range_write_no_row_of_others(lens, Hq, Hkv, Dh):
    T = Batch(lens, Hq, Hkv, Dh, 32, seed=4, gap=3).T
    # starts, and the rows that each request then has (None: the starts do not say)
    for starts, rows in (([0, 5, 5, 45, 10 ** 9], [(0, 5), (5, 0), (5, 40), (45, T - 45)]),
                         ([-100, 5, 5, 45, 46], [None, (5, 0), (5, 40), (45, 1)]),
                         ([0, 5, 5, T + 9, T + 9], [(0, 5), (5, 0), (5, T - 5), (T, 0)]),
                         ([T, T, T, T, T], [(T, 0)] * 4),
                         ([0, 60, 3, 45, 46], None), ([90, 80, 70, 60, 50], None), ([-9, -8, -7, -6, -5], None)):
        for with_len in (False, True):
            b = Batch(lens, Hq, Hkv, Dh, 32, seed=4, gap=3)
            b.q_start = np.array(starts, np.int32)
            if rows is not None:
                n = np.array([0 if x is None else x[1] for x in rows], np.int32)
                if with_len:  # lengths past the room there is are cut to it
                    n = np.minimum(n, b.q_len)
                    given = [10 ** 9 if x is not None and x[1] <= y else int(y) for x, y in zip(rows, b.q_len)]
            log(f"paged guarded starts={starts} Hq={Hq} Dh={Dh} q_len={with_len}")
            got = run_guarded(b, 1, (b.q_len if rows is None else given) if with_len else None)
            if rows is None:
                continue
            b.q_start, b.q_len = np.array([max(0, min(s, T)) for s in starts], np.int32), n
            o, a, mine = b.expected(1)
            assert np.all((np.abs(got - o) <= paged_ref.attention_tolerance(a))[mine])
            sure = ~mine
            if rows[0] is None:
                sure[:5] = False
            assert np.all(got[sure] == OLD)
