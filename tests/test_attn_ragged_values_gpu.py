"""Infinities and NaN in V of a part of the key axis whose weight vanishes beside another part's (ragged attentions)."""
import numpy as np
import pytest

import paged_ref
from gpu_helpers import log
from paged_ref import Batch
from ragged_plans import plan
from test_attn_ragged_gpu import OLD, cross_case, run_cross, run_paged

pytestmark = pytest.mark.gpu

SHAPES = [([(1, 1500), (2, 900)], 8, 2, 128, False), ([(1, 1500), (2, 900)], 8, 2, 128, True), ([(3, 2000)], 5, 5, 64, False),
          ([(150, 2600)], 32, 32, 64, False), ([(150, 2600)], 32, 32, 128, True), ([(1, 700), (140, 2600), (140, 2500)], 32, 16, 64, False)]


def check_finite_and_not(got, o, a, mine):
    """The same places are finite; there within the tolerance.  (What is not finite may be NaN where the formula has an
    infinity: its weight is 0 in 32 bits.)"""
    at = mine[:, None, None] & np.isfinite(o)
    assert np.array_equal(np.isfinite(got[mine]), np.isfinite(o[mine]))
    assert np.all(np.abs(got[at] - o[at]) <= paged_ref.attention_tolerance(a)[at])
    assert np.all(got[~mine] == OLD)


@pytest.mark.parametrize("lens,Hq,Hkv,Dh,fp8", SHAPES)
@pytest.mark.parametrize("low_first", [True, False])
def test_values_not_finite_under_a_weight_that_vanishes(lens, Hq, Hkv, Dh, fp8, low_first):
    """Half of the key axis scores at about -45 (Dh 64: -64), the rest at 90 (128): further apart than the 88 nats that a
    weight of 32 bits spans.  A NaN (and infinities) of V in the low half reaches every row, whatever its weight."""
    import torch
    b = Batch(lens, Hq, Hkv, Dh, 16, seed=61 + Dh, fp8=fp8)
    p = plan(len(lens), b.T, Hq, Hkv, Dh, b.width * 16)
    assert p["splits"] > 1 and p["keys"] < max(m for _, m in lens)
    amp = 8 if Dh == 128 else 16  # scores: q.k / sqrt(Dh) = 8 or 16 * sqrt(Dh) * (K's value)
    b.q = (amp + 0.5 * torch.randn(b.T, Hq, Dh, generator=torch.Generator().manual_seed(3))).bfloat16()
    for r, (n, m) in enumerate(lens):
        for j in range(m):
            pg, row = b.table[r, j // 16], j % 16
            low = (j < m // 2) == low_first
            if fp8:
                b.k[pg, row], b.k_exp[pg, row] = (0xB0 if low else 0x38), 127  # -0.5, 1
                b.v[pg, row] = 0x30 + (j & 7)
            else:
                b.k[pg, row] = (-0.5 if low else 1.0)
                b.v[pg, row] = 0.5 + 0.0625 * (j & 7)
        j = m // 4 if low_first else m - m // 4
        pg, row = b.table[r, j // 16], j % 16
        for dim, val in ((3, float("nan")), (5, float("inf")), (9, float("-inf")), (Dh - 1, float("nan"))):
            b.v[pg, row, :, dim] = 0x7F if fp8 else val
    log(f"paged low part not finite {lens} Hq={Hq} Dh={Dh} fp8={fp8} low_first={low_first}")
    with np.errstate(invalid="ignore"):
        check_finite_and_not(run_paged(b, 0), *b.expected(0))


@pytest.mark.parametrize("q_lens,k_lens,Hq,Hkv,Dh", [([2, 1], [1600, 900], 4, 2, 128), ([260], [2400], 20, 4, 64)])
def test_cross_values_not_finite_under_a_weight_that_vanishes(q_lens, k_lens, Hq, Hkv, Dh):
    q, kv, qs, ks, S, _ = cross_case(q_lens, k_lens, Hq, Hkv, Dh, 71)
    assert plan(len(q_lens), len(q), Hq, Hkv, Dh, S)["splits"] > 1
    q[:] = 8 if Dh == 128 else 16
    for r, m in enumerate(k_lens):
        kv[ks[r]:ks[r] + m // 2, 0], kv[ks[r] + m // 2:ks[r] + m, 0] = -0.5, 1.0
        kv[ks[r] + m // 4, 1, :, 7] = float("nan")
        kv[ks[r] + m // 4, 1, :, 8] = float("inf")
    log(f"cross low part not finite {q_lens} {k_lens} Hq={Hq} Dh={Dh}")
    x, y = q.double().numpy(), kv.double().numpy()
    o, a, mine = np.zeros(q.shape), np.zeros(q.shape), np.zeros(len(q), bool)
    with np.errstate(invalid="ignore"):
        for r, (n, m) in enumerate(zip(q_lens, k_lens)):
            rows, keys = slice(qs[r], qs[r] + n), slice(ks[r], ks[r] + m)
            mine[rows] = True
            for h in range(Hq):
                hk = h // (Hq // Hkv)
                o[rows, h], a[rows, h] = paged_ref.attend(x[rows, h], y[keys, 0, hk], y[keys, 1, hk], np.ones((n, m), bool), Dh ** -0.5)
    check_finite_and_not(run_cross(q, kv, qs, ks), o, a, mine)


@pytest.mark.parametrize("lens,Hq,Hkv,Dh", [([(1, 1), (3, 40)], 4, 2, 128), ([(1, 1500)], 8, 2, 64), ([(150, 400)], 2, 1, 128), ([(150, 2600)], 32, 32, 64)])
def test_rows_without_a_score_above_minus_infinity(lens, Hq, Hkv, Dh):
    """Every key of KV head 0 scores -infinity: its rows are 0, as of a row that sees no key; the other heads' are as ever."""
    b = Batch(lens, Hq, Hkv, Dh, 16, seed=81 + Dh)
    b.q[..., 5] = 1
    o, a, mine = b.expected(1)
    b.k[..., 0, 5] = float("-inf")
    log(f"paged scores of -infinity {lens} Hq={Hq} Dh={Dh}")
    got, G = run_paged(b, 1), Hq // Hkv
    assert np.all(got[mine][:, :G] == 0)
    o, a, rest = o[:, G:], a[:, G:], got[:, G:]
    assert np.all((np.abs(rest - o) <= paged_ref.attention_tolerance(a))[mine]) and np.all(got[~mine] == OLD)
