"""wam_verify_tree: the sums do not depend on the number of passes; rows that do not sum to one."""
import numpy as np
import pytest

import branch_ref
from gpu_helpers import log
from test_verify_tree_gpu import OLD, check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [4, 10, 20, 40])
def test_a_sum_is_the_same_in_every_pass(T):
    """The last sum decides in its last bit: P holds a one, six entries of 2^-53 that are lost one by one beside it and not together,
    and (1 + 2^-52) before them; all halved.  Both children are rejected, so the last sum is the second pass: of all workgroups or of
    the last one, by the rows of the call (here those of no request)."""
    V, t = 8192, 2.0 ** -53
    p, q = np.zeros((T, V), np.float32), np.zeros((T, V), np.float32)
    p[0, 0], p[0, 1], p[0, 4096] = 0.5, t, 0.5
    p[0, 4096 + 256 * np.array([1, 2, 3, 5, 6, 7])] = t / 2
    q[0, [8190, 8191]] = 0.5
    p[3, 7] = 1.0
    tokens, parent = np.array([0, 8190, 8191, 0] + [0] * (T - 4)), np.array([-1, 0, 0, -1] + [-1] * (T - 4))
    log(f"verify order of a sum T={T}")
    assert branch_ref.verify(p[:3], q[:3], tokens, parent, [0.5] * 3, 0.5) == ([0], 4096)
    check(p, q, tokens, parent, np.full(T, 0.5), [0.5, 0.5], [0, 3, 4])


def test_chosen_drafts_and_rows_that_do_not_sum_to_one():
    """s is one minus what was rejected, whatever the row sums to: 0.55 (1 - 0.5) >= 0.25 rejects (0.55 * 0.375 would not)."""
    p = np.array([[0.5, 0.25, 0.125, 0.0]] * 4, np.float32)
    for u in (0.55, 0.45):
        log(f"verify chosen, sum 0.875, u={u}")
        check(p, None, [0, 0, 1, 2], [-1, 0, 0, 0], [0.0, 0.6, u, 0.9], [0.4], [0, 4])
    path, _, _, _ = run(p, None, [0, 0, 1, 2], [-1, 0, 0, 0], [0.0, 0.6, 0.55, 0.9], [0.4], [0, 4])
    assert path[:2] == [0, OLD]
