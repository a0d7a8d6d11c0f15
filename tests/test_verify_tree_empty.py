"""wam_verify_tree of a batch without rows: the tensors of its rows hold nothing and have no address."""
import numpy as np
import pytest

from gpu_helpers import log
from test_branch_abi_host import verify


def test_without_rows_q_may_be_null():
    assert verify(dict(R=0, T=0), p=0, q=0, tokens=0, parent=0, u=0, path=0) [0] == 0
    assert verify(dict(R=0, T=0)) [0] == 0
    for desc, ptrs in ((dict(R=0), dict(q=0)), (dict(R=0, T=0, drawn=0), {}), (dict(R=0, drawn=0), {})):
        status, says = verify(desc, **ptrs)
        assert status == 1 and "drawn is 1" in says


@pytest.mark.gpu
@pytest.mark.parametrize("drawn", [False, True])
def test_batches_without_rows(drawn):
    from test_verify_tree_gpu import run
    V = 50
    p = np.zeros((0, V), np.float32)
    log(f"verify without rows drawn={drawn}")
    for R in (3, 0):
        path, n_path, nxt, cache = run(p, p if drawn else None, [], [], [], [0.5] * R, [0] * (R + 1), kv_len=[7, 0, 9][:R])
        assert (path, n_path, nxt, cache) == ([], [0] * R, [-1] * R, [7, 0, 9][:R])
