"""wam_verify_tree: hundreds of children of one node."""
import numpy as np
import pytest

from gpu_helpers import log, workspace
from test_verify_tree_gpu import check, f32, i32, softmax

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [64, 65, 130, 700, 1024])
def test_many_siblings(n):
    """Chosen drafts: hundreds of children of the root, some tokens twice (never taken the second time, also hundreds of nodes
    later), others' children with the same tokens between them (which reject nothing)."""
    V = 3000
    for seed in range(3):
        g = np.random.default_rng(100 * n + seed)
        p = softmax(g.normal(size=(n, V)) * 0.5)
        tokens, parent, u = g.permutation(V)[:n], np.zeros(n, int), (0.9 + 0.1 * g.random(n)).astype(np.float32)
        parent[0] = -1
        for i in g.integers(2, n, n // 8):  # a sibling's token again, and a random number that takes whatever has a chance
            tokens[i], u[i] = tokens[g.integers(1, i)], 0.0
        others = np.setdiff1d(g.integers(2, n, n // 8), [n - 1])
        parent[others] = [g.integers(1, i) for i in others]
        if seed == 1:  # one whose token only another node's child had before
            i = int(others[len(others) // 2])
            tokens[n - 1], u[n - 1], parent[n - 1] = tokens[i], 0.0, 0
        log(f"verify siblings n={n} seed={seed}")
        check(p, None, tokens, parent, u, [0.37], [0, n], kv_len=[n + 5])


def test_the_time_of_many_siblings():
    """1023 rejected children of the root: the walk looks at 64 earlier siblings at a time."""
    import torch
    import paper_2602_15922_amd as w
    n, V = 1024, 2000
    args = (f32(np.full((n, V), 1.0 / V)), None, i32(np.arange(n)), i32([-1] + [0] * (n - 1)), f32(np.full(n, 1 - 2.0 ** -24)), f32([0.5]), i32([0, n]))
    outs = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in (n, 1, 1)]
    ws = workspace(w.wam_verify_tree_workspace_bytes(1, n, V, False))
    log("verify time of siblings")
    best = float("inf")
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        w.wam_verify_tree(*args, *outs, ws)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    print(f"{best:.3f} ms")
    assert outs[1].tolist() == [1] and best < 5.0
