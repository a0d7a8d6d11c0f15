"""wam_verify_tree against its definition in exact fractions (whole numbers: equal), and its distribution in closed form."""
import numpy as np
import pytest

import branch_ref
from gpu_helpers import log, workspace

pytestmark = pytest.mark.gpu
OLD = 77


def i32(x):
    import torch
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def f32(x):
    import torch
    return torch.tensor(np.asarray(x, np.float32), device="cuda")


def run(p, q, tokens, parent, u, u_next, q_start, q_len=None, kv_len=None, gap=0, stream=None):
    """The call; returns (path, n_path, next, cache_len).  gap: floats between the rows of p and q."""
    import torch
    import paper_2602_15922_amd as w
    T, V = p.shape
    R = len(u_next)

    def rows(x):
        if x is None:
            return None
        big = torch.full((T, V + gap), float("nan"), device="cuda")
        big[:, :V] = f32(x)
        return big[:, :V]

    old = lambda n: torch.full((n,), OLD, dtype=torch.int32, device="cuda")  # noqa: E731
    path, n_path, nxt, cache = old(T + 1), old(R + 1), old(R + 1), old(R + 1)
    ws = workspace(w.wam_verify_tree_workspace_bytes(R, T, V, q is not None)).fill_(0xFF)
    args = rows(p), rows(q), i32(tokens), i32(parent), f32(u), f32(u_next), i32(q_start)
    for _ in range(2):
        w.wam_verify_tree(*args, path[:T], n_path[:R], nxt[:R], ws, q_len=i32(q_len), kv_len=i32(kv_len),
                          cache_len=None if kv_len is None else cache[:R])
    torch.cuda.synchronize()
    for x, n in ((path, T), (n_path, R), (nxt, R), (cache, R if kv_len is not None else 0)):
        assert (x[n:] == OLD).all()
    return path[:T].tolist(), n_path[:R].tolist(), nxt[:R].tolist(), cache[:R].tolist()


def check(p, q, tokens, parent, u, u_next, q_start, q_len=None, kv_len=None, gap=0):
    path, n_path, nxt, cache = run(p, q, tokens, parent, u, u_next, q_start, q_len, kv_len, gap)
    want = [OLD] * len(p)
    for r, (at, n) in enumerate(branch_ref.rows_of(q_start, q_len, len(p))):
        s = slice(at, at + n)
        nodes, token = branch_ref.verify(np.float32(p)[s], None if q is None else np.float32(q)[s], tokens[s], parent[s], np.float32(u)[s],
                                         np.float32(u_next)[r])
        assert (n_path[r], nxt[r]) == (len(nodes), token), (r, n_path[r], nodes, nxt[r], token)
        want[at:at + len(nodes)] = nodes
        if kv_len is not None:
            assert cache[r] == kv_len[r] - n + len(nodes)
    assert path == want


def softmax(z):
    e = np.exp(z - z.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


def case(seed, sizes, V, drawn, wide=3, noise=0.7, spread=2.0, tail=2):
    """Trees of `sizes` nodes; drafts from a distribution near the target's, or its likeliest tokens."""
    g = np.random.default_rng(seed)
    T = sum(sizes) + tail
    z = g.normal(size=(T, V)) * spread
    p, q = softmax(z), softmax(z + noise * g.normal(size=(T, V)))
    q_start = np.concatenate([[0], np.cumsum(sizes)])
    tokens, parent = g.integers(0, V, T), np.full(T, -1)
    for at, n in zip(q_start, sizes):
        kids = np.zeros(n, int)
        for i in range(1, n):
            at_most = [j for j in range(max(0, i - 5), i) if kids[j] < wide] or [i - 1]
            j = int(g.choice(at_most))
            row = q[at + j].astype(np.float64)
            tokens[at + i] = g.choice(V, p=row / row.sum()) if drawn else np.argsort(-row, kind="stable")[min(kids[j], V - 1)]
            parent[at + i] = j
            kids[j] += 1
    return p, q if drawn else None, tokens, parent, g.random(T).astype(np.float32), g.random(len(sizes)).astype(np.float32), q_start


SIZES = [[1], [2, 1, 0, 3], [5, 9, 1, 20, 0, 7], [33, 64, 65, 2]]


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("V", [1, 2, 3, 61, 300])
@pytest.mark.parametrize("sizes", SIZES)
def test_trees(sizes, V, drawn):
    for seed, wide in ((1, 1), (2, 3), (3, 8), (4, 3)):
        log(f"verify sizes={sizes} V={V} drawn={drawn} wide={wide}")
        c = case(seed, sizes, V, drawn, wide, noise=(0.3, 3.0)[seed % 2])
        check(*c, kv_len=np.arange(len(sizes)) * 7 + np.array(sizes) + 3, gap=seed % 3)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("V", [4095, 4096, 4097, 9001])
def test_vocabularies_of_more_than_one_slice(V, drawn):
    log(f"verify V={V} drawn={drawn}")
    check(*case(V, [4, 1, 6, 9], V, drawn, noise=1.5, spread=0.3), kv_len=[10, 20, 30, 40])


@pytest.mark.parametrize("drawn", [False, True])
def test_a_large_vocabulary(drawn):
    """262147 entries, the last ones and slice borders among the tokens drawn."""
    V, n = 262147, 6
    g = np.random.default_rng(3)
    p = np.zeros((n, V), np.float32)
    hot = np.array([0, 3, 4095, 4096, 8191, V // 2, V - 2, V - 1])
    p[:, hot] = softmax(g.normal(size=(n, len(hot))))
    q = np.roll(p, 1, 0) if drawn else None
    starts = np.arange(n + 1)
    log(f"verify large drawn={drawn}")
    for u in (0.0, 0.2, 0.45, 0.7, 0.95, 1 - 2.0 ** -24):
        check(p, q, np.zeros(n, int), np.full(n, -1), np.zeros(n), np.full(n, u), starts)
    check(p, q, g.choice(hot, n), np.arange(n) - 1, np.full(n, 0.9), [0.5], [0, n])


def test_greedy_rows():
    """One-hot targets and drafts: a child is taken exactly if it is the target's token."""
    n, V = 12, 50
    g = np.random.default_rng(1)
    best = g.integers(0, V, n)
    p = np.eye(V, dtype=np.float32)[best]
    parent = np.array([-1, 0, 0, 0, 1, 2, 2, 3, 3, 6, 6, 7])
    for drawn in (False, True):
        for trial in range(6):
            tokens = g.integers(0, V, n)
            for i in range(1, n):
                if g.random() < 0.5:
                    tokens[i] = best[parent[i]]
            # (a node's draft is one-hot, so a drawn tree's children share a token)
            q = None
            if drawn:
                d = np.array([tokens[list(parent).index(i)] if i in parent else 0 for i in range(n)])
                tokens[1:] = d[parent[1:]]
                q = np.eye(V, dtype=np.float32)[d]
            log(f"verify greedy drawn={drawn}")
            check(p, q, tokens, parent, g.random(n), [g.random()], [0, n])


def test_nothing_is_left():
    """The residual is empty (p below q everywhere it matters, or all of it rejected): the token comes from p; p empty: -1."""
    p = np.array([[0.5, 0.25, 0.25, 0.0]] * 4 + [[0, 0, 0, 0]] * 2, np.float32)
    q = np.array([[0.5, 0.25, 0.25, 1.0]] * 6, np.float32)
    for u_next in (0.0, 0.3, 0.6, 0.9):
        log("verify nothing left")
        check(p, q, [0, 3, 3, 3, 0, 0], [-1, 0, 0, 0, -1, 0], np.full(6, 0.9), [u_next, u_next], [0, 4, 6])
        # chosen drafts: every token of p rejected (u = 1 is past the range, and never taken)
        check(p, None, [0, 0, 1, 2, 1, 3], [-1, 0, 0, 0, -1, 0], np.full(6, 1.0), [u_next, u_next], [0, 4, 6])


def test_equal_tokens_and_equal_distributions():
    """The same token twice among chosen drafts; drafts drawn from the target itself are all taken."""
    g = np.random.default_rng(5)
    p = softmax(g.normal(size=(6, 20)))
    for u in (0.0, 0.5, 0.999):
        check(p, None, [0, 7, 7, 3, 7, 3], [-1, 0, 0, 0, 0, 0], np.full(6, u), [u], [0, 6])
    tokens = [0] + [int(np.argmax(p[i])) for i in range(5)]
    path, n, _, _ = run(p, p, tokens, np.arange(6) - 1, np.full(6, 1 - 2.0 ** -24), [0.5], [0, 6])
    assert path == list(range(6)) and n == [6]


def test_bad_nodes_are_never_taken():
    p = np.full((9, 4), 0.25, np.float32)
    tokens = [0, -1, 4, 2 ** 31 - 1, -2 ** 31, 1, 2, 3, 1]
    parent = [-1, 0, 0, 0, 0, 5, 7, 2 ** 31 - 1, -2 ** 31]
    log("verify bad nodes")
    for q in (None, p):
        check(p, q, tokens, parent, np.zeros(9), [0.6], [0, 9])
        check(p, q, [1] * 9, [-1, 0, 1, 2, 4, 4, 4, 6, 0], np.zeros(9), [0.6], [0, 9])


def test_probabilities_that_are_none():
    """Negative entries and NaN count as 0, in draws and for drafted tokens."""
    p = np.array([[0.5, -0.25, np.nan, 0.5]] * 3, np.float32)
    for u in (0.0, 0.49, 0.5, 0.99):
        log("verify NaN entries")
        check(p, None, [0, 1, 2], [-1, 0, 0], np.zeros(3), [u], [0, 3])
        check(p, None, [0, 1, 3], [-1, 0, 0], np.full(3, 0.7), [u], [0, 3])
        q = np.array([[0.75, -0.5, 0.25, np.nan]] * 3, np.float32)
        for tokens in ([0, 0, 1], [0, 3, 0], [0, 2, 2]):
            check(p, q, tokens, [-1, 0, 0], np.full(3, 0.9), [u], [0, 3])


def test_padded_and_starts_out_of_range():
    c = case(8, [5, 0, 9, 3], 40, True)
    log("verify padded")
    check(*c, q_len=[3, 0, 9, 2], kv_len=[9, 9, 9, 9])
    check(*c, q_len=[10 ** 9, -4, 1, 0], kv_len=[100, 9, 9, 9])
    for starts in ([0, 5, 5, 14, 10 ** 9], [-7, 5, 5, 14, 17], [3, 3, 3, 3, 3], [90, 80, 70, 60, 50], [-9, -8, -7, -6, -5], [0, 12, 3, 14, 17]):
        log(f"verify starts {starts}")
        c = (*c[:6], np.array(starts))
        if all(0 <= a <= b for a, b in zip(starts, starts[1:])):
            check(*c, kv_len=[50] * 4)
        else:
            run(*c, kv_len=[50] * 4)


def test_many_nodes():
    """More than 64 nodes, all children of one; and more than are looked at."""
    g = np.random.default_rng(6)
    n, V = 1100, 7
    p = softmax(g.normal(size=(n, V)))
    u = np.full(n, 1.0)  # nothing is taken, but
    for hit in (70, 640, 1023, 1024, 1090):
        u[hit] = 0.0
        tokens = np.zeros(n, int)
        tokens[hit] = 5
        log(f"verify many nodes, {hit}")
        check(p, None, tokens, [-1] + [0] * (n - 1), u, [0.3], [0, n], kv_len=[2000])
        u[hit] = 1.0


@pytest.mark.parametrize("drawn", [False, True])
def test_many_requests(drawn):
    g = np.random.default_rng(2)
    sizes = [int(x) for x in g.integers(0, 6, 150)]
    log(f"verify many requests drawn={drawn}")
    check(*case(11, sizes, 30, drawn), kv_len=np.array(sizes) + 1)


def test_outcomes_follow_the_targets_distribution():
    """A root with two children over 4 tokens, over a grid of random numbers and of all drafts.  Every threshold of these
    probabilities (1/2 and 1/4 for the first child, 1/2 or none for the second, 5/6 or 1/2 for the last draw) lies between two of the 12
    points a side, so the share of each first token that comes out is the target's probability of it, up to the 64-bit sums."""
    p, q = np.array([1 / 2, 1 / 4, 1 / 8, 1 / 8], np.float32), np.array([1 / 8, 1 / 8, 1 / 4, 1 / 2], np.float32)
    grid = (np.arange(12) + 0.5) / 12
    U = np.stack(np.meshgrid(grid, grid, grid, indexing="ij"), -1).reshape(-1, 3)
    R = len(U)
    P, Q, u = np.tile(p, (3 * R, 1)), np.tile(q, (3 * R, 1)), np.stack([np.zeros(R), U[:, 0], U[:, 1]], 1).ravel()
    log("verify distribution")

    def add(share, a, b, drawn, weight):
        path, n_path, nxt, _ = run(P, Q if drawn else None, np.tile([0, a, b], R), np.tile([-1, 0, 0], R), u, U[:, 2], np.arange(R + 1) * 3)
        for r in range(R):
            share[nxt[r] if n_path[r] == 1 else (a, b)[path[3 * r + 1] - 1]] += weight / R

    share = np.zeros(4)
    for a in range(4):
        for b in range(4):
            add(share, a, b, True, float(q[a]) * float(q[b]))
    assert np.allclose(share, p, rtol=0, atol=1e-9), share
    for a, b in ((0, 1), (1, 0)):  # chosen drafts, whatever they are (thresholds 1/2, 1/4; 1/2, 2/3; 1/2)
        share = np.zeros(4)
        add(share, a, b, False, 1.0)
        assert np.allclose(share, p, rtol=0, atol=1e-9), share


def test_streams_and_graphs():
    """Replayed from a graph with other inputs in the same buffers, the program's own work between; two calls at once."""
    import torch
    import paper_2602_15922_amd as w
    sizes, V = [6, 9, 1], 5000
    T, R = sum(sizes) + 2, len(sizes)
    cases = [case(s, sizes, V, True, spread=1.0, noise=1.0) for s in range(4)]
    bufs = [f32(cases[0][0]), f32(cases[0][1]), *(i32(x) for x in cases[0][2:4]), f32(cases[0][4]), f32(cases[0][5]), i32(cases[0][6])]
    outs = [[torch.zeros(n, dtype=torch.int32, device="cuda") for n in (T, R, R)] for _ in range(2)]
    ws = [workspace(w.wam_verify_tree_workspace_bytes(R, T, V, True)).fill_(0xFF) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    log("verify streams and graph")
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            w.wam_verify_tree(*bufs, *outs[i], ws[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        w.wam_verify_tree(*bufs, *outs[0], ws[0])
    for c in cases[1:] + cases[:1]:
        for buf, x in zip(bufs, c):
            buf.copy_(torch.as_tensor(np.asarray(x)))
        outs[0][0].fill_(OLD)
        g.replay()
        torch.cuda.synchronize()
        for r, at in enumerate(c[6][:-1]):
            s = slice(at, c[6][r + 1])
            nodes, token = branch_ref.verify(c[0][s], c[1][s], c[2][s], c[3][s], c[4][s], c[5][r])
            assert outs[0][0][at:at + len(nodes)].tolist() == nodes and outs[0][1][r] == len(nodes) and outs[0][2][r] == token
