"""wam_attn_tree against its definition in 64 bits, element by element (the tolerance is the paged attention's: the same
arithmetic over other keys)."""
import numpy as np
import pytest

import branch_ref
import paged_ref
from gpu_helpers import host, log, workspace
from paged_ref import Batch

pytestmark = pytest.mark.gpu
OLD = 5.0


def masks(b, kind, seed, words=None):
    """Mask rows [T][words] int32 of a batch: trees, separate branches, random bits, causal, all, none, only itself."""
    g = np.random.default_rng(seed)
    most = max([n for n, _ in b.lens] + [1])
    words = -(-most // 32) if words is None else words
    out = g.integers(-2 ** 31, 2 ** 31, (b.T, words)).astype(np.int32)  # (rows of nobody, bits past the last token: anything)
    for at, (n, _) in zip(b.q_start, b.lens):
        full = -(-max(n, 1) // 32)
        rows = np.zeros((n, full), np.uint32)
        if kind == "tree":
            rows = branch_ref.ancestors([-1 if i == 0 else int(g.integers(max(0, i - 6), i)) for i in range(n)], full).view(np.uint32)
        elif kind != "random":
            sees = {"branches": lambda i, j: i * 3 // max(n, 1) == j * 3 // max(n, 1), "causal": lambda i, j: j <= i, "all": lambda i, j: True,
                    "none": lambda i, j: False, "self": lambda i, j: i == j}[kind]
            for i in range(n):
                for j in range(n):
                    rows[i, j // 32] |= np.uint32(sees(i, j) << (j % 32))
        else:
            rows = g.integers(0, 2 ** 32, (n, full)).astype(np.uint32)
        if n % 32:
            rows[:, -1] |= np.uint32(0xFFFFFFFF) << np.uint32(n % 32)  # bits of tokens that there are not
        out[at:at + n, :min(full, words)] = rows.view(np.int32)[:, :words]
    return out


def expected(b, mask, scale=None, max_kv=None):
    scale = b.Dh ** -0.5 if scale is None else scale
    o, a, mine = np.zeros((b.T, b.Hq, b.Dh)), np.zeros((b.T, b.Hq, b.Dh)), np.zeros(b.T, bool)
    q = b.q.double().numpy()
    for r, n in enumerate(b.q_len):
        at, m = int(b.q_start[r]), int(b.kv_len[r])
        mine[at:at + n] = True
        k, v, there = b.kv64(r)
        seen = branch_ref.tree_seen(mask, at, n, m, len(there)) & there if m > 0 else np.zeros((n, len(there)), bool)
        if max_kv is not None:
            seen[:, max_kv:] = False
        for h in range(b.Hq):
            hk = h // (b.Hq // b.Hkv)
            o[at:at + n, h], a[at:at + n, h] = paged_ref.attend(q[at:at + n, h], k[:, hk], v[:, hk], seen, scale)
    return o, a, mine


def run_tree(b, mask, max_kv=None, q_len=None, scale=0.0, cache=None, gap=1):
    import torch
    import paper_2602_15922_amd as w
    c = cache or b.cache()
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    wide = torch.full((b.T, b.Hq + 1, b.Dh), OLD, dtype=torch.bfloat16, device="cuda")
    bits = torch.full((b.T, mask.shape[1] + gap), -1, dtype=torch.int32, device="cuda")
    bits[:, :mask.shape[1]] = i32(mask)
    n = w.wam_attn_tree_workspace_bytes(c, R=len(b.lens), T=b.T, Hq=b.Hq, max_kv=b.width * b.ps if max_kv is None else max_kv)
    ws = workspace(n).fill_(0xFF)
    w.wam_attn_tree(c, b.q.cuda(), i32(b.table), i32(b.q_start), i32(b.kv_len), bits[:, :mask.shape[1]], wide[:, :b.Hq], ws, max_kv=max_kv,
                    q_len=None if q_len is None else i32(q_len), scale=scale)
    torch.cuda.synchronize()
    assert (wide[:, b.Hq:] == OLD).all()
    return host(wide[:, :b.Hq])


def check(got, ref, what=""):
    o, a, mine = ref
    assert np.isfinite(got).all(), what
    worst = np.abs(got - o)[mine] - paged_ref.attention_tolerance(a)[mine]
    assert worst.max(initial=-1) <= 0, (what, float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))
    assert np.all(got[~mine] == OLD), what


KINDS = ["tree", "branches", "random", "causal", "all", "none", "self"]
MIXED = [(1, 1), (1, 63), (0, 30), (3, 3), (4, 64), (31, 65), (32, 40), (33, 300), (1, 129), (65, 66), (2, 0), (5, 3), (7, 700)]


@pytest.mark.parametrize("Hq,Hkv,Dh,ps,layout,fp8", [
    (1, 1, 128, 16, "nhd", False), (8, 2, 128, 48, "hnd", False), (3, 3, 64, 64, "kv", False), (16, 1, 64, 16, "nhd", False), (6, 2, 64, 1024, "hnd", False),
    (1, 1, 128, 16, "nhd", True), (8, 2, 128, 48, "hnd", True), (5, 5, 128, 32, "kv", True)])
def test_mixed_lengths(Hq, Hkv, Dh, ps, layout, fp8):
    b = Batch(MIXED, Hq, Hkv, Dh, ps, seed=Hq + ps, fp8=fp8, layout=layout)
    for kind in KINDS:
        mask = masks(b, kind, Hq)
        log(f"tree mixed Hq={Hq} Hkv={Hkv} Dh={Dh} ps={ps} {layout} fp8={fp8} {kind}")
        check(run_tree(b, mask), expected(b, mask), kind)


# (few rows: the streaming kernel with 16 and 32 rows to a workgroup; many: tiles; one request: eight wavefronts; split and whole)
AXIS = [([(n, n + h) for n in (1, 2, 5, 16) for h in (0, 1, 15, 16, 31, 100, 511, 1025)], 1, 1, 128, 16), ([(8, 5000)], 2, 2, 128, 64),
        ([(4, 3001), (2, 17), (1, 2999)], 20, 5, 64, 16), ([(33, 2100)], 2, 1, 128, 16), ([(128, 1300), (129, 129)], 2, 2, 128, 64),
        ([(257, 700)], 3, 1, 64, 48), ([(64, 4000)], 1, 1, 128, 32), ([(500, 1100)], 1, 1, 128, 16), ([(200, 200), (300, 301), (1, 900)], 2, 1, 64, 16),
        ([(16, 700)] * 9, 2, 1, 128, 16)]


@pytest.mark.parametrize("lens,Hq,Hkv,Dh,ps,fp8", [(*x, f) for x in AXIS for f in (False, True) if x[3] == 128 or not f])
def test_lengths_of_history_and_tree(lens, Hq, Hkv, Dh, ps, fp8):
    b = Batch(lens, Hq, Hkv, Dh, ps, seed=3, fp8=fp8)
    for kind in ("tree", "branches", "random"):
        mask = masks(b, kind, 5)
        log(f"tree lengths {lens[:3]} Hq={Hq} Hkv={Hkv} Dh={Dh} ps={ps} fp8={fp8} {kind}")
        check(run_tree(b, mask), expected(b, mask), kind)


@pytest.mark.parametrize("lens,Hq,Hkv,Dh", [([(20, 150), (5, 1500)], 4, 4, 128), ([(140, 1000), (3, 50)], 2, 1, 64), ([(300, 900)], 1, 1, 128)])
def test_causal_mask_is_the_causal_attention(lens, Hq, Hkv, Dh):
    """The same keys by mask and by chunk 1: within both tolerances; all new tokens visible: as with chunk 0."""
    from test_attn_ragged_gpu import run_paged
    b = Batch(lens, Hq, Hkv, Dh, 16, seed=17)
    log(f"tree against paged {lens}")
    for kind, chunk in (("causal", 1), ("all", 0)):
        got, want, (_, a, mine) = run_tree(b, masks(b, kind, 1)), run_paged(b, chunk), b.expected(chunk)
        assert np.all((np.abs(got - want) <= 2 * paged_ref.attention_tolerance(a))[mine])


def bits_of(sees):
    """Mask rows of a truth table [n][n]."""
    n = len(sees)
    out = np.zeros((n, -(-n // 32) * 32), np.uint8)
    out[:, :n] = sees
    return np.packbits(out, axis=1, bitorder="little").view(np.int32)


@pytest.mark.parametrize("lens,Hq,Hkv,Dh,fp8", [([(2600, 2700), (40, 300)], 1, 1, 64, False), ([(1500, 1531), (70, 70)], 2, 1, 128, False),
                                                ([(1700, 2300), (3, 100)], 1, 1, 128, True), ([(1300, 1400), (1290, 1290), (1500, 3000)], 1, 1, 64, False),
                                                ([(1300, 1400)], 24, 24, 64, False)])
def test_long_masks(lens, Hq, Hkv, Dh, fp8):
    """Masks of thousands of tokens, whose rows see nothing of long stretches: before their own branch, behind it, or of all new
    tokens; with pages missing, and values that are not finite in what is not seen."""
    from ragged_plans import plan
    b = Batch(lens, Hq, Hkv, Dh, 16, seed=19, fp8=fp8)
    assert b.T >= 512 * len(lens) and plan(len(lens), b.T, Hq, Hkv, Dh, b.width * 16)["groups"] == 1
    i = {n: np.arange(n) for n, _ in lens}
    kinds = {
        "branches": lambda n: i[n][:, None] * 2 // n == i[n] * 2 // n, "late": lambda n: (i[n] >= n - 40) & (i[n][:, None] % 3 > 0),
        "early": lambda n: (i[n] < 5) & (i[n][:, None] < 2000), "none": lambda n: np.zeros((n, n), bool), "self": lambda n: np.eye(n, dtype=bool),
        "apart": lambda n: (i[n] % 1100 == 7) & (i[n] <= i[n][:, None]), "causal": lambda n: i[n] <= i[n][:, None],
        "all": lambda n: np.ones((n, n), bool), "shifted": lambda n: (i[n] >= 77) & (i[n] < n - 90) & (i[n][:, None] >= 0)}
    for name, sees in kinds.items():
        if Hq > 2 and name not in ("late", "branches", "shifted"):
            continue
        mask = np.zeros((b.T, max(-(-n // 32) for n, _ in lens)), np.int32)
        for at, (n, _) in zip(b.q_start, lens):
            rows = bits_of(sees(n))
            mask[at:at + n, :rows.shape[1]] = rows
        log(f"tree long masks {lens} Hq={Hq} Dh={Dh} fp8={fp8} {name}")
        check(run_tree(b, mask), expected(b, mask), name)
    table = b.table.copy()  # (the last kind: new tokens from the 78th on, seen by all)
    b.table[0, 20:60] = -1
    check(run_tree(b, mask), expected(b, mask), "absent")
    b.table = table
    n, m = lens[0]
    for back in (n - 100, 900, 3):
        j = m - back  # tokens that only some rows see, or none
        b.v[b.table[0, j // 16], j % 16] = 0x7F if fp8 else float("nan")
    mask[:] = 0
    for at, (n, _) in zip(b.q_start, lens):
        rows = bits_of(kinds["branches"](n))
        mask[at:at + n, :rows.shape[1]] = rows
    log(f"tree long masks {lens} not finite")
    got, (o, a, mine) = run_tree(b, mask), expected(b, mask)
    assert np.array_equal(np.isnan(got), np.isnan(o) & mine[:, None, None])
    fin = mine[:, None, None] & np.isfinite(o)
    assert np.all(np.abs(got[fin] - o[fin]) <= paged_ref.attention_tolerance(a)[fin])


def test_words_of_the_mask():
    """Fewer words than tokens (the rest is seen by nobody), more, none; rows apart."""
    b = Batch([(70, 200), (3, 100), (33, 33)], 4, 2, 128, 16, seed=6)
    for words in (0, 1, 2, 3, 7):
        mask = masks(b, "all", 2, words)
        log(f"tree words={words}")
        check(run_tree(b, mask, gap=words % 2 + (words == 0)), expected(b, mask), str(words))


@pytest.mark.parametrize("fp8", [False, True])
def test_absent_pages_max_kv_and_lengths(fp8):
    for lens in ([(4, 200), (2, 100), (9, 700)], [(60, 200), (70, 100), (150, 300)], [(90, 1300)]):
        b = Batch(lens, 4, 2, 128, 16, seed=8, fp8=fp8)
        b.table[0, 3], b.table[0, 12] = -1, b.n_pages
        if len(lens) > 1:
            b.table[1, :], b.table[2, 1::2] = -2 ** 31, 2 ** 31 - 1
        mask = masks(b, "random", 3)
        log(f"tree absent pages {lens} fp8={fp8}")
        check(run_tree(b, mask), expected(b, mask))
        for most in (48, 190, 0):
            check(run_tree(b, mask, max_kv=most), expected(b, mask, max_kv=most), str(most))
        b.kv_len[:] = [-5, 0, -2 ** 31][:len(lens)]
        got = run_tree(b, mask)
        assert np.all(got[:-3] == 0) and np.all(got[-3:] == OLD)


def test_more_rows_than_tokens():
    """kv_len below the rows: the first rows' own keys do not exist, the bits still count from the first row."""
    for lens in ([(40, 25), (5, 2)], [(200, 130)], [(12, 7)] * 4):
        b = Batch(lens, 2, 1, 64, 16, seed=23)
        for kind in ("causal", "random"):
            mask = masks(b, kind, 4)
            log(f"tree more rows than tokens {lens} {kind}")
            check(run_tree(b, mask), expected(b, mask), kind)


def test_padded_batches_and_starts_out_of_range():
    b = Batch([(5, 30), (0, 9), (40, 200), (1, 1)], 6, 3, 64, 32, seed=4, gap=3)
    mask = masks(b, "tree", 9)
    log("tree padded")
    check(run_tree(b, mask, q_len=b.q_len), expected(b, mask))
    for starts in ([0, 5, 5, 45, 10 ** 9], [-100, 5, 5, 45, 46], [0, 60, 3, 45, 46], [90, 80, 70, 60, 50], [-9, -8, -7, -6, -5]):
        log(f"tree starts {starts}")
        b.q_start = np.array(starts, np.int32)
        run_tree(b, mask)
    b.kv_len[:] = 2 ** 31 - 1  # positions past the table
    b.k.nan_to_num_(0.0), b.v.nan_to_num_(0.0)
    log("tree kv_len past the width")
    run_tree(b, mask)


@pytest.mark.parametrize("lens,Hq,Hkv,Dh,fp8", [
    ([(6, 70), (3, 129), (9, 9)], 2, 2, 64, False), ([(6, 70), (3, 129)], 2, 2, 128, False), ([(5, 700), (4, 90)], 8, 2, 128, False),
    ([(6, 170), (5, 64)], 4, 2, 128, True), ([(150, 200), (40, 140), (3, 65)], 4, 2, 128, False), ([(100, 190), (65, 65)], 4, 2, 128, True),
    ([(140, 1000)], 2, 1, 128, False), ([(300, 300)], 1, 1, 64, False), ([(90, 800)], 2, 2, 128, True)])
@pytest.mark.parametrize("kind", ["tree", "branches", "self"])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(lens, Hq, Hkv, Dh, fp8, kind):
    b = Batch(lens, Hq, Hkv, Dh, 16, seed=sum(n + m for n, m in lens) + Dh, fp8=fp8)
    for r, (n, m) in enumerate(lens):
        for i, dims, val in ((n - 1, slice(None), float("nan")), (n // 2, 3, float("inf")), (n // 2, 5, float("-inf")), (n // 3, 3, float("-inf")),
                             (n // 4, 17, float("inf")), (1, Dh - 1, float("-inf"))):
            j = m - n + i
            b.v[b.table[r, j // 16], j % 16, :, dims] = 0x7F if fp8 else val
    mask = masks(b, kind, 7)
    log(f"tree values not finite {lens} Hq={Hq} Dh={Dh} fp8={fp8} {kind}")
    with np.errstate(invalid="ignore"):
        got, (o, a, mine) = run_tree(b, mask), expected(b, mask)
    fin = np.isfinite(o)
    at = mine[:, None, None] & ~fin
    assert np.array_equal(np.isnan(got[at]), np.isnan(o[at]))
    inf = at & np.isinf(o)
    assert np.array_equal(got[inf], o[inf])
    ok = mine[:, None, None] & fin
    assert np.isfinite(got[ok]).all()
    assert np.all(np.abs(got[ok] - o[ok]) <= paged_ref.attention_tolerance(a)[ok])


def test_nan_keys_that_a_row_does_not_see():
    for lens, Hq in (([(9, 60)], 2), ([(150, 400)], 2)):
        b = Batch(lens, Hq, Hq, 64, 16, seed=13)
        n, m = lens[0]
        mask = masks(b, "self", 1)
        for i in (0, n // 2, n - 1):
            j = m - n + i
            b.k[b.table[0, j // 16], j % 16] = (float("nan"), float("inf"))[i % 2]
        log(f"tree NaN keys {lens}")
        got, (o, a, mine) = run_tree(b, mask), expected(b, mask)
        rows = np.setdiff1d(np.arange(n), [0, n // 2, n - 1])
        assert np.all((np.abs(got - o) <= paged_ref.attention_tolerance(a))[rows])


def test_offsets_past_32_bits():
    """Pages more than 4 GiB apart, and mask rows more than 2^31 words in all."""
    import torch
    import paper_2602_15922_amd as w
    b = Batch([(1, 40), (33, 50)], 2, 1, 128, 16, seed=14)
    n, span = b.n_pages, 400_000_000
    log("tree far pages and masks")
    big = torch.empty(n * span, dtype=torch.bfloat16, device="cuda")
    k = torch.as_strided(big, (n, 16, 1, 128), (span, 128, 128, 1))
    v = torch.as_strided(big, (n, 16, 1, 128), (span, 128, 128, 1), storage_offset=16 * 128)
    k.copy_(b.k), v.copy_(b.v)
    mask = masks(b, "random", 2)
    check(run_tree(b, mask, cache=w.make_paged_cache(k, v), gap=70_000_000), expected(b, mask))
    del big, k, v
    torch.cuda.empty_cache()


@pytest.mark.parametrize("lens", [[(3, 900), (5, 77)], [(140, 900), (3, 77)], [(200, 700)]])
def test_streams_graphs_and_repeats(lens):
    """On another stream, again (bit for bit), two calls at once, and replayed with other masks and lengths."""
    import torch
    import paper_2602_15922_amd as w
    b = Batch(lens, 8, 2, 128, 16, seed=31)
    log(f"tree graph {lens}")
    b.k.nan_to_num_(0.0), b.v.nan_to_num_(0.0)
    c, q = b.cache(), b.q.cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, qs, kv, first = i32(b.table), i32(b.q_start), i32(b.kv_len), masks(b, "tree", 1)
    mask = i32(first)
    o = torch.full((2, b.T, 8, 128), OLD, dtype=torch.bfloat16, device="cuda")
    n = w.wam_attn_tree_workspace_bytes(c, R=len(lens), T=b.T, Hq=8, max_kv=b.width * 16)
    ws, streams = [workspace(n).fill_(0xFF) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            w.wam_attn_tree(c, q, table, qs, kv, mask, o[i], ws[i], stream=s)
    torch.cuda.synchronize()
    check(host(o[0]), expected(b, first))
    assert torch.equal(o[0], o[1])
    want = o[0].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        w.wam_attn_tree(c, q, table, qs, kv, mask, o[0], ws[0])
    full = b.kv_len.copy()
    for kind, less in (("branches", 0), ("random", 13), ("self", 40), ("tree", 0)):
        bits = masks(b, kind, 1)
        b.kv_len = np.maximum(full - less, 0).astype(np.int32)
        mask.copy_(i32(bits)), kv.copy_(i32(b.kv_len))
        g.replay()
        torch.cuda.synchronize()
        check(host(o[0]), expected(b, bits), kind)
    assert torch.equal(o[0], want)
