"""wam_attn_paged and wam_attn_cross against their definitions in 64 bits, element by element."""
import numpy as np
import pytest

import paged_ref
from gpu_helpers import host, log, workspace
from paged_ref import Batch

pytestmark = pytest.mark.gpu
OLD = 5.0  # what the output held before


def run_paged(b, chunk, max_kv=None, q_len=None, scale=0.0, cache=None, q=None):
    """The call on the device; o rows wider than the heads, to see that nothing else is written."""
    import torch
    import paper_2602_15922_amd as w
    c = cache or b.cache()
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    wide = torch.full((b.T, b.Hq + 1, b.Dh), OLD, dtype=torch.bfloat16, device="cuda")
    n = w.wam_attn_paged_workspace_bytes(c, R=len(b.lens), T=b.T, Hq=b.Hq, max_kv=b.width * b.ps if max_kv is None else max_kv)
    ws = workspace(n).fill_(0xFF)
    w.wam_attn_paged(c, b.q.cuda() if q is None else q, i32(b.table), i32(b.q_start), i32(b.kv_len), wide[:, :b.Hq], ws, max_kv=max_kv,
                     chunk=chunk, q_len=None if q_len is None else i32(q_len), scale=scale)
    torch.cuda.synchronize()
    assert (wide[:, b.Hq:] == OLD).all()
    return host(wide[:, :b.Hq])


def check(got, ref, what=""):
    o, a, mine = ref
    assert np.isfinite(got).all(), what
    worst = np.abs(got - o)[mine] - paged_ref.attention_tolerance(a)[mine]
    assert worst.max(initial=-1) <= 0, (what, float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))
    assert np.all(got[~mine] == OLD), what


MIXED = [(1, 1), (1, 63), (0, 30), (3, 3), (1, 64), (1, 65), (17, 40), (40, 300), (1, 129), (130, 131), (2, 0), (5, 3), (1, 700)]


@pytest.mark.parametrize("Hq,Hkv,Dh,ps,layout,fp8", [
    (1, 1, 128, 16, "nhd", False), (8, 2, 128, 48, "hnd", False), (3, 3, 64, 64, "kv", False), (16, 1, 64, 16, "nhd", False),
    (5, 5, 128, 32, "kv", False), (40, 1, 128, 16, "nhd", False), (6, 2, 64, 1024, "hnd", False), (1, 1, 128, 16, "nhd", True),
    (8, 2, 128, 48, "hnd", True), (5, 5, 128, 32, "kv", True), (40, 1, 128, 16, "nhd", True)])
def test_mixed_lengths(Hq, Hkv, Dh, ps, layout, fp8):
    b = Batch(MIXED, Hq, Hkv, Dh, ps, seed=Hq + ps, fp8=fp8, layout=layout)
    for chunk in (0, 1, 7):
        log(f"paged mixed Hq={Hq} Hkv={Hkv} Dh={Dh} ps={ps} {layout} fp8={fp8} chunk={chunk}")
        check(run_paged(b, chunk), b.expected(chunk), f"chunk={chunk}")


AXIS = [([(1, n) for n in (1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 127, 128, 255, 256, 257, 511, 513, 1023, 1025)], 4, 1, 128, 16, 1),
        ([(1, 5000)], 8, 8, 128, 64, 0), ([(1, 3001), (1, 17), (2, 2999)], 5, 5, 64, 16, 1), ([(33, 2100)], 2, 1, 128, 16, 1),
        ([(128, 1300), (129, 129)], 2, 2, 128, 64, 32), ([(257, 700)], 3, 1, 64, 48, 257), ([(64, 4000)], 1, 1, 128, 32, 0)]


@pytest.mark.parametrize("lens,Hq,Hkv,Dh,ps,chunk,fp8", [(*x, f) for x in AXIS for f in (False, True) if x[3] == 128 or not f])
def test_key_axis_lengths(lens, Hq, Hkv, Dh, ps, chunk, fp8):
    b = Batch(lens, Hq, Hkv, Dh, ps, seed=3, fp8=fp8)
    log(f"paged lengths {lens[:3]} Hq={Hq} Hkv={Hkv} Dh={Dh} ps={ps} chunk={chunk} fp8={fp8}")
    check(run_paged(b, chunk), b.expected(chunk))


@pytest.mark.parametrize("fp8", [False, True])
def test_absent_pages_are_not_seen(fp8):
    for lens in ([(1, 200), (1, 100), (1, 700)], [(60, 200), (70, 100), (150, 300)]):
        b = Batch(lens, 4, 2, 128, 16, seed=8, fp8=fp8)
        b.table[0, 3], b.table[0, 12], b.table[1, :], b.table[2, 1::2] = -1, b.n_pages, -2 ** 31, 2 ** 31 - 1
        for chunk in (0, 1):
            log(f"paged absent pages {lens} fp8={fp8} chunk={chunk}")
            check(run_paged(b, chunk), b.expected(chunk))


@pytest.mark.parametrize("n,m,G,Dh,fp8", [(100, 1500, 1, 128, False), (300, 1300, 2, 64, False), (90, 2000, 1, 128, True),
                                          (40, 900, 3, 128, False), (3, 2500, 4, 128, True), (1, 300, 1, 64, False)])
def test_one_request_with_holes(n, m, G, Dh, fp8):
    """One request (the eight-wavefront form where its rows are many): pages missing at the start, in the middle, at the
    end, and whole parts of the key axis without any."""
    b = Batch([(n, m)], 2 * G, 2, Dh, 16, seed=n + m, fp8=fp8, tail=1)
    b.table[0, :2], b.table[0, 30:70], b.table[0, -1], b.table[0, 5] = -1, b.n_pages, -1, 2 ** 30
    for chunk in (0, 1):
        log(f"paged one request n={n} m={m} G={G} Dh={Dh} fp8={fp8} chunk={chunk}")
        check(run_paged(b, chunk), b.expected(chunk), f"chunk={chunk}")
    b.table[:] = -1
    got = run_paged(b, 0)
    assert np.all(got[:n] == 0) and np.all(got[n:] == OLD)


@pytest.mark.parametrize("Hq,Hkv,Dh", [(2, 1, 128), (3, 3, 64)])
def test_many_requests(Hq, Hkv, Dh):
    """Hundreds of requests, empty ones among them: more than one pass of a wavefront over their starts."""
    g = np.random.default_rng(Hq)
    for new in (2, 40):
        lens = []
        for _ in range(300):
            n = int(g.integers(0, new + 1))
            lens.append((n, n + int(g.integers(0, 60))))
        b = Batch(lens, Hq, Hkv, Dh, 16, seed=1, tail=70)
        log(f"paged many requests Hq={Hq} Dh={Dh} new<={new}")
        check(run_paged(b, 1), b.expected(1))


def test_two_calls_at_once():
    """Two streams, two workspaces, one cache: neither disturbs the other."""
    import torch
    import paper_2602_15922_amd as w
    bs = [Batch([(1, 1500), (2, 900)], 8, 2, 128, 16, seed=41), Batch([(200, 700)], 8, 2, 128, 16, seed=42)]
    log("paged two streams")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    args, streams = [], [torch.cuda.Stream() for _ in bs]
    for b in bs:
        c = b.cache()
        n = w.wam_attn_paged_workspace_bytes(c, R=len(b.lens), T=b.T, Hq=8, max_kv=b.width * 16)
        args.append((c, b.q.cuda(), i32(b.table), i32(b.q_start), i32(b.kv_len),
                     torch.full((b.T, 8, 128), OLD, dtype=torch.bfloat16, device="cuda"), workspace(n)))
    torch.cuda.synchronize()
    for _ in range(20):
        for a, s in zip(args, streams):
            w.wam_attn_paged(*a, chunk=1, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(args, bs):
        check(host(a[5]), b.expected(1))


def test_lengths_past_the_table_and_max_kv():
    b = Batch([(4, 100), (1, 40), (50, 90)], 4, 2, 64, 16, seed=2)
    log("paged max_kv")
    check(run_paged(b, 0, max_kv=48), b.expected(0, max_kv=48))
    check(run_paged(b, 1, max_kv=90), b.expected(1, max_kv=90))
    check(run_paged(b, 1, max_kv=0), b.expected(1, max_kv=0))
    b.kv_len[1] = 10 ** 9  # past the table's width: its keys end there, and the position counts
    b.table[1] = b.table[0]
    b.k.nan_to_num_(0.0), b.v.nan_to_num_(0.0)
    log("paged kv_len past the width")
    check(run_paged(b, 0), b.expected(0))
    b.kv_len[:] = [-5, 0, -2 ** 31]
    got = run_paged(b, 0)
    assert np.all(got[:55] == 0) and np.all(got[55:] == OLD)


def test_padded_batches_and_starts_out_of_range():
    b = Batch([(5, 30), (0, 9), (40, 200), (1, 1)], 6, 3, 64, 32, seed=4, gap=3)
    ref = b.expected(1)
    log("paged padded")
    check(run_paged(b, 1, q_len=b.q_len), ref)
    check(run_paged(b, 1, q_len=b.q_len), ref)
    # starts past T, negative and falling: cut, never outside the buffers
    for starts in ([0, 5, 5, 45, 10 ** 9], [-100, 5, 5, 45, 46], [0, 60, 3, 45, 46], [90, 80, 70, 60, 50], [-9, -8, -7, -6, -5]):
        log(f"paged starts {starts}")
        b.q_start = np.array(starts, np.int32)
        run_paged(b, 1)


def test_strides_of_q_and_scale():
    import torch
    b = Batch([(3, 50), (70, 70)], 4, 4, 64, 16, seed=6)
    qkv = torch.zeros(b.T, 12 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    qkv[:, 64:64 + 256] = b.q.cuda().flatten(1)
    log("paged strided q")
    check(run_paged(b, 1, q=qkv[:, 64:64 + 256].unflatten(1, (4, 64)), scale=0.3), b.expected(1, scale=0.3))


def test_large_scores():
    """Scores of hundreds, whose maximum moves from tile to tile: one key takes the whole weight."""
    b = Batch([(1, 900), (40, 500)], 2, 1, 128, 16, seed=12, junk=np.inf)
    b.q *= 16
    log("paged large scores")
    o, a, mine = b.expected(1)
    # a score of size s <= 1024 is off by s 2^-24 * sqrt(128) in fp32, its weight by the same factor: 2^-10.5 of it
    got = run_paged(b, 1)
    tol = paged_ref.attention_tolerance(a) + 2.0 ** -10 * a
    assert np.isfinite(got).all() and np.all((np.abs(got - o) <= tol)[mine])


def test_infinite_keys_in_masked_places():
    """Keys (not values) that a causal row does not see may hold anything."""
    b = Batch([(6, 70)], 2, 2, 64, 16, seed=13)
    pg, row = b.table[0, 69 // 16], 69 % 16
    b.k[pg, row] = float("inf")  # the last token's key: only the last row sees it
    log("paged infinite key")
    got, (o, a, mine) = run_paged(b, 1), b.expected(1)
    assert np.all((np.abs(got - o) <= paged_ref.attention_tolerance(a))[:5])


@pytest.mark.parametrize("lens,Hq,Hkv,Dh,chunk,fp8", [
    ([(6, 70), (2, 2), (9, 40)], 2, 2, 64, 1, False), ([(6, 70), (3, 129)], 2, 2, 128, 1, False), ([(5, 700), (4, 90)], 8, 2, 128, 1, False),
    ([(7, 70), (8, 333)], 8, 2, 64, 3, False), ([(6, 170), (5, 64)], 4, 2, 128, 1, True), ([(150, 200), (40, 140), (3, 65)], 4, 2, 128, 1, False),
    ([(150, 200), (200, 240)], 3, 3, 64, 7, False), ([(100, 190), (65, 65)], 4, 2, 128, 1, True), ([(130, 400)], 1, 1, 128, 1, False),
    ([(140, 2000)], 2, 1, 128, 32, False), ([(300, 300)], 1, 1, 64, 1, False), ([(90, 1500)], 2, 2, 128, 1, True)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(lens, Hq, Hkv, Dh, chunk, fp8):
    """V of keys that some rows of a request see and others do not: NaN over a whole row, infinities of both signs in
    some dims.  The rows that see none are as ever; the others hold what the formula gives, dim by dim."""
    b = Batch(lens, Hq, Hkv, Dh, 16, seed=sum(n + m for n, m in lens) + Dh, fp8=fp8)
    for r, (n, m) in enumerate(lens):
        for back, dims, val in ((1, slice(None), float("nan")), (2, 3, float("inf")), (2, 5, float("-inf")), (3, 3, float("-inf")),
                                ((n + 1) // 2, 17, float("inf")), ((n + 1) // 2, 18, float("nan")), (n - 1, Dh - 1, float("-inf"))):
            j = m - max(1, min(back, n - 1))
            b.v[b.table[r, j // 16], j % 16, :, dims] = 0x7F if fp8 else val
    log(f"paged values not finite {lens} Hq={Hq} Hkv={Hkv} Dh={Dh} chunk={chunk} fp8={fp8}")
    with np.errstate(invalid="ignore"):
        got, (o, a, mine) = run_paged(b, chunk), b.expected(chunk)
    fin = np.isfinite(o)
    at = mine[:, None, None] & ~fin
    assert np.array_equal(np.isnan(got[at]), np.isnan(o[at]))
    inf = at & np.isinf(o)
    assert np.array_equal(got[inf], o[inf])
    ok = mine[:, None, None] & fin
    assert np.isfinite(got[ok]).all()
    assert np.all(np.abs(got[ok] - o[ok]) <= paged_ref.attention_tolerance(a)[ok])
    assert np.all(got[~mine] == OLD)


@pytest.mark.parametrize("lens,Hq,Hkv,Dh", [([(1, 1), (1, 5000), (1, 90)], 8, 8, 128), ([(3, 3000), (2, 40)], 5, 5, 64),
                                            ([(100, 4000)], 1, 1, 128), ([(20, 3000)] * 30, 16, 2, 128), ([(150, 400)], 2, 1, 64)])
def test_keys_that_are_nan_make_the_rows_that_see_them_nan(lens, Hq, Hkv, Dh):
    """One key, and the first half of a request's keys: whole parts of a split key axis whose scores are all NaN."""
    for first in (False, True):
        b = Batch(lens, Hq, Hkv, Dh, 16, seed=21 + Dh)
        o, a, mine = b.expected(1)
        ref = np.broadcast_to(mine[:, None, None], o.shape).copy()  # rows that see none
        for r, (n, m) in enumerate(lens):
            if r % 2 == 1:
                continue
            keys = range(0, (m + 1) // 2) if first else [m - 1]
            for j in keys:
                b.k[b.table[r, j // 16], j % 16, Hkv - 1] = float("nan")
            at = b.q_start[r] + np.arange(n)
            ref[at if first else at[-1:], Hq - Hq // Hkv:] = False
        log(f"paged NaN keys {lens[:2]} Hq={Hq} first={first}")
        got = run_paged(b, 1)
        assert np.isfinite(got[ref]).all()
        assert np.isnan(got[mine[:, None, None] & ~ref]).all()
        assert np.all(np.abs(got[ref] - o[ref]) <= paged_ref.attention_tolerance(a)[ref])


def test_offsets_past_32_bits():
    """Pages whose rows lie more than 4 GiB apart in elements and bytes."""
    import torch
    import paper_2602_15922_amd as w
    b = Batch([(1, 40), (33, 50)], 2, 1, 128, 16, seed=14)
    n, span = b.n_pages, 400_000_000  # elements between pages: 8 of them pass 2^32 bytes and elements alike
    log("paged far pages")
    big = torch.empty(n * span, dtype=torch.bfloat16, device="cuda")
    k = torch.as_strided(big, (n, 16, 1, 128), (span, 128, 128, 1))
    v = torch.as_strided(big, (n, 16, 1, 128), (span, 128, 128, 1), storage_offset=16 * 128)
    k.copy_(b.k), v.copy_(b.v)
    assert n * span * 2 > 2 ** 32
    check(run_paged(b, 1, cache=w.make_paged_cache(k, v)), b.expected(1))
    del big, k, v
    torch.cuda.empty_cache()


# ---- cross-attention ----
def cross_case(q_lens, k_lens, Hq, Hkv, Dh, seed, k_at=None, gap=0, tail=3):
    import torch
    g = torch.Generator().manual_seed(seed)
    q_start = np.cumsum([0] + [n + gap for n in q_lens])
    k_start = np.cumsum([0] + list(k_lens)) if k_at is None else np.array(list(k_at) + [0])
    S = int(max([a + n for a, n in zip(k_start, k_lens)] + [0])) + 2
    T = int(q_start[-1]) + tail
    q = torch.randn(T, Hq, Dh, generator=g).bfloat16()
    kv = torch.randn(S, 2, Hkv, Dh, generator=g).bfloat16()
    used = torch.zeros(S, dtype=torch.bool)
    for a, n in zip(k_start, k_lens):
        used[a:a + n] = True
    kv[~used] = float("nan")
    o, a, mine = np.zeros((T, Hq, Dh)), np.zeros((T, Hq, Dh)), np.zeros(T, bool)
    x, y = q.double().numpy(), kv.double().numpy()
    for r, (n, m) in enumerate(zip(q_lens, k_lens)):
        at = int(q_start[r])
        mine[at:at + n] = True
        for h in range(Hq):
            kk, vv = y[k_start[r]:k_start[r] + m, 0, h // (Hq // Hkv)], y[k_start[r]:k_start[r] + m, 1, h // (Hq // Hkv)]
            o[at:at + n, h], a[at:at + n, h] = paged_ref.attend(x[at:at + n, h], kk, vv, np.ones((n, m), bool), Dh ** -0.5)
    return q, kv, q_start, k_start, S, (o, a, mine)


def run_cross(q, kv, q_start, k_start, max_k=None, q_len=None, k_len=None):
    import torch
    import paper_2602_15922_amd as w
    i32 = lambda x: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    T, Hq, Dh = q.shape
    wide = torch.full((T, Hq + 1, Dh), OLD, dtype=torch.bfloat16, device="cuda")
    d = kv.cuda()
    n = w.wam_attn_cross_workspace_bytes(R=len(q_start) - 1, T=T, Hq=Hq, Hkv=kv.shape[2], Dh=Dh, max_k=kv.shape[0] if max_k is None else max_k)
    ws = workspace(n).fill_(0xFF)
    w.wam_attn_cross(q.cuda(), d[:, 0], d[:, 1], i32(q_start), i32(k_start), wide[:, :Hq], ws, max_k=max_k, q_len=i32(q_len), k_len=i32(k_len))
    torch.cuda.synchronize()
    assert (wide[:, Hq:] == OLD).all()
    return host(wide[:, :Hq])


@pytest.mark.parametrize("q_lens,k_lens,Hq,Hkv,Dh", [
    ([144, 1, 30], [32, 0, 77], 8, 8, 64), ([1] * 9, [1, 2, 63, 64, 65, 300, 0, 700, 1500], 8, 2, 128),
    ([200, 130], [512, 77], 3, 3, 128), ([1, 0, 2, 129], [5, 3, 33, 640], 20, 4, 64), ([1], [1], 1, 1, 128),
    ([16, 31], [2000, 31], 4, 1, 128), ([150], [700], 2, 2, 128), ([500], [300], 6, 2, 64)])
def test_cross(q_lens, k_lens, Hq, Hkv, Dh):
    log(f"cross {q_lens} {k_lens} Hq={Hq} Hkv={Hkv} Dh={Dh}")
    q, kv, qs, ks, S, ref = cross_case(q_lens, k_lens, Hq, Hkv, Dh, 5)
    check(run_cross(q, kv, qs, ks), ref, "packed")
    check(run_cross(q, kv, qs, ks[:-1], max_k=max(k_lens), k_len=k_lens), ref, "lengths")
    q, kv, qs, ks, S, ref = cross_case(q_lens, k_lens, Hq, Hkv, Dh, 6, gap=5, k_at=[7 * i % 4 for i in range(len(k_lens))])
    check(run_cross(q, kv, qs, ks[:-1], q_len=q_lens, k_len=k_lens), ref, "padded rows, shared keys")


def test_cross_starts_and_lengths_out_of_range():
    q, kv, qs, ks, S, (o, a, mine) = cross_case([5, 70], [30, 90], 4, 2, 64, 7)
    kv = kv.nan_to_num(0.0)
    for at, n in (([0, 10 ** 9], [30, 90]), ([-50, 30], [30, 10 ** 9]), ([0, 0], [-1, -2 ** 31]), ([S - 1, S], [2 ** 31 - 1, 5])):
        log(f"cross starts {at} lengths {n}")
        got = run_cross(q, kv, qs, at, k_len=n)
        assert np.isfinite(got).all() and np.all(got[~mine] == OLD)
    import torch
    empty = torch.zeros(0, 2, 2, 64, dtype=torch.bfloat16)
    log("cross no keys at all")
    got = run_cross(q, empty, qs, [0, 0], k_len=[3, 0])
    assert np.all(got[mine] == 0) and np.all(got[~mine] == OLD)


def test_agrees_with_the_attention_over_one_block():
    """One history for the batch, one head each: the same as wam_attn_blockcausal, within both tolerances."""
    import torch
    import paper_2602_15922_amd as w
    b = Batch([(96, 288)], 4, 4, 128, 32, seed=21)
    log("paged against one block")
    k, v, _ = b.kv64(0)
    dk, dv = (torch.from_numpy(x).to(torch.bfloat16).cuda()[None] for x in (k, v))
    o = torch.empty(1, 96, 4, 128, dtype=torch.bfloat16, device="cuda")
    w.wam_attn_blockcausal(b.q[:96].cuda()[None], dk, dv, o, w.append_chunks([96 * 2], [48, 48]))
    torch.cuda.synchronize()
    got, (_, a, mine) = run_paged(b, 48), b.expected(48)
    assert np.all(np.abs(got[:96] - host(o[0])) <= 2 * paged_ref.attention_tolerance(a)[:96])


@pytest.mark.parametrize("lens", [[(1, 900), (1, 77)], [(140, 900), (3, 77)]])
def test_streams_graphs_and_repeats(lens):
    """The same call on another stream, again (bit for bit), and replayed with other lengths in the same buffers."""
    import torch
    import paper_2602_15922_amd as w
    b = Batch(lens, 8, 2, 128, 16, seed=31)
    log(f"paged graph {lens}")
    c, q = b.cache(), b.q.cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, qs, kv = i32(b.table), i32(b.q_start), i32(b.kv_len)
    o = torch.full((b.T, 8, 128), OLD, dtype=torch.bfloat16, device="cuda")
    ws = workspace(w.wam_attn_paged_workspace_bytes(c, R=2, T=b.T, Hq=8, max_kv=b.width * 16)).fill_(0xFF)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    w.wam_attn_paged(c, q, table, qs, kv, o, ws, chunk=1, stream=s)
    s.synchronize()
    check(host(o), b.expected(1))
    first = o.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        w.wam_attn_paged(c, q, table, qs, kv, o, ws, chunk=1)
    for m in ([900, 77], [640, 70], [lens[0][0], 80], [900, 77]):
        b.kv_len = np.array(m, np.int32)
        b.k.nan_to_num_(0.0), b.v.nan_to_num_(0.0)
        b.dk.copy_(b.k), b.dv.copy_(b.v)
        kv.copy_(torch.tensor(m, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        check(host(o), b.expected(1), str(m))
    assert torch.equal(o, first)
