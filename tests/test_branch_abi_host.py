"""The entry points of requests that branch refuse bad arguments on the host, before any launch (fake device addresses, no
GPU needed: every call here is refused or has nothing to do); the host helper for trees."""
import ctypes as C
import itertools

import numpy as np
import pytest

import branch_ref
from test_paged_abi_host import cache, lib


def refused(status_says, status, says):
    got, text = status_says
    assert got == status and says in text, text


# ---- page fork ----
FR, FN, FPAGES, FW, FSTRIDE = 4, 3, 30, 8, 20
FORK = dict(src=FN, dst=FN, first=FN, len=FN, held=FR, n_free=1, block_table=(FR - 1) * FSTRIDE + FW, free_list=FPAGES, held_out=FR,
            n_free_out=1, copies=3 * FN, status=2)
FORK_READ = ("src", "dst", "first", "len", "held", "n_free", "free_list")


def fork(desc=(), **moved):
    _, b, L = lib()
    d = b.wam_page_fork_desc(R=FR, N=FN, page_size=16, n_pages=FPAGES, max_pages=FW, table_stride=FSTRIDE)
    for k, v in dict(desc).items():
        setattr(d, k, v)
    at = {n: 4096 * (i + 1) for i, n in enumerate(FORK)} | moved
    return L.wam_page_fork(C.byref(d), *(at[n] for n in FORK), None), L.wam_last_error().decode()


@pytest.mark.parametrize("desc,ptrs,status,says", [
    (dict(R=-1), {}, 1, "negative"), (dict(N=-1), {}, 1, "N=-1"), (dict(R=4097), {}, 2, "exceeds"), (dict(N=4097), {}, 2, "exceeds"),
    (dict(page_size=8), {}, 2, "page_size"), (dict(n_pages=-1), {}, 1, "n_pages"), (dict(max_pages=-1), {}, 1, "negative"),
    (dict(max_pages=1 << 30, table_stride=1 << 30), {}, 2, "2^31"), (dict(table_stride=7), {}, 1, "table_stride"),
    *(({}, {n: 0}, 1, f"{n} is NULL") for n in FORK if n != "first"), *(({}, {n: 4098}, 1, f"{n} is not 4-byte") for n in FORK)])
def test_fork_refusals(desc, ptrs, status, says):
    refused(fork(desc, **ptrs), status, says)


def pairs(sizes, read):
    return [p for p in itertools.combinations(sizes, 2) if not set(p) <= set(read)]


def check_overlaps(call, sizes, a, b):
    """b at a's first int, on a's last one, and ending on a's first one."""
    at = 4096 * (1 + list(sizes).index(a))
    for where in (at, at + 4 * (sizes[a] - 1), at - 4 * (sizes[b] - 1)):
        status, says = call(**{b: where})
        assert status == 1 and "overlap" in says and a in says and b in says, (where - at, says)


@pytest.mark.parametrize("a,b", pairs(FORK, FORK_READ))
def test_fork_overlaps(a, b):
    check_overlaps(fork, FORK, a, b)


# ---- page collect ----
COLLECT = dict(cache_len=FR, held=FR, block_table=(FR - 1) * FSTRIDE + FW, free_list=FPAGES, held_out=FR, n_free_out=1, status=2)


def collect(desc=(), **moved):
    _, b, L = lib()
    d = b.wam_page_collect_desc(R=FR, page_size=16, n_pages=FPAGES, max_pages=FW, table_stride=FSTRIDE)
    for k, v in dict(desc).items():
        setattr(d, k, v)
    at = {n: 4096 * (i + 1) for i, n in enumerate(COLLECT)} | moved
    return L.wam_page_collect(C.byref(d), *(at[n] for n in COLLECT), None), L.wam_last_error().decode()


@pytest.mark.parametrize("desc,ptrs,status,says", [
    (dict(R=-1), {}, 1, "negative"), (dict(R=4097), {}, 2, "exceeds"), (dict(page_size=24), {}, 2, "page_size"),
    (dict(n_pages=(1 << 20) + 1), {}, 2, "exceeds"), (dict(max_pages=-2), {}, 1, "negative"), (dict(table_stride=3), {}, 1, "table_stride"),
    *(({}, {n: 0}, 1, f"{n} is NULL") for n in COLLECT), *(({}, {n: 4097}, 1, f"{n} is not 4-byte") for n in COLLECT)])
def test_collect_refusals(desc, ptrs, status, says):
    refused(collect(desc, **ptrs), status, says)


@pytest.mark.parametrize("a,b", pairs(COLLECT, ("cache_len", "held", "block_table")))
def test_collect_overlaps(a, b):
    check_overlaps(collect, COLLECT, a, b)


# ---- page copy ----
@pytest.mark.parametrize("bad,N,ptr,status,says", [
    ({}, -1, 4096, 1, "N=-1"), ({}, 3, 0, 1, "copies is NULL"), ({}, 3, 4099, 1, "copies is not"), (dict(Dh=32), 3, 4096, 2, "Dh=32"),
    (dict(page_size=4096, page_stride=4096 * 256), (1 << 31) - 1, 4096, 2, "one launch")])
def test_copy_refusals(bad, N, ptr, status, says):
    _, _, L = lib()
    c = cache(**bad)
    refused((L.wam_page_copy(C.byref(c), N, ptr, None), L.wam_last_error().decode()), status, says)


# ---- compact ----
@pytest.mark.parametrize("bad,desc,ptrs,status,says", [
    ({}, dict(R=-1), {}, 1, "negative"), ({}, dict(T=-1), {}, 1, "T=-1"), ({}, dict(max_pages=-1), {}, 1, "negative"),
    ({}, dict(table_stride=2), {}, 1, "table_stride"), (dict(v=0), {}, {}, 1, "cache v"), (dict(k_exp=12290, v_scale=1.0), {}, {}, 1, "k_exp"),
    (dict(Hkv=4096, head_stride=128, tok_stride=1 << 19, page_size=16, page_stride=1 << 24), dict(R=1 << 20, max_pages=3), {}, 2, "one launch"),
    *(({}, {}, {n: 0}, 1, f"{n} is NULL") for n in ("block_table", "q_start", "kv_len", "keep", "n_keep")),
    *(({}, {}, {n: 4098}, 1, f"{n} is not") for n in ("block_table", "q_start", "q_len", "kv_len", "keep", "n_keep"))])
def test_compact_refusals(bad, desc, ptrs, status, says):
    _, b, L = lib()
    c = cache(**bad)
    d = b.wam_cache_compact_desc(R=2, T=5, max_pages=3, table_stride=3)
    for k, v in desc.items():
        setattr(d, k, v)
    p = dict(block_table=4096, q_start=4096, q_len=None, kv_len=4096, keep=4096, n_keep=4096) | ptrs
    refused((L.wam_cache_compact(C.byref(d), C.byref(c), *p.values(), None), L.wam_last_error().decode()), status, says)


# ---- tree attention ----
@pytest.mark.parametrize("bad,desc,ptrs,status,says", [
    ({}, dict(R=-1), {}, 1, "negative"), ({}, dict(Hq=3), {}, 1, "multiple of Hkv"), ({}, dict(max_kv=(1 << 30) + 1), {}, 2, "2^30"),
    ({}, dict(T=1 << 30), {}, 2, "2^31"), ({}, dict(scale=float("nan")), {}, 1, "scale"), ({}, dict(table_stride=2), {}, 1, "table_stride"),
    ({}, dict(mask_words=-1), {}, 1, "mask_words"), ({}, dict(mask_stride=0), {}, 1, "mask_stride"), ({}, dict(q_tok_stride=256), {}, 1, "strides"),
    ({}, dict(o_tok_stride=516), {}, 1, "strides"), ({}, dict(mask_stride=1 << 60), {}, 1, "mask_stride"), (dict(Dh=96), {}, {}, 2, "Dh=96"),
    *(({}, {}, {n: 0}, 1, f"{n} is NULL") for n in ("q", "block_table", "q_start", "kv_len", "mask", "o")),
    *(({}, {}, {n: 4098}, 1, f"{n} is not") for n in ("q", "block_table", "q_start", "q_len", "kv_len", "mask", "o")),
    ({}, dict(max_kv=100000, max_pages=3000, table_stride=3000), dict(ws=0), 3, "workspace"),
    ({}, dict(max_kv=100000, max_pages=3000, table_stride=3000), dict(ws=4096 + 128), 3, "workspace")])
def test_tree_refusals(bad, desc, ptrs, status, says):
    _, b, L = lib()
    c = cache(**bad)
    d = b.wam_attn_tree_desc(R=2, T=5, Hq=4, max_pages=3, max_kv=100, mask_words=1, table_stride=3, q_tok_stride=512, o_tok_stride=512,
                             mask_stride=1, scale=0.0)
    for k, v in desc.items():
        setattr(d, k, v)
    p = dict(q=4096, block_table=4096, q_start=4096, q_len=None, kv_len=4096, mask=4096, o=8192, ws=1 << 20) | ptrs
    refused((L.wam_attn_tree(C.byref(d), C.byref(c), *p.values(), 1 << 40, None), L.wam_last_error().decode()), status, says)


# ---- verification ----
VR, VT, VV = 2, 6, 50
VERIFY = dict(p=VT * VV, q=VT * VV, tokens=VT, parent=VT, u=VT, u_next=VR, q_start=VR + 1, q_len=VR, kv_len=VR, path=VT, n_path=VR,
              next_token=VR, cache_len=VR)
VERIFY_READ = ("p", "q", "tokens", "parent", "u", "u_next", "q_start", "q_len", "kv_len")


def verify(desc=(), ws=1 << 30, bytes_=1 << 40, **moved):
    _, b, L = lib()
    d = b.wam_verify_tree_desc(R=VR, T=VT, V=VV, drawn=1, p_stride=VV, q_stride=VV)
    for k, v in dict(desc).items():
        setattr(d, k, v)
    at = {n: 65536 * (i + 1) for i, n in enumerate(VERIFY)} | moved
    return L.wam_verify_tree(C.byref(d), *(at[n] for n in VERIFY), ws, bytes_, None), L.wam_last_error().decode()


@pytest.mark.parametrize("desc,ptrs,status,says", [
    (dict(R=-1), {}, 1, "negative"), (dict(T=-1), {}, 1, "negative"), (dict(V=0), {}, 1, "V=0"), (dict(V=(1 << 20) + 1, p_stride=1 << 21, q_stride=1 << 21), {}, 2, "exceeds"),
    (dict(drawn=2), {}, 1, "drawn=2"), (dict(p_stride=49), {}, 1, "strides"), (dict(q_stride=49), {}, 1, "strides"),
    (dict(p_stride=1 << 61), {}, 1, "overflows"), (dict(q_stride=1 << 61), {}, 1, "overflows"), (dict(R=(1 << 31) - 1), {}, 2, "one launch"),
    ({}, dict(q=0), 1, "drawn is 1"), (dict(drawn=0), {}, 1, "drawn is 1"), ({}, dict(kv_len=0), 1, "both"), ({}, dict(cache_len=0), 1, "both"),
    *(({}, {n: 0}, 1, f"{n} is NULL") for n in VERIFY if n not in ("q", "q_len", "kv_len", "cache_len")),
    *(({}, {n: 65538}, 1, f"{n} is not 4-byte") for n in VERIFY),
    ({}, dict(ws=0), 3, "workspace"), ({}, dict(ws=1 << 30 | 16), 3, "workspace"), ({}, dict(bytes_=10), 3, "workspace")])
def test_verify_refusals(desc, ptrs, status, says):
    refused(verify(desc, **ptrs), status, says)


@pytest.mark.parametrize("a,b", pairs(VERIFY, VERIFY_READ))
def test_verify_overlaps(a, b):
    check = {**VERIFY}
    at = 65536 * (1 + list(VERIFY).index(a))
    for where in (at, at + 4 * (check[a] - 1), at - 4 * (check[b] - 1)):
        status, says = verify(**{b: where})
        assert status == 1 and "overlap" in says and a in says and b in says, says


def test_nothing_to_do():
    """Calls of no requests, tokens or copies end before a launch."""
    _, b, L = lib()
    c = cache()
    assert L.wam_page_copy(C.byref(c), 0, None, None) == 0
    d = b.wam_cache_compact_desc(R=0, T=5, max_pages=3, table_stride=3)
    assert L.wam_cache_compact(C.byref(d), C.byref(c), None, None, None, None, None, None, None) == 0
    d = b.wam_attn_tree_desc(R=2, T=0, Hq=4, max_pages=3, max_kv=100, mask_words=0, table_stride=3, q_tok_stride=512, o_tok_stride=512)
    assert L.wam_attn_tree(C.byref(d), C.byref(c), None, None, None, None, None, None, None, None, 0, None) == 0
    assert verify(dict(R=0)) [0] == 0


# ---- the mask of a tree ----
@pytest.mark.parametrize("n,words", [(0, 0), (1, 1), (32, 1), (33, 2), (70, 5)])
def test_tree_mask(n, words):
    w, _, _ = lib()
    g = np.random.default_rng(n)
    parent = [-1 if i == 0 or g.random() < 0.1 else int(g.integers(0, i)) for i in range(n)]
    assert np.array_equal(w.wam_tree_mask(parent, words).numpy(), branch_ref.ancestors(parent, words))


def test_tree_mask_refusals():
    w, _, L = lib()
    for parent, words in (([0], 1), ([-1, 1], 1), ([-1, -2], 1), ([-1] * 33, 1), ([-1], 0)):
        with pytest.raises(w.WamError):
            w.wam_tree_mask(parent, words)
    assert L.wam_tree_mask(None, 3, 1, None) == 1 and b"NULL" in L.wam_last_error()
