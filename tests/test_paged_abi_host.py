"""The paged cache's entry points refuse bad arguments on the host, before any launch (fake device addresses, no
GPU needed); the reference functions of the GPU tests against brute force."""
import ctypes as C

import numpy as np
import pytest

import paged_ref


def lib():
    import paper_2602_15922_amd as w
    return w, w.binding, w.lib()


def cache(**kw):
    _, b, _ = lib()
    c = b.wam_paged_cache(k=4096, v=8192, k_exp=None, page_stride=64 * 256, tok_stride=256, head_stride=128, n_pages=10,
                          page_size=64, Hkv=2, Dh=128, v_scale=0.0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


FP8 = dict(k_exp=12288, v_scale=1.0)


@pytest.mark.parametrize("bad,status,says", [
    (dict(Dh=96), 2, b"Dh=96"), (dict(Dh=64, head_stride=64, **FP8), 2, b"FP8"), (dict(Hkv=0), 1, b"Hkv"),
    (dict(page_size=24), 2, b"page_size"), (dict(page_size=0), 2, b"page_size"), (dict(n_pages=-1), 1, b"n_pages"),
    (dict(n_pages=1 << 26), 2, b"2^31"), (dict(k=0), 1, b"cache k is NULL"), (dict(v=8200), 1, b"aligned"),
    (dict(tok_stride=100), 1, b"strides"), (dict(tok_stride=250), 1, b"multiples of 8"), (dict(head_stride=0), 1, b"strides"),
    (dict(page_stride=-256), 1, b"strides"), (dict(tok_stride=1 << 25), 2, b"2^31"), (dict(head_stride=1 << 33), 2, b"2^31"),
    (dict(page_stride=1 << 61), 1, b"overflows"), (dict(k_exp=12290, v_scale=1.0), 1, b"aligned"),
    (dict(k_exp=12288, v_scale=0.0), 1, b"v_scale"), (dict(k_exp=12288, v_scale=float("inf")), 1, b"v_scale"),
    (dict(tok_stride=264, page_stride=64 * 264, **FP8), 1, b"multiples of 128"),
])
def test_cache_refusals(bad, status, says):
    w, b, L = lib()
    c = cache(**bad)
    d = b.wam_attn_paged_desc(R=2, T=5, Hq=4, max_pages=3, max_kv=100, chunk=0, table_stride=3, q_tok_stride=512,
                              o_tok_stride=512, scale=0.0)
    assert L.wam_attn_paged(C.byref(d), C.byref(c), 4096, 8192, 4096, None, 4096, 8192, 1 << 20, 1 << 40, None) == status
    assert says in L.wam_last_error()
    r = b.wam_rope_paged_desc(T=5, Hq=4, n_axes=1, halves=0, theta=1e4, qkv_tok_stride=1024, q_tok_stride=512)
    r.pairs[0] = 64
    assert L.wam_rope_qkv_paged(C.byref(r), C.byref(c), 4096, 4096, 4096, 8192, None) == status
    assert says in L.wam_last_error()


@pytest.mark.parametrize("bad,ptrs,status,says", [
    (dict(R=-1), {}, 1, b"negative"), (dict(T=-1), {}, 1, b"negative"), (dict(max_kv=-1), {}, 1, b"negative"),
    (dict(Hq=3), {}, 1, b"multiple of Hkv"), (dict(Hq=0), {}, 1, b"Hq"), (dict(Hq=8192), {}, 1, b"Hq"),
    (dict(chunk=-1), {}, 1, b"chunk"), (dict(table_stride=2), {}, 1, b"table_stride"), (dict(max_pages=-1), {}, 1, b"max_pages"),
    (dict(max_kv=(1 << 30) + 1), {}, 2, b"2^30"), (dict(T=1 << 30), {}, 2, b"2^31"), (dict(R=1 << 30), {}, 2, b"2^31"),
    (dict(scale=float("inf")), {}, 1, b"scale"), (dict(scale=float("nan")), {}, 1, b"scale"),
    (dict(q_tok_stride=256), {}, 1, b"strides"), (dict(o_tok_stride=516), {}, 1, b"strides"),
    ({}, dict(q=0), 1, b"q is NULL"), ({}, dict(q=4100), 1, b"aligned"), ({}, dict(o=0), 1, b"o is NULL"),
    ({}, dict(table=0), 1, b"block_table is NULL"), ({}, dict(q_start=0), 1, b"q_start is NULL"),
    ({}, dict(q_len=4098), 1, b"q_len"), ({}, dict(kv_len=0), 1, b"kv_len is NULL"), ({}, dict(kv_len=4097), 1, b"aligned"),
])
def test_attn_paged_refusals(bad, ptrs, status, says):
    w, b, L = lib()
    d = b.wam_attn_paged_desc(R=2, T=5, Hq=4, max_pages=3, max_kv=100, chunk=1, table_stride=3, q_tok_stride=512,
                              o_tok_stride=512, scale=0.0)
    for k, v in bad.items():
        setattr(d, k, v)
    p = dict(q=4096, table=8192, q_start=4096, q_len=None, kv_len=4096, o=8192) | ptrs
    c = cache()
    assert L.wam_attn_paged(C.byref(d), C.byref(c), p["q"], p["table"], p["q_start"], p["q_len"], p["kv_len"], p["o"],
                            1 << 20, 1 << 40, None) == status
    assert says in L.wam_last_error()


@pytest.mark.parametrize("bad,ptrs,status,says", [
    (dict(Dh=80), {}, 2, b"Dh=80"), (dict(S=-1), {}, 1, b"S="), (dict(max_k=-2), {}, 1, b"negative"),
    (dict(Hkv=3), {}, 1, b"multiple of Hkv"), (dict(kv_tok_stride=128), {}, 1, b"kv_tok_stride"),
    (dict(kv_tok_stride=260), {}, 1, b"kv_tok_stride"), (dict(kv_tok_stride=1 << 26), {}, 1, b"kv_tok_stride"),
    (dict(scale=float("inf")), {}, 1, b"scale"), ({}, dict(k=0), 1, b"k is NULL"), ({}, dict(v=4104), 1, b"aligned"),
    ({}, dict(k_start=0), 1, b"k_start is NULL"), ({}, dict(k_len=2), 1, b"k_len"), ({}, dict(o=8), 1, b"aligned"),
])
def test_attn_cross_refusals(bad, ptrs, status, says):
    w, b, L = lib()
    d = b.wam_attn_cross_desc(R=2, T=5, S=9, Hq=4, Hkv=2, Dh=128, max_k=9, q_tok_stride=512, kv_tok_stride=256,
                              o_tok_stride=512, scale=0.0)
    for k, v in bad.items():
        setattr(d, k, v)
    p = dict(q=4096, k=4096, v=8192, q_start=4096, q_len=None, k_start=4096, k_len=None, o=8192) | ptrs
    assert L.wam_attn_cross(C.byref(d), p["q"], p["k"], p["v"], p["q_start"], p["q_len"], p["k_start"], p["k_len"],
                            p["o"], 1 << 20, 1 << 40, None) == status
    assert says in L.wam_last_error()


@pytest.mark.parametrize("bad,pairs,ptrs,status,says", [
    (dict(T=-1), [64], {}, 1, b"T=-1"), (dict(n_axes=0), [64], {}, 1, b"n_axes"), (dict(n_axes=5), [64], {}, 1, b"n_axes"),
    ({}, [65], {}, 1, b"pairs[0]=65"), (dict(n_axes=2), [40, 30], {}, 1, b"pairs[1]=30"), ({}, [-1], {}, 1, b"pairs[0]"),
    (dict(theta=0.0), [64], {}, 1, b"theta"), (dict(theta=float("nan")), [64], {}, 1, b"theta"),
    (dict(halves=2), [64], {}, 1, b"halves"), (dict(halves=1), [20], {}, 2, b"halves"),
    (dict(qkv_tok_stride=1000), [64], {}, 1, b"qkv_tok_stride"), (dict(q_tok_stride=504), [64], {}, 1, b"q_tok_stride"),
    ({}, [64], dict(qkv=0), 1, b"qkv is NULL"), ({}, [64], dict(pos=0), 1, b"pos is NULL"),
    ({}, [64], dict(slots=4097), 1, b"slots"), ({}, [64], dict(q_out=8), 1, b"q_out"),
])
def test_rope_paged_refusals(bad, pairs, ptrs, status, says):
    w, b, L = lib()
    d = b.wam_rope_paged_desc(T=5, Hq=4, n_axes=1, halves=0, theta=1e4, qkv_tok_stride=1024, q_tok_stride=512)
    d.pairs[:len(pairs)] = pairs
    for k, v in bad.items():
        setattr(d, k, v)
    p = dict(qkv=4096, pos=4096, slots=4096, q_out=8192) | ptrs
    c = cache()
    assert L.wam_rope_qkv_paged(C.byref(d), C.byref(c), p["qkv"], p["pos"], p["slots"], p["q_out"], None) == status
    assert says in L.wam_last_error()


def test_rope_halves_of_an_fp8_cache_need_whole_blocks():
    w, b, L = lib()
    d = b.wam_rope_paged_desc(T=5, Hq=4, n_axes=1, halves=1, theta=1e4, qkv_tok_stride=1024, q_tok_stride=512)
    d.pairs[0] = 40
    c = cache(**FP8)
    assert L.wam_rope_qkv_paged(C.byref(d), C.byref(c), 4096, 4096, 4096, 8192, None) == b.WAM_EUNSUPPORTED
    assert b"multiple of 32" in L.wam_last_error()


@pytest.mark.parametrize("bad,ptrs,status,says", [
    (dict(R=-1), {}, 1, b"negative"), (dict(R=5000), {}, 2, b"exceeds"), (dict(T=-1), {}, 1, b"negative"),
    (dict(page_size=40), {}, 2, b"page_size"), (dict(n_pages=-1), {}, 1, b"n_pages"), (dict(n_pages=1 << 27), {}, 2, b"2^31"),
    (dict(table_stride=7), {}, 1, b"table_stride"), (dict(max_pages=1 << 30, table_stride=1 << 30), {}, 2, b"max_pages"),
    ({}, dict(cache_len=0), 1, b"cache_len"), ({}, dict(new_len=2), 1, b"new_len"), ({}, dict(held=0), 1, b"held"),
    ({}, dict(n_free=0), 1, b"n_free"), ({}, dict(table=0), 1, b"block_table"), ({}, dict(free_list=0), 1, b"free_list"),
    ({}, dict(slots=0), 1, b"slots"), ({}, dict(status=0), 1, b"status"), ({}, dict(token_pos=1), 1, b"token_pos"),
    ({}, dict(held_out=4096 + 8), 1, b"overlap"), ({}, dict(n_free_out=20480), 1, b"overlap"),
])
def test_page_plan_refusals(bad, ptrs, status, says):
    w, b, L = lib()
    d = b.wam_page_plan_desc(R=4, T=50, page_size=16, n_pages=30, max_pages=8, table_stride=8)
    for k, v in bad.items():
        setattr(d, k, v)
    p = dict(cache_len=8192, new_len=12288, held=4096, n_free=20480, table=24576, free_list=28672, held_out=32768,
             n_free_out=36864, q_start=40960, kv_len=45056, slots=49152, token_pos=None, status=53248) | ptrs
    assert L.wam_page_plan(C.byref(d), *p.values(), None) == status
    assert says in L.wam_last_error()


def test_nothing_to_do_is_not_an_error():
    w, b, L = lib()
    c = cache()
    d = b.wam_attn_paged_desc(R=0, T=5, Hq=4, max_pages=0, max_kv=0, chunk=0, table_stride=0, q_tok_stride=512,
                              o_tok_stride=512, scale=0.0)
    assert L.wam_attn_paged(C.byref(d), C.byref(c), None, None, None, None, None, None, None, 0, None) == b.WAM_OK
    d = b.wam_attn_cross_desc(R=2, T=0, S=0, Hq=4, Hkv=2, Dh=128, max_k=0)
    assert L.wam_attn_cross(C.byref(d), *[None] * 9, 0, None) == b.WAM_OK
    d = b.wam_rope_paged_desc(T=0, Hq=4, n_axes=1, theta=1e4)
    assert L.wam_rope_qkv_paged(C.byref(d), C.byref(c), None, None, None, None, None) == b.WAM_OK
    for f in (L.wam_attn_paged, L.wam_attn_cross, L.wam_rope_qkv_paged, L.wam_page_plan):
        n = len(f.argtypes)
        args = [0 if t is C.c_size_t else None for t in f.argtypes]
        assert len(args) == n and f(*args) == b.WAM_EINVAL
    assert L.wam_attn_paged_workspace_bytes(None, None) == 0 and L.wam_attn_cross_workspace_bytes(None) == 0


def test_binding_checks_tensor_layouts():
    import torch
    w, b, L = lib()
    k = torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="share"):
        w.make_paged_cache(k, torch.zeros(4, 16, 3, 128, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="contiguous"):
        w.make_paged_cache(k.transpose(2, 3), k.transpose(2, 3))
    with pytest.raises(ValueError, match="exponent"):
        w.make_paged_cache(k, k, k_exp=torch.zeros(4, 16, 4, dtype=torch.int32)[:, :, ::2], v_scale=1.0)


def test_binding_takes_any_stride_of_a_single_entry():
    import torch
    w, b, L = lib()
    buf = torch.zeros(16, 128, dtype=torch.bfloat16)
    k = torch.as_strided(buf, (1, 16, 1, 128), (7, 128, 3, 1))
    v = torch.as_strided(buf, (1, 16, 1, 128), (0, 128, 0, 1))
    c = w.make_paged_cache(k, v)
    assert (c.page_stride, c.tok_stride, c.head_stride) == (16 * 128, 128, 128)


def test_reference_rotation_and_chunk_rule():
    pos = np.array([[3, 5], [0, 0], [7, 1]])
    x = np.random.default_rng(0).standard_normal((3, 1, 8))
    for halves in (False, True):
        y = paged_ref.rotate(x, paged_ref.angles(pos, [2, 1], 100.0), halves)
        for t in range(3):
            for p, ang in enumerate([pos[t, 0], pos[t, 0] * 100.0 ** -0.5, pos[t, 1]]):
                i, j = (p, p + 3) if halves else (2 * p, 2 * p + 1)
                z = complex(x[t, 0, i], x[t, 0, j]) * complex(np.cos(ang), np.sin(ang))
                assert np.allclose([y[t, 0, i], y[t, 0, j]], [z.real, z.imag])
        assert np.array_equal(y[..., 6:], x[..., 6:]) and np.array_equal(y[1], x[1])
    assert paged_ref.chunk_seen(2, 5, 1).tolist() == [[1, 1, 1, 1, 0], [1, 1, 1, 1, 1]]
    assert paged_ref.chunk_seen(3, 7, 3).sum(1).tolist() == [6, 6, 7] and paged_ref.chunk_seen(2, 3, 0).all()
    assert paged_ref.chunk_seen(4, 2, 1).sum(1).tolist() == [0, 0, 1, 2]
    assert paged_ref.E4M3[0x7E] == 448 and paged_ref.E4M3[1] == 2.0 ** -9 and paged_ref.E4M3[0xB8] == -1


def test_reference_plan_by_hand():
    table = np.array([[5, 6, 7, -1], [1, -1, -1, -1], [-1] * 4], np.int32)
    free = np.array([9, 8, 0, 0, 0, 0, 0, 0, 0, 0], np.int32)
    # request 0 ends (gives 5, 6, 7), 1 grows from one page to two, 2 begins with 17 tokens
    r = paged_ref.plan([0, 10, 0], [0, 10, 17], [3, 1, 0], free, 2, table, 16, 10, 30)
    assert r["table"].tolist() == [[5, 6, 7, -1], [1, 7, -1, -1], [6, 5, -1, -1]]
    assert r["held_out"] == [0, 2, 2] and r["n_free_out"] == [2] and r["free_list"].tolist() == free.tolist()
    assert r["q_start"] == [0, 0, 10, 27] and r["kv_len"] == [0, 20, 17] and r["status"] == [0, 0, 0, 0]
    assert r["slots"][:10].tolist() == [26, 27, 28, 29, 30, 31, 112, 113, 114, 115]
    assert r["slots"][26] == 80 and r["slots"][27:].tolist() == [-1] * 3 and r["token_pos"][9:11].tolist() == [19, 0]
