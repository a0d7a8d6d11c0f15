"""Sizes whose launch would have 2^32 threads or more are refused with the reason (fake addresses; no call here reaches a
launch)."""
import ctypes as C

import pytest

import paper_2602_15922_amd as w


def cache(Hkv, Dh):
    return w.binding.wam_paged_cache(k=4096, v=8192, page_stride=16 * Hkv * Dh, tok_stride=Hkv * Dh, head_stride=Dh, n_pages=10, page_size=16,
                                     Hkv=Hkv, Dh=Dh)


@pytest.mark.parametrize("T,Hq,Hkv,Dh", [(1 << 24, 40, 40, 128), (1 << 25, 8, 2, 128), (1 << 26, 1, 1, 64), (2 ** 31 - 1, 1, 1, 64)])
def test_rotary_append(T, Hq, Hkv, Dh):
    """256, 128 and 64 threads per token."""
    b, L, c = w.binding, w.lib(), cache(Hkv, Dh)
    width = (Hq + 2 * Hkv) * Dh
    d = b.wam_rope_paged_desc(T=T, Hq=Hq, n_axes=1, theta=1e4, qkv_tok_stride=width, q_tok_stride=Hq * Dh)
    d.pairs[0] = 32
    assert L.wam_rope_qkv_paged(C.byref(d), C.byref(c), 4096, 4096, 4096, 8192, None) == b.WAM_EUNSUPPORTED
    assert b"2^32" in L.wam_last_error()


@pytest.mark.parametrize("R,Hkv", [((1 << 24) + 1, 1), (1 << 21, 8)])
def test_attentions_of_millions_of_requests(R, Hkv):
    b, L, c = w.binding, w.lib(), cache(Hkv, 64)
    d = b.wam_attn_paged_desc(R=R, T=R, Hq=Hkv, max_pages=1, max_kv=16, table_stride=1, q_tok_stride=64 * Hkv, o_tok_stride=64 * Hkv)
    assert L.wam_attn_paged(C.byref(d), C.byref(c), 4096, 8192, 4096, None, 4096, 8192, 1 << 20, 1 << 40, None) == b.WAM_EUNSUPPORTED
    assert b"2^32" in L.wam_last_error()
    d = b.wam_attn_cross_desc(R=R, T=R, S=9, Hq=Hkv, Hkv=Hkv, Dh=64, max_k=9, q_tok_stride=64 * Hkv, kv_tok_stride=64 * Hkv,
                              o_tok_stride=64 * Hkv)
    assert L.wam_attn_cross(C.byref(d), 4096, 4096, 8192, 4096, None, 4096, None, 8192, 1 << 20, 1 << 40, None) == b.WAM_EUNSUPPORTED
    assert b"2^32" in L.wam_last_error()
