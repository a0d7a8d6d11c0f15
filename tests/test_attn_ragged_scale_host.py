"""A softmax scale that is finite but whose factor of the exponent of 2 is not, is refused (fake addresses; no call here
reaches a launch)."""
import ctypes as C

import pytest


@pytest.mark.parametrize("scale", [3.0e38, 2.4e38, 3.4028234e38])
def test_scale_past_the_range_of_its_exponent(scale):
    import paper_2602_15922_amd as w
    b, L = w.binding, w.lib()
    c = b.wam_paged_cache(k=4096, v=8192, page_stride=64 * 256, tok_stride=256, head_stride=128, n_pages=10, page_size=64, Hkv=2, Dh=128)
    d = b.wam_attn_paged_desc(R=2, T=5, Hq=4, max_pages=3, max_kv=100, chunk=1, table_stride=3, q_tok_stride=512, o_tok_stride=512,
                              scale=scale)
    assert L.wam_attn_paged(C.byref(d), C.byref(c), 4096, 8192, 4096, None, 4096, 8192, 1 << 20, 1 << 40, None) == b.WAM_EINVAL
    assert b"scale" in L.wam_last_error()
    d = b.wam_attn_cross_desc(R=2, T=5, S=9, Hq=4, Hkv=2, Dh=128, max_k=9, q_tok_stride=512, kv_tok_stride=256, o_tok_stride=512,
                              scale=scale)
    assert L.wam_attn_cross(C.byref(d), 4096, 4096, 8192, 4096, None, 4096, None, 8192, 1 << 20, 1 << 40, None) == b.WAM_EINVAL
    assert b"scale" in L.wam_last_error()
