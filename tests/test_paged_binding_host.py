"""The binding of the paged operators refuses tensors whose addresses would be misread: another type, order, size or device.
(Host tensors: every call ends before the library.)"""
import pytest
import torch

import paper_2602_15922_amd as w

I = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
B = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
R, T, HQ, HKV, DH, PS, PAGES, WIDTH, S = 3, 10, 4, 2, 128, 16, 6, 5, 20


def cache():
    return w.make_paged_cache(B(PAGES, PS, HKV, DH), B(PAGES, PS, HKV, DH))


def plan_args():
    return dict(cache_len=I(R), new_len=I(R), held=I(R), n_free=I(1), block_table=I(R, WIDTH), free_list=I(PAGES), held_out=I(R),
                n_free_out=I(1), q_start=I(R + 1), kv_len=I(R), slots=I(T), status=I(4), page_size=PS, token_pos=I(T))


def rope_args():
    return dict(cache=cache(), qkv=B(T, (HQ + 2 * HKV) * DH), pos=I(T, 2), slots=I(T), q_out=B(T, HQ, DH), pairs=[32, 32])


def paged_args():
    return dict(cache=cache(), q=B(T, HQ, DH), block_table=I(R, WIDTH), q_start=I(R + 1), kv_len=I(R), o=B(T, HQ, DH),
                ws=torch.zeros(1 << 16, dtype=torch.uint8), q_len=I(R))


def cross_args():
    return dict(q=B(T, HQ, DH), k=B(S, HKV, DH), v=B(S, HKV, DH), q_start=I(R + 1), k_start=I(R), o=B(T, HQ, DH),
                ws=torch.zeros(1 << 16, dtype=torch.uint8), q_len=I(R), k_len=I(R))


CALLS = dict(plan=(w.wam_page_plan, plan_args), rope=(w.wam_rope_qkv_paged, rope_args), paged=(w.wam_attn_paged, paged_args),
             cross=(w.wam_attn_cross, cross_args))


def refused(call, match, **bad):
    f, args = CALLS[call]
    with pytest.raises(ValueError, match=match):
        f(**{**args(), **bad})


@pytest.mark.parametrize("call", list(CALLS))
def test_host_tensors(call):
    """Everything in order but the device."""
    refused(call, "on the GPU")


INTS = [(c, n) for c, (f, args) in CALLS.items() for n, t in args().items()
        if isinstance(t, torch.Tensor) and t.dtype == torch.int32]


@pytest.mark.parametrize("call,name", INTS)
def test_index_tensors(call, name):
    t = CALLS[call][1]()[name]
    refused(call, f"{name} must", **{name: t.long()})
    refused(call, f"{name} must", **{name: t.float()})
    if t.dim() == 1 and t.numel() > 1:
        refused(call, f"{name} must", **{name: I(2 * t.numel())[::2]})
    if t.dim() == 1 and (call, name) not in (("plan", "free_list"), ("plan", "slots"), ("cross", "q_start")):  # (they say the sizes)
        refused(call, f"{name} must", **{name: I(t.numel() - 1)})
    if t.dim() == 2:
        refused(call, f"{name} must", **{name: I(t.shape[1], t.shape[0]).t()})


def test_starts_from_a_cumulative_sum():
    """torch.cumsum of int32 is int64."""
    starts = torch.cat([I(1), torch.cumsum(torch.ones(R, dtype=torch.int32), 0)])
    assert starts.dtype == torch.int64
    refused("paged", "q_start must be a contiguous int32", q_start=starts)


def test_starts_of_the_keys_without_lengths():
    refused("cross", "k_start must", k_len=None)  # R + 1 of them then


@pytest.mark.parametrize("call,name", [("paged", "q"), ("paged", "o"), ("cross", "q"), ("cross", "o"), ("cross", "k"), ("cross", "v"), ("rope", "q_out")])
def test_rows_of_heads(call, name):
    t = CALLS[call][1]()[name]
    n, H, _ = t.shape
    refused(call, "must", **{name: t.half()})
    refused(call, "must", **{name: B(n, H, DH + 8)[..., :DH]})       # heads apart
    refused(call, "must", **{name: B(n, DH, H).transpose(1, 2)})     # heads innermost
    refused(call, "must", **{name: B(H, n, DH).transpose(0, 1)})     # heads outermost
    if name not in ("q", "k"):                                       # (those say the sizes)
        refused(call, "must", **{name: B(n - 1, H, DH)})
        refused(call, "must", **{name: B(n, H - 1, DH)})
    if (call, name) != ("cross", "q"):
        refused(call, "must", **{name: B(n, H, 64)})


def test_fused_projection():
    refused("rope", "whole heads", qkv=B(T, (HQ + 2 * HKV) * DH + 8))
    refused("rope", "qkv must", qkv=B((HQ + 2 * HKV) * DH, T).t())
    refused("rope", "qkv must", qkv=B(T, (HQ + 2 * HKV) * DH).float())
    refused("rope", "row per token", pos=I(T - 1, 2))
    refused("rope", "row per token", pos=I(2 * T))


def test_workspaces():
    for call in ("paged", "cross"):
        refused(call, "ws must", ws=torch.zeros(1 << 17, dtype=torch.uint8)[::2])


def test_cache_types():
    k, c8, e = B(PAGES, PS, HKV, DH), torch.zeros(PAGES, PS, HKV, DH, dtype=torch.uint8), I(PAGES, PS, HKV)
    for bad in (dict(k=k.half(), v=k.half()), dict(k=k, v=k.half()), dict(k=c8, v=c8), dict(k=k, v=k, k_exp=e),
                dict(k=c8, v=c8, k_exp=e.float()), dict(k=c8, v=c8, k_exp=I(PAGES - 1, PS, HKV)), dict(k=c8, v=c8, k_exp=e.long())):
        with pytest.raises(ValueError):
            w.make_paged_cache(v_scale=1.0, **bad)
    assert w.make_paged_cache(c8, c8, k_exp=e, v_scale=1.0).tok_stride == HKV * DH
    f8 = c8.view(torch.float8_e4m3fn)
    assert w.make_paged_cache(f8, f8, k_exp=e, v_scale=1.0).n_pages == PAGES
