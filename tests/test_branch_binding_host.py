"""The binding of the operators of requests that branch refuses tensors whose addresses would be misread: another type, order,
size or device.  (Host tensors: every call ends before the library.)"""
import pytest
import torch

import paper_2602_15922_amd as w

I = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
B = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
F = lambda *s: torch.zeros(s)  # noqa: E731
R, N, T, HQ, HKV, DH, PS, PAGES, WIDTH, WORDS, V = 3, 4, 10, 4, 2, 128, 16, 6, 5, 2, 40


def cache():
    return w.make_paged_cache(B(PAGES, PS, HKV, DH), B(PAGES, PS, HKV, DH))


def bytes_(n=1 << 16):
    return torch.zeros(n, dtype=torch.uint8)


ARGS = dict(
    fork=(w.wam_page_fork, lambda: dict(src=I(N), dst=I(N), first=I(N), length=I(N), held=I(R), n_free=I(1), block_table=I(R, WIDTH),
                                        free_list=I(PAGES), held_out=I(R), n_free_out=I(1), copies=I(N, 3), status=I(2), page_size=PS)),
    copy=(w.wam_page_copy, lambda: dict(cache=cache(), copies=I(N, 3))),
    collect=(w.wam_page_collect, lambda: dict(cache_len=I(R), held=I(R), block_table=I(R, WIDTH), free_list=I(PAGES), held_out=I(R),
                                              n_free_out=I(1), status=I(2), page_size=PS)),
    compact=(w.wam_cache_compact, lambda: dict(cache=cache(), block_table=I(R, WIDTH), q_start=I(R + 1), kv_len=I(R), keep=I(T), n_keep=I(R),
                                               q_len=I(R))),
    tree=(w.wam_attn_tree, lambda: dict(cache=cache(), q=B(T, HQ, DH), block_table=I(R, WIDTH), q_start=I(R + 1), kv_len=I(R), mask=I(T, WORDS),
                                        o=B(T, HQ, DH), ws=bytes_(), q_len=I(R))),
    verify=(w.wam_verify_tree, lambda: dict(p=F(T, V), q=F(T, V), tokens=I(T), parent=I(T), u=F(T), u_next=F(R), q_start=I(R + 1), path=I(T),
                                            n_path=I(R), next_token=I(R), ws=bytes_(), q_len=I(R), kv_len=I(R), cache_len=I(R))))
SAY_SIZES = {("fork", "src"), ("fork", "free_list"), ("collect", "free_list"), ("compact", "keep"), ("verify", "p"), ("verify", "u_next")}


def refused(call, match, **bad):
    f, args = ARGS[call]
    with pytest.raises(ValueError, match=match):
        f(**{**args(), **bad})


@pytest.mark.parametrize("call", list(ARGS))
def test_host_tensors(call):
    """Everything in order but the device."""
    refused(call, "on the GPU")


INTS = [(c, n) for c, (_, args) in ARGS.items() for n, t in args().items() if isinstance(t, torch.Tensor) and t.dtype == torch.int32]


@pytest.mark.parametrize("call,name", INTS)
def test_index_tensors(call, name):
    t = ARGS[call][1]()[name]
    refused(call, f"{name} must", **{name: t.long()})
    refused(call, f"{name} must", **{name: t.float()})
    if t.dim() == 1 and t.numel() > 1:
        refused(call, f"{name} must", **{name: I(2 * t.numel())[::2]})
    if t.dim() == 1 and (call, name) not in SAY_SIZES:
        refused(call, f"{name} must", **{name: I(t.numel() - 1)})
    if t.dim() == 2:
        refused(call, f"{name} must", **{name: I(t.shape[1], t.shape[0]).t()})


def test_columns_and_rows():
    refused("copy", "three columns", copies=I(N, 4))
    refused("copy", "three columns", copies=I(3 * N))
    refused("tree", "mask must", mask=I(T - 1, WORDS))
    refused("tree", "mask must", mask=I(T * WORDS))


@pytest.mark.parametrize("name", ["q", "o"])
def test_rows_of_heads(name):
    refused("tree", "must", **{name: B(T, HQ, DH).half()})
    refused("tree", "must", **{name: B(T, HQ, DH + 8)[..., :DH]})
    refused("tree", "must", **{name: B(T, HQ, 64)})


@pytest.mark.parametrize("name", ["p", "q", "u", "u_next"])
def test_probabilities(name):
    t = ARGS["verify"][1]()[name]
    refused("verify", f"{name} must", **{name: t.double()})
    refused("verify", f"{name} must", **{name: t.bfloat16()})
    if t.dim() == 1:
        refused("verify", f"{name} must", **{name: F(2 * t.numel())[::2]})
    else:
        refused("verify", f"{name} must", **{name: F(V, T).t()})
    if name != "p":
        refused("verify", "must", **{name: t[:-1]})


def test_workspaces():
    for call in ("tree", "verify"):
        refused(call, "ws must", ws=bytes_(1 << 17)[::2])
