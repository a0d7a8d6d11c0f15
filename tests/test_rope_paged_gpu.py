"""wam_rope_qkv_paged against the rotation in 64 bits, in every layout of pairs, heads and pages."""
import numpy as np
import pytest

import paged_ref
from gpu_helpers import host, log

pytestmark = pytest.mark.gpu
FAR = 2 ** 31 - 1


def setup(T, Hq, Hkv, Dh, ps, axes, seed, fp8=False, far=5000, layout="nhd", pad=16, skip=0.1, shift=0):
    """Inputs with rows wider than the projection, slots in random pages, some of them skipped."""
    import torch
    g = torch.Generator().manual_seed(seed)
    n_pages = -(-T // ps) + 2
    d = {"T": T, "Hq": Hq, "Hkv": Hkv, "Dh": Dh, "ps": ps, "n_pages": n_pages}
    width = (Hq + 2 * Hkv) * Dh
    d["x"] = torch.randn(T, width, generator=g).bfloat16()
    wide = torch.full((T, width + pad), float("nan"), dtype=torch.bfloat16)
    wide[:, :width] = d["x"]
    d["qkv"] = wide.cuda()[:, :width]
    d["pos"] = torch.randint(-far if shift else 0, far + 1, (T, axes), generator=g, dtype=torch.int64).int()
    if T:
        d["pos"][-1] = far
    slots = torch.randperm(n_pages * ps, generator=g)[:T].int()
    out = torch.rand(T, generator=g) < skip
    slots[out] = torch.tensor([-1, n_pages * ps, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)[torch.arange(int(out.sum())) % 4]
    d["slots"], d["ok"] = slots, (~out).numpy()
    kind = torch.uint8 if fp8 else torch.bfloat16
    shape = {"nhd": (n_pages, ps, Hkv, Dh), "hnd": (n_pages, Hkv, ps, Dh), "kv": (n_pages, 2, ps, Hkv, Dh)}[layout]

    def page(dtype, *last):
        s = shape[:-1] + last
        if layout == "kv":
            both = torch.full(s, 0x5B, dtype=torch.uint8).cuda() if dtype == torch.uint8 else torch.full(s, 7, dtype=dtype).cuda()
            return both[:, 0], both[:, 1]
        t = [torch.full(s, 0x5B if dtype == torch.uint8 else 7, dtype=dtype).cuda() for _ in range(2)]
        return [y.transpose(1, 2) for y in t] if layout == "hnd" else t
    d["k"], d["v"] = page(kind, Dh)
    d["ex"] = page(torch.int32)[0] if fp8 else None
    d["q_out"] = torch.full((T, Hq + 1, Dh), 9.0, dtype=torch.bfloat16).cuda()
    return d


def call(d, pairs, halves=False, theta=10000.0, v_scale=0.02, q=True, stream=None):
    import paper_2602_15922_amd as w
    c = w.make_paged_cache(d["k"], d["v"], k_exp=d["ex"], v_scale=v_scale)
    w.wam_rope_qkv_paged(c, d["qkv"], d["pos"].cuda(), d["slots"].cuda(), d["q_out"][:, :d["Hq"]] if q else None, pairs=pairs,
                         halves=halves, theta=theta, stream=stream)


def reference(d, pairs, halves, theta):
    x = d["x"].double().numpy().reshape(d["T"], -1, d["Dh"])
    heads = d["Hq"] + d["Hkv"]
    y = paged_ref.rotate(x[:, :heads], paged_ref.angles(d["pos"].numpy(), pairs, theta), halves)
    return x, y, x[:, heads:]


def tolerance(x, y):
    """One rounding to bf16 (2^-8 of the value), and the fp32 rotation: cosine and sine to 2^-21 of 1, two products and a
    sum, each to 2^-24, of a pair's two values (both at most the head's largest)."""
    return 2.0 ** -8 * np.abs(y) + 2.0 ** -20 * np.abs(x).max(-1, keepdims=True)


def check_cache(d, ok_slots, k, v, kx, untouched=True):
    rows = lambda t: host(t).reshape(-1, d["Hkv"], d["Dh"])  # noqa: E731
    gk, gv = rows(d["k"]), rows(d["v"])
    assert np.all(np.abs(gk[ok_slots] - k) <= tolerance(kx, k)), "k"
    assert np.array_equal(gv[ok_slots], v), "v"
    rest = np.ones(len(gk), bool)
    rest[ok_slots] = False
    assert np.all(gk[rest] == 7) and np.all(gv[rest] == 7)


@pytest.mark.parametrize("T,Hq,Hkv,Dh,ps,pairs,halves,layout,far", [
    (1, 1, 1, 128, 16, [64], False, "nhd", 10), (3, 40, 40, 128, 64, [22, 21, 21], False, "nhd", 4000),
    (77, 8, 2, 64, 48, [12, 10, 10], False, "hnd", 300), (33, 5, 5, 128, 16, [1, 30, 20, 13], True, "kv", FAR),
    (130, 32, 8, 128, 64, [64], True, "nhd", 1000000), (61, 8, 1, 64, 16, [32], True, "hnd", FAR),
    (19, 4, 2, 128, 32, [16, 16], True, "nhd", 99), (19, 4, 2, 128, 32, [16, 15], False, "nhd", 99),
    (19, 3, 3, 64, 32, [0, 7, 0], False, "kv", 99), (9, 2, 2, 64, 16, [8], True, "nhd", 99),
    (5, 2, 2, 64, 16, [0], False, "nhd", 99), (600, 1, 1, 64, 1024, [16, 16], False, "nhd", 70)])
def test_rope_bf16(T, Hq, Hkv, Dh, ps, pairs, halves, layout, far):
    import torch
    log(f"rope T={T} Hq={Hq} Hkv={Hkv} Dh={Dh} ps={ps} pairs={pairs} halves={halves} {layout} far={far}")
    for theta, shift in ((10000.0, 0), (500000.0, 1)):
        d = setup(T, Hq, Hkv, Dh, ps, len(pairs), T + Hq, layout=layout, far=far, shift=shift)
        call(d, pairs, halves, theta)
        torch.cuda.synchronize()
        x, y, v = reference(d, pairs, halves, theta)
        ok = d["ok"]
        q = host(d["q_out"])
        assert np.all(np.abs(q[ok, :Hq] - y[ok, :Hq]) <= tolerance(x[ok, :Hq], y[ok, :Hq])), "q"
        assert np.all(q[~ok] == 9) and np.all(q[:, Hq:] == 9)
        check_cache(d, d["slots"].numpy()[ok], y[ok, Hq:], v[ok], x[ok, Hq:Hq + Hkv])


@pytest.mark.parametrize("T,Hq,Hkv,ps,pairs,halves,layout", [
    (1, 1, 1, 16, [64], False, "nhd"), (50, 40, 40, 64, [22, 21, 21], False, "nhd"), (61, 32, 8, 16, [64], True, "hnd"),
    (40, 6, 3, 48, [20, 12], True, "kv"), (23, 4, 1, 16, [30], False, "nhd")])
def test_rope_fp8(T, Hq, Hkv, ps, pairs, halves, layout):
    """Codes: the block's exponent by the rule (from the value rotated in 64 bits, or its neighbour where the largest
    value lies within 2^-18 of a border), each code within half a step of E4M3 (2^-4 relative, 2^-10 among its
    subnormals) and the fp32 rotation."""
    import torch
    log(f"rope fp8 T={T} Hq={Hq} Hkv={Hkv} ps={ps} pairs={pairs} halves={halves} {layout}")
    d = setup(T, Hq, Hkv, 128, ps, len(pairs), T + 7, fp8=True, layout=layout)
    call(d, pairs, halves, v_scale=0.02)
    torch.cuda.synchronize()
    x, y, v = reference(d, pairs, halves, 10000.0)
    ok, at = d["ok"], d["slots"].numpy()[d["ok"]]
    q = host(d["q_out"])
    assert np.all(np.abs(q[ok, :Hq] - y[ok, :Hq]) <= tolerance(x[ok, :Hq], y[ok, :Hq])) and np.all(q[~ok] == 9)
    rows = lambda t: t.cpu().contiguous().numpy().reshape((-1, Hkv) + t.shape[3:])  # noqa: E731
    kc, vc, ex = rows(d["k"]), rows(d["v"]), rows(d["ex"])
    e = (ex[at].astype(np.int64)[..., None] >> (8 * np.arange(4))) & 255
    want = y[ok, Hq:].reshape(len(at), Hkv, 4, 32)
    top = np.abs(want).max(-1)
    rule = lambda m: np.ceil(np.log2(np.maximum(m, 1e-300) / 448.0))  # noqa: E731
    lo, hi = rule(top * (1 - 2.0 ** -18)), rule(top * (1 + 2.0 ** -18))
    assert np.all((e - 127 >= lo) & (e - 127 <= hi)), "exponents"
    step = 2.0 ** (e - 127)[..., None]
    got = paged_ref.E4M3[kc[at]].reshape(want.shape) * step
    slack = 2.0 ** -20 * np.abs(x[ok, Hq:Hq + Hkv]).max(-1)[..., None, None]
    assert np.all(np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * step) + slack), "k"
    u = (v[ok].astype(np.float32) * np.float32(1.0 / np.float32(0.02))).astype(np.float64)
    assert np.all(np.abs(paged_ref.E4M3[vc[at]] - np.clip(u, -448, 448)) <= np.maximum(2.0 ** -4 * np.abs(u), 2.0 ** -10)), "v"
    rest = np.ones(len(kc), bool)
    rest[at] = False
    assert np.all(kc[rest] == 0x5B) and np.all(vc[rest] == 0x5B) and np.all(ex[rest] == 7)


def test_agrees_with_the_table_form():
    """The split and positions of wam_rope_qkv: the same values up to one rounding of a table entry (2^-24 of 1)."""
    import torch
    import paper_2602_15922_amd as w
    T, H, Dh = 2 * 8 * 8 + 16, 4, 128
    log("rope paged against tables")
    pos = w.wam_chunk_positions(3, 2, 8, 8, 16)
    d = setup(T, H, H, Dh, 16, 3, 1, skip=0.0)
    d["pos"] = torch.from_numpy(pos)
    d["slots"] = torch.arange(T, dtype=torch.int32)
    call(d, [22, 21, 21])
    cos, sin = (torch.from_numpy(t).cuda() for t in w.wam_rope_tables(pos, Dh))
    q = torch.empty(1, T, H, Dh, dtype=torch.bfloat16, device="cuda")
    kc, vc = torch.empty_like(q), torch.empty_like(q)
    w.wam_rope_qkv(d["qkv"].contiguous().view(1, T, -1), cos, sin, q, kc, vc, 0, H, Dh)
    torch.cuda.synchronize()
    x = d["x"].double().numpy().reshape(T, -1, Dh)
    flat = lambda t: host(t).reshape(-1, H, Dh)[:T]  # noqa: E731
    for a, b, i in ((d["q_out"][:, :H], q[0], 0), (d["k"], kc[0], H)):
        a, b = flat(a.contiguous()), flat(b)
        assert np.all(np.abs(a - b) <= 2.0 ** -7 * np.abs(b) + 2.0 ** -20 * np.abs(x[:, i:i + H]).max(-1, keepdims=True))
    assert np.array_equal(flat(d["v"]), flat(vc[0]))


def test_without_q_and_kept_dims_beside_infinities():
    import torch
    log("rope without q, infinities")
    d = setup(12, 3, 2, 64, 16, 1, 4, skip=0.0)
    d["qkv"][:, 3 * 64 + 40] = float("inf")   # a kept dim of the first key head (20 pairs turn dims 0 to 39)
    call(d, [20], q=False)
    torch.cuda.synchronize()
    assert (d["q_out"] == 9).all()
    rows = d["k"].reshape(-1, 2, 64)[d["slots"].long().cuda()].float()
    x = d["qkv"].float()[:, 192:320].reshape(12, 2, 64)
    assert torch.equal(rows[:, :, 40:], x[:, :, 40:])
    assert torch.isfinite(rows[:, :, :40]).all()


def test_another_stream_and_a_graph():
    import torch
    log("rope on a stream and replayed")
    d = setup(40, 4, 4, 128, 16, 2, 9)
    pos, slots, s = d["pos"].cuda(), d["slots"].cuda(), torch.cuda.Stream()
    import paper_2602_15922_amd as w
    c = w.make_paged_cache(d["k"], d["v"])
    s.wait_stream(torch.cuda.current_stream())
    w.wam_rope_qkv_paged(c, d["qkv"], pos, slots, d["q_out"][:, :4], pairs=[32, 32], stream=s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        w.wam_rope_qkv_paged(c, d["qkv"], pos, slots, d["q_out"][:, :4], pairs=[32, 32])
    for k in range(3):
        pos.add_(1000 * k)
        d["pos"] = pos.cpu()
        g.replay()
        torch.cuda.synchronize()
        x, y, _ = reference(d, [32, 32], False, 10000.0)
        ok = d["ok"]
        assert np.all(np.abs(host(d["q_out"])[ok, :4] - y[ok, :4]) <= tolerance(x[ok, :4], y[ok, :4]))
