"""wam_rope_qkv_paged at the far end of its positions for frequencies that fall slowly, and with q written in place."""
import numpy as np
import pytest

from gpu_helpers import host, log

pytestmark = pytest.mark.gpu
PI = np.longdouble("3.14159265358979323846264338327950288")


def near_multiples_of_pi(theta, pairs, tokens, seed):
    """Positions close to 2^31, each one whose angle of some pair lies within 2^-12 of a multiple of pi (64-bit
    mantissas: 2^31 revolutions there are exact to 2^-32)."""
    rng = np.random.default_rng(seed)
    out = []
    while len(out) < tokens:
        pos = int(rng.integers(2 ** 31 - 2 ** 27, 2 ** 31))
        i = int(rng.integers(pairs // 4, pairs))
        w = np.longdouble(theta) ** (-np.longdouble(i) / pairs)
        for k in range(4096):  # neighbours
            half = (pos - k) * w / PI
            if abs(float(half - np.rint(half))) < 2.0 ** -14:
                out.append(pos - k)
                break
    return np.array(out, np.int64)


@pytest.mark.parametrize("theta,pairs", [(10000.0, 64), (100.0, 64), (2.0, 64), (1.1, 64), (1.1, 32)])
def test_far_positions_are_as_exact_as_near_ones(theta, pairs):
    """x = (1, 0) in every pair: the outputs are the cosine and sine themselves, and where they are small their absolute
    error shows.  Tolerance: one rounding to bf16 (2^-8 of the value) and 2^-20: the angle to 2^31 * 2^-53 * 2 (the product's
    rounding and the frequency's, each half a step of a value below 2^31 rad, one step allowed), its reduction to 32 bits,
    the cosine and sine to 2^-22."""
    import torch
    import paper_2602_15922_amd as w
    T, Dh = 160, 128
    pos = near_multiples_of_pi(theta, pairs, T, 11)
    log(f"rope far theta={theta} pairs={pairs}")
    qkv = torch.zeros(T, 3 * Dh, dtype=torch.bfloat16)
    qkv[:, 0:2 * Dh:2] = 1
    k, v = (torch.zeros(T // 16, 16, 1, Dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(T, 1, Dh, dtype=torch.bfloat16, device="cuda")
    w.wam_rope_qkv_paged(w.make_paged_cache(k, v), qkv.cuda(), torch.tensor(pos, dtype=torch.int32, device="cuda")[:, None],
                         torch.arange(T, dtype=torch.int32, device="cuda"), q, pairs=[pairs], theta=theta)
    torch.cuda.synchronize()
    freq = np.longdouble(theta) ** (-np.arange(pairs).astype(np.longdouble) / pairs)
    ang = pos[:, None] * freq
    want = np.zeros((T, Dh))
    want[:, 0:2 * pairs:2], want[:, 1:2 * pairs:2] = np.cos(ang), np.sin(ang)
    want[:, 2 * pairs::2] = 1
    assert (np.abs(want) < 2.0 ** -11).sum() >= T  # the small ones that tell
    for got in (host(q)[:, 0], host(k).reshape(T, Dh)):
        off = np.abs(got - want) - 2.0 ** -8 * np.abs(want)
        assert off.max() <= 2.0 ** -20, float(np.log2(off.max()))


@pytest.mark.parametrize("Hq,Hkv,Dh,halves,fp8", [(8, 2, 64, False, False), (40, 40, 128, True, False), (3, 3, 128, True, True), (1, 1, 64, True, False)])
def test_q_in_its_own_place(Hq, Hkv, Dh, halves, fp8):
    """q_out at q's address in qkv, with its stride: the same values as elsewhere, and K and V of qkv as they were."""
    import torch
    import paper_2602_15922_amd as w
    T, n = 333, Dh // 2
    g = torch.Generator().manual_seed(Hq)
    x = torch.randn(T, (Hq + 2 * Hkv) * Dh, generator=g).bfloat16().cuda()
    pos, slots = torch.randint(0, 9000, (T, 1), generator=g).int().cuda(), torch.randperm(T + 19, generator=g).int()[:T].cuda()
    kind = torch.uint8 if fp8 else torch.bfloat16
    log(f"rope in place Hq={Hq} Dh={Dh} halves={halves} fp8={fp8}")
    outs = []
    for place in (False, True):
        k, v = (torch.zeros(22, 16, Hkv, Dh, dtype=kind, device="cuda") for _ in range(2))
        ex = torch.zeros(22, 16, Hkv, dtype=torch.int32, device="cuda") if fp8 else None
        qkv = x.clone()
        q = qkv[:, :Hq * Dh].unflatten(1, (Hq, Dh)) if place else torch.zeros(T, Hq, Dh, dtype=torch.bfloat16, device="cuda")
        w.wam_rope_qkv_paged(w.make_paged_cache(k, v, k_exp=ex, v_scale=0.02), qkv, pos, slots, q, pairs=[n], halves=halves)
        torch.cuda.synchronize()
        assert torch.equal(qkv[:, Hq * Dh:], x[:, Hq * Dh:])
        outs.append((q.clone(), k, v))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
