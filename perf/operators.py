"""The operators of serving requests with histories of their own, as cases that can be timed and compared:
the page plan (block tables and slot maps from request lengths), rotary positions with the append into a
paged KV cache, attention of new tokens over that cache, and cross-attention to states of other lengths.

`listed` gives the cases, `draw` more of the same ranges; `prepare` builds what a program holds before
the call, `run` is one pass: the plain form in elementary torch operations, or, where `own` is set, the
library's entry point; `exact` is the definition in 64 bits, `work` the bytes and operations a pass
cannot do without.
"""
import math

import torch

own = False

THETA = 10000.0
V_SCALE = 8.0 / 448.0  # an FP8 value cache's calibrated scale: these values stay below 8


def listed():
    return [
        # a language-conditioned policy's shared-head decoder: one new token for each of 48 requests of very
        # different histories
        dict(name="paged_tokens_gqa", kind="paged", R=48, q_lo=1, q_hi=1, unit=1, kv_lo=200, kv_hi=16000, Hq=32, Hkv=8,
             Dh=128, ps=16, chunk=1, fp8=False, pad=0),
        # the same from an E4M3 cache, longer histories
        dict(name="paged_tokens_fp8", kind="paged", R=64, q_lo=1, q_hi=1, unit=1, kv_lo=1000, kv_hi=32000, Hq=40,
             Hkv=8, Dh=128, ps=64, chunk=1, fp8=True, pad=0),
        # one robot's 32 action tokens against a short history, one rank's 5 heads of the 14B class: latency
        dict(name="paged_actions_5heads", kind="paged", R=1, q_lo=32, q_hi=32, unit=1, kv_lo=1088, kv_hi=1088, Hq=5,
             Hkv=5, Dh=128, ps=64, chunk=0, fp8=False, pad=0),
        # two robots' 480p chunks, 14B class, two and four cached chunks behind them
        dict(name="paged_chunk_14b", kind="paged", R=2, q_lo=3152, q_hi=3152, unit=3152, kv_lo=6304, kv_hi=12608,
             Hq=40, Hkv=40, Dh=128, ps=64, chunk=3152, fp8=False, pad=0),
        # ragged causal prefill of a small model, shared heads of 64, pages that end inside a tile, rows behind the
        # last request
        dict(name="paged_prefill_odd", kind="paged", R=12, q_lo=1, q_hi=901, unit=1, kv_lo=1, kv_hi=2500, Hq=8, Hkv=2,
             Dh=64, ps=48, chunk=1, fp8=False, pad=37),
        # two samples' 480p chunks against instructions of 512 and fewer tokens, 14B class
        dict(name="cross_text_14b", kind="cross", R=2, q_lo=3152, q_hi=3152, k_lo=77, k_hi=512, Hq=40, Hkv=40, Dh=128,
             padded=True, pad=0),
        # one token each of 32 requests against an encoder's states, shared heads
        dict(name="cross_tokens_gqa", kind="cross", R=32, q_lo=1, q_hi=1, k_lo=300, k_hi=4000, Hq=32, Hkv=8, Dh=128,
             padded=False, pad=0),
        # the small test model's rows against short and absent texts: latency
        dict(name="cross_d512_odd", kind="cross", R=5, q_lo=1, q_hi=144, k_lo=0, k_hi=77, Hq=8, Hkv=8, Dh=64,
             padded=False, pad=11),
        # one 480p chunk and its actions: three axes, every row of the fused projection moved once
        dict(name="rope_chunk_14b", kind="rope", T=3152, axes=3, pairs="22,21,21", halves=False, Hq=40, Hkv=40, Dh=128,
             ps=64, fp8=False, pad=0, far=4096),
        # single tokens at far positions of one axis into an E4M3 cache, shared heads, pairs in two halves
        dict(name="rope_tokens_fp8", kind="rope", T=61, axes=1, pairs="64", halves=True, Hq=32, Hkv=8, Dh=128, ps=16,
             fp8=True, pad=3, far=1000000),
        # a few robots' next chunks: latency
        dict(name="plan_robots", kind="plan", R=6, lo=0, hi=12608, n_lo=0, n_hi=3152, ps=64, spare=100, pad=32),
        # a busy server: a thousand requests between one token and a long prefill, some ending
        dict(name="plan_server", kind="plan", R=1000, lo=0, hi=16000, n_lo=1, n_hi=1500, ps=16, spare=0, pad=500),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 4e12, w["flops"] / 5e14)


def draw(rng):
    """One more case: any operator, sizes over the whole range (over their logarithm), odd ones among them."""
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["paged", "paged", "paged", "cross", "cross", "rope", "plan"])
        Dh = rng.choice([64, 128, 128])
        Hkv = rng.choice([1, 2, 3, 5, 8, 16, 40])
        Hq = Hkv * (rng.choice([1, 1, 2, 3, 4, 5, 8]) if Hkv <= 8 else 1)
        heads = dict(Hq=Hq, Hkv=Hkv, Dh=Dh)
        pad = rng.choice([0, 0, rng.randint(1, 50)])
        if kind == "paged":
            hi = _log(rng, 1, 3152) if rng.random() < 0.6 else 1
            kv = _log(rng, 20, 32000)
            c = dict(kind=kind, R=_log(rng, 1, 64), q_lo=rng.choice([1, hi]), q_hi=hi, unit=1,
                     kv_lo=rng.randint(1, kv), kv_hi=kv, **heads, ps=16 * _log(rng, 1, 16),
                     chunk=rng.choice([0, 1, 1, hi, 7]), fp8=Dh == 128 and rng.random() < 0.4, pad=pad)
        elif kind == "cross":
            hi = _log(rng, 1, 3152)
            k = _log(rng, 8, 4000)
            c = dict(kind=kind, R=_log(rng, 1, 32), q_lo=rng.choice([1, hi]), q_hi=hi, k_lo=rng.choice([0, k // 4, k]),
                     k_hi=k, **heads, padded=rng.random() < 0.5, pad=pad)
        elif kind == "rope":
            axes = rng.randint(1, 4)
            halves = rng.random() < 0.5
            total = Dh // 2 if rng.random() < 0.7 else 32
            cut = sorted(rng.randint(1, total - 1) for _ in range(axes - 1))
            pairs = [b - a for a, b in zip([0] + cut, cut + [total])]
            if min(pairs) < 1:
                continue
            c = dict(kind=kind, T=_log(rng, 1, 8000), axes=axes, pairs=",".join(map(str, pairs)), halves=halves, **heads,
                     ps=16 * _log(rng, 1, 16), fp8=Dh == 128 and rng.random() < 0.4, pad=pad,
                     far=_log(rng, 100, 1000000))
        else:
            c = dict(kind=kind, R=_log(rng, 1, 2000), lo=0, hi=_log(rng, 50, 16000), n_lo=rng.randint(0, 1),
                     n_hi=_log(rng, 2, 3152), ps=16 * _log(rng, 1, 16), spare=rng.choice([0, 100]), pad=pad)
            if c["R"] * c["n_hi"] > 1500000:
                continue
        if _cost(c) <= most and _room(c):
            return c


def _room(c):
    """Whether the plain form's scores and widened keys fit beside the rest (a limit of the plain form alone)."""
    if c["kind"] not in ("paged", "cross"):
        return True
    q, k = _lens(c)
    scores, keys = c["R"] * c["Hq"] * max(q) * max(k) * 4, c["R"] * max(k) * c["Hkv"] * c["Dh"] * 4
    return scores <= 20e9 and keys <= 9e9


# ---- lengths: spread over the case's range (over its logarithm), the largest first ----
def _spread(n, lo, hi, turn):
    """n whole numbers of [lo, hi], the first hi, the others at steps of the golden ratio."""
    a, b = math.log(max(lo, 0) + 1), math.log(hi + 1)
    return [hi if i == 0 else max(lo, int(math.exp(a + (b - a) * ((i * 0.6180339887 + turn) % 1.0))) - 1)
            for i in range(n)]


def _lens(c):
    """Queries and keys of every request; a paged request's keys are its history and its queries."""
    q = _spread(c["R"], c["q_lo"], c["q_hi"], 0.31)
    if c["kind"] == "cross":
        return q, _spread(c["R"], c["k_lo"], c["k_hi"], 0.0)
    u = c["unit"]
    hist = _spread(c["R"], c["kv_lo"], c["kv_hi"], 0.0)
    if u > 1:
        hist = [c["kv_hi"] if i == 0 else max(c["kv_lo"], h // u * u) for i, h in enumerate(hist)]
    return q, [h + n for h, n in zip(hist, q)]


def _seen(c):
    """(query, key) pairs of every head that a request's rule lets a query see."""
    q, k = _lens(c)
    ch = c.get("chunk", 0)
    if not ch:
        return sum(a * b for a, b in zip(q, k))
    n = 0
    for a, b in zip(q, k):
        for first in range((b - a) // ch * ch, b, ch):  # the positions of one chunk see the same keys
            n += (min(first + ch, b) - max(first, b - a)) * min(first + ch, b)
    return n


def _plan_lens(c):
    """(cached, new, held pages) of every request: most keep their cache and grow, every seventh has ended."""
    cache = _spread(c["R"], c["lo"], c["hi"], 0.0)
    new = _spread(c["R"], c["n_lo"], c["n_hi"], 0.47)
    held = [-(-n // c["ps"]) for n in cache]
    for i in range(6, c["R"], 7):
        cache[i] = new[i] = 0
    return cache, new, held


def work(c):
    if c["kind"] in ("paged", "cross"):
        q, k = _lens(c)
        per_key = c["Hkv"] * ((2 * c["Dh"] + 4) if c.get("fp8") else 4 * c["Dh"])
        return {"bytes": sum(q) * c["Hq"] * c["Dh"] * 4 + sum(k) * per_key, "flops": 4 * c["Dh"] * c["Hq"] * _seen(c)}
    if c["kind"] == "rope":
        kv_out = c["Hkv"] * ((2 * c["Dh"] + 4) if c["fp8"] else 4 * c["Dh"])
        return {"bytes": c["T"] * ((2 * c["Hq"] + 2 * c["Hkv"]) * c["Dh"] * 2 + kv_out + 4 * c["axes"] + 4),
                "flops": c["T"] * (c["Hq"] + c["Hkv"]) * c["Dh"] * 3}
    cache, new, held = _plan_lens(c)
    moved = sum(abs(-(-(a + b) // c["ps"]) - h) for a, b, h in zip(cache, new, held))
    return {"bytes": 20 * c["R"] + 8 * moved + 8 * (sum(new) + c["pad"]), "flops": 0}


# ---- inputs ----
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(n):
    s = [0]
    for x in n:
        s.append(s[-1] + x)
    return s


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _mx(x):
    """E4M3 codes (as float8) and biased exponents of blocks of 32: the smallest e with max <= 448 * 2^e."""
    b = x.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)  # amax = m 2^e with m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(amax > 0, (e - 9 + (m > 0.875)).clamp(-127, 127), torch.zeros_like(e))
    codes = torch.ldexp(b, -e).to(torch.float8_e4m3fn).flatten(-2)
    return codes, (e.squeeze(-1) + 127).to(torch.uint8)


def _scaled(x):
    inv = torch.tensor(1.0 / V_SCALE, dtype=torch.float32, device=x.device)
    return (x * inv).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _cache(c, g, n_pages):
    """A pool of pages, K and V: normal values, channels of unequal size as a projection gives them."""
    H, D = c["Hkv"], c["Dh"]
    size = torch.exp(0.4 * _normal(g, 1, 1, H, D))
    k, v = _normal(g, n_pages, c["ps"], H, D) * size, _normal(g, n_pages, c["ps"], H, D)
    if not c["fp8"]:
        return {"k": k.bfloat16(), "v": v.bfloat16(), "k_exp": None}
    codes, ex = _mx(k)
    return {"k": codes.view(torch.uint8), "v": _scaled(v).view(torch.uint8), "k_exp": ex.view(torch.int32).squeeze(-1)}


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"c": c}
    if c["kind"] == "paged":
        q, kv = _lens(c)
        pages = [-(-n // c["ps"]) for n in kv]
        n_pages, width = sum(pages) + 3, max(pages)
        ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        table = torch.full((c["R"], width), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(width, device="cuda")[None] < _ints(pages)[:, None]] = ids[: sum(pages)]
        T = sum(q) + c["pad"]
        st |= _cache(c, g, n_pages)
        st |= {"q": _normal(g, T, c["Hq"], c["Dh"]).bfloat16(), "table": table, "q_start": _ints(_starts(q)),
               "kv_len": _ints(kv), "o": torch.zeros(T, c["Hq"], c["Dh"], dtype=torch.bfloat16, device="cuda")}
        c["mq"], c["mk"] = max(q), max(kv)
        if own:
            import paper_2602_15922_amd as wam
            st["cache"] = wam.make_paged_cache(st["k"], st["v"], k_exp=st["k_exp"], v_scale=V_SCALE)
            n = wam.wam_attn_paged_workspace_bytes(st["cache"], R=c["R"], T=T, Hq=c["Hq"], max_kv=c["mk"])
            st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    elif c["kind"] == "cross":
        q, k = _lens(c)
        q_at, k_at = _starts(q), _starts(k)
        if c["padded"]:  # [R][longest] rows, each sample's own first
            q_at, k_at = [i * max(q) for i in range(c["R"] + 1)], [i * max(k) for i in range(c["R"] + 1)]
        T, S = q_at[-1] + c["pad"], k_at[-1]
        kv = _normal(g, max(S, 1), 2, c["Hkv"], c["Dh"]).bfloat16()  # the two halves of one projection
        st |= {"q": _normal(g, T, c["Hq"], c["Dh"]).bfloat16(), "k": kv[:S, 0], "v": kv[:S, 1], "q_start": _ints(q_at),
               "k_start": _ints(k_at), "q_len": _ints(q), "k_len": _ints(k),
               "o": torch.zeros(T, c["Hq"], c["Dh"], dtype=torch.bfloat16, device="cuda")}
        c["mq"], c["mk"] = max(q), max(k)
        if own:
            import paper_2602_15922_amd as wam
            n = wam.wam_attn_cross_workspace_bytes(R=c["R"], T=T, Hq=c["Hq"], Hkv=c["Hkv"], Dh=c["Dh"], max_k=c["mk"])
            st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    elif c["kind"] == "rope":
        T = c["T"] + c["pad"]
        n_pages = -(-T // c["ps"]) + 2
        st |= _cache(c, g, n_pages)
        st["qkv"] = _normal(g, T, (c["Hq"] + 2 * c["Hkv"]) * c["Dh"]).bfloat16()
        st["pos"] = torch.randint(0, c["far"] + 1, (T, c["axes"]), generator=g, device="cuda", dtype=torch.int32)
        # the rows of a page lie together, the pages anywhere
        perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        t = torch.arange(T, device="cuda")
        slots = perm[t // c["ps"]] * c["ps"] + (t % c["ps"]).to(torch.int32)
        slots[c["T"]:] = -1
        st["slots"] = slots
        st["q_out"] = torch.zeros(T, c["Hq"], c["Dh"], dtype=torch.bfloat16, device="cuda")
        st["pairs"] = [int(p) for p in c["pairs"].split(",")]
        if own:
            import paper_2602_15922_amd as wam
            st["cache"] = wam.make_paged_cache(st["k"], st["v"], k_exp=st["k_exp"], v_scale=V_SCALE)
    else:
        cache, new, held = _plan_lens(c)
        need = [-(-(a + b) // c["ps"]) for a, b in zip(cache, new)]
        free = max(0, sum(n - h for n, h in zip(need, held))) + 5 + c["spare"]
        n_pages, width = sum(held) + free, max(max(need), max(held), 1)
        ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        table = torch.full((c["R"], width), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(width, device="cuda")[None] < _ints(held)[:, None]] = ids[: sum(held)]
        stack = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        stack[:free] = ids[sum(held):]
        T = sum(new) + c["pad"]
        order = torch.randperm(c["R"], generator=g, device="cuda")
        st |= {"cache_len": _ints(cache)[order], "new_len": _ints(new)[order], "held": _ints(held)[order],
               "table": table[order].contiguous(), "free_list": stack, "n_free": _ints([free]), "T": T}
        for name, n in (("held_out", c["R"]), ("n_free_out", 1), ("q_start", c["R"] + 1), ("kv_len", c["R"]),
                        ("slots", T), ("token_pos", T), ("status", 4)):
            st[name] = torch.zeros(n, dtype=torch.int32, device="cuda")
    return st


# ---- one pass ----
def run(st):
    c = st["c"]
    if c["kind"] == "plan":
        names = ("table", "free_list", "held_out", "n_free_out", "q_start", "kv_len", "slots", "token_pos", "status")
        _plan_own(st) if own else _plan_plain(st)
        return {n: st[n] for n in names}
    if c["kind"] == "rope":
        _rope_own(st) if own else _rope_plain(st)
        if c["fp8"]:
            return {"q": st["q_out"], "k": st["k"].view(torch.float8_e4m3fn), "v": st["v"].view(torch.float8_e4m3fn),
                    "k_exp": st["k_exp"].view(torch.float8_e8m0fnu)}
        return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    if c["kind"] == "paged":
        _paged_own(st) if own else _paged_plain(st)
    else:
        _cross_own(st) if own else _cross_plain(st)
    return st["o"]


def _paged_own(st):
    import paper_2602_15922_amd as wam
    c = st["c"]
    wam.wam_attn_paged(st["cache"], st["q"], st["table"], st["q_start"], st["kv_len"], st["o"], st["ws"],
                       max_kv=c["mk"], chunk=c["chunk"])


def _cross_own(st):
    import paper_2602_15922_amd as wam
    wam.wam_attn_cross(st["q"], st["k"], st["v"], st["q_start"], st["k_start"], st["o"], st["ws"], max_k=st["c"]["mk"],
                       q_len=st["q_len"], k_len=st["k_len"])


def _rope_own(st):
    import paper_2602_15922_amd as wam
    wam.wam_rope_qkv_paged(st["cache"], st["qkv"], st["pos"], st["slots"], st["q_out"], pairs=st["pairs"],
                           halves=st["c"]["halves"], theta=THETA)


def _plan_own(st):
    import paper_2602_15922_amd as wam
    wam.wam_page_plan(st["cache_len"], st["new_len"], st["held"], st["n_free"], st["table"], st["free_list"],
                      st["held_out"], st["n_free_out"], st["q_start"], st["kv_len"], st["slots"], st["status"],
                      page_size=st["c"]["ps"], token_pos=st["token_pos"])


def _attend(q, k, v, seen):
    """q [R, mq, Hq, D], k and v [R, mk, Hkv, D] in 32 bits, seen [R, mq, mk]: softmax attention, 0 where a
    row sees nothing."""
    R, mq, Hq, D = q.shape
    Hkv = k.shape[2]
    q = q.view(R, mq, Hkv, -1, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, -1, D)
    s = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(1.0 / math.sqrt(D))
    s = s.view(R, Hkv, -1, mq, k.shape[1])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(R, Hkv, -1, k.shape[1]), v.permute(0, 2, 1, 3).contiguous())
    o = o.view(R, Hkv, -1, mq, D) / torch.where(total > 0, total, torch.ones_like(total))
    return o.permute(0, 3, 1, 2, 4).reshape(R, mq, Hq, D)


def _rows(start, n, most):
    """Row numbers [R, most] of ragged sequences, and which of them there are."""
    i = torch.arange(most, device=start.device)
    return start[:, None].long() + i, i < n[:, None]


def _paged_plain(st):
    c, ps = st["c"], st["c"]["ps"]
    q_len = st["q_start"][1:] - st["q_start"][:-1]
    rows, here = _rows(st["q_start"][:-1], q_len, c["mq"])
    q = st["q"][rows.clamp(max=st["q"].shape[0] - 1)].float()
    j = torch.arange(c["mk"], device=q.device)
    page = st["table"][:, j // ps].long().clamp(min=0)
    k, v = st["k"][page, j % ps], st["v"][page, j % ps]
    there = j < st["kv_len"][:, None]
    if c["fp8"]:
        ex = st["k_exp"].unsqueeze(-1).view(torch.uint8)[page, j % ps].int() - 127
        k = k.view(torch.float8_e4m3fn).float()
        k = torch.ldexp(k.unflatten(-1, (-1, 32)), ex.unsqueeze(-1)).flatten(-2)
        v = v.view(torch.float8_e4m3fn).float() * V_SCALE
    k, v = k.float(), torch.where(there[..., None, None], v.float(), 0.0)
    p = (st["kv_len"] - q_len)[:, None] + torch.arange(c["mq"], device=q.device)
    end = st["kv_len"][:, None].expand_as(p)
    if c["chunk"]:
        end = torch.minimum(end, (torch.div(p, c["chunk"], rounding_mode="floor") + 1) * c["chunk"])
    o = _attend(q, k, v, j < end[..., None])
    st["o"][rows[here]] = o[here].to(st["o"].dtype)


def _cross_plain(st):
    c = st["c"]
    rows, here = _rows(st["q_start"][:-1], st["q_len"], c["mq"])
    q = st["q"][rows.clamp(max=st["q"].shape[0] - 1)].float()
    keys, there = _rows(st["k_start"][:-1], st["k_len"], c["mk"])
    keys = keys.clamp(max=st["k"].shape[0] - 1)
    k, v = st["k"][keys].float(), torch.where(there[..., None, None], st["v"][keys].float(), 0.0)
    o = _attend(q, k, v, there[:, None].expand(-1, c["mq"], -1))
    st["o"][rows[here]] = o[here].to(st["o"].dtype)


def _rope_plain(st):
    c, D = st["c"], st["c"]["Dh"]
    n = sum(st["pairs"])
    w = torch.tensor([THETA ** (-i / p) for p in st["pairs"] for i in range(p)], dtype=torch.float64, device="cuda")
    axis = torch.tensor([a for a, p in enumerate(st["pairs"]) for _ in range(p)], device="cuda")
    ang = st["pos"].double()[:, axis] * w  # 64 bits: a far position's angle
    cos, sin = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    x = st["qkv"].float().view(-1, c["Hq"] + 2 * c["Hkv"], D)
    r, v = x[:, : c["Hq"] + c["Hkv"]].clone(), x[:, c["Hq"] + c["Hkv"]:]
    if c["halves"]:
        a, b = x[:, : r.shape[1], :n], x[:, : r.shape[1], n: 2 * n]
        r[..., :n], r[..., n: 2 * n] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[:, : r.shape[1], : 2 * n: 2], x[:, : r.shape[1], 1: 2 * n: 2]
        r[..., : 2 * n: 2], r[..., 1: 2 * n: 2] = a * cos - b * sin, a * sin + b * cos
    ok = st["slots"] >= 0
    s = st["slots"][ok].long()
    st["q_out"][ok] = r[ok, : c["Hq"]].to(st["q_out"].dtype)
    k = r[ok, c["Hq"]:]
    put = lambda to, x: to.view(-1, *to.shape[2:]).index_copy_(0, s, x)  # noqa: E731
    if c["fp8"]:
        codes, ex = _mx(k)
        put(st["k"], codes.view(torch.uint8))
        put(st["k_exp"], ex.view(torch.int32).squeeze(-1))
        put(st["v"], _scaled(v[ok]).view(torch.uint8))
    else:
        put(st["k"], k.to(st["k"].dtype))
        put(st["v"], v[ok].to(st["v"].dtype))


def _plan_plain(st):
    ps, (R, width), T = st["c"]["ps"], st["table"].shape, st["T"]
    n_pages = st["free_list"].numel()
    cache, new, held = st["cache_len"].long(), st["new_len"].long(), st["held"].long()
    whole = (cache + new + ps - 1) // ps
    need = whole.clamp(max=width)
    take, back = (need - held).clamp(min=0), (held - need).clamp(min=0)
    take_at, back_at = take.cumsum(0) - take, back.cumsum(0) - back
    free, backs, takes = st["n_free"].long(), back.sum(), take.sum()
    col = torch.arange(width, device=cache.device)
    # the stack with the surplus pages on it, in request order; pages leave it from the top
    spot = torch.where((col >= need[:, None]) & (col < held[:, None]), free + back_at[:, None] + col - need[:, None],
                       n_pages)
    stack = torch.cat([st["free_list"], st["free_list"][:1]])
    stack.scatter_(0, spot.clamp(max=n_pages).flatten(), st["table"].flatten())
    top = free + backs
    at = top - 1 - (take_at[:, None] + col - held[:, None])
    given = torch.where(at >= 0, stack[at.clamp(0, n_pages - 1)], -1)
    st["table"].copy_(torch.where((col >= held[:, None]) & (col < need[:, None]), given, st["table"]))
    left = (top - takes).clamp(min=0)
    i = torch.arange(n_pages, device=cache.device)
    st["free_list"].copy_(torch.where((i >= free) & (i < left), stack[:n_pages], st["free_list"]))
    granted = torch.minimum(take, (top - take_at).clamp(min=0))
    st["held_out"].copy_(torch.minimum(held, need) + granted)
    st["n_free_out"].copy_(left)
    ends = new.cumsum(0).clamp(max=T)
    st["q_start"][0] = 0
    st["q_start"][1:] = ends
    st["kv_len"].copy_(cache + ends - torch.cat([ends.new_zeros(1), ends[:-1]]))
    t = torch.arange(T, device=cache.device)
    r = torch.searchsorted(ends, t, right=True)
    inside = r < R
    r = r.clamp(max=R - 1)
    p = cache[r] + t - st["q_start"][r]
    page = st["table"][r, (p // ps).clamp(max=width - 1)].long()
    ok = inside & (p // ps < width) & (page >= 0)
    st["slots"].copy_(torch.where(ok, page * ps + p % ps, -1))
    st["token_pos"].copy_(torch.where(inside, p, -1))
    st["status"].copy_(torch.stack([(takes - granted.sum()), (whole - need).sum(), (new.sum() - ends[-1]),
                                    torch.zeros_like(takes)]))


# ---- the definition in 64 bits ----
def exact(case, seed):
    if case["kind"] == "plan":
        return None
    st = prepare(case, seed)
    c = st["c"]
    return _exact_rope(st) if c["kind"] == "rope" else _exact_attention(st)


def _exact_attention(st):
    """Request by request, KV head by KV head: weights from the log of the summed exponentials."""
    c, G = st["c"], st["c"]["Hq"] // st["c"]["Hkv"]
    out = st["o"].double()
    at = st["q_start"].tolist()
    paged = c["kind"] == "paged"
    if paged:
        q_len = [b - a for a, b in zip(at, at[1:])]
        k_len = st["kv_len"].tolist()
    else:
        q_len, k_len, k_at = st["q_len"].tolist(), st["k_len"].tolist(), st["k_start"].tolist()
    for r in range(c["R"]):
        n, m = q_len[r], k_len[r]
        if n == 0 or m == 0:
            continue
        for h in range(c["Hkv"]):
            if paged:
                used = st["table"][r, : -(-m // c["ps"])].long()
                k, v = (st[x][used, :, h].flatten(0, 1)[:m] for x in ("k", "v"))
                if c["fp8"]:
                    bits = st["k_exp"][used, :, h].flatten()[:m].long()
                    e = torch.stack([(bits >> (8 * b)) & 255 for b in range(4)], 1).double() - 127
                    k = k.view(torch.float8_e4m3fn).double() * torch.exp2(e).repeat_interleave(32, 1)
                    v = v.view(torch.float8_e4m3fn).double() * V_SCALE
            else:
                k, v = (st[x][k_at[r]: k_at[r] + m, h] for x in ("k", "v"))
            q = st["q"][at[r]: at[r] + n, h * G: (h + 1) * G].double()
            s = torch.tensordot(q, k.double(), dims=([2], [1])) * c["Dh"] ** -0.5
            if paged and c["chunk"]:
                first = torch.arange(m - n, m, device=s.device) // c["chunk"] * c["chunk"]
                s[(torch.arange(m, device=s.device)[None] >= first[:, None] + c["chunk"])[:, None].expand_as(s)] = -math.inf
            w = torch.exp(s - torch.logsumexp(s, -1, keepdim=True))
            out[at[r]: at[r] + n, h * G: (h + 1) * G] = torch.tensordot(w, v.double(), dims=([2], [0]))
    return out


def _exact_rope(st):
    """The rotation as a complex product."""
    c, D, n = st["c"], st["c"]["Dh"], sum(st["pairs"])
    heads = c["Hq"] + c["Hkv"]
    x = st["qkv"].double().view(-1, heads + c["Hkv"], D)
    parts = [st["pos"][:, a: a + 1].double() / THETA ** (torch.arange(p, device=x.device, dtype=torch.float64) / p)
             for a, p in enumerate(st["pairs"])]
    turn = torch.polar(torch.ones_like(torch.cat(parts, 1)), torch.cat(parts, 1))[:, None]
    y = x[:, :heads].clone()
    if c["halves"]:
        z = torch.complex(y[..., :n].contiguous(), y[..., n: 2 * n].contiguous()) * turn
        y[..., :n], y[..., n: 2 * n] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., : 2 * n].unflatten(-1, (n, 2)).contiguous()) * turn
        y[..., : 2 * n] = torch.view_as_real(z).flatten(-2)
    ok = st["slots"] >= 0
    q = st["q_out"].double()
    q[ok] = y[ok, : c["Hq"]]
    if c["fp8"]:
        return {"q": q, "k": None, "v": None, "k_exp": None}
    k, v = st["k"].double(), st["v"].double()
    s = st["slots"][ok].long()
    k[s // c["ps"], s % c["ps"]] = y[ok, c["Hq"]:]
    v[s // c["ps"], s % c["ps"]] = x[ok, heads:]
    return {"q": q, "k": k, "v": v}
