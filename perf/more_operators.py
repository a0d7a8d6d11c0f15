"""The operators of requests that branch over a paged KV cache, as cases that can be timed and compared: forking
a history (shared pages, the last one copied), collecting the pages that no request names any more, attention of a
tree of new tokens over the cache, the choice among drafted tokens from given random numbers, and moving the chosen
branch's rows together.

`listed` gives the cases, `draw` more of the same ranges; `prepare` builds what a program holds before
the call, `run` is one pass: the plain form in elementary torch operations, or, where `own` is set, the
library's entry points; `exact` is the definition in 64 bits, `work` the bytes and operations a pass
cannot do without.
"""
import math
import random

import numpy as np
import torch

own = False

V_SCALE = 8.0 / 448.0  # an FP8 value cache's calibrated scale: these values stay below 8


def listed():
    return [
        # 16 drafted tokens of one request, one rank's 5 heads of the 14B class: latency
        dict(name="tree_one_5heads", kind="attn", R=1, n_lo=16, n_hi=16, kv_lo=1088, kv_hi=1088, Hq=5, Hkv=5, Dh=128,
             ps=64, fp8=False, branches=0, pad=0),
        # a shared-head decoder's drafted trees over very different histories
        dict(name="tree_gqa", kind="attn", R=16, n_lo=24, n_hi=64, kv_lo=200, kv_hi=16000, Hq=32, Hkv=8, Dh=128, ps=16,
             fp8=False, branches=0, pad=0),
        # small trees over long histories in an E4M3 cache
        dict(name="tree_fp8", kind="attn", R=48, n_lo=1, n_hi=12, kv_lo=1000, kv_hi=32000, Hq=40, Hkv=8, Dh=128, ps=64,
             fp8=True, branches=0, pad=5),
        # two futures of one robot's 480p chunk, 14B class, over two cached chunks: each sees the history and itself
        dict(name="branches_14b", kind="attn", R=1, n_lo=6304, n_hi=6304, kv_lo=6304, kv_hi=6304, Hq=40, Hkv=40, Dh=128,
             ps=64, fp8=False, branches=2, pad=0),
        # one robot's history forked for 8 candidate action chunks, 14B class
        dict(name="fork_candidates_14b", kind="fork", R=1, per=8, kv_lo=12640, kv_hi=12640, Hkv=40, Dh=128, ps=64,
             fp8=False),
        # a server's 64 requests, four branches of each, large pages
        dict(name="fork_server", kind="fork", R=64, per=4, kv_lo=200, kv_hi=8000, Hkv=16, Dh=128, ps=128, fp8=False),
        # the pages of a few robots' histories and branches
        dict(name="collect_robots", kind="collect", R=12, lo=1000, hi=16000, ps=64, shared=0.5, spare=1000),
        # a server's: 1000 requests, small pages, some ended, some shortened
        dict(name="collect_server", kind="collect", R=1000, lo=0, hi=16000, ps=16, shared=0.3, spare=40000),
        # accepted paths of drafted trees
        dict(name="compact_paths", kind="compact", R=16, n_lo=24, n_hi=64, keep=0.1, kv_lo=200, kv_hi=16000, Hkv=8,
             Dh=128, ps=16, fp8=False, pad=0),
        # half of the tokens of four 480p chunks kept, 14B class
        dict(name="compact_chunk_14b", kind="compact", R=4, n_lo=3152, n_hi=3152, keep=0.5, kv_lo=0, kv_hi=3152, Hkv=40,
             Dh=128, ps=64, fp8=False, pad=0),
        # trees of chosen (not drawn) drafts
        dict(name="verify_chosen", kind="verify", R=4, n_lo=24, n_hi=24, V=32000, drawn=False, wide=3, pad=0),
        # trees of drafts drawn from the draft's distribution, a large vocabulary
        dict(name="verify_drawn", kind="verify", R=48, n_lo=8, n_hi=32, V=100000, drawn=True, wide=3, pad=0),
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
        kind = rng.choice(["attn", "attn", "attn", "fork", "collect", "compact", "verify", "verify"])
        Dh = rng.choice([64, 128, 128])
        Hkv = rng.choice([1, 2, 3, 5, 8, 16, 40])
        heads = dict(Hkv=Hkv, Dh=Dh)
        fp8 = Dh == 128 and rng.random() < 0.4
        pad = rng.choice([0, 0, rng.randint(1, 50)])
        ps = 16 * _log(rng, 1, 16)
        if kind == "attn":
            Hq = Hkv * (rng.choice([1, 1, 2, 3, 4, 5, 8]) if Hkv <= 8 else 1)
            branches = rng.choice([0, 0, 2, 3, 8])
            hi = _log(rng, 1, 3000 if branches else 200)
            kv = _log(rng, 20, 32000)
            c = dict(kind=kind, R=_log(rng, 1, 64), n_lo=rng.choice([1, hi]), n_hi=hi, kv_lo=rng.randint(0, kv),
                     kv_hi=kv, Hq=Hq, **heads, ps=ps, fp8=fp8, branches=branches, pad=pad)
        elif kind == "fork":
            kv = _log(rng, 20, 16000)
            c = dict(kind=kind, R=_log(rng, 1, 64), per=_log(rng, 1, 8), kv_lo=rng.randint(1, kv), kv_hi=kv, **heads,
                     ps=ps, fp8=fp8)
        elif kind == "collect":
            c = dict(kind=kind, R=_log(rng, 1, 2000), lo=0, hi=_log(rng, 50, 16000), ps=ps,
                     shared=rng.choice([0.0, 0.3, 0.9]), spare=_log(rng, 1, 60000))
        elif kind == "compact":
            hi = _log(rng, 1, 3152)
            kv = _log(rng, 20, 16000)
            c = dict(kind=kind, R=_log(rng, 1, 64), n_lo=rng.choice([1, hi]), n_hi=hi, keep=rng.choice([0.05, 0.3, 0.9]),
                     kv_lo=rng.randint(0, kv), kv_hi=kv, **heads, ps=ps, fp8=fp8, pad=pad)
        else:
            hi = _log(rng, 1, 64)
            c = dict(kind=kind, R=_log(rng, 1, 64), n_lo=rng.choice([1, hi]), n_hi=hi, V=_log(rng, 1000, 200000),
                     drawn=rng.random() < 0.6, wide=rng.choice([1, 2, 4]), pad=pad)
        if _cost(c) <= most and _room(c):
            return c


def _room(c):
    """Whether a state, and the plain form beside it, fits (the scores and widened keys are limits of the plain form
    alone)."""
    if c["kind"] == "collect":
        return c["R"] * c["hi"] // c["ps"] <= 4000000
    if c["kind"] == "verify":
        return sum(_lens(c)[0]) * c["V"] <= 2e8
    n, kv = _lens(c)
    pool = (sum(kv) + c["R"] * c.get("per", 1) * c["ps"]) * c["Hkv"] * c["Dh"] * 4
    if c["kind"] == "attn":
        scores, keys = c["R"] * c["Hq"] * max(n) * max(kv) * 4, c["R"] * max(kv) * c["Hkv"] * c["Dh"] * 4
        return scores <= 20e9 and keys <= 9e9 and pool <= 9e9
    return pool <= 9e9


# ---- lengths: spread over the case's range (over its logarithm), the largest first ----
def _spread(n, lo, hi, turn):
    """n whole numbers of [lo, hi], the first hi, the others at steps of the golden ratio."""
    a, b = math.log(max(lo, 0) + 1), math.log(hi + 1)
    return [hi if i == 0 else max(lo, int(math.exp(a + (b - a) * ((i * 0.6180339887 + turn) % 1.0))) - 1)
            for i in range(n)]


def _lens(c):
    """New tokens and all tokens of every request: a history and the new ones (none for a fork)."""
    if c["kind"] == "verify":
        n = _spread(c["R"], c["n_lo"], c["n_hi"], 0.31)
        return n, n
    hist = _spread(c["R"], c["kv_lo"], c["kv_hi"], 0.0)
    n = [0] * c["R"] if c["kind"] == "fork" else _spread(c["R"], c["n_lo"], c["n_hi"], 0.31)
    return n, [h + a for h, a in zip(hist, n)]


def _kept(c):
    """New tokens that each request keeps, and those of them that move (the first two of them lie in place)."""
    n = _lens(c)[0]
    m = [max(1, int(a * c["keep"])) for a in n]
    return m, [max(0, k - 2) if k < a else 0 for k, a in zip(m, n)]


def _collect_lens(c):
    """Tokens that every request keeps and pages that it holds: every seventh has ended, every third lost some."""
    had = _spread(c["R"], c["lo"], c["hi"], 0.0)
    held = [-(-h // c["ps"]) for h in had]
    keep = [0 if i % 7 == 6 else h * 2 // 3 if i % 3 == 1 else h for i, h in enumerate(had)]
    return keep, held


def _blocks(n, branches):
    """Rows of each branch."""
    at = [n * b // branches for b in range(branches + 1)]
    return [(a, b) for a, b in zip(at, at[1:])]


def _parents(c, seed):
    """Every request's tree: node 0 the root, a node's parent before it, at most `wide` children (attention: any)."""
    rng = random.Random(seed)
    out = []
    for n in _lens(c)[0]:
        par, kids = [-1] * min(n, 1), [0] * n
        for i in range(1, n):
            while True:
                p = rng.randrange(max(0, i - 8), i)
                if kids[p] < c.get("wide", n) or i - p == 1:
                    break
            kids[p] += 1
            par.append(p)
        out.append(par)
    return out


def _bits(c, seed):
    """Every request's rows of visible new tokens, as whole numbers of one bit each."""
    if c["branches"]:
        return [[(1 << b) - (1 << a) for a, b in _blocks(n, c["branches"]) for _ in range(a, b)] for n in _lens(c)[0]]
    rows = []
    for par in _parents(c, seed):
        m = []
        for i, p in enumerate(par):
            m.append((m[p] if p >= 0 else 0) | 1 << i)
        rows.append(m)
    return rows


def work(c):
    n, kv = _lens(c) if c["kind"] != "collect" else (None, None)
    if c["kind"] == "collect":
        keep, held = _collect_lens(c)
        used = sum(min(h, -(-k // c["ps"])) for k, h in zip(keep, held))
        return {"bytes": 4 * (used + sum(held) - used + c["spare"]) + 12 * c["R"], "flops": 0}
    if c["kind"] == "verify":
        rows = c["R"] * c["V"] * (2 if c["drawn"] else 1)
        return {"bytes": 4 * rows + 16 * sum(n) + 12 * c["R"], "flops": 3 * c["R"] * c["V"]}
    row = c["Hkv"] * ((2 * c["Dh"] + 4) if c["fp8"] else 4 * c["Dh"])
    if c["kind"] == "fork":
        tails = sum(k % c["ps"] for k in kv) * c["per"]
        return {"bytes": 2 * tails * row + 8 * c["per"] * sum(-(-k // c["ps"]) for k in kv), "flops": 0}
    if c["kind"] == "compact":
        return {"bytes": 2 * sum(_kept(c)[1]) * row + 8 * sum(_kept(c)[0]), "flops": 0}
    seen = 0
    for a, b in zip(n, kv):
        if c["branches"]:
            own_part = sum((y - x) ** 2 for x, y in _blocks(a, c["branches"]))
        else:
            own_part = a * (1 + min(a, 8)) // 2  # (a tree's depth, about)
        seen += a * (b - a) + own_part
    return {"bytes": sum(n) * c["Hq"] * c["Dh"] * 4 + sum(kv) * row, "flops": 4 * c["Dh"] * c["Hq"] * seen}


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
    return torch.ldexp(b, -e).to(torch.float8_e4m3fn).flatten(-2), (e.squeeze(-1) + 127).to(torch.uint8)


def _cache(c, g, n_pages):
    """A pool of pages, K and V: normal values, channels of unequal size as a projection gives them."""
    H, D = c["Hkv"], c["Dh"]
    size = torch.exp(0.4 * _normal(g, 1, 1, H, D))
    if not c["fp8"]:
        k = (_normal(g, n_pages, c["ps"], H, D) * size).bfloat16()
        return {"k": k, "v": _normal(g, n_pages, c["ps"], H, D).bfloat16(), "k_exp": None}
    codes, ex = _mx(_normal(g, n_pages, c["ps"], H, D) * size)
    v = (_normal(g, n_pages, c["ps"], H, D) / V_SCALE).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return {"k": codes.view(torch.uint8), "v": v.view(torch.uint8), "k_exp": ex.view(torch.int32).squeeze(-1)}


def _table(g, pages, width, n_pages):
    """A table of scattered pages, -1 past each request's last; the pages left over."""
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(pages), width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda")[None] < _ints(pages)[:, None]] = ids[: sum(pages)]
    return table, ids[sum(pages):]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"c": c}
    if c["kind"] == "verify":
        return _prepare_verify(c, g, seed)
    if c["kind"] == "collect":
        return _prepare_collect(c, g)
    n, kv = _lens(c)
    pages = [-(-k // c["ps"]) for k in kv]
    forks = c["R"] * c["per"] if c["kind"] == "fork" else 0
    n_pages, width = sum(pages) + 3 + forks, max(max(pages), 1)
    st["table"], left = _table(g, pages, width, n_pages)
    st |= _cache(c, g, n_pages)
    if own:
        import paper_2602_15922_amd as wam
        st["cache"] = wam.make_paged_cache(st["k"], st["v"], k_exp=st["k_exp"], v_scale=V_SCALE if c["fp8"] else 0.0)
    if c["kind"] == "fork":
        # the branches' rows follow the requests'; they hold nothing yet
        st["table"] = torch.cat([st["table"], st["table"].new_full((forks, width), -1)])
        st |= {"src": torch.arange(c["R"], dtype=torch.int32, device="cuda").repeat_interleave(c["per"]),
               "dst": c["R"] + torch.randperm(forks, generator=g, device="cuda").to(torch.int32),
               "len": _ints(kv).repeat_interleave(c["per"]), "held": _ints(pages + [0] * forks),
               "free_list": torch.cat([left, left.new_full((n_pages - left.numel(),), -1)]), "n_free": _ints([left.numel()])}
        for name, size in (("held_out", (c["R"] + forks,)), ("n_free_out", (1,)), ("copies", (forks, 3)), ("status", (2,))):
            st[name] = torch.zeros(size, dtype=torch.int32, device="cuda")
        return st
    T = sum(n) + c["pad"]
    st |= {"q_start": _ints(_starts(n)), "kv_len": _ints(kv)}
    c["mq"], c["mk"] = max(n), max(kv)
    if c["kind"] == "compact":
        rng, keep = np.random.RandomState(seed % (1 << 32)), np.zeros(T, np.int32)
        for at, a, m in zip(_starts(n), n, _kept(c)[0]):
            # the first two lie in place, the others anywhere after them
            first = np.arange(min(m, 2))
            rest = np.sort(rng.permutation(np.arange(len(first), a))[: m - len(first)])
            keep[at: at + m] = np.concatenate([first, rest])
        st |= {"keep": _ints(keep.tolist()), "n_keep": _ints(_kept(c)[0])}
        return st
    words = -(-max(n) // 32)
    rows = b"".join(m.to_bytes(4 * words, "little") for req in _bits(c, seed) for m in req) + bytes(4 * words * c["pad"])
    mask = np.frombuffer(rows, np.int32).reshape(T, words).copy()
    st |= {"mask": torch.from_numpy(mask).cuda(), "q": _normal(g, T, c["Hq"], c["Dh"]).bfloat16(),
           "o": torch.zeros(T, c["Hq"], c["Dh"], dtype=torch.bfloat16, device="cuda")}
    if own:
        size = wam.wam_attn_tree_workspace_bytes(st["cache"], R=c["R"], T=T, Hq=c["Hq"], max_kv=c["mk"])
        st["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return st


def _prepare_collect(c, g):
    keep, held = _collect_lens(c)
    width = max(max(held), 1)
    # some requests begin with another's pages
    rows = torch.arange(c["R"], device="cuda")
    n_pages = sum(held) + c["spare"]
    table, _ = _table(g, held, width, n_pages)
    other = torch.randint(0, c["R"], (c["R"],), generator=g, device="cuda")
    both = torch.minimum(_ints(held), _ints(held)[other]) // 2
    takes = (torch.rand(c["R"], generator=g, device="cuda") < c["shared"]) & (other < rows)
    part = takes[:, None] & (torch.arange(width, device="cuda") < both[:, None])
    table = torch.where(part, table[other], table)
    st = {"c": c, "table": table, "cache_len": _ints(keep), "held": _ints(held),
          "free_list": torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")}
    for name, size in (("held_out", c["R"]), ("n_free_out", 1), ("status", 2)):
        st[name] = torch.zeros(size, dtype=torch.int32, device="cuda")
    return st


def _prepare_verify(c, g, seed):
    n, V = _lens(c)[0], c["V"]
    T = sum(n) + c["pad"]
    at, par = _starts(n), _parents(c, seed)
    z = _normal(g, T, V).mul_(2.5)
    near = torch.softmax(z + _normal(g, T, V), -1)  # the draft: the target's scores, off by something
    parent = [p for req in par for p in req] + [-1] * c["pad"]
    row = torch.tensor([a + max(p, 0) for a, req in zip(at, par) for p in req] + [0] * c["pad"], device="cuda")
    if c["drawn"]:
        tokens = torch.multinomial(near[row], 1, generator=g)[:, 0]
    else:  # a node's children: its likeliest tokens, in order
        turn, kids = [], {}
        for t in range(T):
            kids[int(row[t])] = kids.get(int(row[t]), -1) + 1
            turn.append(kids[int(row[t])] if parent[t] >= 0 else 0)
        top = near[row].topk(min(V, max(turn) + 1), -1).indices
        tokens = top[torch.arange(T, device="cuda"), torch.tensor(turn, device="cuda")]
    st = {"c": c, "p": torch.softmax(z, -1), "q": near if c["drawn"] else None, "tokens": tokens.to(torch.int32),
          "parent": _ints(parent), "u": torch.rand(T, generator=g, device="cuda"),
          "u_next": torch.rand(c["R"], generator=g, device="cuda"), "q_start": _ints(at),
          "kv_len": _ints([1000 + a for a in n])}
    for name, size in (("path", T), ("n_path", c["R"]), ("next", c["R"]), ("cache_len", c["R"])):
        st[name] = torch.zeros(size, dtype=torch.int32, device="cuda")
    c["mq"] = max(n)
    if own:
        import paper_2602_15922_amd as wam
        size = wam.wam_verify_tree_workspace_bytes(R=c["R"], T=T, V=V, drawn=c["drawn"])
        st["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return st


# ---- one pass ----
def run(st):
    kind = st["c"]["kind"]
    (_OWN if own else _PLAIN)[kind](st)
    if kind == "attn":
        return st["o"]
    if kind == "collect":
        return {n: st[n] for n in ("free_list", "held_out", "n_free_out", "status")}
    if kind == "verify":
        return {n: st[n] for n in ("path", "n_path", "next", "cache_len")}
    out = {n: st[n] for n in ("table", "held_out", "n_free_out", "copies", "status")} if kind == "fork" else {}
    if st["c"]["fp8"]:
        return out | {"k": st["k"].view(torch.float8_e4m3fn), "v": st["v"].view(torch.float8_e4m3fn),
                      "k_exp": st["k_exp"].view(torch.float8_e8m0fnu)}
    return out | {"k": st["k"], "v": st["v"]}


def _attn_own(st):
    import paper_2602_15922_amd as wam
    wam.wam_attn_tree(st["cache"], st["q"], st["table"], st["q_start"], st["kv_len"], st["mask"], st["o"], st["ws"],
                      max_kv=st["c"]["mk"])


def _fork_own(st):
    import paper_2602_15922_amd as wam
    wam.wam_page_fork(st["src"], st["dst"], None, st["len"], st["held"], st["n_free"], st["table"], st["free_list"],
                      st["held_out"], st["n_free_out"], st["copies"], st["status"], page_size=st["c"]["ps"])
    wam.wam_page_copy(st["cache"], st["copies"])


def _collect_own(st):
    import paper_2602_15922_amd as wam
    wam.wam_page_collect(st["cache_len"], st["held"], st["table"], st["free_list"], st["held_out"], st["n_free_out"],
                         st["status"], page_size=st["c"]["ps"])


def _compact_own(st):
    import paper_2602_15922_amd as wam
    wam.wam_cache_compact(st["cache"], st["table"], st["q_start"], st["kv_len"], st["keep"], st["n_keep"])


def _verify_own(st):
    import paper_2602_15922_amd as wam
    wam.wam_verify_tree(st["p"], st["q"], st["tokens"], st["parent"], st["u"], st["u_next"], st["q_start"], st["path"],
                        st["n_path"], st["next"], st["ws"], kv_len=st["kv_len"], cache_len=st["cache_len"])


def _rows(start, n, most):
    """Row numbers [R, most] of ragged sequences, and which of them there are."""
    i = torch.arange(most, device=start.device)
    return start[:, None].long() + i, i < n[:, None]


def _attn_plain(st):
    c, ps = st["c"], st["c"]["ps"]
    q_len = st["q_start"][1:] - st["q_start"][:-1]
    rows, here = _rows(st["q_start"][:-1], q_len, c["mq"])
    rows = rows.clamp(max=st["q"].shape[0] - 1)
    q = st["q"][rows].float()
    j = torch.arange(c["mk"], device=q.device)
    page = st["table"][:, j // ps].long().clamp(min=0)
    k, v = st["k"][page, j % ps], st["v"][page, j % ps]
    there = j < st["kv_len"][:, None]
    if c["fp8"]:
        ex = st["k_exp"].unsqueeze(-1).view(torch.uint8)[page, j % ps].int() - 127
        k = torch.ldexp(k.view(torch.float8_e4m3fn).float().unflatten(-1, (-1, 32)), ex.unsqueeze(-1)).flatten(-2)
        v = v.view(torch.float8_e4m3fn).float() * V_SCALE
    k, v = k.float(), torch.where(there[..., None, None], v.float(), 0.0)
    # the history, and of the new tokens those whose bit is set
    bit = torch.arange(32, device=q.device, dtype=torch.int32)
    new = ((st["mask"][rows].unsqueeze(-1) >> bit) & 1).flatten(-2).bool()  # [R, mq, 32 words]
    i = j - (st["kv_len"] - q_len)[:, None]
    seen = (i < 0)[:, None] | new.gather(2, i.clamp(0, new.shape[2] - 1)[:, None].expand(-1, c["mq"], -1))
    seen = seen & there[:, None]
    R, mq, Hq, D = q.shape
    Hkv = k.shape[2]
    q = q.view(R, mq, Hkv, -1, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, -1, D)
    s = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(1.0 / math.sqrt(D)).view(R, Hkv, -1, mq, c["mk"])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(R, Hkv, -1, c["mk"]), v.permute(0, 2, 1, 3).contiguous()).view(R, Hkv, -1, mq, D)
    o = (o / torch.where(total > 0, total, torch.ones_like(total))).permute(0, 3, 1, 2, 4).reshape(R, mq, Hq, D)
    st["o"][rows[here]] = o[here].to(st["o"].dtype)


def _fork_plain(st):
    ps, width, table = st["c"]["ps"], st["table"].shape[1], st["table"]
    src, dst, length = st["src"].long(), st["dst"].long(), st["len"]
    whole, tail = length // ps, length % ps
    has = (tail > 0).int()
    at = st["n_free"] - 1 - (has.cumsum(0) - has)  # a page for each tail, in order, from the top of the stack
    page = torch.where((has > 0) & (at >= 0), st["free_list"][at.clamp(min=0).long()], -1)
    col = torch.arange(width, device=src.device)
    row = torch.where(col < whole[:, None], table[src], table[dst])
    row = torch.where((col == whole[:, None]) & (has[:, None] > 0), page[:, None], row)
    last = table[src, whole.clamp(max=width - 1).long()]
    table[dst] = row
    there = (has > 0) & (page >= 0)
    st["copies"].copy_(torch.stack([torch.where(there, last, -1), torch.where(there, page, -1), tail * there], 1))
    st["held_out"].copy_(st["held"])
    st["held_out"][dst] = whole.int() + there.int()
    st["n_free_out"].copy_((st["n_free"] - has.sum()).clamp(min=0))
    st["status"].copy_(torch.stack([(has - there.int()).sum(), torch.zeros_like(has).sum()]))
    # the copies: all of the pages' rows at once
    i = torch.arange(ps, device=src.device)
    mine = i < st["copies"][:, 2:3]
    a = (st["copies"][:, :1].long() * ps + i)[mine]
    b = (st["copies"][:, 1:2].long() * ps + i)[mine]
    _move(st, a, b)


def _move(st, a, b):
    """Rows (slots) a of the cache to b, all of them read first."""
    for x in (st["k"], st["v"], st["k_exp"]):
        if x is not None:
            y = x.view(-1, *x.shape[2:])
            y.index_copy_(0, b, y[a])


def _collect_plain(st):
    ps, width, n_pages = st["c"]["ps"], st["table"].shape[1], st["free_list"].numel()
    need = ((st["cache_len"] + ps - 1) // ps).clamp(max=width)
    kept = torch.minimum(st["held"], need)
    mine = torch.arange(width, device=need.device) < kept[:, None]
    there = mine & (st["table"] >= 0) & (st["table"] < n_pages)
    used = torch.zeros(n_pages + 1, dtype=torch.bool, device=need.device)
    used.scatter_(0, torch.where(there, st["table"], n_pages).flatten().long(), True)
    free = ~used[:n_pages]
    at = torch.where(free, free.cumsum(0) - 1, n_pages)
    out = torch.cat([st["free_list"], st["free_list"][:1]])
    out.scatter_(0, at, torch.arange(n_pages, dtype=torch.int32, device=need.device))
    st["free_list"].copy_(out[:n_pages])
    st["held_out"].copy_(kept)
    st["n_free_out"].copy_(free.sum())
    st["status"].copy_(torch.stack([(mine & ~there).sum(), torch.zeros_like(kept[0])]))


def _compact_plain(st):
    c, ps = st["c"], st["c"]["ps"]
    q_len = st["q_start"][1:] - st["q_start"][:-1]
    rows, _ = _rows(st["q_start"][:-1], q_len, c["mq"])
    i = torch.arange(c["mq"], device=rows.device)
    first = (st["kv_len"] - q_len)[:, None]
    slots = []
    for x in (st["keep"][rows.clamp(max=st["keep"].shape[0] - 1)], i):
        p = (first + x).clamp(max=st["table"].shape[1] * ps - 1).long()
        slots.append(st["table"].gather(1, p // ps).long() * ps + p % ps)
    moved = (i < st["n_keep"][:, None]) & (slots[0] != slots[1])
    _move(st, slots[0][moved], slots[1][moved])


def _verify_plain(st):
    c, V = st["c"], st["c"]["V"]
    at = st["q_start"][:-1].long()
    n = st["q_start"][1:].long() - at
    R, dev = n.numel(), n.device
    last = st["p"].shape[0] - 1
    cur, count = torch.zeros_like(n), (n > 0).long()
    s, take = torch.ones(R, dtype=torch.float64, device=dev), torch.zeros(R, dtype=torch.float64, device=dev)
    gone = torch.zeros(R, V, dtype=torch.bool, device=dev)
    path = torch.cat([st["path"], st["path"].new_zeros(1)])
    path[torch.where(n > 0, at, last + 1)] = 0

    def left():
        """What is left of the target's probabilities at each request's node."""
        row = (at + cur).clamp(max=last)
        p = st["p"][row].double()
        if st["q"] is None:
            return torch.where(gone, 0.0, p)
        return torch.relu(p - take[:, None] * st["q"][row].double())

    rest = left()
    for i in range(1, c["mq"]):
        row = (at + i).clamp(max=last)
        token = st["tokens"][row].long()
        mine = (i < n) & (st["parent"][row] == cur) & (token >= 0) & (token < V)
        token = token.clamp(0, V - 1)
        chance = rest.gather(1, token[:, None])[:, 0]
        drafted = 1.0 if st["q"] is None else st["q"][(at + cur).clamp(max=last), token].double()
        yes = mine & (st["u"][row].double() * s * drafted < chance)
        no = mine & ~yes
        cur = torch.where(yes, i, cur)
        path[torch.where(yes, at + count, last + 1)] = i
        count = count + yes.long()
        take = torch.where(no, take + s, torch.where(yes, 0.0, take))
        if st["q"] is None:
            gone = torch.where(yes[:, None], False, gone)
            gone.scatter_(1, token[:, None], gone.gather(1, token[:, None]) | no[:, None])
        rest = left()
        fewer = s - chance if st["q"] is None else rest.sum(-1)
        s = torch.where(no, fewer, torch.where(yes, 1.0, s))
    whole = st["p"][(at + cur).clamp(max=last)].double()
    rest = torch.where(rest.sum(-1, keepdim=True) > 0, rest, whole)
    sums = rest.cumsum(-1)
    hit = sums > st["u_next"].double()[:, None] * sums[:, -1:]
    index = torch.arange(V, device=dev)
    first = torch.where(hit, index, V).amin(-1)
    final = torch.where(rest > 0, index, -1).amax(-1)
    st["path"].copy_(path[:-1])
    st["n_path"].copy_(count)
    st["next"].copy_(torch.where(n > 0, torch.minimum(first, final), -1))
    st["cache_len"].copy_(st["kv_len"] - n + count)


_PLAIN = dict(attn=_attn_plain, fork=_fork_plain, collect=_collect_plain, compact=_compact_plain, verify=_verify_plain)
_OWN = dict(attn=_attn_own, fork=_fork_own, collect=_collect_own, compact=_compact_own, verify=_verify_own)


# ---- the definition in 64 bits ----
def exact(case, seed):
    """Attention request by request, KV head by KV head, weights from the log of the summed exponentials.  The other
    operators' outputs are whole numbers and bits moved."""
    if case["kind"] != "attn":
        return None
    st = prepare(case, seed)
    c, G = st["c"], st["c"]["Hq"] // st["c"]["Hkv"]
    out = st["o"].double()
    at, kv = st["q_start"].tolist(), st["kv_len"].tolist()
    for r, bits in enumerate(_bits(case, seed)):
        n, m = len(bits), kv[r]
        if n == 0:
            continue
        words = -(-n // 8)
        sees = np.unpackbits(np.frombuffer(b"".join(b.to_bytes(words, "little") for b in bits), np.uint8), bitorder="little")
        sees = torch.from_numpy(sees.reshape(n, 8 * words)[:, :n].astype(bool)).cuda()
        hidden = torch.cat([sees.new_zeros(n, m - n), ~sees], 1)[:, None]
        used = st["table"][r, : -(-m // c["ps"])].long()
        for h in range(c["Hkv"]):
            k, v = (st[x][used, :, h].flatten(0, 1)[:m] for x in ("k", "v"))
            if c["fp8"]:
                e8 = st["k_exp"][used, :, h].flatten()[:m].long()
                e = torch.stack([(e8 >> (8 * b)) & 255 for b in range(4)], 1).double() - 127
                k = k.view(torch.float8_e4m3fn).double() * torch.exp2(e).repeat_interleave(32, 1)
                v = v.view(torch.float8_e4m3fn).double() * V_SCALE
            q = st["q"][at[r]: at[r] + n, h * G: (h + 1) * G].double()
            s = torch.tensordot(q, k.double(), dims=([2], [1])) * c["Dh"] ** -0.5
            s.masked_fill_(hidden, -math.inf)
            w = torch.exp(s - torch.logsumexp(s, -1, keepdim=True))
            out[at[r]: at[r] + n, h * G: (h + 1) * G] = torch.tensordot(w, v.double(), dims=([2], [0]))
    return out
