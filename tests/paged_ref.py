"""Plain 64-bit definitions of the paged operators (numpy, loops), and inputs for their tests."""
import math

import numpy as np

E4M3 = np.array([(-1) ** (b >> 7) * (math.ldexp(b & 7, -9) if not b >> 3 & 15 else math.ldexp(8 + (b & 7), (b >> 3 & 15) - 10))
                 for b in range(256)])
E4M3[[0x7F, 0xFF]] = np.nan


def plan(cache, new, held, free, n_free, table, ps, n_pages, T):
    """The page plan step by step with a Python list as the stack.  Returns the outputs by name."""
    R, width = table.shape
    table, free_list = table.copy(), free.copy()
    bad = sum(c < 0 or n < 0 or not 0 <= h <= width for c, n, h in zip(cache, new, held)) + (not 0 <= n_free <= n_pages)
    cache, new = [max(0, int(c)) for c in cache], [max(0, int(n)) for n in new]
    held = [min(max(0, int(h)), width) for h in held]
    n_free = min(max(0, int(n_free)), n_pages)
    whole = [-(-(c + n) // ps) for c, n in zip(cache, new)]
    need = [min(w, width) for w in whole]
    stack = [int(x) for x in free[:n_free]]
    for r in range(R):
        stack += [int(x) for x in table[r, need[r]:held[r]]]
    missing, held_out = 0, [min(h, n) for h, n in zip(held, need)]
    for r in range(R):
        for e in range(held[r], need[r]):
            if stack:
                table[r, e] = stack.pop()
                held_out[r] += 1
            else:
                table[r, e] = -1
                missing += 1
    left = len(stack)
    for i in range(n_free, min(left, n_pages)):
        free_list[i] = stack[i]
    q_start = [0]
    for n in new:
        q_start.append(min(q_start[-1] + n, T))
    slots, pos = np.full(T, -1), np.full(T, -1)
    kv = []
    for r in range(R):
        for t in range(q_start[r], q_start[r + 1]):
            p = cache[r] + t - q_start[r]
            pos[t] = p
            if p // ps < width and 0 <= table[r, p // ps] < n_pages:
                slots[t] = table[r, p // ps] * ps + p % ps
        kv.append(cache[r] + q_start[r + 1] - q_start[r])
    return dict(table=table, free_list=free_list, held_out=held_out, n_free_out=[min(left, n_pages)], q_start=q_start,
                kv_len=kv, slots=slots, token_pos=pos,
                status=[missing, sum(w - n for w, n in zip(whole, need)), sum(new) - q_start[-1], bad])


def angles(pos, pairs, theta):
    """[T, sum pairs] angles of positions [T, axes]."""
    cols = [pos[:, a:a + 1].astype(np.float64) * theta ** (-np.arange(p) / max(p, 1)) for a, p in enumerate(pairs)]
    return np.concatenate(cols, 1)


def rotate(x, ang, halves):
    """x [T, H, Dh] float64 turned pair by pair."""
    n = ang.shape[1]
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    y = x.copy()
    i, j = (slice(0, n), slice(n, 2 * n)) if halves else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
    return y


def attend(q, k, v, seen, scale):
    """One request and head: q [n, D], k, v [m, D], seen [n, m] -> (o [n, D], weighted mean of |v|).  Keys
    that a row does not see do not enter its sums, whatever they hold."""
    o, a = np.zeros((len(q), v.shape[1])), np.zeros((len(q), v.shape[1]))
    for i in range(len(q)):
        j = np.flatnonzero(seen[i])
        if len(j):
            s = k[j] @ q[i] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            o[i], a[i] = w @ v[j], w @ np.abs(v[j])
    return o, a


def chunk_seen(n, m, chunk):
    """[n, m]: which of m keys the last n tokens see."""
    p, j = m - n + np.arange(n)[:, None], np.arange(m)[None]
    return (j < (p // chunk + 1) * chunk) if chunk else np.ones((n, m), bool)


# ---- a ragged batch over a paged cache ----
class Batch:
    """Requests (q_len, kv_len) with their pages scattered over a pool; every cache row that holds no key, and every
    page of no request, is filled with `junk`."""

    def __init__(self, lens, Hq, Hkv, Dh, ps, seed, junk=np.nan, fp8=False, layout="nhd", spare=2, tail=3, gap=0):
        import torch
        g = torch.Generator().manual_seed(seed)
        self.lens, self.Hq, self.Hkv, self.Dh, self.ps, self.fp8 = lens, Hq, Hkv, Dh, ps, fp8
        R = len(lens)
        pages = [-(-max(m, 0) // ps) for _, m in lens]
        self.n_pages, self.width = sum(pages) + spare, max(pages + [1])
        ids = torch.randperm(self.n_pages, generator=g).tolist()
        self.table = np.full((R, self.width), -1, np.int32)
        self.q_start = np.zeros(R + 1, np.int32)
        for r, (n, _) in enumerate(lens):
            self.table[r, :pages[r]] = [ids.pop() for _ in range(pages[r])]
            self.q_start[r + 1] = self.q_start[r] + n + gap
        self.T = int(self.q_start[-1]) + tail
        self.q_len = np.array([n for n, _ in lens], np.int32)
        self.kv_len = np.array([m for _, m in lens], np.int32)
        self.q = torch.randn(self.T, Hq, Dh, generator=g).bfloat16()
        used = torch.zeros(self.n_pages, ps, dtype=torch.bool)
        for r, (_, m) in enumerate(lens):
            for j in range(m):
                used[self.table[r, j // ps], j % ps] = True
        shape = (self.n_pages, ps, Hkv, Dh)
        if fp8:
            self.k, self.v = (torch.randint(0, 256, shape, generator=g, dtype=torch.uint8) for _ in range(2))
            for x in (self.k, self.v):
                x[(x & 0x7F) == 0x7F] = 0x3A  # no NaN among the keys; magnitudes to 448
                x[~used] = 0x7F               # NaN codes where no key is
            self.k_exp = torch.randint(117, 122, shape[:3] + (4,), generator=g, dtype=torch.uint8)
            self.v_scale = 0.011
        else:
            self.k, self.v = torch.randn(shape, generator=g).bfloat16(), torch.randn(shape, generator=g).bfloat16()
            self.k[~used], self.v[~used] = junk, junk
            self.k_exp, self.v_scale = None, 0.0
        self.layout = layout

    def kv64(self, r):
        """Keys and values [m, Hkv, Dh] of request r, absent pages as None rows in `there`."""
        m = min(int(self.kv_len[r]), self.width * self.ps)
        k, v, there = np.zeros((m, self.Hkv, self.Dh)), np.zeros((m, self.Hkv, self.Dh)), np.zeros(m, bool)
        for j in range(m):
            pg, row = int(self.table[r, j // self.ps]), j % self.ps
            if 0 <= pg < self.n_pages:
                there[j] = True
                if self.fp8:
                    e = 2.0 ** (self.k_exp[pg, row].numpy().astype(np.float64) - 127)
                    k[j] = E4M3[self.k[pg, row].numpy()] * np.repeat(e, 32, axis=1)
                    v[j] = E4M3[self.v[pg, row].numpy()] * float(np.float32(self.v_scale))
                else:
                    k[j], v[j] = self.k[pg, row].double().numpy(), self.v[pg, row].double().numpy()
        return k, v, there

    def expected(self, chunk, scale=None, max_kv=None):
        """(o [T, Hq, Dh], weighted |v| mean, rows that are written)."""
        scale = self.Dh ** -0.5 if scale is None else scale
        o, a = np.zeros((self.T, self.Hq, self.Dh)), np.zeros((self.T, self.Hq, self.Dh))
        mine = np.zeros(self.T, bool)
        q = self.q.double().numpy()
        for r, n in enumerate(self.q_len):
            at, m = int(self.q_start[r]), int(self.kv_len[r])
            mine[at:at + n] = True
            k, v, there = self.kv64(r)
            seen = chunk_seen(n, m, chunk)[:, :len(there)] & there
            if max_kv is not None:
                seen[:, max_kv:] = False
            for h in range(self.Hq):
                hk = h // (self.Hq // self.Hkv)
                o[at:at + n, h], a[at:at + n, h] = attend(q[at:at + n, h], k[:, hk], v[:, hk], seen, scale)
        return o, a, mine

    def cache(self):
        """The device cache in this batch's layout; keeps its tensors."""
        import torch

        import paper_2602_15922_amd as w
        k, v, ex = self.k, self.v, None if self.k_exp is None else self.k_exp.view(torch.int32).squeeze(-1)
        if self.layout == "hnd":  # [page][head][token][Dh]
            k, v = (x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (k, v))
            ex = None if ex is None else ex.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        elif self.layout == "kv":  # halves of one buffer
            both = torch.stack([k, v], 1).cuda()
            k, v = both[:, 0], both[:, 1]
            if ex is not None:
                ex = torch.stack([ex, ex], 1).cuda()[:, 0]
        else:
            k, v, ex = k.cuda(), v.cuda(), None if ex is None else ex.cuda()
        self.dk, self.dv, self.dex = k, v, ex
        return w.make_paged_cache(k, v, k_exp=ex, v_scale=self.v_scale)


def attention_tolerance(a):
    """Per element: the probabilities and their sum are each off by at most half a bf16 step (2^-8 relative), and so is
    the stored output: 3 * 2^-8 of the weighted mean of |v|; 2^-11 of it more for fp32 scores, exponentials and sums
    (a score of size 64 in fp32 steps of 2^-18 moves its weight by 2^-18 / 2; sums of thousands of terms stay below
    2^-12)."""
    return (3 * 2.0 ** -8 + 2.0 ** -11) * a + 1e-30
