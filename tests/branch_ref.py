"""Plain definitions of the operators of requests that branch (Python loops, fractions and 64 bits)."""
from fractions import Fraction

import numpy as np


def fork(src, dst, first, length, held, n_free, table, free_list, ps, n_pages):
    """The forks one after another.  Returns the outputs by name."""
    R, width = table.shape
    table = table.copy()
    bad = sum(not 0 <= h <= width for h in held) + (not 0 <= n_free <= n_pages)
    held = [min(max(0, int(h)), width) for h in held]
    left = n_free = min(max(0, int(n_free)), n_pages)
    held_out, copies, missing, named = list(held), [], 0, set()
    for i, (s, d, n) in enumerate(zip(src, dst, length)):
        f = int(first[i]) if first is not None else 0
        inside = 0 <= d < R
        ok = inside and d not in named and held[d] == 0 and 0 <= s < R and f >= 0 and n >= 0
        if inside:
            named.add(int(d))
        if not ok or f * ps + n > held[s] * ps:
            bad += 1
            copies.append((-1, -1, 0))
            continue
        w, tail = divmod(int(n), ps)
        table[d, :w] = table[s, f:f + w]
        held_out[d] = w
        copy = (-1, -1, 0)
        if tail:
            page = -1
            if left > 0:
                left -= 1
                page = int(free_list[left])
                held_out[d] += 1
                copy = (int(table[s, f + w]), page, tail)
            else:
                missing += 1
            table[d, w] = page
        copies.append(copy)
    return dict(table=table, held_out=held_out, n_free_out=[left], copies=np.array(copies).reshape(-1, 3), status=[missing, bad])


def collect(cache_len, held, table, free_list, ps, n_pages):
    R, width = table.shape
    used, missing, bad, out = set(), 0, 0, []
    for r in range(R):
        bad += cache_len[r] < 0 or not 0 <= held[r] <= width
        kept = min(min(max(0, int(held[r])), width), -(-max(0, int(cache_len[r])) // ps))
        out.append(kept)
        for p in table[r, :kept]:
            if 0 <= p < n_pages:
                used.add(int(p))
            else:
                missing += 1
    free = [p for p in range(n_pages) if p not in used]
    free_list = free_list.copy()
    free_list[:len(free)] = free
    return dict(free_list=free_list, held_out=out, n_free_out=[len(free)], status=[missing, bad])


def rows_of(q_start, q_len, T):
    """(first row, rows) of each request, cut to T."""
    out = []
    for r in range(len(q_start) - 1):
        a, b = int(q_start[r]), min(max(int(q_start[r + 1]), 0), T)
        room = b - a if 0 <= a < b else 0
        out.append((a, room if q_len is None else min(max(int(q_len[r]), 0), room)))
    return out


def place(table, n_pages, ps, r, p):
    """(page, row) of position p, or None."""
    if p < 0 or p // ps >= table.shape[1] or not 0 <= table[r, p // ps] < n_pages:
        return None
    return int(table[r, p // ps]), p % ps


def compact(x, table, q_start, q_len, kv_len, keep, n_keep, ps):
    """x [n_pages, ps, ...] after the call: all rows read before any is written."""
    y = x.clone()
    for r, (at, n) in enumerate(rows_of(q_start, q_len, len(keep))):
        hist = int(kv_len[r]) - n
        for i in range(min(max(int(n_keep[r]), 0), n)):
            k = int(keep[at + i])
            if i < k < n:
                a, b = place(table, len(x), ps, r, hist + k), place(table, len(x), ps, r, hist + i)
                if a and b:
                    y[b] = x[a]
    return y


def tree_seen(mask, first, n, m, width):
    """[n, min(m, width)]: which keys n rows from row `first` of the mask on see; the last n of m keys are theirs."""
    seen = np.zeros((n, m), bool)
    hist = m - n
    words = mask.astype(np.int64) & 0xFFFFFFFF
    for i in range(n):
        seen[i, :max(hist, 0)] = True
        for j in range(max(0, -hist), min(n, 32 * words.shape[1])):
            seen[i, hist + j] = words[first + i, j // 32] >> (j % 32) & 1
    return seen[:, :width]


def ancestors(parent, words):
    """Rows of the mask for one tree."""
    out = np.zeros((len(parent), words), np.uint32)
    for i in range(len(parent)):
        j = i
        while j >= 0:
            out[i, j // 32] |= np.uint32(1 << (j % 32))
            j = parent[j]
    return out.view(np.int32)


def verify(p, q, tokens, parent, u, u_next, max_nodes=1024):
    """One tree, in exact fractions: p, q [n][V] (q None: the drafts were chosen).  Returns (path, next token)."""
    n = len(p)
    if n == 0:
        return [], -1
    F = lambda x: Fraction(float(x)) if x > 0 else Fraction(0)  # noqa: E731
    row = lambda x: {int(v): Fraction(float(x[v])) for v in np.flatnonzero(np.asarray(x) > 0)}  # noqa: E731
    V = len(p[0])
    cur, path = 0, [0]
    left, s = None, Fraction(1)  # left: what is left of the target (entries above 0) where it is no longer p itself
    for i in range(1, min(n, max_nodes)):
        x = int(tokens[i])
        if int(parent[i]) != cur or not 0 <= x < V:
            continue
        chance = left.get(x, Fraction(0)) if left is not None else F(p[cur][x])
        draft = F(q[cur][x]) if q is not None else Fraction(1)
        if Fraction(float(u[i])) * s * draft < chance:
            cur, left, s = i, None, Fraction(1)
            path.append(i)
            continue
        left = row(p[cur]) if left is None else left
        if q is not None:
            left = {v: a - s * F(q[cur][v]) for v, a in left.items()}
            left = {v: a for v, a in left.items() if a > 0}
            s = sum(left.values())
        else:
            s -= chance
            left.pop(x, None)
    left = row(p[cur]) if not left else left
    total = sum(left.values())
    if total == 0:
        return path, -1
    goal, at = Fraction(float(u_next)) * total, Fraction(0)
    for v in sorted(left):
        at += left[v]
        if at > goal:
            return path, v
    return path, max(left)
