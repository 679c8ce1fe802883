"""fp64 numpy oracle of the operators around a round of speculative decoding: 8-bit matrices with block scales and their
products, rows and pages of a round, verification of drafted tokens, commit of accepted rows.  Shares no code with the library."""
import math

import numpy as np

from oracle.decode_oracle import round_e4m3


# ---- matrices in 8 bits
def quantise_rows(x):
    """x [rows, k] -> (codes as numbers [rows, k], exponent bytes [rows, ceil(k / 128)]); 255: the block has a NaN or an infinity."""
    x = np.asarray(x, np.float64)
    rows, k = x.shape
    codes, marks = np.zeros_like(x), np.full((rows, -(-k // 128)), 127)
    for r in range(rows):
        for b in range(0, k, 128):
            v = x[r, b:b + 128]
            a = np.abs(v).max()
            if not np.isfinite(a):
                marks[r, b // 128] = 255
                continue
            if a == 0:
                continue
            m, e = math.frexp(a / 448.0)  # the least power of two >= a / 448 is 2^e, or 2^(e - 1) where m is 0.5
            e = max(e - 1 if m == 0.5 else e, -126)
            codes[r, b:b + 128] = round_e4m3(v / 2.0 ** e)
            marks[r, b // 128] = e + 127
    return codes, marks


def values(codes, marks):
    s = np.where(np.asarray(marks) == 255, np.nan, 2.0 ** (np.asarray(marks, np.float64) - 127))
    return np.asarray(codes, np.float64) * np.repeat(s, 128, axis=1)[:, :codes.shape[1]]


def gelu(y):
    return np.array([0.5 * v * math.erfc(-v / math.sqrt(2.0)) for v in y.ravel()]).reshape(y.shape)


# ---- rows and pages of a round
def page_plan(ring, head, count, table, held, lengths, new_rows, n_rows, page, ended=None):
    """One round, step by step.  Changes ring, table, held and lengths (lists or arrays) in place; returns
    (head, count, cu, row_seq, row_pos, row_slot, sequences that were put off)."""
    n, N = len(new_rows), len(ring)
    free = [(head + i) % N for i in range(count)]      # places of the free pages
    back, put_off, want, need = [], [], [], []
    for s in range(n):
        l, h = int(lengths[s]), int(held[s])
        if ended is not None and ended[s]:
            back += [int(table[s][i]) for i in range(h)]
            lengths[s], held[s], l, h = 0, 0, 0, 0
        want.append(int(new_rows[s]))
        need.append(max(0, -(-(l + want[s]) // page) - h) if want[s] else 0)
    cu, used = [0], 0
    for s in range(n):
        rows_so_far, pages_so_far = sum(want[:s + 1]), sum(need[:s + 1])
        ok = rows_so_far <= n_rows and (need[s] == 0 or pages_so_far <= count)
        if not ok and want[s]:
            put_off.append(s)
        cu.append(cu[-1] + (want[s] if ok else 0))
        if ok:
            for i in range(need[s]):
                table[s][held[s] + i] = ring[free[used]]
                used += 1
            held[s] += need[s]
    for i, x in enumerate(back):
        ring[(head + count + i) % N] = x
    seq, pos, slot = (np.full(n_rows, -1, np.int64) for _ in range(3))
    for s in range(n):
        for i in range(cu[s + 1] - cu[s]):
            p = int(lengths[s]) + i
            seq[cu[s] + i], pos[cu[s] + i] = s, p
            slot[cu[s] + i] = int(table[s][p // page]) * page + p % page
    return (head + used) % N, count - used + len(back), np.array(cu), seq, pos, slot, put_off


# ---- verification of drafted tokens
def distribution(x, t):
    """softmax(x / t) in float64; t = 0: all of it on the first largest.  None where there is none."""
    x = np.asarray(x, np.float64)
    top = x.max() if not np.isnan(x).any() else np.nan
    if not np.isfinite(top):
        return None
    if t == 0:
        p = np.zeros(len(x))
        p[int(np.argmax(x))] = 1.0
        return p
    e = np.exp((x - top) / t)
    return e / e.sum()


def draft_verify(logits, tokens, parents, u, u_last, t=1.0, draft=None):
    """One sequence: logits [n, V], tokens and parents [n] (row 0 is the last token; a parent that does not fit: never tried).  Returns
    (tokens that are new, rows that stay, margin): how near to a border the nearest decision was, relative to what decides it."""
    n = len(tokens)
    if n == 0:
        return [], [], math.inf
    V = logits.shape[1]
    out, path, cur, margin = [], [0], 0, math.inf
    while True:
        p = distribution(logits[cur], t)
        if p is None:
            return out + [-1], path, margin
        kept = None
        for i in range(cur + 1, n):
            if parents[i] != cur or not 0 <= parents[i] < i or not 0 <= tokens[i] < V:
                continue
            x = int(tokens[i])
            if t == 0:
                if p[x] == 1.0:
                    kept = i
                    break
                continue
            q = np.asarray(draft[cur], np.float64) if draft is not None else None
            chance = float(u[i]) * (q[x] if q is not None else 1.0)
            margin = min(margin, abs(chance - p[x]) / max(p[x], 1e-300) * 1e6 if p[x] > 0 else math.inf)
            if chance < p[x]:
                kept = i
                break
            rest = np.where(p - q > 0, p - q, 0.0) if q is not None else np.where(np.arange(V) == x, 0.0, p)
            if rest.sum() > 0:
                p = rest / rest.sum()
        if kept is None:
            break
        out.append(int(tokens[kept]))
        path.append(kept)
        cur = kept
    if t == 0:
        return out + [int(np.argmax(p))], path, margin
    sums = np.cumsum(p)
    target = float(u_last) * sums[-1]
    some = np.flatnonzero(p > 0)
    hit = some[sums[some] > target]
    v = int(hit[0] if len(hit) else some[-1])
    margin = min(margin, min(abs(sums[v] - target), abs((sums[v] - p[v]) - target) if v > some[0] else math.inf) * 1e11)
    return out + [v], path, margin


# ---- commit
def commit(k, table, start, path, page):
    """k [pages, heads, page, d] of one side of a cache, in place: the rows of `path` (a list) move behind `start`."""
    at = lambda p: (int(table[p // page]), p % page)
    rows = [k[at(start + r)[0], :, at(start + r)[1]].copy() for r in path]
    for i, row in enumerate(rows):
        pg, w = at(start + i)
        k[pg, :, w] = row
