"""fp64 numpy oracle of the decoding-stage operators: cache number formats, attention of drafted tokens over a cache,
beam selection and reordering of beam states.  Shares no code with the library."""
import math

import numpy as np


# ---- number formats of a cache
def e4m3_grid():
    """Non-negative e4m3 values: 3 mantissa bits, exponent bias 7, subnormals, largest 448."""
    v = [m / 8.0 * 2.0 ** -6 for m in range(8)]
    for e in range(1, 16):
        for m in range(8):
            if not (e == 15 and m == 7):  # that code is NaN
                v.append((1 + m / 8.0) * 2.0 ** (e - 7))
    return np.array(v)


_GRID = e4m3_grid()


def round_e4m3(x):
    """Nearest grid value, ties to the even code, by search (|x| <= 448)."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_GRID, a), 1, len(_GRID) - 1)
    lo = hi - 1
    down, up = a - _GRID[lo], _GRID[hi] - a
    pick = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.copysign(_GRID[pick], x)


def bf16_up(x):
    """The least bfloat16 not below a positive float32 number."""
    bits = np.float32(x).view(np.uint32)
    return float(np.uint32((int(bits) + 0xFFFF) & 0xFFFF0000).view(np.float32))


def quantise(x, fmt):
    """x [..., d] float64 holding values of the path's type -> (codes as numbers, scales)."""
    x = np.asarray(x, np.float64)
    flat = x.reshape(-1, x.shape[-1])
    codes, scales = np.zeros_like(flat), np.ones(len(flat))
    for i, vec in enumerate(flat):
        a = np.abs(vec).max()
        if not np.isfinite(a):
            scales[i] = np.nan
            continue
        if a == 0:
            continue
        if fmt == "e4m3":
            e = math.frexp(a / 448.0)  # m in [0.5, 1): the least power of two >= a / 448 is 2^e, or 2^(e - 1) if m is 0.5
            s = 2.0 ** max(e[1] - 1 if e[0] == 0.5 else e[1], -126)
            codes[i] = round_e4m3(vec / s)
        else:
            s = max(bf16_up(np.float32(a) / np.float32(127)), 2.0 ** -126)
            codes[i] = np.rint(vec / s)
        scales[i] = s
    return codes.reshape(x.shape), scales.reshape(x.shape[:-1])


def stored(x, fmt):
    """What vectors are worth after the cache."""
    if fmt == "path":
        return np.asarray(x, np.float64)
    codes, s = quantise(x, fmt)
    return codes * s[..., None]


# ---- attention of the rows of one sequence
def visible(start, n, tail, bits=None):
    """[n, positions] truth values: which cache positions each of n rows sees.  bits: [n, >= n] truth values."""
    if tail == "none":
        return np.ones((n, start), bool)
    see = np.ones((n, start + n), bool)
    see[:, start:] = np.tril(np.ones((n, n), bool)) if tail == "causal" else np.asarray(bits)[:, :n]
    return see


def attend(q, k, v, see, scale):
    """q [n, H, d], k / v [positions, Hk, d], see [n, positions] -> (out [n, H, d], lse [n, H]).  What a row does not
    see has no influence on it, whatever it holds."""
    n, H, d = q.shape
    G = H // k.shape[1]
    out, lse = np.zeros((n, H, d)), np.full((n, H), -np.inf)
    for i in range(n):
        at = np.nonzero(see[i])[0]
        if not len(at):
            continue
        for h in range(H):
            s = k[at, h // G] @ q[i, h] * scale
            m = s.max()
            p = np.exp(s - m)
            out[i, h] = p @ v[at, h // G] / p.sum()
            lse[i, h] = m + np.log(p.sum())
    return out, lse


# ---- beam search
def beam_select(logits, scores, keep, beams=None, finished=None, end_token=-1, suppressed=None):
    """logits [B, W, V], scores [B, W] -> (scores, parents, tokens, finished) [B, keep]."""
    B, W, V = logits.shape
    out = (np.full((B, keep), -np.inf), np.full((B, keep), -1, np.int64), np.full((B, keep), -1, np.int64), np.zeros((B, keep), np.int64))
    for b in range(B):
        found = []
        for w in range(W if beams is None else int(beams[b])):
            if finished is not None and finished[b, w]:
                found.append((float(scores[b, w]), w, end_token))
                continue
            x = np.array(logits[b, w], np.float64)
            if suppressed is not None:
                x[suppressed] = -np.inf
            if np.isnan(x).any() or x.max() == np.inf or x.max() == -np.inf:
                continue
            m = x.max()
            c = float(scores[b, w]) + (x - (m + np.log(np.exp(x - m).sum())))
            found += [(c[t], w, t) for t in range(V) if c[t] > -np.inf]
        found = [f for f in found if f[0] > -np.inf]
        found.sort(key=lambda f: (-f[0], f[1], f[2]))
        for i, (c, w, t) in enumerate(found[:keep]):
            done = t == end_token or (finished is not None and bool(finished[b, w]))
            out[0][b, i], out[1][b, i], out[2][b, i], out[3][b, i] = c, w, t, done
    return out


def beam_sources(parents):
    """Row whose state each row of a [B * W, ...] state takes over."""
    B, W = parents.shape
    p = np.where(parents < 0, np.arange(W)[None], parents)
    return (p + W * np.arange(B)[:, None]).reshape(-1)
