"""The decoding-stage kernels at batch sizes that choose their variants for large calls: units of attention shared by two warps or
one, several heads of a cache row per group of lanes, selections with more blocks than SMs.  Against the fp64 oracle."""
import numpy as np
import pytest

from oracle import decode_oracle as O
from tests.test_decode_attention import Case
from tests.test_decode_cache import _layout, _values

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _decoder(**kw):
    from paper_2412_11272_b200.binding import Decoder
    return Decoder(**{**dict(n_head=4, d_head=64, dtype="bf16", cache_format="e4m3", page_size=16), **kw})


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda:0", dtype)


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# ---- attention: many sequences that read a few histories
def _attend_all(q, k, v, see, scale):
    """O.attend for many sequences with one history: q [b, n, H, d], k / v [positions, Hk, d], see [n, positions]."""
    b, n, H, d = q.shape
    Hk = k.shape[1]
    x = np.einsum("bnkgd,pkd->bnkgp", q.reshape(b, n, Hk, H // Hk, d), k, optimize=True) * scale
    x = np.where(see[None, :, None, None], x, -np.inf)
    m = x.max(-1, initial=-np.inf, keepdims=True)
    p = np.exp(x - np.where(np.isinf(m), 0, m))
    total = p.sum(-1)
    out = np.einsum("bnkgp,pkd->bnkgd", p, v, optimize=True) / np.where(total == 0, 1, total)[..., None]
    with np.errstate(divide="ignore"):
        lse = m[..., 0] + np.log(total)
    return out.reshape(b, n, H, d), lse.reshape(b, n, H)


class Batch(Case):
    """``copies`` sequences for every history of a Case: their own queries, the same pages."""

    def __init__(self, rng, dec, rows, starts, tail, copies):
        super().__init__(rng, dec, rows, starts, tail)
        self.copies, self.base_rows, self.base_starts = copies, rows, starts
        S = len(rows)
        self.of = rng.permutation(np.repeat(np.arange(S), copies))                   # the history of each sequence
        if tail == "mask":
            self.mask = np.concatenate([self.mask[self.cu[h]:self.cu[h + 1]] for h in self.of])
        self.rows, self.starts, self.table = [rows[h] for h in self.of], [starts[h] for h in self.of], self.table[self.of]
        self.cu = np.concatenate([[0], np.cumsum(self.rows)])
        self.n = int(self.cu[-1])
        self.q = torch.as_tensor((1.5 * rng.normal(size=(self.n, dec.n_head, dec.d_head))).astype(np.float32)).to(dec.torch_dtype)

    def want(self):
        d = self.dec
        out, lse = np.zeros((self.n, d.n_head, d.d_head)), np.full((self.n, d.n_head), -np.inf)
        for h, n in enumerate(self.base_rows):
            if n == 0:
                continue
            k, v = (O.stored(x[self.first[h]:self.first[h + 1]].double().numpy(), d.cache_format) for x in (self.k, self.v))
            see = O.visible(self.base_starts[h], n, self.tail, self.bits[h])
            at = self.cu[np.nonzero(self.of == h)[0]][:, None] + np.arange(n)
            out[at], lse[at] = _attend_all(self.q.double().numpy()[at], k, v, see, d.d_head ** -0.5)
            one, one_lse = O.attend(self.q[at[0]].double().numpy(), k, v, see, d.d_head ** -0.5)
            assert np.allclose(out[at[0]], one, atol=1e-12) and np.allclose(lse[at[0]], one_lse, atol=1e-12)
        return out, lse


@pytest.mark.parametrize("warps", [2, 1])
@pytest.mark.parametrize("d,group,top", [(64, 2, 4), (64, 2, 8), (64, 3, 10), (128, 2, 4), (128, 2, 8)])
@pytest.mark.parametrize("fmt", ["path", "e4m3", "int8"])
def test_units_shared_by_fewer_warps(fmt, d, group, top, warps):
    """Tiles of 8, 16 and 32 query rows (``top`` rows of ``group`` heads); twice (four times) as many units as warps of four fit the SMs."""
    rng = np.random.default_rng([d, group, top, warps])
    heads = 20
    tile = 8 if group * top <= 8 else 16 if group * top <= 16 or d == 128 else 32
    resident = _sms() * (16 if tile == 8 else 12 if tile == 16 and d == 64 else 8)
    need = (2 if warps == 2 else 4) * resident                                       # units: one tile of every head and sequence
    rows, starts = [top, 1, 0, 3, 2, top - 1], [0, 37, 12, 150, 0, 64]
    copies = -(-need // (heads * len(rows)))
    units = heads * len(rows) * copies
    assert units >= need and (warps == 1 or units < 2 * need)
    dec = _decoder(n_head=heads * group, n_kv_head=heads, d_head=d, cache_format=fmt, page_size=32)
    for tail in ("causal", "none") if top % 2 else ("mask", "none"):
        c = Batch(rng, dec, rows, starts, tail, copies)
        assert dec.tree_attention_workspace(len(c.rows), c.n, top, c.max_len) == 0   # one split
        got = c.run()
        c.check(got, c.want())
        again = c.run()
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("fmt,d", [("e4m3", 64), ("path", 128)])
def test_single_tokens_of_many_beams(fmt, d):
    """One token for each of 64 x 5 beams of 20 heads, values that are not finite in places that nothing sees."""
    rng = np.random.default_rng(d)
    dec = _decoder(n_head=20, d_head=d, cache_format=fmt, page_size=16)
    c = Batch(rng, dec, [1] * 5, [0, 1, 15, 16, 219], "causal", 64)
    got, want = c.run(), c.want()
    c.check(got, want)
    # the same as the sequences one at a time give (units shared by four warps, other orders of the sums)
    for s in range(0, 320, 71):
        one = dec.wf_tree_attention(c.cache, _dev(c.table[s:s + 1]), _dev([0, 1]), _dev(c.starts[s:s + 1]), c.q[s:s + 1].cuda(), 1, c.max_len)
        # each answer within the tolerance of Case.check of the oracle's
        assert (one[0].double() - got[0][s:s + 1].double()).abs().max() <= 2 * (2.0 ** -7 + 1e-4) * float(c.v.double().abs().max())
        assert torch.isfinite(one[0]).all()


# ---- cache: rows enough for four heads (write) and two (read) per group of lanes
@pytest.mark.parametrize("fmt", ["path", "e4m3", "int8"])
@pytest.mark.parametrize("d,H", [(64, 5), (64, 6), (128, 3), (128, 7)])
def test_large_writes_and_reads(fmt, d, H):
    """16-bit rows from 2^20 groups of eight elements on: head counts that are no multiples of four or two, sequences that end inside a
    warp's rows, rows behind the last one, strides, and pages that are not the cache's."""
    from paper_2412_11272_b200.binding import STATUS_BAD_PAGE
    rng = np.random.default_rng([d, H])
    n_min = -(-(1 << 20) // (H * d // 8))
    rows, starts, page = [n_min - 4000, 0, 1, 2503, 0, 1501], [11, 3, 40, 0, 5, 77], 64
    n, pad = sum(rows), 9
    assert (n + pad) * H * (d // 8) >= 1 << 20
    dec = _decoder(n_head=H, d_head=d, cache_format=fmt, page_size=page)
    table, total = _layout(starts, rows, page, rng)
    cu = np.concatenate([[0], np.cumsum(rows)])
    pool = _values(rng, 499, H, d, "bf16")                                            # the rows' contents repeat
    of = [torch.as_tensor(rng.integers(0, 499, size=n)) for _ in range(2)]
    wide = torch.full((n + pad, 3 * H * d), 7.0, dtype=torch.bfloat16)
    sides = [wide[:, i * H * d:(i + 1) * H * d].unflatten(1, (H, d)) for i in (0, 2)]
    for side, pick in zip(sides, of):
        side[:n] = pool[pick]
    wide = wide.cuda()
    k, v = (wide[:, i * H * d:(i + 1) * H * d].unflatten(1, (H, d)) for i in (0, 2))
    stored = torch.as_tensor(O.stored(pool.double().numpy(), fmt)).to(torch.bfloat16)
    want = [stored[pick] for pick in of]

    def go(table, cache):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        args = (_dev(table), _dev(cu), _dev(starts))
        dec.wf_cache_write(cache, *args, k, v, status=status)
        back = torch.full((n + pad, 3 * H * d), 9.0, dtype=torch.bfloat16, device="cuda")
        gk, gv = (back[:, i * H * d:(i + 1) * H * d].unflatten(1, (H, d)) for i in (1, 2))
        dec.wf_cache_read(cache, *args, n + pad, k=gk, v=gv, status=status)
        assert (back[:, :H * d] == 9).all() and (gk[n:] == 9).all() and (gv[n:] == 9).all()
        return gk[:n].cpu(), gv[:n].cpu(), int(status)

    cache = dec.cache(total)
    gk, gv, status = go(table, cache)
    assert status == 0 and torch.equal(gk, want[0]) and torch.equal(gv, want[1])
    # small calls (one head per group of lanes) write the same bytes
    other = dec.cache(total)
    for a in range(0, n, 1000):
        b = min(n, a + 1000)
        here = np.clip(cu, a, b) - a
        first = np.array(starts) + np.maximum(a - cu[:-1], 0)
        dec.wf_cache_write(other, _dev(table), _dev(here), _dev(first), k[a:b], v[a:b])
    for x, y in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), (other.k, other.v, other.k_scale, other.v_scale)):
        if x is not None:
            wrote = x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)
            assert torch.equal(wrote, y.view(wrote.dtype))
    # a page of the first sequence that is not the cache's: its rows stay as they were, on both sides
    bad = table.copy()
    bad[0, 2] = total
    gk, gv, status = go(bad, dec.cache(total))
    gone = torch.zeros(n, dtype=torch.bool)
    gone[2 * page - starts[0]:3 * page - starts[0]] = True
    assert status == STATUS_BAD_PAGE and (gk[gone] == 9).all() and (gv[gone] == 9).all()
    assert torch.equal(gk[~gone], want[0][~gone]) and torch.equal(gv[~gone], want[1][~gone])


# ---- selection: more blocks than SMs
def _select(logits, scores, keep, beams, finished, end, off):
    """O.beam_select for large vocabularies: every sequence's candidates sorted stably."""
    B, W = scores.shape
    V = logits.shape[-1]
    out = (np.full((B, keep), -np.inf), np.full((B, keep), -1, np.int64), np.full((B, keep), -1, np.int64), np.zeros((B, keep), np.int64))
    for b in range(B):
        c = np.full((W, V), -np.inf)
        for w in range(int(beams[b])):
            if finished[b, w]:
                c[w, end] = scores[b, w]
                continue
            x = np.where(off, -np.inf, logits[b, w])
            m = x.max()
            c[w] = scores[b, w] + (x - (m + np.log(np.exp(x - m).sum())))
        order = np.argsort(-c.reshape(-1), kind="stable")[:keep]
        for i, f in enumerate(order):
            w, t = divmod(int(f), V)
            if c[w, t] > -np.inf:
                out[0][b, i], out[1][b, i], out[2][b, i], out[3][b, i] = c[w, t], w, t, t == end or bool(finished[b, w])
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,W,V,keep", [(40, 5, 9001, 10), (64, 5, 20_011, 5), (160, 3, 2600, 6), (160, 5, 30_003, 10), (330, 2, 700, 4)])
def test_selections_with_more_blocks_than_sms(dtype, B, W, V, keep):
    rng = np.random.default_rng([B, V])
    dec = _decoder()
    logits = torch.as_tensor((3 * rng.normal(size=(B * W, V))).astype(np.float32)).to(dtype)
    scores = (-5 * rng.random((B, W))).astype(np.float32)
    beams = np.where(rng.random(B) < 0.3, rng.integers(0, W + 1, size=B), W)
    finished = rng.random((B, W)) < 0.15
    off = rng.random(V) < 0.02
    end = V - 1
    off[end] = False
    bits = np.zeros(-(-V // 32) * 32, bool)
    bits[:V] = off
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (logits.cuda(), _dev(scores, torch.float32), keep, _dev(beams), _dev(finished, torch.uint8), end,
            torch.from_numpy(np.packbits(bits, bitorder="little").view(np.int32)).cuda())
    got = dec.wf_beam_select(*args, status=status)
    assert int(status) == 0
    x = logits.double().numpy().reshape(B, W, V)
    want = _select(x, scores.astype(np.float64), keep, beams, finished, end, off)
    one = O.beam_select(x[:1], scores[:1].astype(np.float64), keep, beams[:1], finished[:1], end, off)
    assert np.allclose(want[0][0], one[0][0], atol=1e-12) and all(np.array_equal(a[0], b[0]) for a, b in zip(want[1:], one[1:]))
    s, fin = got[0].double().cpu().numpy(), np.isfinite(want[0])
    assert np.array_equal(fin, np.isfinite(s))
    # one rounding to float32 and the log-sum's float32 error, 2e-6 of the sum at most
    assert (np.abs(s[fin] - want[0][fin]) <= 2.0 ** -23 * np.abs(want[0][fin]) + 2e-6).all()
    # candidates nearer to a neighbour than twice that error may change places with it, the last one with the first that is left out;
    # equal logits of one beam have equal scores on both sides, and the lower token first
    gap = np.abs(np.diff(np.where(fin, want[0], -1e30), axis=1))
    near = (gap <= 5e-6) & ~((gap == 0) & (want[1][:, 1:] == want[1][:, :-1]))
    sure = np.ones_like(fin)
    sure[:, 1:] &= ~near
    sure[:, :-1] &= ~near
    sure[:, -1] = False
    assert sure[:, :-1].mean() > 0.9
    for g, w in zip(got[1:], want[1:]):
        assert np.array_equal(g.cpu().numpy()[sure], w[sure])
    again = dec.wf_beam_select(*args)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


# ---- 128-row tiles: magnitudes and scores far apart
@pytest.mark.parametrize("fmt", ["path", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [200, 2500])
def test_many_rows_with_vectors_of_very_different_sizes(fmt, d, T):
    """Values from 1e-30 to 1e30 and keys down to 1e-30 beside ordinary ones, in one split and in several."""
    rng = np.random.default_rng([d, T])
    dec = _decoder(n_head=2, n_kv_head=1, d_head=d, cache_format=fmt, page_size=64)
    k, v = (rng.normal(size=(T, 1, d)) for _ in range(2))
    v *= 10.0 ** rng.integers(-30, 30, size=(T, 1, 1))
    k[::3] *= 1e-30
    k, v = (torch.as_tensor(x.astype(np.float32)).to(torch.bfloat16) for x in (k, v))
    c = Case(rng, dec, rows=[50], starts=[T - 50], tail="causal", k=k, v=v)
    out, lse = c.run()
    wo, wl = c.want()
    assert np.abs(lse.cpu().double().numpy() - wl).max() <= 1e-4
    see = O.visible(T - 50, 50, "causal")
    ks, vs = (O.stored(x.double().numpy(), fmt) for x in (k, v))
    bound, _ = O.attend(c.q.double().numpy(), ks, np.abs(vs), see, d ** -0.5)
    # of the sum of p |v| of each row and channel: half a step, 2^-8, for the weight's rounding and as much for the output's; the float32 part
    # as in Case.check
    assert (np.abs(out.double().cpu().numpy() - wo) <= (2.0 ** -7 + 1e-4) * bound).all()


@pytest.mark.parametrize("fmt", ["path", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [400, 2500])
def test_many_rows_with_scores_that_keep_growing(fmt, d, T):
    """Rows whose largest score comes last, first or nowhere in particular, from -1e4 to 1e4: the reference is raised in every step, in none,
    or in some rows of a tile only."""
    rng = np.random.default_rng([d, T, 1])
    dec = _decoder(n_head=2, n_kv_head=2, d_head=d, cache_format=fmt, page_size=32)
    k = torch.zeros(T, 2, d)
    # within a bfloat16 step of one another where unquantised, whole numbers where codes are to be exact
    k[:, :, 0] = torch.linspace(-100, 100, T)[:, None] if fmt == "path" else (torch.arange(T)[:, None] * 97 // T - 48.0)
    k[:, :, 1] = torch.as_tensor(rng.integers(-8, 9, size=(T, 2)).astype(np.float32))
    k = k.to(torch.bfloat16)
    v = torch.as_tensor(rng.normal(size=(T, 2, d)).astype(np.float32)).to(torch.bfloat16)
    rows = 70
    c = Case(rng, dec, rows=[rows], starts=[T - rows], tail="causal", k=k, v=v)
    c.q = torch.zeros(rows, 2, d)
    c.q[:, :, 0] = torch.as_tensor(rng.choice([800.0, -800.0, 8.0, -8.0, 0.5, 0.0, 100.0, -100.0], size=(rows, 2)).astype(np.float32))
    c.q[:, :, 1] = torch.as_tensor(rng.choice([0.0, 1.0, -2.0], size=(rows, 2)).astype(np.float32))
    c.q = c.q.to(torch.bfloat16)
    (out, lse), (wo, wl) = c.run(), c.want()
    # scores of up to 1e4: their float32 roundings (the products are exact, 2^-22 of the value covers the scale and log2(e)) move lse, and the
    # weights by the same relative amount: 1e4 2^-22 = 2.4e-3
    lse_tol = 1e-4 + 2.0 ** -22 * np.abs(wl)
    assert (np.abs(lse.cpu().double().numpy() - wl) <= lse_tol).all()
    assert (np.abs(out.double().cpu().numpy() - wo) <= (2.0 ** -7 + 1e-4 + 2 * lse_tol[..., None]) * float(v.abs().max())).all()


@pytest.mark.parametrize("dtype,fmt,d,H,Hk", [("bf16", "e4m3", 64, 3, 1), ("bf16", "path", 128, 2, 2), ("f32", "int8", 64, 2, 1), ("f32", "path", 128, 1, 1)])
def test_prompts_of_thousands_of_rows(dtype, fmt, d, H, Hk):
    """A long causal prompt behind a committed prefix, beside a single token and a short prompt: many row tiles of one sequence, none of others."""
    rng = np.random.default_rng([d, H])
    dec = _decoder(n_head=H, n_kv_head=Hk, d_head=d, dtype=dtype, cache_format=fmt, page_size=256)
    c = Batch(rng, dec, [2111, 1, 37], [45, 900, 0], "causal", 1)
    got = c.run()
    c.check(got, c.want())
    again = c.run()
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
