"""wf_tree_attention against the fp64 oracle: formats, head layouts, trees, lengths around the tile, page and split borders,
empty rows, values that must not leak, and its refusals."""
import ctypes as C

import numpy as np
import pytest

from oracle import decode_oracle as O

torch = pytest.importorskip("torch")


def _decoder(**kw):
    from paper_2412_11272_b200.binding import Decoder
    return Decoder(**{**dict(n_head=4, d_head=64, dtype="bf16", cache_format="e4m3", page_size=16), **kw})


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda:0", dtype)


# ---- refusals (no GPU is needed)
def test_refusals_at_the_c_entry():
    from paper_2412_11272_b200 import binding as Bn
    d = _decoder()
    P = 1 << 20
    base = dict(h=d.handle, cache=Bn.wf_cache(P, P, P, P, 3), rows=Bn.wf_rows(2, 8, P, P, P, 4), q=P, qs=256, scale=0.125, tail=1, mask=None,
                words=0, max_rows=4, max_len=64, out=P, os=256, lse=None, ws=None, wsb=0, status=None, stream=None)

    def call(**kw):
        a = {**base, **kw}
        return d.lib.wf_tree_attention(*(a[k] for k in base))

    nan, inf = float("nan"), float("inf")
    for bad in (dict(h=None), dict(cache=None), dict(rows=None), dict(cache=Bn.wf_cache(P, P, None, None, 3)), dict(cache=Bn.wf_cache(P, P + 8, P, P, 3)),
                dict(rows=Bn.wf_rows(2, 8, None, P, P, 4)), dict(q=None), dict(out=None), dict(q=P + 2), dict(out=P + 8), dict(qs=252), dict(qs=248),
                dict(os=260), dict(tail=3), dict(tail=-1), dict(tail=2), dict(tail=2, mask=P, words=0), dict(tail=2, mask=P, words=1, max_rows=33),
                dict(scale=nan), dict(scale=inf), dict(max_rows=-1), dict(max_len=-1), dict(max_len=65)):
        assert call(**bad) == 1, bad
    assert call(max_rows=70000) == 4 and call(rows=Bn.wf_rows(65536, 8, P, P, P, 4)) == 4
    assert call(max_rows=0) == 0 and call(rows=Bn.wf_rows(0, 8, None, None, None, 0)) == 0 and call(rows=Bn.wf_rows(2, 0, None, None, None, 0)) == 0
    n = C.c_size_t(5)
    assert d.lib.wf_tree_attention_workspace(d.handle, 0, 0, 0, 0, C.byref(n)) == 0 and n.value == 0
    assert d.lib.wf_tree_attention_workspace(d.handle, -1, 0, 0, 0, C.byref(n)) == 1
    assert d.lib.wf_tree_attention_workspace(d.handle, 1, 1, 1, 1, None) == 1
    assert d.lib.wf_tree_attention_workspace(None, 1, 1, 1, 1, C.byref(n)) == 1


def test_oracle_attention_pins():
    k = np.ones((5, 1, 4))
    v = np.arange(20.0).reshape(5, 1, 4)
    out, lse = O.attend(np.ones((2, 2, 4)), k, v, O.visible(3, 2, "causal"), 0.5)
    assert np.allclose(out[0, 1], v[:4, 0].mean(0)) and np.allclose(out[1, 0], v[:, 0].mean(0))       # identical keys: the mean
    assert np.allclose(lse[0], 2 + np.log(4)) and np.allclose(lse[1], 2 + np.log(5))
    see = O.visible(0, 3, "mask", np.array([[1, 0, 0], [0, 0, 0], [1, 0, 1]], bool))
    out, lse = O.attend(np.ones((3, 1, 4)), k[:3], v[:3], see, 0.5)
    assert np.allclose(out[0, 0], v[0, 0]) and (out[1] == 0).all() and lse[1, 0] == -np.inf and np.allclose(out[2, 0], (v[0, 0] + v[2, 0]) / 2)


# ---- on the GPU
def _random_tree(n, rng):
    bits = np.zeros((n, n), bool)
    for i in range(n):
        parent = int(rng.integers(-1, i)) if i else -1
        if parent >= 0:
            bits[i] = bits[parent]
        bits[i, i] = True
    return bits


def _pack(bits, words):
    n = len(bits)
    full = np.zeros((n, words * 32), bool)
    full[:, :bits.shape[1]] = bits
    return np.packbits(full, axis=1, bitorder="little").view(np.uint32).view(np.int32)


class Case:
    """A batch in a cache that the library wrote, and the oracle's answer from the same stored values."""

    def __init__(self, rng, dec, rows, starts, tail, bits=None, peaked=1.5, pad=0, k=None, v=None):
        self.dec, self.rows, self.starts, self.tail = dec, rows, starts, tail
        H, Hk, d, page = dec.n_head, dec.n_kv_head, dec.d_head, dec.page_size
        self.n, self.pad = sum(rows), pad
        total = [s + (n if tail != "none" else 0) for s, n in zip(starts, rows)]
        each = [-(-t // page) for t in total]
        n_pages = sum(each) + 3
        order = rng.permutation(n_pages)
        self.table = np.full((len(rows), max(max(each), 1)), 10 ** 6, np.int32)      # entries behind the last page lead nowhere
        at = 0
        for i, e in enumerate(each):
            self.table[i, :e] = order[at:at + e]
            at += e
        self.cu = np.concatenate([[0], np.cumsum(rows)])
        self.max_len = max(max(total), 1)

        def data(*shape, size=1.0):
            return torch.as_tensor((size * rng.normal(size=shape)).astype(np.float32)).to(dec.torch_dtype)

        T = sum(total)
        self.cache = dec.cache(n_pages)
        for t in (self.cache.k, self.cache.v):                                        # what nobody wrote is NaN
            t.view(torch.uint8).fill_(0xFF)
        for s in (self.cache.k_scale, self.cache.v_scale):
            if s is not None:
                s.fill_(float("nan"))
        k = data(max(T, 1), Hk, d)[:T] if k is None else k
        v = (data(max(T, 1), Hk, d)[:T].float() * torch.exp(0.7 * torch.as_tensor(rng.normal(size=(1, Hk, d)).astype(np.float32)))).to(dec.torch_dtype) if v is None else v
        self.k, self.v = k, v
        if T:
            args = (self.cache, _dev(self.table), _dev(np.concatenate([[0], np.cumsum(total)])), _dev(np.zeros(len(rows))), k.cuda(), v.cuda())
            dec.wf_cache_write(*args)
        self.first = np.concatenate([[0], np.cumsum(total)])
        self.q = data(self.n + pad, H, d, size=peaked)
        self.words = -(-max(max(rows), 1) // 32)
        self.bits = bits if bits is not None else [_random_tree(n, rng) for n in rows]
        self.mask = np.concatenate([_pack(b, self.words) if n else np.zeros((0, self.words), np.int32) for b, n in zip(self.bits, rows)]
                                   + [np.full((pad, self.words), -1, np.int32)])

    def run(self, **kw):
        d = self.dec
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kw = {**dict(max_rows=max(max(self.rows), 1), max_len=self.max_len, tail=self.tail, mask=_dev(self.mask) if self.tail == "mask" else None,
                     status=status), **kw}
        out = d.wf_tree_attention(self.cache, _dev(self.table), _dev(self.cu), _dev(self.starts), self.q.cuda(), **kw)
        assert int(kw["status"]) == 0
        return out

    def want(self):
        d = self.dec
        out, lse = np.zeros((self.n, d.n_head, d.d_head)), np.full((self.n, d.n_head), -np.inf)
        for s, n in enumerate(self.rows):
            at, to = self.first[s], self.first[s + 1]
            if n == 0:
                continue
            k, v = (O.stored(x[at:to].double().numpy(), d.cache_format) for x in (self.k, self.v))
            see = O.visible(self.starts[s], n, self.tail, self.bits[s])
            out[self.cu[s]:self.cu[s + 1]], lse[self.cu[s]:self.cu[s + 1]] = O.attend(
                self.q[self.cu[s]:self.cu[s + 1]].double().numpy(), k, v, see, d.d_head ** -0.5)
        return out, lse

    def check(self, got, want):
        """Tolerances.  Every output is a mean of values with weights p: an error of relative size e in every weight moves it by at
        most e times the sum of p |v|, so errors are counted against B = max |v| of the sequence.
        float32: scores are sums of d products (relative 2^-24 each step, |q||k| scale <= 60 here): absolute error under
        60 d 2^-24 / 8 in a score (random signs; 5e-5 for d = 128), the same relative error in p; sums and products add less.
        bf16: bfloat16 has 8 significant bits, half a step is at most eps / 2 = 2^-8 of the value (the step of [1, 2) is 2^-7).  The
        weight is rounded once (2^-8 B at most) and the output once (2^-8 |o|, |o| <= B): 2^-7 B + the float32 part.  lse is never
        rounded to 16 bits: the score's error alone."""
        (out, lse), (wo, wl) = got, want
        out, lse = out[:self.n].double().cpu().numpy(), lse[:self.n].double().cpu().numpy()
        assert np.array_equal(np.isneginf(lse), np.isneginf(wl)), "empty rows"
        fin = ~np.isneginf(wl)
        assert (out[~fin] == 0).all()
        if fin.any():
            assert np.abs(lse[fin] - wl[fin]).max() <= 1e-4
        B = float(self.v.double().abs().max()) if len(self.v) else 1.0
        tol = (2.0 ** -7 + 1e-4) * B if self.dec.dtype == "bf16" else 1e-4 * B
        assert np.abs(out - wo).max() <= tol
        # on the whole the rounding is smaller: uniform within half a step, 2^-8 / sqrt(3) in the root mean square, for the output and for the
        # weights (where few carry the sum): together at most 2^-8 sqrt(2 / 3)
        if fin.any():
            rel = np.linalg.norm(out - wo) / np.linalg.norm(wo)
            assert rel <= (2.0 ** -8 if self.dec.dtype == "bf16" else 2e-5)


_FORMATS = [("bf16", "path"), ("bf16", "e4m3"), ("bf16", "int8"), ("f32", "path"), ("f32", "e4m3"), ("f32", "int8")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt", _FORMATS)
@pytest.mark.parametrize("H,Hk,d,page", [(4, 4, 64, 16), (8, 2, 128, 64), (5, 1, 64, 256), (6, 6, 128, 32)])
@pytest.mark.parametrize("tail", ["none", "causal", "mask"])
def test_formats_heads_and_tails(dtype, fmt, H, Hk, d, page, tail):
    rng = np.random.default_rng([H, d, page, len(tail)])
    dec = _decoder(n_head=H, n_kv_head=Hk, d_head=d, dtype=dtype, cache_format=fmt, page_size=page)
    c = Case(rng, dec, rows=[1, 5, 0, 9, 2, 17], starts=[0, 3, 7, 130, 64, 300], tail=tail, pad=2)
    c.check(c.run(), c.want())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["path", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_around_every_border(dtype, fmt):
    rng = np.random.default_rng(11)
    starts = sorted({0, 1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 95, 96, 127, 128, 129, 191, 255, 256, 257, 300, 511, 512, 513})
    dec = _decoder(n_head=2, dtype=dtype, cache_format=fmt, page_size=32)
    for tail in ("none", "causal"):
        c = Case(rng, dec, rows=[1 + i % 3 for i in range(len(starts))], starts=starts, tail=tail)
        c.check(c.run(), c.want())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt", _FORMATS)
@pytest.mark.parametrize("n", [8, 9, 16, 31, 32, 33, 48, 64, 65, 100, 200])
def test_big_trees(dtype, fmt, n):
    rng = np.random.default_rng(n)
    for H, Hk, d in ((2, 2, 64), (4, 1, 128)):
        dec = _decoder(n_head=H, n_kv_head=Hk, d_head=d, dtype=dtype, cache_format=fmt, page_size=64)
        c = Case(rng, dec, rows=[n, 3, max(1, n - 1)], starts=[70, 0, 190], tail="mask")
        c.check(c.run(), c.want())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt", _FORMATS)
def test_long_histories_are_split_and_joined(dtype, fmt):
    rng = np.random.default_rng(5)
    dec = _decoder(n_head=4, n_kv_head=2, d_head=64, dtype=dtype, cache_format=fmt, page_size=128)
    c = Case(rng, dec, rows=[2, 1], starts=[9001, 4], tail="causal", peaked=2.0)
    assert dec.tree_attention_workspace(2, 3, 2, c.max_len) > 0
    got, want = c.run(), c.want()
    c.check(got, want)
    # the same from a workspace full of NaN, and bit for bit
    ws = torch.full((dec.tree_attention_workspace(2, 3, 2, c.max_len) // 4,), float("nan"), device="cuda").view(torch.uint8)
    again = c.run(workspace=ws)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt", _FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_masks_that_leave_rows_empty(dtype, fmt, d):
    rng = np.random.default_rng(6)
    dec = _decoder(n_head=2, d_head=d, dtype=dtype, cache_format=fmt)
    bits = [np.zeros((4, 4), bool), np.eye(3, dtype=bool), np.zeros((2, 2), bool), np.zeros((40, 40), bool)]
    bits[0][2, 1] = True
    bits[3][39, 0] = bits[3][1, 39] = True
    c = Case(rng, dec, rows=[4, 3, 2, 40], starts=[0, 0, 20, 0], tail="mask", bits=bits)
    c.check(c.run(), c.want())
    c = Case(rng, dec, rows=[2, 1], starts=[0, 0], tail="none")
    out, lse = c.run()
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt", _FORMATS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("d,n", [(64, 5), (128, 5), (64, 40), (128, 70)])
def test_what_a_row_does_not_see_cannot_reach_it(dtype, fmt, bad, d, n):
    """One drafted token has keys and values that are not finite: rows that see it are not finite, the others are untouched."""
    rng = np.random.default_rng(7)
    dec = _decoder(n_head=2, d_head=d, dtype=dtype, cache_format=fmt)
    rows, starts = [n, n, 2], [33, 0, 50]
    T = sum(rows) + sum(starts)
    k, v = (torch.as_tensor(rng.normal(size=(T, 2, d)).astype(np.float32)).to(dec.torch_dtype) for _ in range(2))
    c = Case(rng, dec, rows=rows, starts=starts, tail="mask", k=k, v=v)
    want = c.run()
    kb, vb = k.clone(), v.clone()
    hit = [2, n - 1]
    for s in range(2):
        at = c.first[s] + starts[s] + hit[s]
        kb[at], vb[at] = bad, bad
    args = (c.cache, _dev(c.table), _dev(c.first), _dev(np.zeros(3)), kb.cuda(), vb.cuda())
    dec.wf_cache_write(*args)
    got = c.run()
    sees = np.zeros(c.n, bool)
    for s in range(2):
        sees[c.cu[s]:c.cu[s + 1]] = c.bits[s][:, hit[s]]
    sees = torch.as_tensor(sees).cuda()
    assert sees.any() and (~sees).any()
    assert torch.equal(got[0][~sees], want[0][~sees]) and torch.equal(got[1][~sees], want[1][~sees])
    assert not torch.isfinite(got[0][sees]).all(-1).any()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["path", "e4m3", "int8"])
@pytest.mark.parametrize("where", ["keys", "values"])
def test_vectors_of_very_different_sizes(fmt, where):
    """Magnitudes from 1e-30 to 1e30 among one sequence's vectors: no scale drowns another one's."""
    rng = np.random.default_rng(9)
    dec = _decoder(n_head=1, cache_format=fmt)
    T = 200
    k, v = (rng.normal(size=(T, 1, 64)) for _ in range(2))
    if where == "values":
        v *= 10.0 ** rng.integers(-30, 30, size=(T, 1, 1))
        k[:, 0] *= 3
    else:
        k[::3] *= 1e-30
    k, v = (torch.as_tensor(x.astype(np.float32)).to(torch.bfloat16) for x in (k, v))
    c = Case(rng, dec, rows=[3], starts=[T - 3], tail="causal", k=k, v=v)
    out, lse = c.run()
    wo, wl = c.want()
    assert np.abs(lse.cpu().double().numpy() - wl).max() <= 1e-4
    # against the sum of p |v| of each row and channel: half a step, 2^-8, for the weight's rounding and as much for the output's
    see = O.visible(T - 3, 3, "causal")
    ks, vs = (O.stored(x.double().numpy(), fmt) for x in (k, v))
    bound, _ = O.attend(c.q.double().numpy(), ks, np.abs(vs), see, 0.125)
    assert (np.abs(out.double().cpu().numpy() - wo) <= (2.0 ** -7 + 1e-4) * bound).all()
    # a large value that a row gives almost no weight must not drown the rest: one key far below the others
    if where == "values":
        k2, v2 = torch.zeros(T, 1, 64, dtype=torch.bfloat16), torch.ones(T, 1, 64, dtype=torch.bfloat16)
        k2[:, 0, 0] = 8.0
        k2[5, 0, 0], v2[5] = -80.0, 1e20
        c = Case(rng, dec, rows=[1], starts=[T - 1], tail="causal", k=k2, v=v2)
        c.q = torch.zeros(1, 1, 64, dtype=torch.bfloat16)
        c.q[0, 0, 0] = 10.0
        out, _ = c.run()                                         # weight of key 5: exp(-110) = 2e-48, times 1e20 is nothing
        assert (out.float() - 1).abs().max() <= 2.0 ** -7       # half a step for the weights (all alike), half a step for the output


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt", _FORMATS)
def test_scores_of_any_size(dtype, fmt):
    """Scores from -1e4 to 1e4: the running maximum carries them."""
    rng = np.random.default_rng(10)
    dec = _decoder(n_head=2, d_head=64, dtype=dtype, cache_format=fmt)
    k = torch.zeros(700, 2, 64)
    k[:, :, 0] = torch.linspace(-100, 100, 700)[:, None] if fmt == "path" else torch.arange(700)[:, None].remainder(97) - 48.0
    k = k.to(dec.torch_dtype)
    v = torch.as_tensor(rng.normal(size=(700, 2, 64)).astype(np.float32)).to(dec.torch_dtype)
    c = Case(rng, dec, rows=[4], starts=[696], tail="causal", k=k, v=v)
    c.q = torch.zeros(4, 2, 64).to(dec.torch_dtype)
    c.q[:, :, 0] = torch.tensor([800.0, -800.0, 8.0, -0.5])[:, None].to(dec.torch_dtype)
    (out, lse), (wo, wl) = c.run(), c.want()
    assert (np.abs(lse.cpu().double().numpy() - wl) <= 1e-4 + 2.0 ** -22 * np.abs(wl)).all()
    assert np.abs(out.cpu().double().numpy() - wo).max() <= (2.0 ** -7 if dtype == "bf16" else 1e-2) * float(v.abs().max())


@pytest.mark.gpu
def test_rows_behind_the_batch_strides_and_given_buffers():
    rng = np.random.default_rng(12)
    dec = _decoder(n_head=4, n_kv_head=2, cache_format="int8")
    c = Case(rng, dec, rows=[3, 6], starts=[10, 40], tail="mask", pad=5)
    want = c.want()
    n = c.n + c.pad
    wide = torch.full((n, 3 * 256), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 256:512] = c.q.cuda().reshape(n, 256)
    out = torch.full((n, 2 * 256), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, 4), 2.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dec.wf_tree_attention(c.cache, _dev(c.table), _dev(c.cu), _dev(c.starts), wide[:, 256:512].unflatten(1, (4, 64)), 6, c.max_len, "mask",
                          _dev(c.mask), out=out[:, 256:].unflatten(1, (4, 64)), lse=lse, status=status)
    assert int(status) == 0
    c.check((out[:, 256:].unflatten(1, (4, 64)), lse), want)
    assert (out[:, :256] == 3).all() and (out[c.n:] == 3).all() and (lse[c.n:] == 2).all()
    # generous bounds give the same answer up to the order of the sums
    loose = c.run(max_rows=30, max_len=c.table.shape[1] * 16)
    c.check(loose, want)
    scaled = c.run(scale=0.01)
    assert not torch.equal(scaled[0], loose[0])


@pytest.mark.gpu
def test_bad_device_data_is_passed_over_and_reported():
    from paper_2412_11272_b200.binding import STATUS_BAD_PAGE, STATUS_BAD_ROWS
    rng = np.random.default_rng(13)
    for fmt, dtype in (("path", "bf16"), ("e4m3", "bf16"), ("path", "f32")):
        dec = _decoder(n_head=2, cache_format=fmt, dtype=dtype)
        c = Case(rng, dec, rows=[2, 2], starts=[30, 14], tail="causal")
        good = c.run()

        def run(table=c.table, cu=c.cu, starts=c.starts, **kw):
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            o, _ = dec.wf_tree_attention(c.cache, _dev(table), _dev(cu), _dev(starts), c.q.cuda(), status=status,
                                         out=torch.zeros(c.n, 2, 64, dtype=dec.torch_dtype, device="cuda"), **{**dict(max_rows=2, max_len=c.max_len), **kw})
            return o, int(status)

        for page in (-1, c.cache.shape[0], 2 ** 31 - 1, -2 ** 31):
            t = c.table.copy()
            t[0, 1] = page                                        # positions 16 .. 31 are absent
            o, st = run(table=t)
            assert st == STATUS_BAD_PAGE and torch.equal(o[2:], good[0][2:]) and torch.isfinite(o).all()
            at, to = c.first[0], c.first[1]
            see = O.visible(30, 2, "causal")
            see[:, 16:32] = False
            k, v = (O.stored(x[at:to].double().numpy(), fmt) for x in (c.k, c.v))
            w, _ = O.attend(c.q[:2].double().numpy(), k, v, see, 0.125)
            assert np.abs(o[:2].double().cpu().numpy() - w).max() <= 2.0 ** -7 * np.abs(v).max()
        assert run(cu=[0, 2, 9])[1] == STATUS_BAD_ROWS and run(cu=[0, -2, 4])[1] & STATUS_BAD_ROWS
        assert run(starts=[-1, 14])[1] == STATUS_BAD_ROWS and run(starts=[2 ** 31 - 1, 14])[1] & STATUS_BAD_ROWS
        o, st = run(max_rows=1)                                    # the sequences' second rows are not computed
        assert st == STATUS_BAD_ROWS and (o[1] == 0).all() and (o[3] == 0).all() and (o[0] != 0).any()
        o, st = run(max_len=20)                                    # the first sequence is cut, the second is whole
        assert st == STATUS_BAD_ROWS and torch.isfinite(o).all()


@pytest.mark.gpu
def test_captured_replayed_and_on_another_stream():
    """A captured write and attention, replayed with other contents in the same buffers; two graphs share nothing."""
    rng = np.random.default_rng(14)
    dec = _decoder(n_head=4, cache_format="e4m3", page_size=64)
    c = Case(rng, dec, rows=[2, 3], starts=[3000, 17], tail="mask")
    table, cu, starts, mask, q = _dev(c.table), _dev(c.cu), _dev(c.starts), _dev(c.mask), c.q.cuda()
    kw = dict(max_rows=3, max_len=c.max_len, tail="mask", mask=mask)
    eager = dec.wf_tree_attention(c.cache, table, cu, starts, q, **kw)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = dec.wf_tree_attention(c.cache, table, cu, starts, q, **kw)
        graphs.append((g, o))
    for g, _ in graphs:
        g.replay()
    torch.cuda.synchronize()
    for _, o in graphs:
        assert torch.equal(o[0], eager[0]) and torch.equal(o[1], eager[1])
    q2 = torch.randn_like(q)
    q.copy_(q2)
    starts.copy_(_dev([1500, 9]))
    graphs[0][0].replay()
    again = dec.wf_tree_attention(c.cache, table, cu, starts, q, **kw)
    assert torch.equal(graphs[0][1][0], again[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = dec.wf_tree_attention(c.cache, table, cu, starts, q, **kw)
    third = dec.wf_tree_attention(c.cache, table, cu, starts, q, **kw, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(other[0], again[0]) and torch.equal(third[0], again[0])


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """A cache of more than 2^31 elements a side: positions in its last pages are found."""
    dec = _decoder(n_head=1, d_head=128, dtype="bf16", cache_format="path", page_size=256)
    pages = (1 << 31) // (256 * 128) + 5
    cache = dec.cache(pages)
    table = torch.arange(pages - 1, pages - 4, -1, dtype=torch.int32, device="cuda")[None]
    k = torch.randn(700, 1, 128, device="cuda").bfloat16()
    cu, zero = _dev([0, 700]), _dev([0])
    dec.wf_cache_write(cache, table, cu, zero, k, k)
    back, _ = dec.wf_cache_read(cache, table, cu, zero, 700)
    assert torch.equal(back, k) and torch.equal(cache.k[-1, 0], k[:256, 0])
    q = torch.randn(1, 1, 128, device="cuda").bfloat16()
    out, _ = dec.wf_tree_attention(cache, table, _dev([0, 1]), _dev([700]), q, 1, 700, tail="none")
    p = torch.softmax((k[:, 0].double() @ q[0, 0].double()) * 128 ** -0.5, 0)
    assert (out[0, 0].double() - p @ k[:, 0].double()).abs().max() <= (2.0 ** -7 + 1e-4) * float(k.abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt", _FORMATS)
@pytest.mark.parametrize("n,H,Hk,d", [(1, 3, 3, 64), (9, 4, 2, 128), (40, 2, 1, 128), (70, 2, 2, 64)])
def test_repeated_calls_agree_bit_for_bit(dtype, fmt, n, H, Hk, d):
    """No result depends on the order in which blocks run: twenty calls in a row, with other work between, give the same bits."""
    rng = np.random.default_rng([n, H, d])
    dec = _decoder(n_head=H, n_kv_head=Hk, d_head=d, dtype=dtype, cache_format=fmt, page_size=32)
    c = Case(rng, dec, rows=[n, 1, max(1, n // 2)] * 6, starts=[700, 5, 1300] * 6, tail="mask")
    table, cu, starts, mask, q = _dev(c.table), _dev(c.cu), _dev(c.starts), _dev(c.mask), c.q.cuda()
    first = None
    for _ in range(20):
        got = dec.wf_tree_attention(c.cache, table, cu, starts, q, n, c.max_len, "mask", mask)
        if first is None:
            first = got
            c.check(got, c.want())
        assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 40])
def test_calls_on_a_given_stream_keep_their_workspace(n):
    """Calls on a side stream with workspaces of their own, while the current stream allocates and overwrites memory."""
    rng = np.random.default_rng(15)
    dec = _decoder(n_head=4, cache_format="int8", page_size=64)
    c = Case(rng, dec, rows=[n, 1], starts=[4000, 17], tail="causal")
    table, cu, starts, q = _dev(c.table), _dev(c.cu), _dev(c.starts), c.q.cuda()
    need = dec.tree_attention_workspace(2, n + 1, n, c.max_len)
    assert need > 0
    want = dec.wf_tree_attention(c.cache, table, cu, starts, q, n, c.max_len, "causal")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(50):
        got = dec.wf_tree_attention(c.cache, table, cu, starts, q, n, c.max_len, "causal", stream=side)
        junk = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]   # on the current stream
        del junk
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
def test_prompts_of_many_rows():
    """A prompt as a call of its own: hundreds of causal rows of ragged sequences, several row tiles."""
    rng = np.random.default_rng(16)
    for fmt, H, Hk, d in (("e4m3", 2, 1, 64), ("path", 2, 2, 128), ("int8", 1, 1, 128)):
        dec = _decoder(n_head=H, n_kv_head=Hk, d_head=d, cache_format=fmt, page_size=128)
        c = Case(rng, dec, rows=[300, 1, 129, 0, 64], starts=[0, 200, 33, 5, 500], tail="causal")
        c.check(c.run(), c.want())
