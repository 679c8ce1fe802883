"""The paged, quantised cache (wf_cache_write / wf_cache_read) and wf_beam_reorder against the oracle, and their refusals."""
import ctypes as C

import numpy as np
import pytest

from oracle import decode_oracle as O

torch = pytest.importorskip("torch")


def _decoder(**kw):
    from paper_2412_11272_b200.binding import Decoder
    return Decoder(**{**dict(n_head=4, d_head=64, dtype="bf16", cache_format="e4m3", page_size=16), **kw})


# ---- the oracle's own number formats (hand-worked)
def test_oracle_e4m3_rounding_pins():
    x = np.array([448.0, 1.0, 1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, -1.06, 0.0])
    # 1.0625 is half way between 1 and 1.125 (even code: 1); 1.1875 between 1.125 and 1.25 (even: 1.25)
    assert O.round_e4m3(x).tolist() == [448.0, 1.0, 1.0, 1.25, 2.0 ** -9, 0.0, 2.0 ** -8, -1.0, 0.0]


def test_oracle_scales():
    for a, s in ((448.0, 1.0), (449.0, 2.0), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7), (2.0 ** -140, 2.0 ** -126)):
        assert O.quantise(np.array([[a, 0.0]]), "e4m3")[1][0] == s
    codes, s = O.quantise(np.array([[127.0, -63.5, 0.5, 1.5]]), "int8")
    assert s[0] == 1.0 and codes[0].tolist() == [127.0, -64.0, 0.0, 2.0]
    assert O.quantise(np.array([[0.0, 0.0]]), "int8")[1][0] == 1.0


# ---- refusals (no GPU is needed: they come before any launch)
def _status(fn, *args):
    return {0: "ok", 1: "invalid", 4: "capacity"}.get(fn(*args))


def test_decoder_create_refusals():
    from paper_2412_11272_b200.binding import WfError
    for bad in (dict(n_head=0), dict(n_head=6, n_kv_head=4), dict(d_head=80), dict(page_size=24), dict(page_size=8), dict(page_size=512),
                dict(dtype="f16"), dict(cache_format="int4"), dict(n_head=2048)):
        with pytest.raises(WfError) as e:
            _decoder(**bad)
        assert e.value.status == "WF_ERR_INVALID_ARG"


def test_cache_and_reorder_refusals_at_the_c_entry():
    from paper_2412_11272_b200 import binding as Bn
    d = _decoder()
    lib, h = d.lib, d.handle
    p = C.c_void_p(1 << 20)                                     # never dereferenced: every call below is refused (or has no work)
    cache = Bn.wf_cache(1 << 20, 1 << 20, 1 << 20, 1 << 20, 3)
    rows = Bn.wf_rows(2, 8, 1 << 20, 1 << 20, 1 << 20, 4)
    ok = (h, cache, rows, p, 256, p, 256, None, None)

    def call(i, value, fn=lib.wf_cache_write):
        a = list(ok)
        a[i] = value
        return _status(fn, *a)

    assert call(0, None) == "invalid"
    for fn in (lib.wf_cache_write, lib.wf_cache_read):
        for i, bad in ((1, Bn.wf_cache(None, 1 << 20, 1 << 20, 1 << 20, 3)), (1, Bn.wf_cache(1 << 20, 1 << 20, None, 1 << 20, 3)),
                       (1, Bn.wf_cache(1 << 20, 1 << 20, 1 << 20, 1 << 20, 0)), (1, Bn.wf_cache((1 << 20) + 8, 1 << 20, 1 << 20, 1 << 20, 3)),
                       (1, Bn.wf_cache(1 << 20, 1 << 20, 1 << 20, (1 << 20) + 4, 3)), (1, None), (2, None),
                       (2, Bn.wf_rows(-1, 8, 1 << 20, 1 << 20, 1 << 20, 4)), (2, Bn.wf_rows(2, -8, 1 << 20, 1 << 20, 1 << 20, 4)),
                       (2, Bn.wf_rows(2, 8, None, 1 << 20, 1 << 20, 4)), (2, Bn.wf_rows(2, 8, 1 << 20, None, 1 << 20, 4)),
                       (2, Bn.wf_rows(2, 8, 1 << 20, 1 << 20, None, 4)), (2, Bn.wf_rows(2, 8, 1 << 20, 1 << 20, 1 << 20, 0)),
                       (3, None), (5, None), (3, C.c_void_p((1 << 20) + 2)), (4, 252), (4, 248), (6, 260), (4, 0)):
            assert call(i, bad, fn) == "invalid", (i, bad)
        assert call(2, Bn.wf_rows(2, (1 << 27) + 1, 1 << 20, 1 << 20, 1 << 20, 4), fn) == "capacity"
        assert call(2, Bn.wf_rows(0, 8, None, None, None, 0), fn) == "ok"      # no sequences: nothing to do
        assert call(2, Bn.wf_rows(2, 0, None, None, None, 0), fn) == "ok"
    assert b"row stride" in lib.wf_decoder_last_error(h) or lib.wf_decoder_last_error(h)

    st = (Bn.wf_beam_state * 1)(Bn.wf_beam_state(1 << 20, 64, 64))
    ca = (Bn.wf_cache * 2)(cache, Bn.wf_cache(1 << 20, 1 << 20, 1 << 20, 1 << 20, 4))

    def reorder(parents=p, B=2, W=4, states=st, ns=1, caches=ca, nc=1, table=p, stride=4, lengths=p):
        return _status(lib.wf_beam_reorder, h, parents, B, W, states, ns, caches, nc, table, stride, lengths, None, None)

    assert reorder(parents=None) == "invalid" and reorder(B=-1) == "invalid" and reorder(W=0) == "invalid" and reorder(W=17) == "invalid"
    assert reorder(B=65536) == "capacity" and reorder(states=None) == "invalid" and reorder(ns=-1) == "invalid"
    assert reorder(caches=None) == "invalid" and reorder(table=None) == "invalid" and reorder(lengths=None) == "invalid" and reorder(stride=0) == "invalid"
    assert reorder(nc=2) == "invalid"                           # different numbers of pages
    assert reorder(states=(Bn.wf_beam_state * 1)(Bn.wf_beam_state(1 << 20, 64, 32))) == "invalid"
    assert reorder(states=(Bn.wf_beam_state * 1)(Bn.wf_beam_state(None, 64, 64))) == "invalid"
    assert reorder(states=(Bn.wf_beam_state * 1)(Bn.wf_beam_state(1 << 20, -1, 64))) == "invalid"
    assert reorder(B=0) == "ok" and reorder(W=1) == "ok"


def test_binding_refuses_host_tensors_and_wrong_shapes():
    from paper_2412_11272_b200.binding import KvCache, WfError
    d = _decoder()
    pages = torch.zeros(3, 4, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale = torch.ones(3, 4, 16, dtype=torch.bfloat16)
    i32 = torch.zeros(2, dtype=torch.int32)
    k = torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    for make in (lambda: KvCache(pages, pages[:2]), lambda: KvCache(pages, pages, scale), lambda: KvCache(pages, pages, scale, scale[:2]),
                 lambda: KvCache(pages, pages, scale.float(), scale.float()), lambda: KvCache(pages.transpose(1, 2), pages.transpose(1, 2)),
                 lambda: d.wf_cache_write(KvCache(pages, pages, scale, scale), i32[None], i32, i32, k, k),          # host memory
                 lambda: d.wf_cache_write(KvCache(pages, pages), i32[None], i32, i32, k, k),                        # no scales
                 lambda: d.wf_cache_read(KvCache(scale.new_zeros(3, 4, 16, 64), scale.new_zeros(3, 4, 16, 64)), i32[None], i32, i32, 1),
                 lambda: d.wf_beam_reorder(i32[None])):
        with pytest.raises(WfError) as e:
            make()
        assert e.value.status == "WF_ERR_INVALID_ARG"


# ---- on the GPU
def _layout(starts, rows, page, rng, extra=2):
    """A page table with pages in no order, and how many pages there are."""
    each = [-(-(s + n) // page) for s, n in zip(starts, rows)]
    total = sum(each) + extra
    table = np.full((len(rows), max(max(each), 1) + 1), -7, np.int32)
    order = rng.permutation(total)
    at = 0
    for i, n in enumerate(each):
        table[i, :n] = order[at:at + n]
        at += n
    return table, total


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda:0", dtype)


def _values(rng, n, H, d, dtype):
    """Vectors over many magnitudes, with ties of both formats, zeros and exact powers of two among them."""
    x = rng.normal(size=(n, H, d)) * np.exp2(rng.integers(-20, 20, size=(n, H, 1)))
    flat = x.reshape(-1, d)
    flat[0] = 0
    if len(flat) > 3:
        flat[1] = np.linspace(-127, 127, d).round() + 0.5 * (np.arange(d) % 2)
        flat[1, 0] = 127
        flat[2] = 448 * np.exp2(-(np.arange(d) % 20.0)) * (1 + (np.arange(d) % 3) / 16)
        flat[3] = np.where(np.arange(d) % 2, 1e-38, 3e38)
    return torch.as_tensor(x.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["path", "e4m3", "int8"])
@pytest.mark.parametrize("d,H,page", [(64, 5, 16), (128, 1, 64), (64, 20, 256), (128, 3, 32)])
def test_cache_write_and_read_match_the_oracle(dtype, fmt, d, H, page):
    rng = np.random.default_rng(d + H + page)
    rows, starts = [3, 0, 1, page + 5, 0, 2 * page], [0, 4, page - 1, 7, 0, page]
    n = sum(rows)
    dec = _decoder(n_head=H, d_head=d, dtype=dtype, cache_format=fmt, page_size=page)
    table, total = _layout(starts, rows, page, rng)
    cu = np.concatenate([[0], np.cumsum(rows)])
    pad = 4                                                      # rows behind the last sequence
    wide = torch.full((n + pad, 3 * H * d), 7.0, dtype=dec.torch_dtype)   # keys and values inside wider rows
    k, v = (wide[:, i * H * d:(i + 1) * H * d].unflatten(1, (H, d)) for i in (0, 2))
    k[:n], v[:n] = _values(rng, n, H, d, dtype), _values(rng, n, H, d, dtype)
    wide = wide.cuda()
    kd, vd = (wide[:, i * H * d:(i + 1) * H * d].unflatten(1, (H, d)) for i in (0, 2))
    cache = dec.cache(total)
    if fmt != "path":
        cache.k_scale.fill_(-3.0)                                # vectors that nothing writes keep theirs
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (_dev(table), _dev(cu), _dev(starts))
    dec.wf_cache_write(cache, *args, kd, vd, status=status)
    gk, gv = (torch.full((n + pad, H, d), 9.0, dtype=dec.torch_dtype, device="cuda") for _ in range(2))
    dec.wf_cache_read(cache, *args, n + pad, k=gk, v=gv, status=status)
    assert int(status) == 0
    assert (gk[n:] == 9).all() and (gv[n:] == 9).all()
    for src, got in ((k, gk), (v, gv)):
        want = torch.as_tensor(O.stored(src[:n].double().numpy(), fmt)).to(dec.torch_dtype)   # one rounding, to nearest even
        assert torch.equal(got[:n].cpu(), want)
    # the codes and scales themselves, at the places that the table names; all else untouched
    seen = torch.zeros(total, page, dtype=torch.bool)
    for s in range(len(rows)):
        for i in range(rows[s]):
            pos = starts[s] + i
            pg, at = int(table[s, pos // page]), pos % page
            seen[pg, at] = True
            if fmt == "path":
                assert torch.equal(cache.k[pg, :, at].cpu(), k[cu[s] + i])
            elif i % 7 == 0:
                codes, scale = O.quantise(k[cu[s] + i].double().numpy(), fmt)
                assert np.array_equal(cache.k[pg, :, at].float().cpu().numpy(), codes)
                assert np.array_equal(cache.k_scale[pg, :, at].float().cpu().numpy(), scale)
    raw = (cache.k.float().cpu() != 0).any(-1).any(1)
    assert not (raw & ~seen).any()
    if fmt != "path":
        assert (cache.k_scale.cpu().permute(0, 2, 1)[~seen] == -3).all()


@pytest.mark.gpu
def test_int8_rounding_borders_are_exact():
    """Quotients on, just above and just below a half: float32 inputs whose quotient a float32 division rounds onto the border."""
    rng = np.random.default_rng(3)
    x = np.zeros((4000, 1, 64), np.float32)
    for i in range(len(x)):
        a = np.float32(127 * np.exp2(rng.uniform(-3, 3)))
        s = np.float32(O.bf16_up(a / np.float32(127)))
        half = (rng.integers(-126, 126, size=63) + 0.5) * np.float64(s)
        x[i, 0, 0] = a
        x[i, 0, 1:] = np.nextafter(half.astype(np.float32), np.float32(np.inf) * np.sign(rng.normal(size=63)).astype(np.float32)) if i % 2 else half
    dec = _decoder(n_head=1, dtype="f32", cache_format="int8")
    cache = dec.cache(250)
    table = _dev(np.arange(250)[None])
    k = torch.as_tensor(x).cuda()
    dec.wf_cache_write(cache, table, _dev([0, 4000]), _dev([0]), k, k)
    codes, _ = O.quantise(x.astype(np.float64), "int8")
    assert np.array_equal(cache.k.cpu().numpy().transpose(0, 2, 1, 3).reshape(4000, 1, 64), codes)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_non_finite_vectors_read_back_as_nan(fmt):
    dec = _decoder(n_head=2, cache_format=fmt)
    cache = dec.cache(1)
    k = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    k[0, 0, 5], k[1, 1, 63], k[2, 0, 0] = float("nan"), float("inf"), float("-inf")
    args = (_dev([[0]]), _dev([0, 3]), _dev([0]))
    dec.wf_cache_write(cache, *args, k, k)
    got, _ = dec.wf_cache_read(cache, *args, 3)
    bad = torch.zeros(3, 2, dtype=torch.bool)
    bad[0, 0] = bad[1, 1] = bad[2, 0] = True
    assert torch.equal(torch.isnan(got).all(-1).cpu(), bad) and (got[~bad.cuda()] == 1).all()
    assert (cache.k.float()[0, 0, 0] == 0).all()


@pytest.mark.gpu
def test_bad_tables_are_passed_over_and_reported():
    from paper_2412_11272_b200.binding import STATUS_BAD_PAGE, STATUS_BAD_ROWS
    dec = _decoder(n_head=1)
    k = torch.ones(20, 1, 64, dtype=torch.bfloat16, device="cuda")

    def run(table, cu, start):
        cache = dec.cache(2)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        dec.wf_cache_write(cache, _dev(table), _dev(cu), _dev(start), k, k, status=status)
        wrote = (cache.k.float() != 0).any(-1)[:, 0].sum(1).tolist()
        out = dec.wf_cache_read(cache, _dev(table), _dev(cu), _dev(start), 20, status=status)
        assert out[0].shape[0] == 20
        return wrote, int(status)

    assert run([[1, 0]], [0, 20], [0]) == ([4, 16], 0)
    assert run([[1, 2]], [0, 20], [0]) == ([0, 16], STATUS_BAD_PAGE)            # page 2 of 2
    assert run([[-1, 0]], [0, 20], [0]) == ([4, 0], STATUS_BAD_PAGE)
    assert run([[1, 0]], [0, 20], [14]) == ([16, 2], STATUS_BAD_ROWS)           # two rows lie behind the table
    assert run([[1, 0]], [0, 20], [-3]) == ([1, 16], STATUS_BAD_ROWS)
    assert run([[1, 0]], [0, 25], [0]) == ([4, 16], STATUS_BAD_ROWS)            # more rows than the arrays have
    assert run([[1, 0]], [0, 20], [2 ** 31 - 2]) == ([0, 0], STATUS_BAD_ROWS)


@pytest.mark.gpu
def test_many_sequences_find_their_rows():
    """More sequences than one step of the 32-way search, empty ones among them."""
    rng = np.random.default_rng(8)
    rows = rng.integers(0, 3, size=1500)
    rows[100:180] = 0
    n = int(rows.sum())
    dec = _decoder(n_head=1, cache_format="path")
    cache = dec.cache(1500)
    k = torch.arange(n, dtype=torch.float32).remainder(251).to(torch.bfloat16).cuda()[:, None, None].expand(n, 1, 64).contiguous()
    args = (_dev(np.arange(1500)[:, None]), _dev(np.concatenate([[0], np.cumsum(rows)])), _dev(rng.integers(0, 13, size=1500)))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dec.wf_cache_write(cache, *args, k, -k, status=status)
    gk, gv = dec.wf_cache_read(cache, *args, n, status=status)
    assert int(status) == 0 and torch.equal(gk, k) and torch.equal(gv, -k)


@pytest.mark.gpu
@pytest.mark.parametrize("W", [1, 2, 4, 5, 8, 13, 16])
def test_reorder_contiguous_states(W):
    rng = np.random.default_rng(W)
    B = 7
    parents = rng.integers(-1, W, size=(B, W)).astype(np.int32)
    parents[0] = (np.arange(W) + 1) % W                         # a cycle: every row is read and written
    if W > 1:
        parents[1] = np.arange(W)[::-1]
    src = O.beam_sources(parents)
    a = torch.randint(-100, 100, (B * W, 33), dtype=torch.int32, device="cuda")                   # 132 bytes: 4-byte units
    wide = torch.randint(-100, 100, (B * W, 4096 + 64), dtype=torch.int8, device="cuda")          # rows inside wider rows: 16-byte units
    c = wide[:, :4096]
    odd = torch.randint(0, 100, (B * W, 7), dtype=torch.uint8, device="cuda")                      # single bytes
    f = torch.randn(B * W, 3, 5, device="cuda")
    flags = torch.randint(0, 2, (B * W,), dtype=torch.uint8, device="cuda")
    before = [t.clone() for t in (a, wide, odd, f, flags)]
    dec = _decoder()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dec.wf_beam_reorder(_dev(parents), states=[a, c, odd, f, flags], status=status)
    want = [t[src] for t in before]
    want[1] = before[1].clone()
    want[1][:, :4096] = before[1][src][:, :4096]
    assert int(status) == 0
    for got, exp in zip((a, wide, odd, f, flags), want):
        assert torch.equal(got, exp)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("int8", "f32"), ("path", "bf16"), ("path", "f32")])
@pytest.mark.parametrize("W,page,d", [(5, 16, 64), (3, 32, 128), (9, 16, 128)])
def test_reorder_paged_caches(fmt, dtype, W, page, d):
    """The values that each beam's table leads to are its parent's afterwards, and no other beam's page is touched."""
    rng = np.random.default_rng(W + page + d)
    lengths = [0, 1, page - 1, page, page + 3, 3 * page, 2 * page + 7]
    B, H, layers = len(lengths), 3, 35                           # 70 sides and the table: more than one launch holds
    P = max(lengths) // page + 1
    dec = _decoder(n_head=H, d_head=d, dtype=dtype, cache_format=fmt, page_size=page)
    table = rng.permutation(B * W * P).reshape(B, P, W).transpose(0, 2, 1).reshape(B * W, P).astype(np.int32)
    for r in range(B * W):                                       # full pages may be shared already
        for j in range(lengths[r // W] // page):
            table[r, j] = table[r // W * W + rng.integers(0, W), j]
    parents = rng.integers(-1, W, size=(B, W)).astype(np.int32)
    src = O.beam_sources(parents)
    caches = []
    for _ in range(layers):
        c = dec.cache(B * W * P)
        for t in (c.k, c.v):
            t.view(torch.uint8).copy_(torch.randint(0, 100, t.view(torch.uint8).shape, dtype=torch.uint8, device="cuda"))
        if c.k_scale is not None:
            c.k_scale.copy_(torch.rand(c.k_scale.shape, device="cuda"))
            c.v_scale.copy_(torch.rand(c.v_scale.shape, device="cuda"))
        caches.append(c)

    def rows(t, tab, r):                                         # positions [0, length) of one beam, page by page
        n = lengths[r // W]
        ids = torch.as_tensor(tab[r, :-(-n // page)].astype(np.int64), device="cuda")
        x = t[ids].transpose(1, 2)
        return x.reshape(-1, *x.shape[2:])[:n]

    checked = [0, 1, layers - 1]
    sides = [t.view(torch.uint8) if t.dtype.itemsize == 1 else t for i in checked for t in (caches[i].k, caches[i].v, caches[i].k_scale, caches[i].v_scale)
             if t is not None]
    before = [t.clone() for t in sides]
    td, status = _dev(table), torch.zeros(1, dtype=torch.int32, device="cuda")
    dec.wf_beam_reorder(_dev(parents), caches=caches, page_table=td, lengths=_dev(lengths), status=status)
    new = td.cpu().numpy()
    assert int(status) == 0
    for r in range(B * W):
        full = lengths[r // W] // page
        assert (new[r, :full] == table[src[r], :full]).all() and (new[r, full:] == table[r, full:]).all()
        for t, old in zip(sides, before):
            assert torch.equal(rows(t, new, r), rows(old, table, src[r]))
    # outside the rows that moved nothing changed
    keep = torch.ones(B * W * P, page, dtype=torch.bool)
    for r in range(B * W):
        n = lengths[r // W]
        if n % page and src[r] != r:
            keep[int(table[r, n // page]), :n % page] = False
    for t, old in zip(sides, before):
        same = (t == old) if t.dim() == 3 else (t == old).all(-1)
        assert same.permute(0, 2, 1)[keep.cuda()].all()


@pytest.mark.gpu
def test_reorder_reports_bad_device_data():
    from paper_2412_11272_b200.binding import STATUS_BAD_PAGE, STATUS_BAD_PARENT, STATUS_BAD_ROWS
    dec = _decoder(n_head=1)

    def run(parents, table, lengths):
        cache = dec.cache(4)
        cache.k.view(torch.uint8).copy_(torch.arange(4, device="cuda", dtype=torch.uint8)[:, None, None, None].expand(4, 1, 16, 64))
        state = torch.arange(2, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        dec.wf_beam_reorder(_dev(parents), states=[state], caches=[cache], page_table=_dev(table), lengths=_dev(lengths), status=status)
        return state.tolist(), cache.k.view(torch.uint8)[:, 0, 0, 0].tolist(), int(status)

    assert run([[1, 0]], [[0], [1]], [3]) == ([1, 0], [1, 0, 2, 3], 0)
    assert run([[2, 0]], [[0], [1]], [3]) == ([0, 0], [0, 0, 2, 3], STATUS_BAD_PARENT)
    assert run([[1, 0]], [[0], [4]], [3]) == ([1, 0], [0, 1, 2, 3], STATUS_BAD_PAGE)
    assert run([[1, 0]], [[0], [1]], [17]) == ([1, 0], [0, 1, 2, 3], STATUS_BAD_ROWS)
    assert run([[1, 0]], [[0], [1]], [-1]) == ([1, 0], [0, 1, 2, 3], STATUS_BAD_ROWS)
    assert run([[1, 0]], [[0], [1]], [16]) == ([1, 0], [0, 1, 2, 3], 0)          # a full page: only its table entry moves
