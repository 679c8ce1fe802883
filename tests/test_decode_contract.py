"""What the header of the decoding-stage operators promises about calls that are wrong: prefix sums that do not fit, messages of refusals,
sizes that a launch cannot hold."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")


def _decoder(**kw):
    from paper_2412_11272_b200.binding import Decoder
    return Decoder(**{**dict(n_head=4, d_head=64, dtype="bf16", cache_format="e4m3", page_size=16), **kw})


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda:0", dtype)


# ---- prefix sums
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_sums_that_do_not_fit_are_reported(dtype):
    """Every cache call reports what wf_tree_attention reports, and writes no place outside the rows' own pages."""
    from paper_2412_11272_b200.binding import STATUS_BAD_ROWS
    dec = _decoder(n_head=1, dtype=dtype)
    k = torch.ones(20, 1, 64, dtype=dec.torch_dtype, device="cuda")

    def run(cu, call):
        n = len(cu) - 1
        cache = dec.cache(2 * n + 1)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        args = (cache, _dev(np.arange(2 * n).reshape(n, 2)), _dev(cu), _dev(np.zeros(n)))
        if call == "write":
            dec.wf_cache_write(*args, k, k, status=status)
        elif call == "read":
            dec.wf_cache_read(*args, 20, status=status)
        else:
            dec.wf_tree_attention(*args, k, 20, 32, "none", status=status)
        assert (cache.k[2 * n].float() == 0).all()                                    # no sequence has the last page
        return int(status), (cache.k.float() != 0).any(-1).any(1)

    many = np.concatenate([np.arange(0, 11).repeat(60), [20]])                        # hundreds of sequences, most of them empty
    for cu, good in (([0, 5, 20], True), ([0, 0, 0, 7], True), (many, True), ([0, 5, 3, 8], False), ([0, 20, 18], False), ([0, 8, 8, 2, 8], False),
                     ([-2, 3], False), ([0, 21], False), (np.concatenate([many[:400], [0], many[400:]]), False),
                     ([0, 2 ** 31 - 1, -2 ** 31, 4], False)):
        for call in ("write", "read", "attention"):
            assert run(cu, call)[0] == (0 if good else STATUS_BAD_ROWS), (cu, call)
    # a sequence whose rows begin before the first has no places: nothing of it is written
    assert not run([-2, 3], "write")[1].any()


# ---- refusals (no GPU is needed)
def _message(d):
    return d.lib.wf_decoder_last_error(d.handle).decode()


def test_refusals_say_what_was_wrong():
    from paper_2412_11272_b200 import binding as Bn
    d = _decoder()
    P = 1 << 20
    cache, rows = Bn.wf_cache(P, P + 4096, P, P, 3), Bn.wf_rows(2, 8, P, P, P, 4)
    for fn, name in ((d.lib.wf_cache_write, "wf_cache_write"), (d.lib.wf_cache_read, "wf_cache_read")):
        assert fn(d.handle, cache, rows, P, 248, P, 256, None, None) == 1
        assert _message(d).startswith(name) and "row stride is shorter than a row of 256" in _message(d)
        assert fn(d.handle, cache, rows, P, 260, P, 256, None, None) == 1 and "16-byte aligned" in _message(d)
        assert fn(d.handle, cache, Bn.wf_rows(2, (1 << 27) + 1, P, P, P, 4), P, 256, P, 256, None, None) == 4 and "2^27 rows" in _message(d)
    with pytest.raises(Bn.WfError) as e:
        _decoder(d_head=80)
    assert "d_head must be 64 or 128" in str(e.value)


def test_workspace_sizes_are_kept_per_device(monkeypatch):
    """The size follows from the device's SMs: "cuda" stands for the device that is current when the question is asked, and one device
    has one remembered size however it is named."""
    import contextlib
    import types
    d = _decoder()
    current, asked = [0], []

    def fake_size(handle, n_seq, n_rows, max_rows, max_len, out):
        asked.append(current[0])
        out._obj.value = 1000 * (current[0] + 1)
        return 0

    @contextlib.contextmanager
    def device(x):
        index = x if isinstance(x, int) else torch.device(x).index
        before, current[0] = current[0], current[0] if index is None else index
        yield
        current[0] = before

    real = d.lib
    d.lib = types.SimpleNamespace(wf_tree_attention_workspace=fake_size, wf_decoder_destroy=real.wf_decoder_destroy)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    sizes = (3, 9, 4, 5000)
    assert d.tree_attention_workspace(*sizes) == 1000
    current[0] = 1                                                                    # another device, with other SMs, is current now
    assert d.tree_attention_workspace(*sizes) == 2000
    assert d.tree_attention_workspace(*sizes, torch.device("cuda")) == 2000 and d.tree_attention_workspace(*sizes, "cuda:0") == 1000
    assert d.tree_attention_workspace(*sizes, torch.device("cuda", 1)) == 2000 and d.tree_attention_workspace(*sizes, 0) == 1000
    assert asked == [0, 1]


# ---- waits that give up
@pytest.mark.gpu
@pytest.mark.parametrize("d,fmt", [(64, "e4m3"), (64, "path"), (128, "int8")])
@pytest.mark.parametrize("hi", [100, 5000])
def test_a_wait_that_gives_up_leaves_no_plausible_numbers(d, fmt, hi):
    """Also where the caller passes no status word: rows are NaN, with one split and with many; rows behind the batch stay."""
    from paper_2412_11272_b200.binding import STATUS_GAVE_UP
    dec = _decoder(n_head=4, n_kv_head=2, d_head=d, cache_format=fmt, page_size=64)
    rows, starts = [40, 0, 33], [hi, 3, 7]
    n, longest = sum(rows), hi + 40
    pages = -(-longest // 64)
    cache = dec.cache(pages)
    for t in (cache.k, cache.v):
        if fmt == "path":
            t.normal_()
        else:
            t.view(torch.uint8).random_(0, 100)
    table = _dev(np.stack([np.arange(pages)] * 3))                                    # the sequences read the same pages
    q = torch.randn(n + 3, 4, d, device="cuda").bfloat16()
    args = (cache, table, _dev(np.concatenate([[0], np.cumsum(rows)])), _dev(starts), q, 40, longest)
    assert (dec.tree_attention_workspace(3, n + 3, 40, longest) > 0) == (hi == 5000)

    def run(**kw):
        out, lse = torch.full((n + 3, 4, d), 5.0, device="cuda").bfloat16(), torch.full((n + 3, 4), 5.0, device="cuda")
        dec.wf_tree_attention(*args, out=out, lse=lse, **kw)
        assert (out[n:] == 5).all() and (lse[n:] == 5).all()
        return out[:n], lse[:n]

    want = run()
    assert torch.isfinite(want[0]).all() and torch.isfinite(want[1]).all()
    dec.wf_selftest_attention_timeout(True)
    for status in (None, torch.zeros(1, dtype=torch.int32, device="cuda")):
        out, lse = run(status=status)
        assert torch.isnan(out).all() and torch.isnan(lse).all()
    assert int(status) == STATUS_GAVE_UP
    dec.wf_selftest_attention_timeout(False)
    status.zero_()
    got = run(status=status)
    assert int(status) == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_calls_that_no_launch_holds_are_refused():
    """A call of 2^32 vectors a side or more (which no cache holds) would need more blocks than a grid counts."""
    from paper_2412_11272_b200 import binding as Bn
    P = 1 << 20
    d = _decoder(n_head=1024, d_head=128, cache_format="path", page_size=16)
    cache = Bn.wf_cache(P, P + 4096, None, None, 3)
    for fn in (d.lib.wf_cache_write, d.lib.wf_cache_read):
        for n in (1 << 27, (1 << 26) + 2, 1 << 22):                                   # (2^26 + 2 rows: 2^32 + 128 blocks)
            assert fn(d.handle, cache, Bn.wf_rows(1, n, P, P, P, 4), P, 1024 * 128, P, 1024 * 128, None, None) == 4, n
            assert "2^32 vectors" in _message(d)


def test_reordering_refuses_memory_given_twice():
    """A state, or a cache, that the call is given twice would be moved twice, in any order."""
    from paper_2412_11272_b200 import binding as Bn
    d = _decoder(n_head=1)
    P = 1 << 20

    def reorder(*states, caches=(), B=2, W=4):
        s = (Bn.wf_beam_state * max(len(states), 1))(*[Bn.wf_beam_state(*x) for x in states])
        c = (Bn.wf_cache * max(len(caches), 1))(*caches)
        return d.lib.wf_beam_reorder(d.handle, P, B, W, s, len(states), c, len(caches), P, 4, P, None, None)

    for bad in (((P, 64, 64), (P, 64, 64)),                                           # the same state
                ((P, 64, 64), (P, 16, 128)),                                          # its first bytes under another stride
                ((P, 64, 256), (P + 32, 64, 256)),                                    # columns that share bytes
                ((P + 32, 64, 256), (P, 64, 256)),
                ((P, 64, 256), (P + 3 * 256 + 63, 8, 256)),
                ((P, 64, 256), (P - 256 + 200, 64, 256)),                             # its last bytes are the other's first
                ((P, 64, 64), (P + 640, 4, 64), (P + 128, 4, 64))):
        assert reorder(*bad) == 1, bad
        assert "share memory" in _message(d)
    one, two = Bn.wf_cache(P, 2 * P, 3 * P, 4 * P, 3), Bn.wf_cache(5 * P, 6 * P, 7 * P, 8 * P, 3)
    for bad in ((one, one), (one, two, one), (Bn.wf_cache(P, P, 3 * P, 4 * P, 3),), (one, Bn.wf_cache(5 * P, 2 * P, 7 * P, 8 * P, 3)),
                (Bn.wf_cache(P, 2 * P, 3 * P, 3 * P, 3),)):
        assert reorder(caches=bad) == 1 and "share memory" in _message(d)
    assert reorder((P, 16, 16), caches=(two,)) == 1 and "share memory" in _message(d)  # the page table, as a state too
    # side by side, interleaved, behind one another or without bytes they are different states: no refusal (without a device they end there)
    fine = (((P, 64, 64), (P + 512, 64, 64)), ((P, 64, 256), (P + 64, 64, 256), (P + 128, 128, 256)), ((P + 128, 128, 256), (P, 64, 256)),
            ((P, 64, 64), (P, 0, 64)), ((P, 64, 256), (P - 256 + 192, 64, 256)))
    if not torch.cuda.is_available():
        for good in fine:
            assert reorder(*good) == 5, good
        assert reorder((2 * P, 16, 16), caches=(one, two)) == 5
    assert reorder(*fine[0], B=0) == 0 and reorder((P, 64, 64), (P, 64, 64), W=1) == 0  # nothing moves


def test_the_tensors_of_a_cache_cannot_be_exchanged():
    """A KvCache stands for the memory it was made with: another tensor needs another KvCache."""
    from paper_2412_11272_b200.binding import KvCache
    pages = torch.zeros(3, 4, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale = torch.ones(3, 4, 16, dtype=torch.bfloat16)
    cache = KvCache(pages, pages.clone(), scale, scale.clone())
    for name in ("k", "v", "k_scale", "v_scale", "device", "shape", "c"):
        with pytest.raises(AttributeError):
            setattr(cache, name, getattr(cache, name))
    with pytest.raises(AttributeError):
        del cache.k
    assert cache.k is pages and cache.c.k == pages.data_ptr() and cache.c.n_pages == 3


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n", [("bf16", 4), ("bf16", 40), ("f32", 4)])
def test_some_sequences_of_a_packed_batch(dtype, n):
    """A slice of the prefix sums (with the starts and the table's rows that belong to it) stands for those sequences: rows in front of
    the first one are padding like the rows behind the last, and nothing about that is wrong."""
    rng = np.random.default_rng(n)
    dec = _decoder(n_head=2, dtype=dtype)
    rows, starts = [n, 3, 0, n - 1, 5], [20, 0, 7, 33, 2]
    cu = np.concatenate([[0], np.cumsum(rows)])
    total = int(cu[-1])
    k, v, q = (torch.as_tensor(rng.normal(size=(total, 2, 64)).astype(np.float32)).to("cuda", dec.torch_dtype) for _ in range(3))
    pages = 5
    table = _dev(rng.permutation(5 * pages).reshape(5, pages))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(a, b, cache):
        """Writes, reads back and attends the sequences a .. b - 1."""
        args = (cache, table[a:b].contiguous(), _dev(cu[a:b + 1]), _dev(starts[a:b]))
        dec.wf_cache_write(*args, k, v, status=status)
        back = [torch.full_like(x, 9.0) for x in (k, v)]
        dec.wf_cache_read(*args, total, k=back[0], v=back[1], status=status)
        out, lse = torch.full_like(q, 9.0), torch.full((total, 2), 9.0, device="cuda")
        dec.wf_tree_attention(*args, q, max(rows), 80, "causal", out=out, lse=lse, status=status)
        return [*back, out, lse]

    whole, part = dec.cache(5 * pages), dec.cache(5 * pages)
    want, got = run(0, 5, whole), [None] * 4
    for a, b in ((0, 1), (1, 4), (4, 5)):
        here = run(a, b, part)
        lo, hi = cu[a], cu[b]
        for x in here:
            assert (x[:lo] == 9).all() and (x[hi:] == 9).all()
        got = [x[lo:hi] if g is None else torch.cat([g, x[lo:hi]]) for g, x in zip(got, here)]
    assert int(status) == 0
    for x, y in ((whole.k, part.k), (whole.v, part.v)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # the cache's values are the same; attention may split the positions otherwise: two answers within the tolerance of rounding
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    tol = 2.0 ** -6 + 2e-4 if dtype == "bf16" else 2e-4
    assert (got[2].double() - want[2].double()).abs().max() <= tol * float(v.double().abs().max()) and (got[3] - want[3]).abs().max() <= 2e-4
