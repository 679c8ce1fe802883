"""wf_beam_select against the fp64 oracle, its refusals, and a decoding round that runs the operators together."""
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


# ---- no GPU is needed
def test_oracle_selection_pins():
    x = np.log(np.array([[[0.5, 0.25, 0.25], [0.1, 0.8, 0.1]]]))
    s, p, t, f = O.beam_select(x, np.array([[0.0, np.log(0.5)]]), 4, end_token=2)
    assert np.allclose(np.exp(s[0]), [0.5, 0.4, 0.25, 0.25]) and p[0].tolist() == [0, 1, 0, 0] and t[0].tolist() == [0, 1, 1, 2]
    assert f[0].tolist() == [0, 0, 0, 1]
    s, p, t, f = O.beam_select(x, np.array([[0.0, -1.0]]), 3, finished=np.array([[0, 1]]), end_token=2, suppressed=np.array([True, False, False]))
    assert np.allclose(s[0], [np.log(0.5), np.log(0.5), -1.0]) and t[0].tolist() == [1, 2, 2] and p[0].tolist() == [0, 0, 1] and f[0].tolist() == [0, 1, 1]
    s, p, t, f = O.beam_select(x, np.array([[0.0, -1.0]]), 3, beams=[0])
    assert (s == -np.inf).all() and (p == -1).all() and (t == -1).all()


def test_select_refusals_at_the_c_entry():
    d = _decoder()
    P = 1 << 20
    base = dict(h=d.handle, x=P, dt=1, ld=100, B=2, W=4, V=100, sc=P, beams=None, fin=None, end=-1, sup=None, keep=4, os=P, op=P, ot=P, of=None,
                status=None, stream=None)

    def call(**kw):
        a = {**base, **kw}
        return d.lib.wf_beam_select(*(a[k] for k in base))

    for bad in (dict(h=None), dict(x=None), dict(x=P + 1), dict(dt=0, x=P + 2), dict(dt=2), dict(ld=99), dict(B=-1), dict(W=0), dict(W=17), dict(V=0),
                dict(V=1 << 27, ld=1 << 27, W=16), dict(sc=None), dict(fin=P), dict(end=100), dict(end=-2), dict(keep=0), dict(keep=33), dict(os=None),
                dict(op=None), dict(ot=None)):
        assert call(**bad) == 1, bad
    assert call(B=(1 << 24) + 1) == 4 and call(V=(1 << 28) + 1, ld=1 << 29, W=1) == 4 and call(B=0) == 0
    from paper_2412_11272_b200.binding import WfError
    x = torch.zeros(4, 100)
    for make in (lambda: d.wf_beam_select(x, torch.zeros(2, 2), 3), lambda: d.wf_beam_select(x.half(), torch.zeros(2, 2), 3)):
        with pytest.raises(WfError) as e:
            make()
        assert e.value.status == "WF_ERR_INVALID_ARG"


# ---- on the GPU
def _check(dec, logits, scores, keep, beams=None, finished=None, end_token=-1, suppressed=None, ld_pad=0, offset=0):
    B, W = scores.shape
    V = logits.shape[-1]
    wide = torch.full((B * W, V + ld_pad + offset), 1e9).to(logits.dtype)
    wide[:, offset:offset + V] = logits.reshape(B * W, V)
    x = wide.cuda()[:, offset:offset + V]
    words = None
    if suppressed is not None:
        bits = np.zeros(-(-V // 32) * 32, bool)
        bits[:V] = suppressed
        words = torch.from_numpy(np.packbits(bits, bitorder="little").view(np.int32)).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = dec.wf_beam_select(x, _dev(scores, torch.float32), keep, beams=None if beams is None else _dev(beams),
                             finished=None if finished is None else _dev(finished, torch.uint8), end_token=end_token, suppress=words, status=status)
    assert int(status) == 0
    want = O.beam_select(logits.double().numpy().reshape(B, W, V), np.asarray(scores, np.float32).astype(np.float64), keep, beams, finished, end_token,
                         suppressed)
    s = got[0].double().cpu().numpy()
    fin = np.isfinite(want[0])
    assert np.array_equal(fin, np.isfinite(s))
    # one rounding to float32 (2^-24 of the score) and the log-sum's error: its exponentials and partial sums in float32,
    # a relative error under 2e-6 of the sum for any vocabulary here
    assert (np.abs(s[fin] - want[0][fin]) <= 2.0 ** -23 * np.abs(want[0][fin]) + 2e-6).all()
    for g, w in zip(got[1:], want[1:]):
        assert np.array_equal(g.cpu().numpy(), w)
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 31, 33, 200, 1000, 1023, 1025, 5001, 40_003])
def test_vocabularies_of_any_size(dtype, V):
    rng = np.random.default_rng(V)
    dec = _decoder()
    for B, W, keep in ((1, 1, 1), (3, 5, 5), (2, 3, 10)):
        logits = torch.as_tensor(rng.normal(size=(B * W, V)).astype(np.float32) * 3).to(dtype)
        # scores far enough apart from the ties of bfloat16 logits: random float32
        _check(dec, logits, -5 * rng.random((B, W)), keep, ld_pad=V % 5, offset=V % 3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("W,keep", [(1, 32), (2, 4), (8, 16), (16, 32), (13, 1)])
def test_beam_counts_finished_and_pruned(dtype, W, keep):
    rng = np.random.default_rng(W * 100 + keep)
    dec = _decoder()
    B, V = 6, 3001
    logits = torch.as_tensor(rng.normal(size=(B * W, V)).astype(np.float32) * 2).to(dtype)
    scores = -4 * rng.random((B, W))
    finished = (rng.random((B, W)) < 0.3).astype(np.uint8)
    finished[0] = 1                                              # every beam has ended
    beams = rng.integers(0, W + 1, size=B)
    beams[:2] = W
    beams[2] = 0
    sup = rng.random(V) < 0.02
    sup[:40] = True
    _check(dec, logits, scores, keep, beams, finished, 17, sup)
    _check(dec, logits, scores, keep, None, finished, V - 1, None)
    _check(dec, logits, scores, keep, beams, None, 3, None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_go_to_the_lowest_index(dtype):
    dec = _decoder()
    # identical rows and equal scores: a tie of every token with itself in all beams; constant rows: all tokens tie
    row = torch.as_tensor(np.random.default_rng(1).normal(size=4000).astype(np.float32)).to(dtype)
    _check(dec, row.expand(6, 4000).clone(), np.zeros((2, 3)), 7)
    _check(dec, torch.zeros(6, 9000).to(dtype), np.zeros((2, 3)), 32)
    few = torch.full((4, 20_000), -8.0)
    few[:, [19_999, 3, 777, 10_000]] = 1.0                       # four ties far apart, then thousands of ties
    _check(dec, few.to(dtype), np.zeros((2, 2)), 12)
    steps = torch.arange(5000).div(50, rounding_mode="floor").float().div(8)    # plateaus, rising: the best lie at the end
    _check(dec, steps.expand(2, 5000).clone().to(dtype), np.zeros((1, 2)), 31)
    _check(dec, steps.flip(0).expand(2, 5000).clone().to(dtype), np.zeros((1, 2)), 31)
    _check(dec, torch.arange(6000.0).expand(1, 6000).clone().div(64).to(dtype), np.zeros((1, 1)), 32)


@pytest.mark.gpu
def test_many_tiles_of_one_row():
    """Rows longer than sixteen tiles of a block of the widest cluster: items keep their best over several tiles."""
    rng = np.random.default_rng(3)
    dec = _decoder()
    V = 300_007
    x = torch.as_tensor(rng.normal(size=(2, V)).astype(np.float32))
    x[0, -40:] = torch.arange(40.0) / 10 + 5                     # the best at the very end
    x[1, ::1000] = 6.0                                           # ties over all tiles
    _check(dec, x, np.array([[0.0, -0.3]]), 32)
    _check(dec, x.bfloat16(), np.array([[0.0], [-0.3]]), 32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_without_continuations(dtype):
    inf, nan = float("inf"), float("nan")
    dec = _decoder()
    V = 2500
    x = torch.as_tensor(np.random.default_rng(4).normal(size=(10, V)).astype(np.float32)).to(dtype)
    x[0] = -inf
    x[1, 2400] = nan
    x[2, 0] = inf
    x[3, :-1] = -inf                                             # a single possible token
    x[4, 5:] = -inf
    scores = np.array([[0, 0, 0, -1, -2], [-inf, -1, -inf, nan, -3]])
    _check(dec, x, scores, 9)
    _check(dec, x, scores, 9, finished=np.array([[0, 0, 0, 0, 1], [1, 1, 0, 1, 0]]), end_token=7)
    _check(dec, x, np.zeros((10, 1)), 3, suppressed=np.arange(V) != 2400)       # only the token that is NaN in one row
    _check(dec, x, np.zeros((10, 1)), 3, suppressed=np.isin(np.arange(V), [0, 2400]))  # NaN and infinity are suppressed
    _check(dec, x, np.zeros((10, 1)), 3, suppressed=np.ones(V, bool))


@pytest.mark.gpu
def test_logits_of_any_size_and_repeated_calls():
    rng = np.random.default_rng(5)
    dec = _decoder()
    x = torch.as_tensor((rng.normal(size=(8, 7001)) * np.array([1e-4, 1, 30, 1e4] * 2)[:, None]).astype(np.float32))
    scores = rng.normal(size=(4, 2)) * 100
    first = _check(dec, x, scores, 8)
    for _ in range(3):
        for a, b in zip(_check(dec, x, scores, 8), first):
            assert torch.equal(a, b)
    x[:, 100] = 1e30                                             # one token far above all others
    _check(dec, x, scores, 2)


@pytest.mark.gpu
def test_beams_outside_the_range_are_cut_and_reported():
    from paper_2412_11272_b200.binding import STATUS_BAD_ROWS
    dec = _decoder()
    x, scores = torch.randn(6, 100, device="cuda"), torch.zeros(2, 3, device="cuda")
    for beams, same in (([9, 3], [3, 3]), ([3, -4], [3, 0])):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = dec.wf_beam_select(x, scores, 4, beams=_dev(beams), status=status)
        want = dec.wf_beam_select(x, scores, 4, beams=_dev(same))
        assert int(status) == STATUS_BAD_ROWS and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_selection_in_a_graph():
    dec = _decoder()
    x, scores = torch.randn(10, 5000, device="cuda"), torch.zeros(2, 5, device="cuda")
    dec.wf_beam_select(x, scores, 5)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = dec.wf_beam_select(x, scores, 5)
    x.copy_(torch.randn(10, 5000, device="cuda"))
    scores.copy_(torch.rand(2, 5, device="cuda"))
    g.replay()
    want = dec.wf_beam_select(x, scores, 5)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
