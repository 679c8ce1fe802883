"""wf_quantise_e4m3 and wf_gemm_e4m3 against the oracle."""
import numpy as np
import pytest

from oracle import speculation_oracle as O

torch = pytest.importorskip("torch")


def _decoder(**kw):
    from paper_2412_11272_b200.binding import Decoder
    return Decoder(**{**dict(n_head=4, d_head=64), **kw})


# ---- no GPU is needed
def test_oracle_pins():
    x = np.zeros((2, 130))
    x[0, :3], x[0, 128:] = [448.0, 1.0, -17.0], [450.0, 2.0 ** -130]
    c, m = O.quantise_rows(x)
    assert m.tolist() == [[127, 128], [127, 127]] and c[0, :3].tolist() == [448, 1, -16] and c[0, 128:].tolist() == [224, 0]
    assert np.array_equal(O.values(c, m)[0, 128:], [448.0, 0.0])
    x[1, 5] = np.inf
    assert O.quantise_rows(x)[1].tolist() == [[127, 128], [255, 127]]
    assert np.allclose(O.gelu(np.array([[0.0, 1.0, -1.0, -30.0]])), [[0, 0.8413447460685429, -0.15865525393145707, 0]], atol=1e-15)


def test_refusals_at_the_c_entry():
    from paper_2412_11272_b200 import binding as Bn
    d = _decoder()
    P = 1 << 20
    ok = Bn.wf_e4m3(P, P, 112, 8)
    base = dict(h=d.handle, x=P, dt=1, ldx=100, rows=8, k=100, out=ok, stream=None)

    def quantise(**kw):
        a = {**base, **kw}
        return d.lib.wf_quantise_e4m3(*(a[k] for k in base))

    bad_codes = [None, Bn.wf_e4m3(None, P, 112, 8), Bn.wf_e4m3(P, None, 112, 8), Bn.wf_e4m3(P + 8, P, 112, 8), Bn.wf_e4m3(P, P + 2, 112, 8),
                 Bn.wf_e4m3(P, P, 104, 8), Bn.wf_e4m3(P, P, 96, 8), Bn.wf_e4m3(P, P, 112, 7)]
    for bad in [dict(h=None), dict(x=None), dict(x=P + 1), dict(dt=0, x=P + 2), dict(dt=2), dict(ldx=99), dict(rows=-1), dict(k=0)] + [dict(out=c) for c in bad_codes]:
        assert quantise(**bad) == 1, bad
    assert quantise(rows=(1 << 27) + 1) == 4 and quantise(k=(1 << 22) + 1, ldx=1 << 23) == 4 and quantise(rows=0) == 0
    gbase = dict(h=d.handle, a=ok, w=ok, bias=None, out=P, dt=1, ldc=8, m=8, n=8, k=100, gelu=0, status=None, stream=None)

    def gemm(**kw):
        a = {**gbase, **kw}
        return d.lib.wf_gemm_e4m3(*(a[k] for k in gbase))

    for bad in [dict(h=None), dict(out=None), dict(out=P + 1), dict(dt=0, out=P + 2), dict(dt=3), dict(ldc=7), dict(m=-1), dict(n=-1), dict(k=0), dict(bias=P + 2)] + \
            [dict(a=c) for c in bad_codes] + [dict(w=c) for c in bad_codes]:
        assert gemm(**bad) == 1, bad
    assert "(w)" in d.lib.wf_decoder_last_error(d.handle).decode()
    assert gemm(m=(1 << 27) + 1) == 4 and gemm(n=(1 << 27) + 1, ldc=1 << 28) == 4 and gemm(k=(1 << 22) + 1) == 4 and gemm(m=0) == 0 and gemm(n=0, ldc=8) == 0


def test_refusals_of_the_binding():
    from paper_2412_11272_b200.binding import ScaledCodes, WfError
    d = _decoder()
    f8 = torch.float8_e4m3fn
    codes, scales = torch.zeros(3, 512).to(f8), torch.full((1, 3, 4), 127, dtype=torch.uint8)
    ok = ScaledCodes(codes, scales)
    assert ok.shape == (3, 512) and ok[1:].shape == (2, 512)
    for make in (lambda: ScaledCodes(codes.float(), scales), lambda: ScaledCodes(codes.t(), scales), lambda: ScaledCodes(codes, scales[0]),
                 lambda: ScaledCodes(codes, scales.int()), lambda: ScaledCodes(codes, torch.zeros(2, 3, 4, dtype=torch.uint8)),
                 lambda: ScaledCodes(codes, torch.zeros(1, 4, 3, dtype=torch.uint8).transpose(1, 2)), lambda: ok[::2],
                 lambda: ScaledCodes.pack(codes, torch.full((3, 4), 3.0)), lambda: ScaledCodes.pack(codes, torch.ones(3, 5)),
                 lambda: ScaledCodes.pack(codes, torch.zeros(3, 4)), lambda: ScaledCodes.pack(codes, -torch.ones(3, 4)),
                 lambda: d.wf_quantise_e4m3(torch.zeros(3, 8)), lambda: d.wf_gemm_e4m3(ok, ok)):
        with pytest.raises(WfError) as e:
            make()
        assert e.value.status == "WF_ERR_INVALID_ARG"
    with pytest.raises(AttributeError):
        ok.codes = codes


def test_packed_codes_mean_what_they_say():
    from paper_2412_11272_b200.binding import ScaledCodes
    g = torch.Generator().manual_seed(1)
    codes = torch.randn(200, 300, generator=g).to(torch.float8_e4m3fn)
    s = 2.0 ** torch.randint(-126, 127, (200, 3), generator=g).float()
    s[3, 1] = float("nan")
    got = ScaledCodes.pack(codes, s)
    want = codes.float() * s.repeat_interleave(128, 1)[:, :300]
    assert torch.equal(got.values().nan_to_num(7.0), want.nan_to_num(7.0)) and got.codes.stride(0) == 304
    assert torch.equal(got[10:50].values(), want[10:50])
    blocks = 2.0 ** torch.randint(-5, 5, (2, 3), generator=g).float()  # one for each 128 x 128 block
    got = ScaledCodes.pack(codes, blocks)
    assert torch.equal(got.values(), codes.float() * blocks.repeat_interleave(128, 0)[:200].repeat_interleave(128, 1)[:, :300])


# ---- codes
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,k,pad,offset", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 127, 0, 0), (5, 129, 0, 0), (7, 1280, 0, 0), (70, 513, 0, 0), (9, 512, 8, 8), (6, 300, 3, 1),
                                               (2, 5000, 0, 0), (300, 40, 0, 0), (33, 640, 5, 3)])
def test_quantise(dtype, rows, k, pad, offset):
    """Codes and scales are the oracle's, bit for bit: sizes of many kinds, blocks of zeros, borders between codes and between scales."""
    g = torch.Generator().manual_seed(k)
    x = torch.randn(rows, k, generator=g) * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g).float())
    x[:, ::7] *= 2.0 ** -9                                            # subnormal codes
    x[rows // 2] = 0
    x[0, : min(k, 6)] = torch.tensor([448.0, 1.0625, 17.0, 1.1875, -0.0, 2.0 ** -10])[: min(k, 6)]  # ties between codes; the largest, exactly
    if k > 140:
        x[rows - 1, 128:140] = 0
        x[rows - 1, 130] = 449.0
    wide = torch.full((rows, k + pad + offset), float("nan")).to(dtype).cuda()
    wide[:, offset:offset + k] = x.to(dtype)
    got = _decoder().wf_quantise_e4m3(wide[:, offset:offset + k])
    codes, marks = O.quantise_rows(x.to(dtype).double().numpy())
    assert np.array_equal(got.codes.float().cpu().numpy(), codes)
    b = got.scales.transpose(0, 1).reshape(rows, -1).cpu().numpy()
    assert np.array_equal(b[:, :marks.shape[1]], marks) and (b[:, marks.shape[1]:] == 127).all()
    assert np.array_equal(got.values().double().cpu().numpy(), O.values(codes, marks))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantise_special_values(dtype):
    """Infinities and NaN, the ends of the range, subnormal numbers."""
    x = torch.zeros(10, 256)
    x[0, 3], x[1, 200], x[2, 5] = float("nan"), float("inf"), -float("inf")
    x[3], x[4, 7], x[5, 9], x[6, 11] = 3.3e38, 2.0 ** -126, 2.0 ** -133, 448 * 2.0 ** -126
    x[7, :128], x[8, 0] = torch.linspace(-3e38, 3e38, 128), 449 * 2.0 ** -126
    x = x.to(dtype)
    got = _decoder().wf_quantise_e4m3(x.cuda())
    codes, marks = O.quantise_rows(x.double().numpy())
    assert np.array_equal(got.codes.float().cpu().numpy(), codes)
    assert np.array_equal(got.scales.transpose(0, 1).reshape(10, -1).cpu().numpy()[:, :2], marks)
    assert marks[0, 0] == marks[1, 1] == marks[2, 0] == 255 and (codes[:3] == 0).all()


@pytest.mark.gpu
def test_quantise_leaves_the_rest():
    """Into the middle of larger arrays: nothing else is written."""
    from paper_2412_11272_b200.binding import ScaledCodes
    codes = torch.full((12, 320), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scales = torch.full((1, 12, 4), 77, dtype=torch.uint8, device="cuda")
    x = torch.randn(5, 300, device="cuda").bfloat16()
    out = _decoder().wf_quantise_e4m3(x, out=ScaledCodes(codes[:, :300], scales)[4:9])
    c, s = codes.view(torch.uint8), scales[0]
    assert (c[:4] == 0x55).all() and (c[9:] == 0x55).all() and (c[:, 300:] == 0x55).all() and (s[:4] == 77).all() and (s[9:] == 77).all()
    assert torch.equal(out.values(), _decoder().wf_quantise_e4m3(x).values())


# ---- products
def _tolerance(a, w, y, out, gelu):
    """The sums: products are exact, each of an instruction's 32 products joins the accumulator with an error of at most a step of float32
    (2^-23) of what is summed in magnitude, a split adds at most eight of the results; the output is rounded by half a step.  GELU changes an error by a
    factor of 1.13 at most; its own: 2.1e-3 |y| (the fit's largest relative error, for bfloat16) and 3e-7, or 1e-6 |x| (erff's half steps)."""
    steps = a.shape[1] / 32 + 32 + 8
    t = steps * 2.0 ** -23 * (np.abs(a) @ np.abs(w).T) * 1.13
    if gelu:
        t = t + (2.1e-3 * np.abs(y) + 3e-7 if out == "bf16" else 1e-6 * np.abs(y) + 1e-6)
    return t + (2.0 ** -8 if out == "bf16" else 2.0 ** -24) * np.abs(y) + 1e-30


def _matrix(rows, k, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, k, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
    return _decoder().wf_quantise_e4m3(x * torch.exp2(torch.randint(-3, 3, (1, k), generator=g, device="cuda").float()))


def _check(m, n, k, out="bf16", bias=True, gelu=False, pad=0, offset=0):
    dec = _decoder()
    a, w = _matrix(m, k, m + k), _matrix(n, k, n + 3 * k)
    A, W = a.values().double(), w.values().double() / (4 * k ** 0.5)
    w = dec.wf_quantise_e4m3(W.float())
    W = w.values().double()
    b = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") if bias else None
    wide = torch.full((m + 2, n + pad + offset), 77.0, device="cuda", dtype=torch.bfloat16 if out == "bf16" else torch.float32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    C = wide[1:m + 1, offset:offset + n]
    got = dec.wf_gemm_e4m3(a, w, bias=b, gelu=gelu, out=C, status=status)
    assert got is C and int(status) == 0
    y = A @ W.T + (0 if b is None else b.double())
    if gelu:
        y = y * torch.special.ndtr(y)
    A, W, y = (t.cpu().numpy() for t in (A, W, y))
    err, tol = np.abs(C.double().cpu().numpy() - y), _tolerance(A, W, y, out, gelu)
    assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index(np.argmax(err / tol), err.shape))
    edge = wide.clone()
    edge[1:m + 1, offset:offset + n] = 77.0
    assert (edge == 77.0).all()                                       # nothing beside C is written


@pytest.mark.gpu
@pytest.mark.parametrize("out,bias,gelu", [("bf16", True, False), ("f32", False, False), ("bf16", True, True), ("f32", True, True)])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 128, 128), (1, 1280, 1280), (3, 5, 130), (16, 129, 513), (17, 640, 512), (20, 50, 5000), (33, 200, 4097), (64, 1280, 1280),
                                   (65, 131, 700), (100, 100, 3000), (129, 1000, 640), (200, 5000, 300), (225, 513, 1300), (320, 1280, 2560), (700, 5120, 256),
                                   (1000, 264, 2000), (2300, 700, 300), (4500, 1030, 129)])
def test_products(m, n, k, out, bias, gelu):
    _check(m, n, k, out, bias, gelu)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(5, 300, 384), (300, 1000, 1000), (3000, 1500, 640)])
@pytest.mark.parametrize("out,pad,offset", [("bf16", 1, 0), ("bf16", 8, 8), ("bf16", 3, 2), ("bf16", 7, 1), ("f32", 1, 0), ("f32", 3, 1), ("f32", 4, 4)])
def test_outputs_at_any_alignment(m, n, k, out, pad, offset):
    _check(m, n, k, out, True, out == "bf16", pad, offset)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(7, 200, 300), (40, 128, 6000), (1500, 2000, 700)])
def test_rows_of_a_larger_matrix(m, n, k):
    """Operands that are rows out of the middle of others; the rest holds NaN."""
    from paper_2412_11272_b200.binding import ScaledCodes
    dec = _decoder()
    sides = []
    for rows in (m, n):
        q, big = _matrix(rows, k, rows), ScaledCodes.empty(rows + 9, k)
        big.codes.view(torch.uint8).fill_(0x7f)
        big.scales.fill_(255)
        big.codes.view(torch.uint8)[4:4 + rows] = q.codes.view(torch.uint8)
        big.scales[:, 4:4 + rows] = q.scales
        sides.append((q, big[4:4 + rows]))
    (a, a2), (w, w2) = sides
    plain = dec.wf_gemm_e4m3(a, w)
    assert torch.isfinite(plain).all() and torch.equal(plain, dec.wf_gemm_e4m3(a2, w2))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [3, 90, 2000])
def test_scales_and_codes_that_are_not_numbers(m):
    """A NaN scale or code reaches the sums that it is part of, and no others; large and small scales meet exactly."""
    from paper_2412_11272_b200.binding import ScaledCodes
    dec, n, k = _decoder(), 600, 900
    a, w = _matrix(m, k, 1), _matrix(n, k, 2)
    plain = dec.wf_gemm_e4m3(a, w, out_dtype="f32")
    a.scales[1, m // 2, 1] = 255                                       # block 5 of a row
    w.codes.view(torch.uint8)[17, 300] = 0x7f
    got = dec.wf_gemm_e4m3(a, w, out_dtype="f32")
    assert got[m // 2].isnan().all() and got[:, 17].isnan().all()
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[m // 2], keep[:, 17] = False, False
    assert torch.equal(got[keep], plain[keep])
    ones = torch.ones(m, 256, device="cuda").to(torch.float8_e4m3fn)
    for sa, sw, want in ((100, -90, 256 * 2.0 ** 10), (-126, 127, 512.0), (-120, -20, 256 * 2.0 ** -140), (127, 100, float("inf")), (-126, -126, 0.0)):
        A = ScaledCodes.pack(ones, torch.full((m, 2), 2.0 ** sa, device="cuda"))
        W = ScaledCodes.pack(ones[:1].expand(130, -1).contiguous(), torch.full((130, 2), 2.0 ** sw, dtype=torch.float64, device="cuda").float())
        c = dec.wf_gemm_e4m3(A, W, out_dtype="f32")
        assert (c == want).all() or (abs(want) < 2.0 ** -126 and (c.abs() <= 2.0 ** -126).all()), (sa, sw, c[0, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m", [2, 3000])
def test_gelu_of_special_values(out, m):
    dec = _decoder()
    zero = dec.wf_quantise_e4m3(torch.zeros(m, 128, device="cuda"))
    w = dec.wf_quantise_e4m3(torch.zeros(300, 128, device="cuda"))
    bias = torch.linspace(-9, 9, 300, device="cuda")
    bias[:4] = torch.tensor([float("inf"), float("nan"), 1e30, -1e30])
    got = dec.wf_gemm_e4m3(zero, w, bias=bias, gelu=True, out_dtype=out).double().cpu().numpy()
    assert np.isposinf(got[:, 0]).all() and np.isnan(got[:, 1]).all() and (np.abs(got[:, 2] / 1e30 - 1) <= 2.0 ** -8).all() and (np.abs(got[:, 3]) < 1e-6).all()
    y = O.gelu(bias[4:].double().cpu().numpy()[None])
    tol = (2.0 ** -8 + 2.1e-3) * np.abs(y) + 3e-7 if out == "bf16" else 2e-6 * np.abs(y) + 1e-6
    assert (np.abs(got[:, 4:] - y) <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 1280, 5120), (320, 1280, 5120), (775, 5120, 1280), (6000, 5120, 640)])
def test_repeated_captured_and_on_another_stream(m, n, k):
    """The same bits each time: split channels are added in order, tiles are nobody else's."""
    dec = _decoder()
    x = torch.randn(m, k, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).bfloat16()
    w, bias = _matrix(n, k, 4), torch.randn(n, device="cuda")
    plain = dec.wf_gemm_e4m3(dec.wf_quantise_e4m3(x), w, bias=bias, gelu=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = dec.wf_gemm_e4m3(dec.wf_quantise_e4m3(x), w, bias=bias, gelu=True)
    for _ in range(5):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, plain)
    x.mul_(2)                                                          # what is replayed takes what the memory holds
    graph.replay()
    torch.cuda.synchronize()
    other = dec.wf_gemm_e4m3(dec.wf_quantise_e4m3(x, stream=side), w, bias=bias, gelu=True, stream=side)
    side.synchronize()
    assert torch.equal(got, other) and not torch.equal(got, plain)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 1280, 5120), (64, 5000, 512), (775, 5120, 1280), (5000, 3000, 640)])
def test_a_wait_that_gives_up_leaves_no_plausible_numbers(m, n, k):
    from paper_2412_11272_b200.binding import STATUS_GAVE_UP
    dec = _decoder()
    a, w = _matrix(m, k, 1), _matrix(n, k, 2)
    plain = dec.wf_gemm_e4m3(a, w)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dec.wf_selftest_attention_timeout(True)
    got = dec.wf_gemm_e4m3(a, w, status=status)
    assert got.isnan().all() and int(status) == STATUS_GAVE_UP
    assert dec.wf_gemm_e4m3(a, w).isnan().all()
    dec.wf_selftest_attention_timeout(False)
    status.zero_()
    assert torch.equal(dec.wf_gemm_e4m3(a, w, status=status), plain) and int(status) == 0


@pytest.mark.gpu
def test_nothing_to_multiply():
    dec = _decoder()
    a, w = _matrix(4, 200, 1), _matrix(6, 200, 2)
    assert dec.wf_gemm_e4m3(a[:0], w).shape == (0, 6) and dec.wf_gemm_e4m3(a, w[:0]).shape == (4, 0)
    assert dec.wf_quantise_e4m3(torch.zeros(0, 33, device="cuda")).shape == (0, 33)


def _gelu_bounds(x):
    """For a bfloat16 output, between which values GELU may lie before it is rounded: the fit's relative error, float32 evaluation included, as found
    for 400,001 arguments in float32 (4.7e-6 up to |x| = 4, 7.7e-6 to 5, 5.3e-5 to 7, 3.7e-3 to 8), with 2^-22 of the exponential and 2^-24 of the last
    sum; further down it may fall faster than the function."""
    y, a = O.gelu(x[None])[0], np.abs(x)
    d = np.select([a <= 5, a <= 7, a <= 8], [7.7e-6, 5.3e-5, 3.7e-3], 3.7e-3) + 2.0 ** -22 + 2.0 ** -24
    one, two = y * (1 - d), y * (1 + d)
    one = np.where(x < -8, 0.0, one)
    return np.minimum(one, two), np.maximum(one, two)


@pytest.mark.gpu
@pytest.mark.parametrize("m,pad", [(1, 0), (3, 1), (300, 0), (300, 1), (5000, 0)])
def test_gelu_is_rounded_once(m, pad):
    """Every bfloat16 value of GELU is the rounding of a value as near to the function as the fit is: over its range, in the tail and behind it."""
    dec, n = _decoder(), 4096
    zero = dec.wf_quantise_e4m3(torch.zeros(m, 128, device="cuda"))
    w = dec.wf_quantise_e4m3(torch.zeros(n, 128, device="cuda"))
    bias = torch.linspace(-17.0, 17.0, n)
    bias[:8] = torch.tensor([float("inf"), -float("inf"), float("nan"), 1e30, -1e30, 3e38, -3e38, 0.0])
    out = torch.empty(m, n + pad, device="cuda", dtype=torch.bfloat16)[:, :n]
    got = dec.wf_gemm_e4m3(zero, w, bias=bias.cuda(), gelu=True, out=out).float()
    assert torch.equal(got.nan_to_num(77.0), got[:1].expand(m, n).nan_to_num(77.0))
    first, wide = got[0].cpu(), dec.wf_gemm_e4m3(zero, w, bias=bias.cuda(), gelu=True, out_dtype="f32")[0].cpu()
    for y in (first, wide):
        assert y[0] == float("inf") and y[1].isnan() and y[2].isnan() and y[4] == 0 and y[6] == 0 and y[7] == 0
    assert first[[3, 5]].tolist() == bias[[3, 5]].bfloat16().float().tolist()
    low, high = (torch.from_numpy(b).bfloat16().double().numpy() for b in _gelu_bounds(bias[8:].double().numpy()))
    y = first[8:].double().numpy()
    off = np.flatnonzero((y < low) | (y > high))
    assert not len(off), (len(off), bias[8 + off[0]], y[off[0]], low[off[0]], high[off[0]])


def _one_warp_gives_up(m, n, k, warp, gelu=False):
    """A call in which at first one warp of every block gives up: it ends, says so, and the handle and the next call are as ever."""
    from paper_2412_11272_b200.binding import STATUS_GAVE_UP
    dec = _decoder()
    a, w = _matrix(m, k, 1), _matrix(n, k, 2)
    plain = dec.wf_gemm_e4m3(a, w, gelu=gelu)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = torch.full_like(plain, 77.0)
    dec.wf_selftest_attention_timeout(-1 - warp)
    for _ in range(3):
        got.fill_(77.0)
        dec.wf_gemm_e4m3(a, w, gelu=gelu, out=got, status=status)
    dec.wf_selftest_attention_timeout(False)
    torch.cuda.synchronize()
    assert int(status) == STATUS_GAVE_UP
    status.zero_()
    assert torch.equal(dec.wf_gemm_e4m3(a, w, gelu=gelu, status=status), plain) and int(status) == 0
    return got, plain


@pytest.mark.gpu
@pytest.mark.parametrize("warp", [16, 19, 20, 21])
@pytest.mark.parametrize("m,n,k", [(1, 128, 512), (1, 1280, 5120), (64, 5000, 512), (775, 5120, 1280), (5000, 3000, 640)])
def test_scales_copies_or_products_that_give_up(m, n, k, warp):
    """Scales, copies or products: nothing is computed.  What is in flight when the products give up, every copy of a tile of few
    channels among it, lands before the block has gone."""
    got, _ = _one_warp_gives_up(m, n, k, warp)
    assert got.isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("warp", range(16))
@pytest.mark.parametrize("m,n,k", [(1, 1280, 5120), (64, 5000, 512), (775, 5120, 1280), (5000, 3000, 640)])
def test_a_warp_of_the_epilogue_that_gives_up(m, n, k, warp):
    """One of the warps that read the accumulator gives up, the others find it complete: those that share barriers with it do not wait for it."""
    got, _ = _one_warp_gives_up(m, n, k, warp, gelu=True)
    assert got.isnan().any() or 8 * (warp // 4) >= m  # (warp w reads columns 8 (w / 4) .. of a tile: rows of A, which may not exist)


@pytest.mark.gpu
@pytest.mark.parametrize("warp", [0, 5, 10, 15])
@pytest.mark.parametrize("m,n,k", [(64, 5000, 512), (64, 5120, 512), (100, 1024, 3000), (775, 5120, 1280), (5000, 3000, 640), (4500, 5120, 256)])
def test_every_value_is_written_where_some_warps_give_up(m, n, k, warp):
    """What was not computed is NaN, whatever the other warps of the tile have stored; nothing is left as it was."""
    got, plain = _one_warp_gives_up(m, n, k, warp)
    assert (got.isnan() | (got == plain)).all(), int((got == 77.0).sum())
    assert got.isnan().any() or m < 100                                # (of small tiles not every warp has rows)
