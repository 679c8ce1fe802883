"""wf_draft_verify and wf_draft_commit against the oracle."""
import numpy as np
import pytest

from oracle import speculation_oracle as O

torch = pytest.importorskip("torch")


def _decoder(**kw):
    from paper_2412_11272_b200.binding import Decoder
    return Decoder(**{**dict(n_head=4, d_head=64, dtype="bf16", cache_format="e4m3", page_size=16), **kw})


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda:0", dtype)


# ---- no GPU is needed
def test_oracle_pins():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.8, 0.1], [0.2, 0.2, 0.6]]))
    assert O.draft_verify(x, [9, 1, 2], [-1, 0, 1], [0, 0.2, 0.05], 0.5)[:2] == ([1, 2, 2], [0, 1, 2])
    assert O.draft_verify(x, [9, 1, 2], [-1, 0, 1], [0, 0.2, 0.2], 0.1)[:2] == ([1, 0], [0, 1])
    assert O.draft_verify(x, [9, 1, 2], [-1, 0, 0], [0, 0.3, 0.34], 0.99)[:2] == ([0], [0])                 # 1 refused, then 2 (1/4 of 3/4)
    assert O.draft_verify(x, [9, 1, 2], [-1, 0, 0], [0, 0.3, 0.33], 0.99)[:2] == ([2, 2], [0, 2])
    q = np.array([[0.2, 0.8, 0.0]] * 3)                                                                     # max(p - q, 0) = 0.3, 0, 0.25
    assert O.draft_verify(x, [9, 1], [-1, 0], [0, 0.32], 0.54, draft=q)[:2] == ([0], [0])
    assert O.draft_verify(x, [9, 1], [-1, 0], [0, 0.32], 0.55, draft=q)[:2] == ([2], [0])
    assert O.draft_verify(x, [9, 0, 1], [-1, 0, 1], [0, 0.9, 0.9], 0.9, t=0)[:2] == ([0, 1, 2], [0, 1, 2])
    assert O.draft_verify(np.full((1, 3), np.nan), [0], [-1], [0], 0.5)[:2] == ([-1], [0])


def test_the_procedure_leaves_the_targets_distribution():
    """What speculative sampling promises, for the oracle: the first new token is distributed as the target's own draws."""
    rng = np.random.default_rng(0)
    p, q = np.array([0.5, 0.3, 0.15, 0.05]), np.array([0.1, 0.2, 0.3, 0.4])
    x, n, found = np.log(np.stack([p] * 3)), 20_000, np.zeros((2, 4))
    for _ in range(n):
        drawn = rng.choice(4, 2, p=q)
        u = rng.random(4)
        found[0, O.draft_verify(x, [0, *drawn], [-1, 0, 0], u[:3], u[3], draft=np.stack([q] * 3))[0][0]] += 1
        found[1, O.draft_verify(x, [0, 1, 3], [-1, 0, 0], u[:3], u[3])[0][0]] += 1
    assert (np.abs(found / n - p) < 5 * np.sqrt(p * (1 - p) / n)).all()


def test_verify_refusals():
    from paper_2412_11272_b200.binding import WfError
    d = _decoder()
    P = 1 << 20
    base = dict(h=d.handle, x=P, dt=1, ld=100, V=100, n=2, rows=8, most=4, cu=P, tok=P, par=None, q=None, qld=0, t=None, u=P, last=P, kept=P, out=P, path=P,
                status=None, stream=None)

    def call(**kw):
        a = {**base, **kw}
        return d.lib.wf_draft_verify(*(a[k] for k in base))

    for bad in (dict(h=None), dict(x=None), dict(x=P + 1), dict(dt=0, x=P + 2), dict(dt=2), dict(ld=99), dict(V=0), dict(n=-1), dict(rows=-1), dict(most=0),
                dict(cu=None), dict(tok=None), dict(q=P, qld=99), dict(q=P + 2, qld=100), dict(u=None), dict(last=None), dict(kept=None), dict(out=None),
                dict(path=None)):
        assert call(**bad) == 1, bad
    assert call(most=1025) == 4 and call(n=(1 << 24) + 1) == 4 and call(rows=(1 << 27) + 1) == 4 and call(V=(1 << 28) + 1, ld=1 << 29) == 4 and call(n=0) == 0
    x, z = torch.zeros(4, 100), torch.zeros(4, dtype=torch.int32)
    for make in (lambda: d.wf_draft_verify(x, z, z, x[0], x[0], 4), lambda: d.wf_draft_verify(x.half(), z, z, x[0], x[0], 4)):
        with pytest.raises(WfError) as e:
            make()
        assert e.value.status == "WF_ERR_INVALID_ARG"


def test_commit_refusals():
    from paper_2412_11272_b200 import binding as Bn
    d = _decoder()
    P = 1 << 20
    cache = lambda i: Bn.wf_cache(P + 64 * i, P + 64 * i + 16, P + 64 * i + 32, P + 64 * i + 48, 3)
    one, two, twice = (Bn.wf_cache * 1)(cache(0)), (Bn.wf_cache * 2)(cache(0), cache(1)), (Bn.wf_cache * 2)(cache(0), cache(0))
    other = (Bn.wf_cache * 2)(cache(0), Bn.wf_cache(P + 640, P + 656, P + 672, P + 688, 4))
    base = dict(h=d.handle, n=2, start=P, kept=P, path=P, stride=4, lengths=P + 64, caches=one, nc=1, table=P, ts=3, status=None, stream=None)

    def call(**kw):
        a = {**base, **kw}
        return d.lib.wf_draft_commit(*(a[k] for k in base))

    for bad in (dict(h=None), dict(n=-1), dict(nc=-1), dict(start=None), dict(kept=None), dict(stride=0), dict(lengths=None), dict(lengths=P + 4), dict(kept=P + 68), dict(caches=None),
                dict(table=None), dict(ts=0), dict(caches=twice, nc=2), dict(caches=other, nc=2), dict(caches=(Bn.wf_cache * 1)(Bn.wf_cache(P, P, P, P + 16, 3)))):
        assert call(**bad) == 1, bad
    assert call(n=65536) == 4 and call(stride=1025) == 4 and call(n=0) == 0 and call(n=0, caches=two, nc=2) == 0


# ---- verification on the GPU
def _run(dec, logits, rows, tokens, parents, u, u_last, t=None, draft=None, max_rows=None, ld_pad=0, offset=0, q_pad=0):
    """Calls the operator on logits that lie inside wider rows, and compares every sequence with the oracle."""
    n, V = logits.shape
    wide = torch.full((n, V + ld_pad + offset), 1e9, device="cuda").to(logits.dtype)
    wide[:, offset:offset + V] = logits
    cu = np.concatenate([[0], np.cumsum(rows)])
    most = max_rows or max([1, *rows])
    q = None
    if draft is not None:
        q = torch.full((n, V + q_pad), 7.0, device="cuda")[:, :V]
        q.copy_(draft)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kept, out, path = (x.cpu().numpy() for x in dec.wf_draft_verify(
        wide[:, offset:offset + V], _dev(cu), _dev(tokens), _dev(u, torch.float32), _dev(u_last, torch.float32), most,
        parents=None if parents is None else _dev(parents), draft=q, temperature=None if t is None else _dev(t, torch.float32), status=status))
    x, undecided = logits.double().cpu().numpy(), 0
    dq = None if draft is None else draft.double().cpu().numpy()
    u, u_last = np.asarray(u, np.float32), np.asarray(u_last, np.float32)
    for b in range(len(rows)):
        r = slice(cu[b], cu[b + 1])
        up = np.arange(-1, rows[b] - 1) if parents is None else np.asarray(parents)[r]
        want, stay, margin = O.draft_verify(x[r], np.asarray(tokens)[r], up, u[r], u_last[b], 1.0 if t is None else float(np.float32(t[b])),
                                            None if dq is None else dq[r])
        if margin < 20:  # within 2e-5 of a decision or 2e-10 of a border between tokens: the float32 sum, or its 64 bits, may decide otherwise
            undecided += 1
            continue
        m = len(stay)
        assert kept[b] == m and out[b].tolist() == want + [-1] * (most - m) and path[b].tolist() == stay + [-1] * (most - m), (b, want, stay, out[b], path[b])
    assert undecided <= max(2, len(rows) // 20)
    return int(status)


def _batch(rng, rows, V, tree, drawn, dtype, siblings=3):
    """Peaked logits, drafts of a model that thinks alike, random numbers."""
    n = int(sum(rows))
    g = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
    x = 1.5 * torch.randn(n, V, generator=g, device="cuda")
    if V > 16:
        x.scatter_(1, torch.randint(0, V, (n, 6), generator=g, device="cuda"), 5.0 + 4.0 * torch.rand(n, 6, generator=g, device="cuda"))
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q = torch.softmax(x.float() + 0.8 * torch.randn(n, V, generator=g, device="cuda"), 1)
    cu = np.concatenate([[0], np.cumsum(rows)])
    parents, tokens = np.full(n, -1), np.zeros(n, np.int64)
    best = torch.topk(q, min(V, siblings), dim=1).indices.cpu().numpy()
    for b, m in enumerate(rows):
        for i in range(1, m):
            up = int(rng.integers(max(0, i - 1 - siblings), i)) if tree else i - 1
            parents[cu[b] + i] = up
            tokens[cu[b] + i] = best[cu[b] + up, rng.integers(0, best.shape[1])]
    if drawn and n:
        at = torch.as_tensor(np.clip(parents, 0, None) + np.repeat(cu[:-1], rows), device="cuda")
        tokens = torch.multinomial(q[at], 1, generator=g).view(-1).cpu().numpy()
    return x, tokens, (parents if tree else None), rng.random(n).astype(np.float32), rng.random(len(rows)).astype(np.float32), (q if drawn else None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("V", [1, 2, 31, 257, 1000, 4099, 50_021])
def test_vocabularies_of_any_size(dtype, tree, drawn, V):
    rng = np.random.default_rng(V)
    rows = [1, 4, 0, 9, 2, 17, 6] if V < 10_000 else [5, 0, 3]
    x, tok, up, u, last, q = _batch(rng, rows, V, tree, drawn, dtype)
    assert _run(_decoder(), x, rows, tok, up, u, last, t=rng.choice([0.0, 0.5, 1.0, 1.7], len(rows)), draft=q) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n_seq", [1, 3, 20, 40, 100, 200])
@pytest.mark.parametrize("drawn", [False, True])
def test_batches_of_any_size(n_seq, drawn):
    """The sizes that choose clusters of eight blocks down to one."""
    rng = np.random.default_rng(n_seq)
    rows = rng.integers(0, 6, n_seq)
    x, tok, up, u, last, q = _batch(rng, rows, 20_011, True, drawn, "bf16")
    assert _run(_decoder(), x, rows.tolist(), tok, up, u, last, draft=q) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,V", [("bf16", 300_007), ("f32", 300_007), ("f32", 1_000_003)])
def test_vocabularies_that_no_block_holds(dtype, V):
    rng = np.random.default_rng(3)
    x, tok, up, u, last, q = _batch(rng, [5, 3], V, True, True, dtype, siblings=4)
    for draft in (q, None):
        assert _run(_decoder(), x, [5, 3], tok, up, u, last, t=[1.0, 0.8], draft=draft) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,offset,q_pad", [(0, 0, 1), (1, 1, 0), (3, 5, 2), (8, 8, 4), (7, 2, 3)])
def test_rows_at_any_alignment(dtype, pad, offset, q_pad):
    rng = np.random.default_rng(pad)
    rows = [6, 3, 1, 8]
    x, tok, up, u, last, q = _batch(rng, rows, 1003, True, True, dtype)
    assert _run(_decoder(), x, rows, tok, up, u, last, draft=q, ld_pad=pad, offset=offset, q_pad=q_pad) == 0


@pytest.mark.gpu
def test_many_drafts():
    """Hundreds of siblings and long chains; every draft of a row refused one after the other."""
    rng = np.random.default_rng(9)
    dec, V, n = _decoder(), 800, 1024
    x, _, _, u, last, _ = _batch(rng, [n, 600], V, True, False, "f32")
    star = np.concatenate([[-1], np.zeros(n - 1), [-1], np.zeros(599)])
    tok = rng.integers(0, V, n + 600)
    u[:] = 1.0 - 2.0 ** -24                                                          # the largest: refused unless p is all there is
    assert _run(dec, x, [n, 600], tok, star, u, last) == 0
    q = torch.softmax(torch.randn(n + 600, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)), 1)
    assert _run(dec, x[:300], [200, 100], tok[:300], np.concatenate([star[:200], star[:100]]), u[:300], last, draft=q[:300]) == 0
    u[:] = 0.0                                                                       # kept wherever p is not zero
    assert _run(dec, x, [n, 600], tok, None, u, last) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_special_values(dtype):
    """Rows without a distribution, tokens of probability zero, equal logits, extreme temperatures, random numbers at the ends."""
    dec, V = _decoder(), 70
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    inf, nan = float("inf"), float("nan")
    x = torch.randn(24, V, generator=torch.Generator().manual_seed(4)).to(tt).cuda()
    x[0, 69] = nan                  # 0: no distribution from the start
    x[2, :] = -inf                  # 1: nothing but -infinity at the second row
    x[2, 5] = -inf
    x[5, 3] = inf                   # 2: +infinity behind the first draft
    x[6, :] = -inf                  # 3: all on one token
    x[6, 11] = -3e38
    x[8, :] = 2.0                   # 4: equals, greedy takes the lowest
    x[10, 7] = -inf                 # 5: a draft of probability zero
    x[12, :] = -inf                 # 6: two tokens, at the first and last place
    x[12, 0], x[12, 69] = 1.0, 1.0
    x[14, :] = 30.0                 # 7 and 8: a temperature near the ends of float32
    x[14, 40] = 31.0
    x[16, 33] = 60.0
    rows = [2] * 12
    tok = np.tile([0, 5], 12)
    tok[[5, 7, 9, 11, 13, 15, 17]] = [4, 11, 0, 7, 69, 40, 33]
    t = np.ones(12, np.float32)
    t[4], t[7], t[8] = 0.0, 1e-38, 1e38
    u, last = np.full(24, 0.25, np.float32), np.full(12, 0.5, np.float32)
    last[[6, 9, 10, 11]] = [0.4999, 0.0, 1.0 - 2.0 ** -24, 0.3]
    assert _run(dec, x, rows, tok, None, u, last, t=t) == 0
    u[:] = 1.0 - 2.0 ** -24
    assert _run(dec, x, rows, tok, None, u, last, t=t) == 0
    last[:] = 0.0
    assert _run(dec, x, rows, tok, None, u, last, t=t) == 0
    # the target's own draws are kept; a draft's distribution that leaves nothing is passed over; one that was never to draw the token too
    clean = x[18:24]
    p = torch.softmax(clean.float(), 1)
    for q, u1 in ((p, 0.99), (torch.full_like(p, 3.0), 0.9), (torch.zeros_like(p), 0.9)):
        assert _run(dec, clean, [3, 3], [0, 3, 9, 0, 1, 2], None, np.full(6, u1), [0.3, 0.7], draft=q) == 0


@pytest.mark.gpu
def test_what_does_not_fit():
    from paper_2412_11272_b200.binding import STATUS_BAD_PARENT, STATUS_BAD_ROWS, STATUS_BAD_VALUE
    rng = np.random.default_rng(1)
    dec, V = _decoder(), 300
    x, tok, up, u, last, _ = _batch(rng, [6, 6, 6], V, True, False, "f32")
    u[:] = 0
    bad = up.copy()
    bad[[2, 8, 15]] = [2, 77, -5]
    assert _run(dec, x, [6, 6, 6], tok, bad, u, last) == STATUS_BAD_PARENT
    worse = tok.copy()
    worse[[1, 9]] = [V, -1]
    assert _run(dec, x, [6, 6, 6], worse, up, u, last) == STATUS_BAD_VALUE
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (_dev(tok), _dev(u, torch.float32), _dev(last, torch.float32))
    for t in (-1.0, float("nan"), float("inf")):
        status.zero_()
        kept, out, path = dec.wf_draft_verify(x, _dev([0, 6, 12, 18]), *args, 6, temperature=_dev([1, t, 1], torch.float32), status=status)
        assert int(status) == STATUS_BAD_VALUE and kept[1] == 0 and (out[1] == -1).all() and (path[1] == -1).all() and kept[0] > 0 and kept[2] > 0
    for cu in ([0, 6, 5, 18], [-1, 6, 12, 18], [0, 6, 12, 19], [0, 6, 2 ** 31 - 1, 18]):
        status.zero_()
        kept, out, path = dec.wf_draft_verify(x, _dev(cu), *args, 6, status=status)
        assert int(status) & STATUS_BAD_ROWS and (kept >= 0).all() and (kept <= 6).all()
    status.zero_()
    kept, out, path = dec.wf_draft_verify(x, _dev([0, 6, 12, 18]), *args, 3, status=status)  # longer ones are cut
    assert int(status) == STATUS_BAD_ROWS and (kept <= 3).all()


@pytest.mark.gpu
def test_drawn_tokens_have_the_targets_distribution():
    """Many sequences of one row each and of drawn drafts: the first new token's frequencies are the target's."""
    dec, V, n = _decoder(), 6, 40_000
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.tensor([1.0, -0.5, 0.3, 2.0, -2.0, 0.0], device="cuda")
    q = torch.tensor([0.3, 0.1, 0.1, 0.1, 0.2, 0.2], device="cuda")
    p = torch.softmax(x.double() / 0.8, 0).cpu().numpy()
    for rows, draft in ((1, None), (3, q), (3, None)):
        tok = torch.multinomial(q.expand(n * rows, V), 1, generator=g).view(-1).int()
        up = torch.zeros(n, rows, dtype=torch.int32, device="cuda")
        kept, out, _ = dec.wf_draft_verify(x.expand(n * rows, V).contiguous(), torch.arange(0, n * rows + 1, rows, device="cuda", dtype=torch.int32), tok,
                                           torch.rand(n * rows, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda"), rows,
                                           parents=up.view(-1), draft=None if draft is None else draft.expand(n * rows, V).contiguous(),
                                           temperature=torch.full((n,), 0.8, device="cuda"))
        found = torch.bincount(out[:, 0], minlength=V).cpu().numpy() / n
        assert (np.abs(found - p) < 5 * np.sqrt(p * (1 - p) / n)).all()


@pytest.mark.gpu
def test_verify_captured_and_on_another_stream():
    rng = np.random.default_rng(6)
    dec, rows = _decoder(), [5, 3, 7]
    cu = _dev([0, 5, 8, 15])
    batches = [_batch(rng, rows, 2003, False, True, "bf16") for _ in range(3)]
    x, tok, _, u, last, q = batches[0]
    held = [x.clone(), _dev(tok), _dev(u, torch.float32), _dev(last, torch.float32), q.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = dec.wf_draft_verify(held[0], cu, held[1], held[2], held[3], 7, draft=held[4])
    for x, tok, _, u, last, q in batches:
        for a, b in zip(held, (x, _dev(tok), _dev(u, torch.float32), _dev(last, torch.float32), q)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            plain = dec.wf_draft_verify(x, cu, _dev(tok), _dev(u, torch.float32), _dev(last, torch.float32), 7, draft=q, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, plain))
        assert _run(dec, x, rows, tok, None, u, last, draft=q) == 0


# ---- commit on the GPU
@pytest.mark.gpu
@pytest.mark.parametrize("fmt,dtype,d,heads,page", [("e4m3", "bf16", 64, 5, 16), ("int8", "bf16", 128, 2, 64), ("path", "bf16", 64, 3, 32), ("path", "f32", 128, 1, 256)])
@pytest.mark.parametrize("layers", [1, 3, 70])
def test_commit(fmt, dtype, d, heads, page, layers):
    """All layers' rows move; what lies elsewhere stays bit for bit; lengths in place and beside."""
    rng = np.random.default_rng(layers)
    dec = _decoder(n_head=heads, d_head=d, dtype=dtype, cache_format=fmt, page_size=page)
    n_seq, most = 7, 40
    start = rng.integers(0, 3 * page, n_seq)
    paths = [[0], [0, 1, 2], [0, 3, 4, 39], [], [0] + sorted(rng.choice(np.arange(1, 40), 20, replace=False).tolist()), list(range(40)),
             [0] + sorted(rng.choice(np.arange(2, 40), 30, replace=False).tolist())]
    pages = [-(-(s + most) // page) for s in start]
    table = np.full((n_seq, max(pages)), -1)
    order = rng.permutation(sum(pages) + 3)
    for b, k in enumerate(pages):
        table[b, :k] = order[sum(pages[:b]):sum(pages[:b]) + k]
    n_pages = sum(pages) + 3
    g = torch.Generator(device="cuda").manual_seed(layers)
    caches, want = [], []
    for _ in range(layers):
        c = dec.cache(n_pages)
        sides = [c.k, c.v] + ([] if fmt == "path" else [c.k_scale, c.v_scale])
        for t in sides:
            flat = t.view(torch.uint8)
            flat.copy_(torch.randint(0, 127, flat.shape, generator=g, device="cuda", dtype=torch.uint8))
        caches.append(c)
        true = [t.view(torch.uint8).cpu().numpy().reshape(n_pages, heads, page, -1).copy() for t in sides]
        for t in true:
            for b in range(n_seq):
                O.commit(t, table[b], start[b], paths[b], page)
        want.append(true)
    path = np.full((n_seq, most), -1)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    kept, status = _dev([len(p) for p in paths]), torch.zeros(1, dtype=torch.int32, device="cuda")
    first = _dev(start)
    in_place = first.clone()
    got = dec.wf_draft_commit(first, kept, _dev(path), caches=caches, page_table=_dev(table), status=status)
    assert got.tolist() == [s + len(p) for s, p in zip(start, paths)] and int(status) == 0 and first.tolist() == start.tolist()
    for c, true in zip(caches, want):
        for t, w in zip([c.k, c.v] + ([] if fmt == "path" else [c.k_scale, c.v_scale]), true):
            assert np.array_equal(t.view(torch.uint8).cpu().numpy().reshape(w.shape), w)
    # rows that lie as they should: nothing moves, in place
    before = [c.k.clone() for c in caches[:1]]
    out = dec.wf_draft_commit(in_place, kept, caches=caches[:1], page_table=_dev(table), lengths=in_place)
    assert out is in_place and in_place.tolist() == got.tolist() and torch.equal(before[0].view(torch.uint8), caches[0].k.view(torch.uint8))
    assert dec.wf_draft_commit(first, kept).tolist() == got.tolist()
    again = first.clone()
    dec.wf_draft_commit(again, kept, _dev(path), caches=caches, page_table=_dev(table), lengths=again)     # the moves read start before it changes
    assert again.tolist() == got.tolist()


@pytest.mark.gpu
def test_commit_of_what_does_not_fit():
    """Nothing outside the rows' own places is written, and each kind is reported."""
    dec = _decoder(n_head=2, cache_format="path", page_size=16)
    cache = dec.cache(4)
    cache.k.normal_()
    cache.v.normal_()
    k, v = cache.k.clone(), cache.v.clone()
    for table, start, kept, path, bits in (
            ([[0, 1]], [3], [3], [[0, 2, 2]], 4),                # not above the one before
            ([[0, 1]], [3], [3], [[0, 0, 1]], 4),
            ([[0, 1]], [3], [2], [[0, -9]], 4),
            ([[0, 1]], [30], [2], [[0, 2]], 2),                  # beyond the table
            ([[0, 1]], [3], [2], [[0, 2 ** 31 - 1]], 2),
            ([[0, 4]], [15], [2], [[0, 3]], 1),                  # pages that do not exist
            ([[-1, 1]], [14], [2], [[0, 9]], 1),
            ([[0, 1]], [3], [-1], [[0, 5]], 2),
            ([[0, 1]], [3], [3], [[0, 5]], 2),                   # more than the path has
            ([[0, 1]], [-4], [2], [[0, 5]], 2),
            ([[0, 1]], [2 ** 31 - 2], [2], [[0, 5]], 2)):
        for in_place in (False, True):
            cache.k.copy_(k)
            cache.v.copy_(v)
            status, first = torch.zeros(1, dtype=torch.int32, device="cuda"), _dev(start)
            got = dec.wf_draft_commit(first, _dev(kept), _dev(path), caches=[cache], page_table=_dev(table), lengths=first if in_place else None, status=status)
            assert int(status) & bits and int(status) & ~bits in (0, 2), (table, start, kept, path, int(status))
            if path[0][:2] == [0, 2]:
                continue                                         # (the second row of those did move)
            assert torch.equal(cache.k, k) and torch.equal(cache.v, v)
            assert got.tolist() == ([start[0]] if bits == 2 and (kept[0] in (-1, 3) or abs(start[0]) > 30 or start[0] < 0) and path != [[0, 2]] else [start[0] + kept[0]])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2, 70, 5000, 50_021])
def test_zeros_of_both_signs_are_equal(dtype, V):
    """The largest logit is zero and occurs with either sign, in one lane, in several, in other warps: the lowest index, greedy or not."""
    rng = np.random.default_rng(V)
    dec, n = _decoder(), 24
    x = -1.0 - torch.rand(n, V, generator=torch.Generator().manual_seed(V))
    tok = np.zeros(n, np.int64)
    for r in range(n):
        at = np.sort(rng.choice(V, min(V, 2 + r % 5), replace=False))
        x[r, at] = torch.tensor([-0.0 if (i + r // 2) % 2 == 0 else 0.0 for i in range(len(at))])
        if r % 2 == 0:
            tok[r + 1] = at[0 if r % 4 == 0 else -1]                 # the draft behind it: the first of the equals, or another one
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    for t in (0.0, 1.0):
        assert _run(dec, x, [2] * (n // 2), tok, None, rng.random(n), rng.random(n // 2), t=[t] * (n // 2)) == 0


def _near(rng, value):
    """A float32 random number within a few steps of `value`, on either side."""
    u = np.float32(min(max(value, 0.0), 1.0 - 2.0 ** -24))
    for _ in range(int(rng.integers(1, 6))):
        u = np.nextafter(u, np.float32(rng.integers(0, 2)))
    return float(min(max(u, np.float32(0)), np.float32(1.0 - 2.0 ** -24)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("V,n_seq", [(40, 12), (3000, 12), (50_021, 8), (300_007, 2)])
def test_decisions_next_to_a_border(dtype, drawn, V, n_seq):
    """Random numbers a few float32 steps beside the probability that they are compared with, for a first child and behind up to seven refusals that
    leave a thousandth of p or less each: decided as in float64."""
    rng = np.random.default_rng(V + n_seq)
    dec, kids, t = _decoder(), 9, 0.75
    rows = [kids] * n_seq
    n, tokens, u = sum(rows), np.zeros(sum(rows), np.int64), np.full(sum(rows), 1.0 - 2.0 ** -24)
    g = torch.Generator().manual_seed(V)
    x = 0.5 * torch.randn(n, V, generator=g) - 40.0
    at = [rng.choice(V, kids, replace=False) for _ in range(n_seq)]
    for b in range(n_seq):
        x[kids * b, at[b]] = torch.tensor([8.0 - i * rng.uniform(1.0, 5.5) for i in range(kids)], dtype=torch.float32)
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q = torch.softmax(x.float() / t + 0.3 * torch.randn(n, V, generator=g), 1) if drawn else None
    for b in range(n_seq):
        i0, depth = kids * b, b % 8 if not drawn else b % 4              # the child whose number lies at the border
        p, qd = O.distribution(x[i0].double().numpy(), np.float32(t)), None if q is None else q[i0].double().numpy()
        order = at[b] if not drawn else rng.choice(at[b], kids)
        tokens[i0 + 1:i0 + kids] = order[:kids - 1]
        for c in range(kids - 1):
            v = int(order[c])
            border = p[v] / (1.0 if qd is None else qd[v])
            if c == depth:
                u[i0 + 1 + c] = _near(rng, border)
                break
            u[i0 + 1 + c] = min(1.0 - 2.0 ** -24, border * 1.5 + 1e-3)
            rest = np.where(np.arange(V) == v, 0.0, p) if qd is None else np.maximum(p - qd, 0.0)
            if np.float32(u[i0 + 1 + c]) * (1.0 if qd is None else qd[v]) >= p[v] and rest.sum() > 0:
                p = rest / rest.sum()
    u, last = u.astype(np.float32), rng.random(n_seq).astype(np.float32)
    star = np.tile([-1] + [0] * (kids - 1), n_seq)
    kept, out, path = (y.cpu().numpy() for y in dec.wf_draft_verify(
        x.cuda(), _dev(np.arange(0, n + 1, kids)), _dev(tokens), _dev(u, torch.float32), _dev(last, torch.float32), kids, parents=_dev(star),
        draft=None if q is None else q.cuda(), temperature=_dev([t] * n_seq, torch.float32)))
    decided = 0
    for b in range(n_seq):
        r = slice(kids * b, kids * (b + 1))
        want, stay, margin = O.draft_verify(x[r].double().numpy(), tokens[r], star[r], u[r], last[b], float(np.float32(t)), None if q is None else q[r].double().numpy())
        if margin < 1e-3:                                              # 1e-9 of a probability: beyond the 64 bits of a small rest
            continue
        decided += 1
        assert kept[b] == len(stay) and out[b, :len(want)].tolist() == want and path[b, :len(stay)].tolist() == stay, (b, want, stay, out[b], path[b], margin)
    assert decided >= n_seq / 2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,V", [("bf16", 300_007), ("f32", 300_007), ("f32", 1_000_003), ("bf16", 50_021)])
@pytest.mark.parametrize("drawn", [False, True])
def test_few_sequences_and_none_left_out(dtype, V, drawn):
    """Two or three sequences of large vocabularies, each of them compared: no decision lies within 1e-9 of its border."""
    rng = np.random.default_rng(V)
    rows = [5, 3] if V > 100_000 else [6, 1, 4]
    x, tok, up, u, last, q = _batch(rng, rows, V, True, drawn, dtype, siblings=4)
    t, cu = [1.0, 0.8, 0.6][:len(rows)], np.concatenate([[0], np.cumsum(rows)])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kept, out, path = (y.cpu().numpy() for y in _decoder().wf_draft_verify(
        x, _dev(cu), _dev(tok), _dev(u, torch.float32), _dev(last, torch.float32), max(rows), parents=_dev(up), draft=q,
        temperature=_dev(t, torch.float32), status=status))
    assert int(status) == 0
    for b, m in enumerate(rows):
        r = slice(cu[b], cu[b + 1])
        want, stay, margin = O.draft_verify(x[r].double().cpu().numpy(), tok[r], up[r], u[r], last[b], float(np.float32(t[b])),
                                            None if q is None else q[r].double().cpu().numpy())
        k = len(stay)
        assert margin >= 1e-3 and kept[b] == k, (b, margin, kept[b], k)
        assert out[b].tolist() == want + [-1] * (max(rows) - k) and path[b].tolist() == stay + [-1] * (max(rows) - k), (b, want, out[b])


@pytest.mark.gpu
def test_commit_reports_rows_that_stay_without_a_place():
    """A row that need not move has a place too: behind the table, or in a page that does not exist, it is reported, and nothing else changes."""
    dec = _decoder(n_head=2, cache_format="path", page_size=16)
    cache = dec.cache(4)
    cache.k.normal_()
    cache.v.normal_()
    k, v = cache.k.clone(), cache.v.clone()
    for table, start, kept, path, bits in (
            ([[0, 1]], [30], [2], [[0, 1]], 0), ([[0, 1]], [31], [2], [[0, 1]], 2), ([[0, 1]], [32], [1], [[0, 7]], 2), ([[0, 1]], [40], [0], [[0, 1]], 0),
            ([[0, -1]], [15], [1], [[0, 1]], 0), ([[0, -1]], [15], [2], [[0, 1]], 1), ([[0, 4]], [16], [1], [[0, 1]], 1),
            ([[0, 1]], [30], [2], None, 0), ([[0, 1]], [30], [3], None, 2), ([[0, 1]], [33], [0], None, 0), ([[0, 1]], [2 ** 31 - 9], [9], None, 2)):
        for in_place in (False, True):
            for caches in ([cache], []):
                status, first = torch.zeros(1, dtype=torch.int32, device="cuda"), _dev(start)
                got = dec.wf_draft_commit(first, _dev(kept), None if path is None else _dev(path), caches=caches, page_table=_dev(table),
                                          lengths=first if in_place else None, status=status)
                want = bits if caches else bits & 2                    # (without caches no page is looked at)
                assert int(status) == want and got.tolist() == [min(start[0] + kept[0], 2 ** 31 - 1) if start[0] + kept[0] < 2 ** 31 else start[0]], \
                    (table, start, kept, path, bool(caches), int(status), got.tolist())
                assert torch.equal(cache.k, k) and torch.equal(cache.v, v)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert dec.wf_draft_commit(_dev([500]), _dev([9]), status=status).tolist() == [509] and int(status) == 0   # no table: nothing to compare with


@pytest.mark.gpu
def test_commit_refuses_a_path_without_rows():
    """A path of no columns is not the same as none (with which all kept rows count)."""
    from paper_2412_11272_b200.binding import WfError
    first, kept = _dev([3, 5]), _dev([2, 1])
    with pytest.raises(WfError) as e:
        _decoder().wf_draft_commit(first, kept, torch.empty(2, 0, dtype=torch.int32, device="cuda"))
    assert e.value.status == "WF_ERR_INVALID_ARG"
    assert _decoder().wf_draft_commit(first, kept, torch.zeros(2, 1, dtype=torch.int32, device="cuda")).tolist() == [3, 6]  # two of one row: none


@pytest.mark.gpu
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("V", [70, 9000])
def test_logits_further_apart_than_float32_holds(drawn, V):
    """Temperatures at which logits of -3e38 beside one of 3e38 have weight: every one of them counts."""
    rng = np.random.default_rng(V)
    n = 16
    x = torch.full((4 * n, V), -3e38)
    x[:, 3], x[::2, 5] = 3e38, 1e38
    tok = np.tile([0, 3, 5, 9], n)
    t = (10.0 ** rng.uniform(37.3, 38.5, n)).astype(np.float32)
    q = torch.rand(4 * n, V, generator=torch.Generator().manual_seed(1)) if drawn else None
    q = None if q is None else (q / q.sum(1, keepdim=True)).cuda()
    u = rng.random(4 * n)
    if not drawn:
        for b in range(n):                                             # beside the border of the first child, where the rest's weight decides
            u[4 * b + 1] = min(O.distribution(x[4 * b].double().numpy(), t[b])[3] * rng.choice([0.98, 1.02]), 0.999)
    assert _run(_decoder(), x.cuda(), [4] * n, tok, np.tile([-1, 0, 0, 0], n), u, rng.random(n), t=t, draft=q) == 0


@pytest.mark.gpu
def test_logits_that_differ_by_subnormal_numbers():
    """Temperatures whose reciprocal float32 does not hold: logits of 0 and -1e-40 differ."""
    n, V = 12, 300
    x = torch.full((2 * n, V), -1e-40)
    x[:, 3] = 0.0
    t = np.tile([1e-39, 1e-40, 1e-42, 1e-45], 3).astype(np.float32)
    u = np.full(2 * n, 0.5)
    for b in range(n):
        u[2 * b + 1] = min(O.distribution(x[2 * b].double().numpy(), float(t[b]))[3] * (0.98, 1.02)[b % 2], 0.999)
    assert _run(_decoder(), x.cuda(), [2] * n, np.tile([0, 3], n), None, u, np.linspace(0.1, 0.9, n), t=t) == 0
