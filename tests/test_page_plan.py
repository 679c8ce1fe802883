"""wf_page_plan against the oracle: sequences that come and go, pools and batches that are too small, numbers that do not fit."""
import numpy as np
import pytest

from oracle import speculation_oracle as O

torch = pytest.importorskip("torch")


def _decoder(page=16):
    from paper_2412_11272_b200.binding import Decoder
    return Decoder(n_head=1, d_head=64, page_size=page)


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda:0", dtype)


# ---- no GPU is needed
def test_oracle_pins():
    ring, table, held, lengths = [7, 8, 9, 5, 6], [[3, -1, -1], [4, -1, -1], [-1, -1, -1]], [1, 1, 0], [16, 3, 0]
    head, count, cu, seq, pos, slot, off = O.page_plan(ring, 3, 3, table, held, lengths, [2, 1, 17], 20, 16, [0, 1, 0])
    # sequence 0 needs a page (5), 1 gives its page back and takes another one (6), 2 asks for two where one is left
    assert table == [[3, 5, -1], [6, -1, -1], [-1, -1, -1]] and held == [2, 1, 0] and lengths == [16, 0, 0] and off == [2]
    assert (head, count) == (0, 2) and ring == [7, 4, 9, 5, 6] and cu.tolist() == [0, 2, 3, 3]
    assert slot[:4].tolist() == [80, 81, 96, -1] and pos[:4].tolist() == [16, 17, 0, -1] and seq[:4].tolist() == [0, 0, 1, -1]


def test_refusals():
    from paper_2412_11272_b200 import binding as Bn
    d = _decoder()
    P = 1 << 20
    base = dict(h=d.handle, pool=Bn.wf_page_pool(P, P, 5), n=2, new=P, ended=None, len=P, held=P, table=P, stride=4, rows=8, cu=P, seq=P, pos=P, slot=P,
                status=None, stream=None)

    def call(**kw):
        a = {**base, **kw}
        return d.lib.wf_page_plan(*(a[k] for k in base))

    for bad in (dict(h=None), dict(pool=None), dict(pool=Bn.wf_page_pool(None, P, 5)), dict(pool=Bn.wf_page_pool(P, None, 5)),
                dict(pool=Bn.wf_page_pool(P, P, 0)), dict(n=-1), dict(rows=-1), dict(new=None), dict(len=None), dict(held=None), dict(table=None),
                dict(stride=0), dict(cu=None)):
        assert call(**bad) == 1, bad
    assert call(n=8193) == 4 and call(rows=(1 << 27) + 1) == 4 and "8192 sequences" in d.lib.wf_decoder_last_error(d.handle).decode()
    pool = Bn.PagePool(torch.arange(4, dtype=torch.int32), torch.tensor([0, 4], dtype=torch.int32))
    z = torch.zeros(2, dtype=torch.int32)
    for make in (lambda: Bn.PagePool(torch.arange(4), torch.zeros(2, dtype=torch.int32)), lambda: Bn.PagePool(torch.arange(4, dtype=torch.int32), z[:1]),
                 lambda: d.wf_page_plan(pool, torch.zeros(2, 3, dtype=torch.int32), z, z, z, 4)):
        with pytest.raises(Bn.WfError) as e:
            make()
        assert e.value.status == "WF_ERR_INVALID_ARG"


# ---- on the GPU
class _State:
    """A batch's pages as they should be, beside the device's."""

    def __init__(self, rng, n_seq, stride, n_pages, lengths, page):
        self.page, self.n_pages = page, n_pages
        self.lengths = np.array(lengths)
        self.held = np.minimum(-(-self.lengths // page) + rng.integers(0, 2, n_seq), stride)
        order = rng.permutation(n_pages)
        self.table = np.full((n_seq, stride), -1)
        at = 0
        for s, h in enumerate(self.held):
            self.table[s, :h] = order[at:at + h]
            at += h
        self.head, self.count = int(rng.integers(0, n_pages)), n_pages - at
        self.ring = np.full(n_pages, -7)
        self.ring[(self.head + np.arange(self.count)) % n_pages] = order[at:]

    def device(self):
        from paper_2412_11272_b200.binding import PagePool
        return (PagePool(_dev(self.ring), _dev([self.head, self.count])), _dev(self.table), _dev(self.held), _dev(self.lengths))

    def plan(self, new, rows, ended):
        out = O.page_plan(self.ring, self.head, self.count, self.table, self.held, self.lengths, new, rows, self.page, ended)
        self.head, self.count = out[:2]
        return out[2:]

    def check(self, dev, got, want, status):
        pool, table, held, lengths = dev
        assert pool.state.tolist() == [self.head, self.count]
        for g, w in ((table, self.table), (held, self.held), (lengths, self.lengths), (got[0], want[0]), (got[1], want[1]), (got[2], want[2]),
                     (got[3], want[3])):
            assert np.array_equal(g.cpu().numpy(), w)
        free = self.ring[(self.head + np.arange(self.count)) % self.n_pages]
        assert np.array_equal(pool.pages.cpu().numpy()[(self.head + np.arange(self.count)) % self.n_pages], free)
        owned = np.concatenate([self.table[s, :h] for s, h in enumerate(self.held)] + [free])
        assert len(np.unique(owned)) == len(owned) == self.n_pages                          # no page is lost and none has two owners
        assert int(status) == (16 if want[4] else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("n_seq,most,page,rows,pages", [
    (1, 1, 16, 1, 1.0), (1, 5000, 16, 6000, 1.0), (3, 40, 32, 200, 0.5), (64, 1, 16, 64, 1.0), (100, 30, 16, 700, 0.4), (300, 9, 64, 5000, 1.0),
    (1000, 3, 256, 1500, 1.0), (8192, 1, 16, 9000, 1.0), (37, 900, 128, 12_000, 0.6)])
def test_rounds(n_seq, most, page, rows, pages):
    """Rounds one after another: rows and pages of one are the next one's state; some sequences end and give their pages back."""
    rng = np.random.default_rng(n_seq + page)
    dec = _decoder(page)
    stride = 4 + -(-(3 * most + 100) // page)
    lengths = rng.integers(0, 100, n_seq) * (rng.random(n_seq) < 0.7)
    st = _State(rng, n_seq, stride, int(n_seq * stride * pages) + int(sum(-(-lengths // page) + 1)), lengths, page)
    dev = st.device()
    pool, table, held, length = dev
    for turn in range(4):
        new = rng.integers(0, most + 1, n_seq)
        ended = (rng.random(n_seq) < 0.3) if turn else None
        if ended is None:
            new = np.minimum(new, stride * page - st.lengths)
        else:
            new = np.minimum(new, np.where(ended, stride * page, stride * page - st.lengths))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = dec.wf_page_plan(pool, table, held, length, _dev(new), rows, ended=None if ended is None else _dev(ended, torch.bool), status=status)
        want = st.plan(new, rows, ended)
        st.check(dev, got, want, status)
        grown = np.diff(want[0])                                                            # every row stays
        st.lengths = st.lengths + grown
        length += got[0][1:] - got[0][:-1]


@pytest.mark.gpu
def test_numbers_that_do_not_fit():
    """A sequence that does not fit is left as it is and gets no rows; the others get theirs; a pool that does not fit gives and takes nothing."""
    from paper_2412_11272_b200.binding import PagePool
    dec = _decoder(16)
    good = dict(lengths=[5, 20, 0], held=[1, 2, 0], new=[3, 4, 5])
    for name, values in (("lengths", [5, -1, 0]), ("lengths", [5, 33, 0]), ("held", [1, -1, 0]), ("held", [1, 4, 0]), ("new", [3, -4, 5]), ("new", [3, 29, 5]),
                         ("new", [3, 2 ** 31 - 1, 5]), ("held", [1, -2 ** 31, 0])):
        for ended in (None, [0, 1, 0]):
            if ended and name == "new" and values[1] == 29:
                continue                                                                    # (they fit where the sequence begins anew)
            a = {**good, name: values}
            table = _dev([[0, -1, -1], [1, 2, -1], [-1, -1, -1]])
            pool = PagePool(_dev([3, 4, 5, -1, -1, -1]), _dev([0, 3]))
            held, lengths, status = _dev(a["held"]), _dev(a["lengths"]), torch.zeros(1, dtype=torch.int32, device="cuda")
            cu, seq, pos, slot = dec.wf_page_plan(pool, table, held, lengths, _dev(a["new"]), 10, ended=None if ended is None else _dev(ended, torch.uint8),
                                                  status=status)
            assert int(status) == 2 and cu.tolist() == [0, 3, 3, 8], (name, values)
            assert seq.tolist() == [0] * 3 + [2] * 5 + [-1] * 2 and pos.tolist()[:8] == [5, 6, 7, 0, 1, 2, 3, 4]
            assert slot.tolist() == [5, 6, 7] + list(range(48, 53)) + [-1] * 2 and table[2].tolist() == [3, -1, -1]
            if ended is None or name != "new":
                assert held.tolist() == [1, a["held"][1], 1] and lengths.tolist() == [5, a["lengths"][1], 0]
                assert table[1].tolist() == [1, 2, -1]
    for state in ([-1, 3], [6, 3], [0, -1], [0, 7]):
        table, held, lengths = _dev([[0, -1, -1], [1, 2, -1], [-1, -1, -1]]), _dev(good["held"]), _dev(good["lengths"])
        pool, status = PagePool(_dev([3, 4, 5, -1, -1, -1]), _dev(state)), torch.zeros(1, dtype=torch.int32, device="cuda")
        cu, seq, _, slot = dec.wf_page_plan(pool, table, held, lengths, _dev(good["new"]), 10, ended=_dev([1, 0, 0], torch.uint8), status=status)
        assert int(status) & 2 and cu.tolist() == [0] * 4 and (seq == -1).all() and (slot == -1).all() and pool.state.tolist() == state
        assert held.tolist() == good["held"] and lengths.tolist() == good["lengths"] and table.tolist() == [[0, -1, -1], [1, 2, -1], [-1, -1, -1]]
        assert pool.pages.tolist() == [3, 4, 5, -1, -1, -1]


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [9, 4000])
def test_pages_outside_the_cache(rows):
    """They are handed out and taken back as they are, reported, and their rows have no place."""
    from paper_2412_11272_b200.binding import PagePool
    dec = _decoder(16)
    table = _dev([[99, -1], [-1, -1]])
    pool, status = PagePool(_dev([3, -2, 0, 0]), _dev([0, 2])), torch.zeros(1, dtype=torch.int32, device="cuda")
    held, lengths = _dev([1, 0]), _dev([3, 0])
    cu, seq, pos, slot = dec.wf_page_plan(pool, table, held, lengths, _dev([2, 20]), max(rows, 22), status=status)
    assert int(status) == 1 and cu.tolist() == [0, 2, 22] and slot[:2].tolist() == [-1, -1] and slot[2:18].tolist() == list(range(48, 64))
    assert slot[18:].tolist() == [-1] * (max(rows, 22) - 18) and pos[18:22].tolist() == [16, 17, 18, 19] and table.tolist() == [[99, -1], [3, -2]]


@pytest.mark.gpu
def test_no_sequences_no_rows_and_rows_that_do_not_fit():
    from paper_2412_11272_b200.binding import STATUS_PUT_OFF
    dec = _decoder(16)
    pool = dec.page_pool(4)
    e = torch.zeros(0, dtype=torch.int32, device="cuda")
    for rows in (5, 3000):
        cu, seq, pos, slot = dec.wf_page_plan(pool, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), e, e, e, rows)
        assert cu.tolist() == [0] and (seq == -1).all() and (pos == -1).all() and (slot == -1).all() and len(slot) == rows
    table, held, lengths = torch.full((3, 4), -1, dtype=torch.int32, device="cuda"), _dev([0, 0, 0]), _dev([0, 0, 0])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cu, *_ = dec.wf_page_plan(pool, table, held, lengths, _dev([0, 0, 0]), 0, status=status)
    assert cu.tolist() == [0] * 4 and int(status) == 0
    cu, seq, *_ = dec.wf_page_plan(pool, table, held, lengths, _dev([3, 4, 2]), 6, status=status)  # the second does not fit, and so the third does not
    assert cu.tolist() == [0, 3, 3, 3] and int(status) == STATUS_PUT_OFF and held.tolist() == [1, 0, 0] and pool.state.tolist() == [1, 3]


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [40, 2500])
def test_captured_and_replayed_on_another_stream(rows):
    """A captured round takes what the arrays hold when it is replayed."""
    rng = np.random.default_rng(5)
    dec = _decoder(16)
    st = _State(rng, 6, 200, 1200, rng.integers(0, 60, 6), 16)
    pool, table, held, lengths = dev = st.device()
    new, ended = _dev([0] * 6), _dev([0] * 6, torch.uint8)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = dec.wf_page_plan(pool, table, held, lengths, new, rows, ended=ended, status=status)
    for turn in range(3):
        w, gone = rng.integers(0, rows // 7, 6), rng.random(6) < 0.4
        new.copy_(_dev(w))
        ended.copy_(_dev(gone, torch.uint8))
        status.zero_()
        graph.replay()
        torch.cuda.synchronize()
        st.check(dev, out, st.plan(w, rows, gone), status)


@pytest.mark.gpu
def test_positions_that_pass_31_bits():
    """A sequence of nearly 2^31 positions: rows up to the last of them, none beyond."""
    from paper_2412_11272_b200.binding import PagePool
    dec, stride, first = _decoder(256), (1 << 23) + 4, 2 ** 31 - 300
    table = torch.arange(stride, dtype=torch.int32, device="cuda")[None].contiguous()
    for new, rows in ((299, 400), (300, 400), (299, 3000), (2000, 3000)):
        pool, held, lengths = PagePool(_dev([0] * (stride + 5)), _dev([0, 0])), _dev([stride]), _dev([first])
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        cu, _, pos, slot = dec.wf_page_plan(pool, table, held, lengths, _dev([new]), rows, status=status)
        if new == 299:
            assert int(status) == 0 and cu.tolist() == [0, 299] and pos[:299].tolist() == list(range(first, first + 299))
            assert slot[:299].tolist() == list(range(first, first + 299)) and (slot[299:] == -1).all()
        else:
            assert int(status) == 2 and cu.tolist() == [0, 0] and (pos == -1).all()
