"""Rounds of speculative decoding that run the operators together, as a server would: rows and pages planned on the device, projections in
8 bits, keys and values into paged caches, attention of the drafted trees over them, logits, verification, the accepted rows committed;
sequences end and others take their places.  Every answer is compared with the oracle's on the state as it should be, which is kept
beside the device's in numpy: for every sequence what its positions hold in every layer."""
import numpy as np
import pytest

from oracle import decode_oracle as O
from oracle import speculation_oracle as S

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

D, H, HK, LAYERS, VOCAB, PAGE = 256, 4, 2, 2, 500, 16


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda:0", dtype)


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("fmt,drawn", [("e4m3", True), ("int8", False), ("path", True)])
def test_rounds_of_speculative_decoding(fmt, drawn):
    from paper_2412_11272_b200.binding import Decoder
    rng = np.random.default_rng(7)
    gen = torch.Generator(device="cuda").manual_seed(7)
    dec = Decoder(H, HK, d_head=64, dtype="bf16", cache_format=fmt, page_size=PAGE)
    n_seq, room, stride = 5, 96, 8
    pool = dec.page_pool(30)
    table, held, lengths = (torch.full((n_seq, stride), -1, dtype=torch.int32, device="cuda"), *(torch.zeros(n_seq, dtype=torch.int32, device="cuda") for _ in range(2)))
    caches = [dec.cache(30) for _ in range(LAYERS)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    embed = normal(VOCAB, D).bfloat16()
    w_qkv = [dec.wf_quantise_e4m3(normal((H + 2 * HK) * 64, D) * D ** -0.5) for _ in range(LAYERS)]
    w_out, bias = dec.wf_quantise_e4m3(normal(VOCAB, H * 64) * 0.3), normal(VOCAB)
    w_exact = [_np(w.values()) for w in w_qkv]
    true = [[(np.zeros((0, HK, 64)), np.zeros((0, HK, 64))) for _ in range(LAYERS)] for _ in range(n_seq)]   # what the positions of a sequence hold
    last, waiting, pages_seen = [0] * n_seq, [True] * n_seq, set()

    for turn in range(9):
        # ---- what every sequence brings: a prompt where its place is new, else its last token and a tree of drafts
        ended = np.array([bool(turn) and not w and rng.random() < 0.2 for w in waiting])
        tokens, parents, new = [], [], []
        for b in range(n_seq):
            if ended[b]:
                true[b] = [(np.zeros((0, HK, 64)), np.zeros((0, HK, 64))) for _ in range(LAYERS)]
            fresh = waiting[b] or ended[b]
            n = int(rng.integers(3, 40)) if fresh else int(rng.integers(1, 9))
            new.append(n)
            tokens.append(rng.integers(0, VOCAB, n) if fresh else np.concatenate([[last[b]], rng.integers(0, VOCAB, n - 1)]))
            parents.append(np.arange(-1, n - 1) if fresh else np.concatenate([[-1], [rng.integers(0, i) for i in range(1, n)]]).astype(int))
            waiting[b] = fresh
        cu, row_seq, row_pos, row_slot = dec.wf_page_plan(pool, table, held, lengths, _dev(new), room, ended=_dev(ended, torch.bool), status=status)
        put_off = int(status)
        assert put_off in (0, 16)
        status.zero_()
        cu_h = cu.cpu().numpy()
        got = np.diff(cu_h)
        assert all(g in (0, m) for g, m in zip(got, new)) and (put_off != 0) == bool((got != new).any())
        live = [b for b in range(n_seq) if got[b]]
        n = int(cu_h[-1])
        assert row_seq[:n].tolist() == np.repeat(np.arange(n_seq), got).tolist() and (row_slot[n:] == -1).all()
        start = lengths.cpu().numpy()
        assert row_pos[:n].tolist() == [start[b] + i for b in live for i in range(got[b])] and all(start[b] == len(true[b][0][0]) for b in range(n_seq))
        pages_seen |= set((row_slot[:n] // PAGE).tolist())

        # ---- the rows through the layers; padding rows are projected too and belong to nobody
        tok = np.zeros(room, np.int64)
        up = np.full(room, -1)
        bits = np.zeros((room, 64), bool)
        for b in live:
            for i in range(got[b]):
                r = cu_h[b] + i
                tok[r], up[r] = tokens[b][i], parents[b][i]
                if parents[b][i] >= 0:
                    bits[r] = bits[cu_h[b] + parents[b][i]]
                bits[r, i] = True
        mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
        x = embed[_dev(tok, torch.int64)]
        for layer in range(LAYERS):
            codes = dec.wf_quantise_e4m3(x)
            qkv = dec.wf_gemm_e4m3(codes, w_qkv[layer]).view(room, H + 2 * HK, 64)
            y = _np(codes.values()) @ w_exact[layer].T
            size = np.abs(_np(codes.values())) @ np.abs(w_exact[layer]).T
            # half a step of the output, and a float32 step of the sums' magnitude for each of eight instructions and 32 products in one
            assert (np.abs(_np(qkv).reshape(room, -1) - y) <= 2.0 ** -8 * np.abs(y) + 40 * 2.0 ** -23 * size).all()
            q, k, v = qkv[:, :H], qkv[:, H:H + HK], qkv[:, H + HK:]
            dec.wf_cache_write(caches[layer], table, cu, lengths, k, v, status=status)
            at = torch.zeros(room, H, 64, dtype=torch.bfloat16, device="cuda")  # (rows of padding are left as they are)
            dec.wf_tree_attention(caches[layer], table, cu, lengths, q, max_rows=max(new), tail="mask", mask=mask, out=at, status=status)
            kn, vn, qn = O.stored(_np(k), fmt), O.stored(_np(v), fmt), _np(q)
            for b in live:
                r = slice(cu_h[b], cu_h[b + 1])
                ks, vs = (np.concatenate([old, fresh_rows[r]]) for old, fresh_rows in zip(true[b][layer], (kn, vn)))
                true[b][layer] = (ks, vs)
                see = O.visible(start[b], got[b], "mask", bits[r])
                want, _ = O.attend(qn[r], ks, vs, see, 0.125)
                # half a step for a probability and half a step for the output, each 2^-8 of the largest value, and float32 sums
                assert np.abs(_np(at[r]) - want).max() <= (2.0 ** -7 + 1e-4) * np.abs(vs).max()
            x = (x.float() + at.reshape(room, -1).float()).bfloat16()
        assert int(status) == 0

        # ---- what the target keeps of the drafts; a prompt's rows all stay, its last one's token is drawn
        logits = dec.wf_gemm_e4m3(dec.wf_quantise_e4m3(x), w_out, bias=bias, out_dtype="f32")
        draft = torch.softmax(logits + normal(room, VOCAB), 1) if drawn else None
        u, u_last = rng.random(room).astype(np.float32), rng.random(n_seq).astype(np.float32)
        for b in live:
            if waiting[b]:
                u[cu_h[b]:cu_h[b + 1]] = 1.0                          # (nothing of a prompt is a draft: its rows go another way, below)
        most = max(new)
        t = _dev(rng.choice([0.0, 0.7, 1.0], n_seq), torch.float32)
        kept, out, path = dec.wf_draft_verify(logits, cu, _dev(tok), _dev(u, torch.float32), _dev(u_last, torch.float32), most, parents=_dev(up), draft=draft,
                                              temperature=t, status=status)
        kept_h, out_h, path_h = kept.cpu().numpy().copy(), out.cpu().numpy(), path.cpu().numpy().copy()
        xn, qn = _np(logits), None if draft is None else _np(draft)
        for b in live:
            r = slice(cu_h[b], cu_h[b + 1])
            if waiting[b]:
                kept_h[b], path_h[b, :got[b]] = got[b], np.arange(got[b])
                last[b] = int(rng.integers(VOCAB))
                continue
            want, stay, margin = S.draft_verify(xn[r], tok[r], up[r], u[r], u_last[b], float(t[b]), None if qn is None else qn[r])
            assert margin > 20, "drawn too near to a border: another seed"
            assert out_h[b, :kept_h[b]].tolist() == want and path_h[b, :kept_h[b]].tolist() == stay
            last[b] = want[-1]
        assert all(kept_h[b] == 0 for b in range(n_seq) if b not in live)

        # ---- the accepted rows become positions
        assert dec.wf_draft_commit(lengths, _dev(kept_h), _dev(path_h), caches=caches, page_table=table, lengths=lengths, status=status) is lengths
        for b in live:
            for layer in range(LAYERS):
                rows = np.concatenate([np.arange(start[b]), start[b] + path_h[b, :kept_h[b]]])
                true[b][layer] = tuple(side[rows] for side in true[b][layer])
            waiting[b] = False
        assert int(status) == 0 and lengths.tolist() == [len(true[b][0][0]) for b in range(n_seq)]
        # ---- what the caches hold is what they should
        count = lengths.cpu().numpy()
        cu_all = _dev(np.concatenate([[0], np.cumsum(count)]))
        for layer in range(LAYERS):
            k, v = dec.wf_cache_read(caches[layer], table, cu_all, torch.zeros_like(lengths), int(count.sum()), status=status)
            for side, got_side in ((0, k), (1, v)):
                whole = np.concatenate([true[b][layer][side] for b in range(n_seq)])
                assert np.array_equal(_np(got_side), _np(torch.from_numpy(whole).to(torch.bfloat16)))
        free = pool.state.tolist()
        owned = np.concatenate([table[b, :held[b]].cpu().numpy() for b in range(n_seq)] +
                               [pool.pages.cpu().numpy()[(free[0] + np.arange(free[1])) % 30]])
        assert sorted(owned.tolist()) == list(range(30))
    assert len(pages_seen) > 15
