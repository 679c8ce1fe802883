"""Rounds of a decoder that run the decoding-stage operators together, next to the encoder's own pieces: cross-attention keys and
values from wf_cross_kv into a quantised cache, self-attention of beams over paged caches, beam widths from the pruner,
selection, reordering, and a last round that verifies a tree of drafted tokens.  Every operator's answer is compared with the oracle's on
the state as it should be; the state (what every beam's cache holds) is kept beside it in numpy."""
import numpy as np
import pytest

from oracle import decode_oracle as O
from paper_2412_11272_b200 import inputs as I
from tests._util import make_encoder

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

D, H, LAYERS, VOCAB, END = 256, 4, 2, 600, 599


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda:0", dtype)


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype,fmt,cross_fmt", [("bf16", "e4m3", "int8"), ("f32", "int8", "path"), ("bf16", "path", "e4m3")])
def test_rounds_of_beam_search_and_a_drafted_tree(dtype, fmt, cross_fmt):
    from paper_2412_11272_b200.binding import BeamPruner, Decoder
    rng = np.random.default_rng(42)
    gen = torch.Generator(device="cuda").manual_seed(42)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(*shape, size=1.0):
        return (size * torch.randn(*shape, generator=gen, device="cuda")).to(tt)

    B, W, page = 2, 3, 16
    R = B * W
    dec = Decoder(H, d_head=64, dtype=dtype, cache_format=fmt, page_size=page)
    cross = Decoder(H, d_head=64, dtype=dtype, cache_format=cross_fmt, page_size=64)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    # bf16: half a step for the weights and half a step for the output (each 2^-8 of the largest value), and float32 sums
    tol = 2.0 ** -7 + 1e-4 if dtype == "bf16" else 1e-4

    # ---- the encoder's output becomes the cross-attention caches, straight out of the rows of the projection of all layers
    shape = I.EncoderShape("r", 80, D, 0, H, 1024, dtype, n_ctx=256)
    enc = make_encoder(shape, I.encoder_weights(0, shape), 8, 1024, 16000)
    frames = [75, 131]
    hidden = normal(sum(frames), D)
    kv = enc.wf_cross_kv(hidden, normal(2 * LAYERS * D, D, size=D ** -0.5), torch.zeros(2 * LAYERS * D, device="cuda"))
    cross_table = _dev([[0, 1, -1], [2, 3, 4]])
    cross_cu, none = _dev(np.concatenate([[0], np.cumsum(frames)])), _dev([0, 0])
    cross_caches, cross_true = [], []
    for layer in range(LAYERS):
        c = cross.cache(5)
        k, v = (kv[:, (2 * layer + i) * D:(2 * layer + i + 1) * D].unflatten(1, (H, 64)) for i in range(2))
        cross.wf_cache_write(c, cross_table, cross_cu, none, k, v, status=status)
        cross_caches.append(c)
        cross_true.append([O.stored(_np(x), cross_fmt) for x in (k, v)])

    # ---- beams
    P = 4
    caches = [dec.cache(R * P) for _ in range(LAYERS)]
    table = _dev(np.arange(R * P).reshape(B, P, W).transpose(0, 2, 1).reshape(R, P))       # n_beam pages for every page index
    tokens = torch.full((R, 64), -1, dtype=torch.int32, device="cuda")
    embed, w_q, w_k, w_v, w_o = normal(VOCAB, D), *(normal(LAYERS, D, D, size=D ** -0.5) for _ in range(4))
    head = normal(VOCAB, D, size=2 * D ** -0.5)
    held = [[[np.zeros((0, H, 64))] * 2 for _ in range(LAYERS)] for _ in range(R)]           # what every beam's caches hold
    said = [[] for _ in range(R)]
    scores = torch.zeros(B, W, device="cuda")
    scores[:, 1:] = -float("inf")                                                               # the first round starts from one beam
    finished = torch.zeros(B, W, dtype=torch.uint8, device="cuda")
    current = _dev(rng.integers(0, VOCAB - 1, size=R))
    pruners = [BeamPruner(rng.integers(0, VOCAB - 1, size=40), np.zeros(VOCAB, np.uint8), full_beam=W) for _ in range(B)]
    beams = np.array([1, 1])
    each = _dev(np.arange(R + 1))
    by_stream, starts_cross = _dev(np.arange(0, R + 1, W)), _dev(frames)

    def block(x, start, cu, max_rows, max_len, tail, mask, check):
        """One decoder layer after another on rows x."""
        for layer in range(LAYERS):
            q, k, v = ((x @ w[layer].T).unflatten(1, (H, 64)) for w in (w_q, w_k, w_v))
            dec.wf_cache_write(caches[layer], table, cu, start, k, v, status=status)
            att, lse = dec.wf_tree_attention(caches[layer], table, cu, start, q, max_rows, max_len, tail, mask, status=status)
            check(layer, q, O.stored(_np(k), fmt), O.stored(_np(v), fmt), att)
            x = x + (att.flatten(1) @ w_o[layer].T)
        return x

    for step in range(20):                                                                      # crosses one page border
        length = step
        x = embed[current.long()]
        starts = _dev([length] * R)

        def check(layer, q, k, v, att):
            for r in range(R):
                mine = held[r][layer]
                mine[0], mine[1] = np.concatenate([mine[0], k[r:r + 1]]), np.concatenate([mine[1], v[r:r + 1]])
                want, _ = O.attend(_np(q[r:r + 1]), mine[0], mine[1], np.ones((1, length + 1), bool), 0.125)
                assert np.abs(_np(att[r]) - want[0]).max() <= tol * np.abs(mine[1]).max(), (step, layer, r)

        x = block(x, starts, each, 1, length + 1, "causal", None, check)
        # the beams of a stream over its one cross-attention cache
        q = x.unflatten(1, (H, 64))
        for layer in range(LAYERS):
            att, _ = cross.wf_tree_attention(cross_caches[layer], cross_table, by_stream, starts_cross, q, W, max(frames), "none", status=status)
            if step % 7 == 0:
                for b in range(B):
                    at, to = int(cross_cu[b]), int(cross_cu[b + 1])
                    k, v = (t[at:to] for t in cross_true[layer])
                    want, _ = O.attend(_np(q[b * W:(b + 1) * W]), k, v, np.ones((W, to - at), bool), 0.125)
                    assert np.abs(_np(att[b * W:(b + 1) * W]) - want).max() <= tol * np.abs(v).max()
            x = x + 0.1 * att.flatten(1)
        logits = x @ head.T
        new = dec.wf_beam_select(logits, scores, W, beams=_dev(beams), finished=finished, end_token=END, status=status)
        want = O.beam_select(_np(logits).reshape(B, W, VOCAB), _np(scores), W, beams, finished.cpu().numpy(), END)
        for g, w in zip(new[1:], want[1:]):
            assert np.array_equal(g.cpu().numpy(), w), step
        scores, parents, chosen, finished = new
        # the states follow: caches, tables, token histories
        tokens[:, step] = current
        for r in range(R):
            said[r].append(int(current[r]))
        dec.wf_beam_reorder(parents, states=[tokens], caches=caches, page_table=table, lengths=_dev([length + 1] * B), status=status)
        src = O.beam_sources(parents.cpu().numpy())
        held = [[[a.copy() for a in layer] for layer in held[s]] for s in src]
        said = [list(said[s]) for s in src]
        for r in range(R):
            assert tokens[r, :step + 1].tolist() == said[r]
        current = chosen.reshape(-1).clamp(min=0)
        beams = np.array([p.step(int(t)) for p, t in zip(pruners, chosen[:, 0].clamp(min=0).tolist())])
        if step in (0, 9, 15, 19):                                                              # what the tables lead to is what the beams hold
            for layer in range(LAYERS):
                gk, gv = dec.wf_cache_read(caches[layer], table, _dev(np.arange(R + 1) * (length + 1)), _dev([0] * R), R * (length + 1), status=status)
                exact = torch.float32 if dtype == "f32" else torch.bfloat16
                for g, i in ((gk, 0), (gv, 1)):
                    want = torch.as_tensor(np.concatenate([held[r][layer][i] for r in range(R)])).to(exact)
                    assert torch.equal(g.cpu(), want), (step, layer)

    # ---- a last round verifies drafts: every beam a tree of its own size, written behind its history and seen along the branches
    sizes = [5, 1, 3, 7, 2, 4]
    cu = np.concatenate([[0], np.cumsum(sizes)])
    n, length = int(cu[-1]), 20
    trees = []
    for m in sizes:
        bits = np.zeros((m, m), bool)
        for i in range(m):
            parent = int(rng.integers(-1, i)) if i else -1
            bits[i] = bits[parent] if parent >= 0 else False
            bits[i, i] = True
        trees.append(bits)
    mask = np.concatenate([np.packbits(np.pad(t, ((0, 0), (0, 32 - len(t)))), axis=1, bitorder="little").view(np.int32) for t in trees])

    def check(layer, q, k, v, att):
        for r in range(R):
            a, b = cu[r], cu[r + 1]
            full = [np.concatenate([held[r][layer][i], s[a:b]]) for i, s in ((0, k), (1, v))]
            want, _ = O.attend(_np(q[a:b]), full[0], full[1], O.visible(length, sizes[r], "mask", trees[r]), 0.125)
            assert np.abs(_np(att[a:b]) - want).max() <= tol * np.abs(full[1]).max(), (layer, r)

    block(embed[_dev(rng.integers(0, VOCAB, size=n)).long()], _dev([length] * R), _dev(cu), max(sizes), length + max(sizes), "tree", _dev(mask), check)
    assert int(status) == 0
    enc.close()
