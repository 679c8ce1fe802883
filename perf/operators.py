"""The decoder-side operators of the framework as cases to be timed, with their plain forms.

Four operators of one decoding round: the quantised paged cache written and read back (``store``), attention of
drafted tokens or beams over it (``attend``), selection over beams and vocabulary (``select``) and the reordering of
the states behind the selected beams (``reorder``)."""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
F8 = torch.float8_e4m3fn
CODES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": F8, "int8": torch.int8}
PATH = {"bf16": torch.bfloat16, "f32": torch.float32}
NBYTES = {"bf16": 2, "f32": 4, "e4m3": 1, "int8": 1}


def listed():
    return [
        # one stream decoding greedily: a single token over its own history (latency)
        dict(name="attend one token", op="attend", seqs=1, rows=1, rows_lo=1, heads=20, kv_heads=20, dim=64, dtype="bf16", fmt="e4m3",
             page=16, lo=150, hi=150, tail="causal"),
        # beam search over the encoder's output: five beams read one buffer's cross-attention keys, 64 streams of 1 .. 15 s
        dict(name="attend cross 64 streams", op="attend", seqs=64, rows=5, rows_lo=1, heads=20, kv_heads=20, dim=64, dtype="bf16", fmt="e4m3",
             page=64, lo=75, hi=775, tail="none"),
        # speculative decoding: trees of drafted tokens, grouped heads, middling histories
        dict(name="attend trees", op="attend", seqs=16, rows=48, rows_lo=2, heads=32, kv_heads=8, dim=128, dtype="bf16", fmt="int8",
             page=64, lo=100, hi=4096, tail="tree"),
        # few sequences with very long histories, a short chain of drafts, unquantised cache
        dict(name="attend long", op="attend", seqs=2, rows=4, rows_lo=3, heads=32, kv_heads=8, dim=128, dtype="bf16", fmt="bf16",
             page=128, lo=98_765, hi=131_000, tail="causal"),
        # the float32 path: a prompt of a few tokens over 30 s buffers
        dict(name="attend float32", op="attend", seqs=8, rows=8, rows_lo=3, heads=6, kv_heads=6, dim=64, dtype="f32", fmt="f32",
             page=32, lo=301, hi=1500, tail="causal"),
        # the cache write of one decoding step, every stream one token
        dict(name="store one token", op="store", seqs=64, rows=1, rows_lo=1, heads=20, dim=64, dtype="bf16", fmt="int8", page=16, at=447),
        # the cross-attention keys and values of a batch of buffers, one layer, out of the projection of all layers
        dict(name="store cross 64 streams", op="store", seqs=64, rows=775, rows_lo=75, heads=20, dim=64, dtype="bf16", fmt="e4m3", page=64, at=0),
        # a long prompt in float32
        dict(name="store float32 prompt", op="store", seqs=3, rows=4001, rows_lo=1, heads=8, dim=128, dtype="f32", fmt="int8", page=128, at=130),
        # one stream's round of beam search (latency)
        dict(name="select one stream", op="select", seqs=1, beams=5, vocab=50_021, dtype="f32", keep=5),
        # the same for a batch, some beams pruned, some finished
        dict(name="select 64 streams", op="select", seqs=64, beams=5, vocab=50_021, dtype="bf16", keep=10),
        # the paged self-attention caches of all layers follow their beams: only the page being filled moves
        dict(name="reorder pages", op="reorder", seqs=16, beams=5, heads=12, dim=64, fmt="e4m3", page=16, length=219, layers=12, row=0, live=0),
        # contiguous per-beam states
        dict(name="reorder rows", op="reorder", seqs=64, beams=5, heads=0, dim=0, fmt="", page=0, length=0, layers=4, row=229_376, live=224_256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "store", "select", "reorder"])
    if op == "attend":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        dim, kv = rng.choice([64, 128]), rng.choice([1, 2, 4, 6, 8, 20])
        heads = kv * rng.choice([1, 1, 2, 4] if kv <= 8 else [1])
        hi = _log(rng, 20, 60_000)
        seqs = min(_log(rng, 1, 96), max(1, 150_000_000 // (hi * kv * dim)))
        rows = max(1, min(_log(rng, 1, 64), 200_000_000 // (seqs * heads * hi)))
        if dtype == "f32":
            rows = min(rows, 16)
            seqs = min(seqs, max(1, 20_000_000 // (hi * kv * dim)))
        return dict(op=op, seqs=seqs, rows=rows, rows_lo=rng.randint(1, rows), heads=heads, kv_heads=kv, dim=dim, dtype=dtype,
                    fmt=rng.choice([dtype, "e4m3", "int8"]), page=rng.choice([16, 32, 64, 128, 256]), lo=rng.randint(1, hi), hi=hi,
                    tail=rng.choice(["none", "causal", "tree"]))
    if op == "store":
        dtype = rng.choice(["bf16", "f32"])
        rows, heads, dim = _log(rng, 1, 4000), rng.choice([1, 4, 6, 8, 20]), rng.choice([64, 128])
        seqs = min(_log(rng, 1, 96), max(1, 60_000_000 // (rows * heads * dim)))
        return dict(op=op, seqs=seqs, rows=rows, rows_lo=rng.randint(1, rows), heads=heads, dim=dim, dtype=dtype,
                    fmt=rng.choice([dtype, "e4m3", "int8"]), page=rng.choice([16, 32, 64, 128, 256]), at=rng.randint(0, 700))
    if op == "select":
        seqs, beams = _log(rng, 1, 64), rng.randint(1, 8)
        vocab = min(_log(rng, 200, 120_000), 16_000_000 // (seqs * beams))
        return dict(op=op, seqs=seqs, beams=beams, vocab=vocab, dtype=rng.choice(["bf16", "f32"]), keep=rng.randint(1, 2 * beams))
    if rng.random() < 0.5:
        return dict(op=op, seqs=_log(rng, 1, 24), beams=rng.randint(2, 8), heads=rng.choice([4, 6, 8, 12]), dim=rng.choice([64, 128]),
                    fmt=rng.choice(["bf16", "e4m3", "int8"]), page=rng.choice([16, 32, 64]), length=rng.randint(1, 250), layers=rng.randint(1, 12),
                    row=0, live=0)
    row = 16 * _log(rng, 1, 8000)
    return dict(op=op, seqs=_log(rng, 1, 64), beams=rng.randint(2, 8), heads=0, dim=0, fmt="", page=0, length=0, layers=rng.randint(1, 4),
                row=row, live=4 * rng.randint(row // 8, row // 4))


# ---- sizes that follow from a case alone (so that the work is known without its inputs)

def _spread(lo, hi, n, step):
    """n whole numbers over [lo, hi], hi among them, in no order."""
    return [hi if i == 0 else lo + int((hi - lo + 1) * ((i * step) % 1.0)) for i in range(n)]


def _sizes(c):
    """(rows, committed positions) of every sequence."""
    rows = _spread(c["rows_lo"], c["rows"], c["seqs"], 0.7548776662)
    if c["op"] == "store":
        return rows, [(c["at"] + 37 * i) % (c["at"] + 1) if i else c["at"] for i in range(c["seqs"])]
    return rows, _spread(c["lo"], c["hi"], c["seqs"], 0.6180339887)


def _parents(c):
    return [[int(w * 0.6 + b % 3) % c["beams"] for w in range(c["beams"])] for b in range(c["seqs"])]


def _lengths(c):
    return [(c["length"] + 5 * b) % (c["length"] + 1) if b else c["length"] for b in range(c["seqs"])]


def work(case):
    c = case
    if c["op"] in ("attend", "store"):
        rows, start = _sizes(c)
        n = sum(rows)
        vec = c["dim"] * NBYTES[c["fmt"]] + (2 if c["fmt"] in ("e4m3", "int8") else 0)
        if c["op"] == "store":
            # each vector read, its codes written and read, and written back as values
            return {"bytes": 2 * n * c["heads"] * (2 * c["dim"] * NBYTES[c["dtype"]] + 2 * vec), "flops": 0}
        tail = 0 if c["tail"] == "none" else 1
        keys = sum(s + tail * r for s, r in zip(start, rows))
        mask = 4 * n * -(-c["rows"] // 32) if c["tail"] == "tree" else 0
        return {"bytes": 2 * keys * c["kv_heads"] * vec + n * c["heads"] * (2 * c["dim"] * NBYTES[c["dtype"]] + 4) + mask,
                "flops": 4 * c["dim"] * c["heads"] * sum(r * (s + tail * r) for s, r in zip(start, rows))}
    if c["op"] == "select":
        rows = sum(_live_beams(c))
        return {"bytes": rows * c["vocab"] * (2 if c["dtype"] == "bf16" else 4) + 13 * c["seqs"] * c["keep"], "flops": 4 * rows * c["vocab"]}
    parents, total = _parents(c), 0
    for p, n in zip(parents, _lengths(c) if c["page"] else [0] * c["seqs"]):
        moved = [w for w, q in enumerate(p) if q != w]
        if c["page"]:
            vec = 2 * c["heads"] * (c["dim"] * NBYTES[c["fmt"]] + (2 if c["fmt"] != "bf16" else 0))
            each = (n % c["page"]) * vec * c["layers"] + 4 * (n // c["page"])
        else:
            each = c["live"] * c["layers"]
        total += each * (len(moved) + len({p[w] for w in moved}))
    return {"bytes": max(total, 16 * c["seqs"] * c["beams"]), "flops": 0}


def _live_beams(c):
    return [c["beams"] if b % 4 else max(1, c["beams"] - b % 8) for b in range(c["seqs"])]


# ---- the cache's number formats

def _scales(x, fmt):
    """The scale of each vector of x (float32, vectors along the last axis)."""
    top = x.abs().amax(-1, keepdim=True)
    if fmt == "e4m3":  # the least power of two with top / scale <= 448
        m, e = torch.frexp(top)
        s = torch.ldexp(torch.ones_like(top), (e - torch.where(m <= 0.875, 9, 8)).clamp(min=-126))
    else:  # top / 127, rounded up to bfloat16
        s = ((top / 127).view(torch.int32) + 0xFFFF).bitwise_and(-65536).view(torch.float32).clamp(min=2.0 ** -126)
    return torch.where(top > 0, s, torch.ones_like(s))


def _quantise(x, fmt):
    """Codes and scales (bfloat16) of float32 vectors; what lies next to a rounding border is decided in 64 bits."""
    s = _scales(x, fmt)
    if fmt == "e4m3":
        return (x / s).to(F8), s.squeeze(-1).bfloat16()
    return torch.round(x.double() / s.double()).to(torch.int8), s.squeeze(-1).bfloat16()


# ---- inputs

def _pages_for(positions, page, g):
    """A page table for sequences of these sizes, its pages in no order, and how many pages there are."""
    each = [-(-p // page) for p in positions]
    n = sum(each)
    table = torch.full((len(each), max(each)), -1, dtype=torch.int32)
    order = torch.randperm(n, generator=g).int()
    at = 0
    for i, k in enumerate(each):
        table[i, :k] = order[at:at + k]
        at += k
    return table.to(DEVICE), n


def _tree(rows, words, g):
    """Bits of the drafted tokens that each one sees: itself and its ancestors in a random tree, as 32-bit words."""
    out = np.zeros((sum(rows), words), np.uint32)
    at = 0
    for n in rows:
        pick = torch.rand(n, generator=g).numpy()
        for i in range(n):
            parent = int(pick[i] * (i + 1)) - 1  # -1: a root
            if parent >= 0:
                out[at + i] = out[at + parent]
            out[at + i, i // 32] |= np.uint32(1 << (i % 32))
        at += n
    return torch.from_numpy(out.view(np.int32)).to(DEVICE)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    c = case
    host = torch.Generator().manual_seed(seed)
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    s = dict(c)
    if c["op"] in ("attend", "store"):
        rows, start = _sizes(c)
        n, positions = sum(rows), [a + b for a, b in zip(rows, start)]
        kv_heads = c.get("kv_heads", c["heads"])
        s["table"], pages = _pages_for(positions, c["page"], host)
        s["cu"], s["start"] = _ints(np.cumsum([0] + rows).tolist()), _ints(start)
        s["n"], s["most"] = n, max(positions)
        shape = (pages, kv_heads, c["page"], c["dim"])
        if c["op"] == "store":
            s["k_pages"], s["v_pages"] = (torch.zeros(shape, device=DEVICE).to(CODES[c["fmt"]]) for _ in range(2))
            s["k_scale"], s["v_scale"] = (torch.ones(shape[:3], dtype=torch.bfloat16, device=DEVICE) for _ in range(2))
            # keys and values of one layer inside the rows of a projection of two layers
            width = c["heads"] * c["dim"]
            size = torch.exp(0.5 * normal(1, 4 * width))  # channels differ in size
            all_kv = (normal(n, 4 * width) * size).to(PATH[c["dtype"]])
            s["k"], s["v"] = (all_kv[:, i * width:(i + 1) * width].unflatten(1, (c["heads"], c["dim"])) for i in (2, 3))
            return s
        sides = []
        for _ in range(2):
            x = normal(*shape)
            x *= torch.exp(0.5 * normal(1, kv_heads, 1, c["dim"]))
            sides.append(_quantise(x, c["fmt"]) if c["fmt"] in ("e4m3", "int8") else (x.to(CODES[c["fmt"]]), None))
            del x
        (s["k_pages"], s["k_scale"]), (s["v_pages"], s["v_scale"]) = sides
        s["q"] = (1.5 * normal(n, c["heads"], c["dim"])).to(PATH[c["dtype"]])
        s["mask"] = _tree(rows, -(-c["rows"] // 32), host) if c["tail"] == "tree" else None
        return s
    if c["op"] == "select":
        B, W, V = c["seqs"], c["beams"], c["vocab"]
        s["logits"] = (3.0 * normal(B * W, V)).to(PATH[c["dtype"]])
        s["scores"] = -10.0 * torch.rand(B, W, generator=g, device=DEVICE)
        s["finished"] = (torch.rand(B, W, generator=g, device=DEVICE) < 0.1).to(torch.uint8)
        s["live"] = _ints(_live_beams(c))
        s["end"] = int(V - 1)
        # a few tokens that are never chosen
        words = torch.zeros(-(-V // 32), dtype=torch.int64)
        words[::50] = 1 << 7
        s["suppress"] = words.int().to(DEVICE)
        return s
    B, W = c["seqs"], c["beams"]
    s["parents"] = _ints(_parents(c))
    s["history"] = torch.randint(0, 50_000, (B * W, 448), generator=g, device=DEVICE, dtype=torch.int32)
    if c["page"]:
        each = c["length"] // c["page"] + 1
        shape = (c["layers"], B * W * each, c["heads"], c["page"], c["dim"])
        s["k_pages"], s["v_pages"] = (normal(*shape).to(CODES[c["fmt"]]) if c["fmt"] != "int8" else
                                      torch.randint(-127, 128, shape, generator=g, device=DEVICE, dtype=torch.int8) for _ in range(2))
        s["k_scale"], s["v_scale"] = (torch.rand(shape[:4], generator=g, device=DEVICE).bfloat16() if c["fmt"] != "bf16" else None for _ in range(2))
        # page p of beam w of sequence b: its own one of the W pages kept for (b, p)
        at = torch.arange(B * W * each).view(B, each, W).transpose(1, 2).reshape(B * W, each)
        s["table"] = torch.randperm(B * W * each, generator=host)[at].int().to(DEVICE)
        s["lengths"] = _ints(_lengths(c))
    else:
        s["rows"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (c["layers"], B * W, -(-c["row"] // 4)), generator=g, device=DEVICE, dtype=torch.int32)
    return s


# ---- one pass

def run(state):
    return {"attend": _attend, "store": _store, "select": _select, "reorder": _reorder}[state["op"]](state)


_kept = {}


def _decoder(s):
    """The framework's handle for these heads and this cache, kept as a program keeps it."""
    from paper_2412_11272_b200.binding import Decoder
    heads = s.get("heads") or 1
    dtype = s.get("dtype") or "bf16"
    key = (heads, s.get("kv_heads") or heads, s.get("dim") or 64, dtype, s.get("fmt") or dtype, s.get("page") or 16)
    if key not in _kept:
        _kept[key] = Decoder(n_head=key[0], n_kv_head=key[1], d_head=key[2], dtype=key[3], cache_format="path" if key[4] == key[3] else key[4],
                             page_size=key[5])
    return _kept[key]


def _caches(s):
    """The framework's views of the state's caches (one, or one for each layer), kept beside them as a program keeps them."""
    if "caches" not in s:
        from paper_2412_11272_b200.binding import KvCache
        parts = [s["k_pages"], s["v_pages"]] + ([s["k_scale"], s["v_scale"]] if s["fmt"] in ("e4m3", "int8") else [])
        s["caches"] = [KvCache(*layer) for layer in (zip(*parts) if s["op"] == "reorder" else [parts])]
    return s["caches"]


def _rows_of(s):
    """Sequence, index in its sequence and position of every row."""
    cu = s["cu"].long()
    row = torch.arange(s["n"], device=DEVICE)
    seq = torch.searchsorted(cu, row, right=True) - 1
    inner = row - cu[seq]
    return seq, inner, s["start"].long()[seq] + inner


def _values(pages, scale, page, at):
    """Vectors of the cache as float32: [..., heads, dim]."""
    x = pages.view(torch.uint8)[page, :, at].view(F8).float() if pages.dtype == F8 else pages[page, :, at].float()
    return x if scale is None else x * scale[page, :, at].float().unsqueeze(-1)


def _attend(s):
    if own:
        return _decoder(s).wf_tree_attention(_caches(s)[0], s["table"], s["cu"], s["start"], s["q"], max_rows=s["rows"], max_len=s["most"],
                                             tail=s["tail"], mask=s["mask"])
    B, Hk, G, D = s["seqs"], s["kv_heads"], s["heads"] // s["kv_heads"], s["dim"]
    scaled = s["fmt"] in ("e4m3", "int8")
    pos = torch.arange(s["most"], device=DEVICE)
    page, at = s["table"].long().clamp(min=0)[:, pos // s["page"]], (pos % s["page"])[None]
    seq, inner, _ = _rows_of(s)
    q = torch.zeros(B, s["rows"], s["heads"], D, device=DEVICE)
    q[seq, inner] = s["q"].float()
    q = q.view(B, s["rows"], Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, s["rows"] * G, D)
    k = _values(s["k_pages"], s["k_scale"] if scaled else None, page, at).permute(0, 2, 3, 1)
    x = torch.matmul(q, k) * (1.0 / math.sqrt(D))  # [B, Hk, rows G, positions]
    del k
    start, count = s["start"].long()[:, None, None], (s["cu"][1:] - s["cu"][:-1]).long()[:, None, None]
    rel = pos[None, None] - start
    seen = (rel < 0).expand(B, s["rows"], -1)
    if s["tail"] == "causal":
        seen = rel <= torch.arange(s["rows"], device=DEVICE)[None, :, None]
    elif s["tail"] == "tree":
        bits = torch.zeros(B, s["rows"], s["mask"].shape[1], dtype=torch.int32, device=DEVICE)
        bits[seq, inner] = s["mask"]
        t = rel.clamp(min=0, max=s["rows"] - 1).expand(B, s["rows"], -1)
        seen = (rel < 0) | ((rel < count) & ((torch.gather(bits, 2, t // 32) >> (t % 32)) & 1).bool())
    x = x.view(B, Hk, s["rows"], G, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m.clamp(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True, dtype=torch.float64)
    v = _values(s["v_pages"], s["v_scale"] if scaled else None, page, at).permute(0, 2, 1, 3)
    o = torch.matmul(p.view(B, Hk, s["rows"] * G, -1), v).view(B, Hk, s["rows"], G, D) / total.clamp(min=1e-300).float()
    lse = (m.double() + total.log()).float().squeeze(-1)
    o, lse = o.permute(0, 2, 1, 3, 4)[seq, inner], lse.permute(0, 2, 1, 3)[seq, inner]
    return o.reshape(s["n"], s["heads"], D).to(s["q"].dtype), lse.reshape(s["n"], s["heads"])


def _store(s):
    """New keys and values into the cache, and the same rows read back (as a prompt's attention takes them)."""
    if own:
        d, cache = _decoder(s), _caches(s)[0]
        d.wf_cache_write(cache, s["table"], s["cu"], s["start"], s["k"], s["v"])
        return d.wf_cache_read(cache, s["table"], s["cu"], s["start"], s["n"])
    seq, _, pos = _rows_of(s)
    page, at = s["table"].long()[seq, pos // s["page"]], pos % s["page"]
    k, v = _put(s, "k", page, at), _put(s, "v", page, at)
    return k.to(s["k"].dtype), v.to(s["v"].dtype)


def _put(s, side, page, at):
    pages, x = s[side + "_pages"], s[side]
    if s["fmt"] not in ("e4m3", "int8"):
        pages[page, :, at] = x
        return _values(pages, None, page, at)
    codes, scale = _quantise(x.float(), s["fmt"])
    pages.view(torch.uint8)[page, :, at] = codes.view(torch.uint8)
    s[side + "_scale"][page, :, at] = scale
    return _values(pages, s[side + "_scale"], page, at)


def _select(s):
    if own:
        return _decoder(s).wf_beam_select(s["logits"], s["scores"], s["keep"], beams=s["live"], finished=s["finished"], end_token=s["end"],
                                          suppress=s["suppress"])
    B, W, V = s["seqs"], s["beams"], s["vocab"]
    v = torch.arange(V, device=DEVICE)
    x = s["logits"].view(B, W, V).double()
    x = x.masked_fill(((s["suppress"][v // 32] >> (v % 32)) & 1).bool(), -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x - (m + (x - m).exp().sum(-1, keepdim=True).log())  # 64 bits: beams are told apart where they nearly tie
    only_end = torch.where(v == s["end"], 0.0, -math.inf).double()
    x = torch.where(s["finished"].bool()[..., None], only_end, x) + s["scores"].double()[..., None]
    x = x.masked_fill((torch.arange(W, device=DEVICE) >= s["live"][:, None])[..., None], -math.inf)
    best, at = torch.sort(x.view(B, W * V), dim=1, descending=True, stable=True)  # ties: the lowest index
    best, at = best[:, :s["keep"]], at[:, :s["keep"]]
    none = best == -math.inf
    parent, token = (at // V).masked_fill(none, -1), (at % V).masked_fill(none, -1)
    done = (torch.gather(s["finished"], 1, parent.clamp(min=0)).bool() | (token == s["end"])) & ~none
    return best.float(), parent.int(), token.int(), done.to(torch.uint8)


def _reorder(s):
    B, W = s["seqs"], s["beams"]
    if own:
        caches = _caches(s) if s["page"] else []
        states = [s["history"]] if s["page"] else [s["history"]] + [r[:, :s["live"] // 4] for r in s["rows"].unbind(0)]
        table = s["table"].contiguous() if s["page"] else None  # (of a single sequence it lies column by column)
        _decoder(s).wf_beam_reorder(s["parents"], states=states, caches=caches, page_table=table, lengths=s["lengths"] if s["page"] else None)
        if s["page"] and table is not s["table"]:
            s["table"].copy_(table)
        return _moved(s)
    source = (s["parents"].long() + W * torch.arange(B, device=DEVICE)[:, None]).view(-1)  # the row whose state each row takes
    s["history"].copy_(s["history"][source])
    if not s["page"]:
        live = s["live"] // 4
        s["rows"][:, :, :live] = s["rows"][:, source, :live]
        return _moved(s)
    page, n = s["page"], s["lengths"].long().repeat_interleave(W)
    full = n // page
    here = s["table"].long().gather(1, full.clamp(max=s["table"].shape[1] - 1)[:, None]).squeeze(1)  # the page being filled
    keep = torch.arange(page, device=DEVICE)[None] < (n % page)[:, None]
    _copy_rows(s["k_pages"].view(torch.uint8) if s["fmt"] != "bf16" else s["k_pages"], here, source, keep)
    _copy_rows(s["v_pages"].view(torch.uint8) if s["fmt"] != "bf16" else s["v_pages"], here, source, keep)
    if s["fmt"] != "bf16":
        _copy_rows(s["k_scale"].unsqueeze(-1), here, source, keep)
        _copy_rows(s["v_scale"].unsqueeze(-1), here, source, keep)
    old = torch.arange(s["table"].shape[1], device=DEVICE)[None] < full[:, None]
    s["table"].copy_(torch.where(old, s["table"][source], s["table"]))
    return _moved(s)


def _copy_rows(pages, here, source, keep):
    """pages [layers, pages, heads, rows, dim]: the kept rows of each beam's page become those of its parent's."""
    new, mine = pages[:, here[source]], pages[:, here]
    pages[:, here] = torch.where(keep[None, :, None, :, None], new, mine)


def _moved(s):
    if not s["page"]:
        return s["history"], s["rows"]
    out = [s["history"], s["table"], s["k_pages"], s["v_pages"]]
    return out if s["fmt"] == "bf16" else out + [s["k_scale"], s["v_scale"]]


# ---- the definitions in 64 bits, sequence by sequence

def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "reorder":
        return None
    if c["op"] == "select":
        B, W, V = c["seqs"], c["beams"], c["vocab"]
        x = s["logits"].double().cpu().numpy().reshape(B, W, V)
        live, done, score = (s[k].cpu().numpy() for k in ("live", "finished", "scores"))
        words = s["suppress"].cpu().numpy().view(np.uint32)
        off = np.unpackbits(words.view(np.uint8), bitorder="little")[:V].astype(bool)
        best = np.full((B, c["keep"]), -np.inf)
        for b in range(B):
            found = []
            for w in range(int(live[b])):
                if done[b, w]:
                    found.append(np.array([np.float64(score[b, w])]))
                    continue
                y = x[b, w][~off]
                top = y.max()
                y = np.float64(score[b, w]) + (y - (top + np.log(np.exp(y - top).sum())))
                found.append(np.sort(y)[::-1][:c["keep"]])
            best_b = np.sort(np.concatenate(found))[::-1][:c["keep"]]
            best[b, :len(best_b)] = best_b
        return torch.from_numpy(best), None, None, None
    rows, start = _sizes(c)
    cu = np.cumsum([0] + rows)
    if c["op"] == "store":
        return tuple(_exact_codes(s[x], c["fmt"]) for x in ("k", "v"))
    H, Hk, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    out = torch.zeros(s["n"], H, D, dtype=torch.float64, device=DEVICE)
    lse = torch.full((s["n"], H), -math.inf, dtype=torch.float64, device=DEVICE)
    for b in range(c["seqs"]):
        n, seen_to = rows[b], start[b] + (rows[b] if c["tail"] != "none" else 0)
        ids = s["table"][b, :-(-seen_to // P)].long()
        for h in range(Hk):
            side = []
            for pages, scale in ((s["k_pages"], s["k_scale"]), (s["v_pages"], s["v_scale"])):
                x = pages[:, h].view(torch.uint8)[ids].view(F8).float().double() if pages.dtype == F8 else pages[ids, h].double()
                x = x * scale[ids, h].double()[..., None] if c["fmt"] in ("e4m3", "int8") else x
                side.append(x.reshape(-1, D)[:seen_to])
            may = torch.ones(n, seen_to, dtype=torch.bool, device=DEVICE)
            if c["tail"] == "causal":
                may[:, start[b]:] = torch.tril(torch.ones(n, n, dtype=torch.bool, device=DEVICE))
            elif c["tail"] == "tree":
                raw = s["mask"][cu[b]:cu[b + 1]].cpu().numpy().view(np.uint8).reshape(n, -1)
                may[:, start[b]:] = torch.from_numpy(np.unpackbits(raw, axis=1, bitorder="little")[:, :n].astype(bool)).to(DEVICE)
            G = H // Hk
            for i in range(h * G, (h + 1) * G):
                z = s["q"][cu[b]:cu[b + 1], i].double() @ side[0].T / math.sqrt(D)
                z = torch.where(may, z, -math.inf)
                some = may.any(1)
                lse[cu[b]:cu[b + 1], i] = torch.logsumexp(z, 1)
                weight = torch.where(some[:, None], torch.softmax(z, 1), 0.0)
                out[cu[b]:cu[b + 1], i] = weight @ side[1]
    return out, lse


def _exact_codes(x, fmt):
    """What vectors are worth after the cache, by the definition: on the host, in 64 bits, step by step."""
    a = x.double().cpu().numpy()
    if fmt not in ("e4m3", "int8"):
        return torch.from_numpy(a)
    top = np.abs(a).max(-1, keepdims=True)
    safe = np.where(top > 0, top, 1.0)
    if fmt == "int8":
        s = (safe.astype(np.float32) / np.float32(127)).astype(np.float32)
        s = ((s.view(np.uint32).astype(np.uint64) + 0xFFFF) & 0xFFFF0000).astype(np.uint32).view(np.float32).astype(np.float64)
        s = np.where(top > 0, np.maximum(s, 2.0 ** -126), 1.0)
        return torch.from_numpy(np.rint(a / s) * s)
    s = np.where(top > 0, 2.0 ** np.maximum(np.ceil(np.log2(safe / 448.0)), -126.0), 1.0)
    y = a / s
    with np.errstate(divide="ignore"):
        e = np.maximum(np.floor(np.log2(np.abs(y))), -6.0)
    step = 2.0 ** (e - 3)
    return torch.from_numpy(np.rint(y / step) * step * s)
