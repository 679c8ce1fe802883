"""Operators around a round of speculative decoding as cases to be timed, with their plain forms.

Four operators: rows and pages of a round planned on the GPU (``plan``), products with 8-bit codes and one scale for each
128 channels of a row (``product``), verification of drafted tokens against the target's distribution (``verify``) and
the accepted rows of every layer's cache moved behind the committed ones (``commit``)."""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
F8 = torch.float8_e4m3fn
PATH = {"bf16": torch.bfloat16, "f32": torch.float32}
NBYTES = {"bf16": 2, "f32": 4, "e4m3": 1, "int8": 1}


def listed():
    return [
        # the projection of a single token, one stream (latency)
        dict(name="product one token", op="product", rows=1, k=1280, n=1280, x="bf16", out="bf16", bias=True, gelu=False),
        # the output projection of 64 streams onto the vocabulary: the weights' bytes, logits in float32
        dict(name="product logits", op="product", rows=64, k=1280, n=50_021, x="bf16", out="f32", bias=False, gelu=False),
        # 64 streams with five drafted tokens each through the second product of a feed-forward block
        dict(name="product drafts", op="product", rows=320, k=5120, n=1280, x="bf16", out="bf16", bias=True, gelu=False),
        # one buffer's rows through the first product of a feed-forward block
        dict(name="product buffer", op="product", rows=775, k=1280, n=5120, x="bf16", out="bf16", bias=True, gelu=True),
        # the same for a batch of 64 buffers
        dict(name="product 64 buffers", op="product", rows=49_600, k=1280, n=5120, x="bf16", out="bf16", bias=True, gelu=True),
        # one stream, a chain of four drafts with the draft's distributions (latency)
        dict(name="verify one stream", op="verify", seqs=1, rows=5, rows_lo=5, vocab=50_021, dtype="f32", tree=False, draft=True, greedy=0),
        # 64 streams with chains, some of them greedy; drafts that were looked up, not drawn
        dict(name="verify 64 streams", op="verify", seqs=64, rows=6, rows_lo=2, vocab=50_021, dtype="bf16", tree=False, draft=False, greedy=4),
        # trees of drawn drafts
        dict(name="verify trees", op="verify", seqs=16, rows=48, rows_lo=2, vocab=50_021, dtype="bf16", tree=True, draft=True, greedy=0),
        # one stream's accepted rows, grouped heads, twelve layers
        dict(name="commit one stream", op="commit", seqs=1, rows=16, keep=4, heads=8, dim=128, fmt="int8", page=64, layers=12, length=219),
        # 64 streams, all layers of a large decoder
        dict(name="commit 64 streams", op="commit", seqs=64, rows=16, keep=6, heads=20, dim=64, fmt="e4m3", page=16, layers=32, length=44),
        # an ordinary round: one token for each of 64 streams, pages of 16
        dict(name="plan one token", op="plan", seqs=64, rows=1, rows_lo=1, lo=0, hi=447, every=0, page=16, spare=2.0),
        # prompts of hundreds of sequences in the places of those that have ended
        dict(name="plan prompts", op="plan", seqs=256, rows=1500, rows_lo=75, lo=75, hi=1900, every=1, page=16, spare=1.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["product", "product", "product", "verify", "verify", "commit", "plan"])
    if op == "product":
        rows, k, n = _log(rng, 1, 30_000), _log(rng, 32, 8000), _log(rng, 8, 60_000)
        rows = max(1, min(rows, 200_000_000_000 // (k * n), 200_000_000 // n))
        if rng.random() < 0.6:
            k, n = max(k // 128, 1) * 128, max(n // 64, 1) * 64
        return dict(op=op, rows=rows, k=k, n=n, x=rng.choice(["bf16", "bf16", "f32"]), out=rng.choice(["bf16", "bf16", "f32"]),
                    bias=rng.random() < 0.7, gelu=rng.random() < 0.4)
    if op == "verify":
        tree = rng.random() < 0.5
        seqs, rows = _log(rng, 1, 96), _log(rng, 2, 60 if tree else 9)
        vocab = min(_log(rng, 300, 150_000), 18_000_000 // (seqs * rows))
        return dict(op=op, seqs=seqs, rows=rows, rows_lo=rng.randint(1, rows), vocab=vocab, dtype=rng.choice(["bf16", "f32"]), tree=tree,
                    draft=rng.random() < 0.5, greedy=rng.choice([0, 0, 2, 5]))
    if op == "commit":
        rows = rng.randint(2, 48)
        return dict(op=op, seqs=_log(rng, 1, 48), rows=rows, keep=rng.randint(1, min(rows, 10)), heads=rng.choice([1, 4, 8, 12]),
                    dim=rng.choice([64, 128]), fmt=rng.choice(["bf16", "e4m3", "int8"]), page=rng.choice([16, 32, 64, 128]), layers=rng.randint(1, 16),
                    length=rng.randint(0, 100))
    rows, hi = _log(rng, 1, 3000), _log(rng, 1, 4000)
    return dict(op=op, seqs=min(_log(rng, 1, 700), max(1, 300_000 // rows)), rows=rows, rows_lo=rng.randint(0, rows), lo=rng.randint(0, hi), hi=hi,
                every=rng.choice([0, 1, 3, 8]), page=rng.choice([16, 32, 64, 128, 256]), spare=rng.choice([0.6, 1.0, 1.7, 3.0]))


# ---- sizes that follow from a case alone (so that the work is known without its inputs)

def _spread(lo, hi, n, step):
    """n whole numbers over [lo, hi], hi among them, in no order."""
    return [hi if i == 0 else lo + int((hi - lo + 1) * ((i * step) % 1.0)) for i in range(n)]


def _rows(c):
    return _spread(c["rows_lo"], c["rows"], c["seqs"], 0.7548776662)


def _lengths(c):
    if c["op"] == "plan":
        return _spread(c["lo"], c["hi"], c["seqs"], 0.6180339887)
    return [(c["length"] + 5 * b) % (c["length"] + 1) if b else c["length"] for b in range(c["seqs"])]


def _paths(c):
    """The rows that stay, of every sequence: the first one and, from there, ever deeper drafts."""
    out = []
    for b in range(c["seqs"]):
        keep = 1 + (c["keep"] - 1 + 3 * b) % c["keep"] if b else c["keep"]
        last = max(keep - 1, c["rows"] - 1 - b % 3)
        out.append([0] + [max(i, i * last // (keep - 1)) for i in range(1, keep)])
    return out


def work(case):
    c = case
    if c["op"] == "product":
        blocks = -(-c["k"] // 128)
        return {"bytes": c["rows"] * c["k"] * NBYTES[c["x"]] + c["n"] * (c["k"] + blocks) + c["rows"] * c["n"] * NBYTES[c["out"]]
                + (4 * c["n"] if c["bias"] else 0), "flops": 2 * c["rows"] * c["k"] * c["n"]}
    if c["op"] == "verify":
        n = sum(_rows(c))
        # every row's logits once, and one row of the draft's distribution for the token that is drawn
        return {"bytes": n * c["vocab"] * NBYTES[c["dtype"]] + (4 * c["vocab"] * c["seqs"] if c["draft"] else 0) + 24 * n, "flops": 4 * n * c["vocab"]}
    if c["op"] == "commit":
        moved = sum(p != i for path in _paths(c) for i, p in enumerate(path))
        vec = c["dim"] * NBYTES[c["fmt"]] + (0 if c["fmt"] == "bf16" else 2)
        return {"bytes": 2 * moved * c["layers"] * 2 * c["heads"] * vec + 8 * c["seqs"] * (c["keep"] + 3), "flops": 0}
    n, page = sum(_rows(c)), c["page"]
    pages = 0
    for i, (r, l) in enumerate(zip(_rows(c), _lengths(c))):
        gone = c["every"] and i % c["every"] == 0
        held = -(-l // page)
        pages += (held if gone else 0) + (max(0, -(-((0 if gone else l) + r) // page) - (0 if gone else held)) if r else 0)
    return {"bytes": 16 * n + 8 * pages + 29 * c["seqs"], "flops": 0}


# ---- the codes: e4m3 with the least power of two that fits as the scale of 128 channels of a row

def _codes(x):
    """x [rows, k] -> codes as float32 values [rows, k] and scales [rows, blocks] (float32, powers of two)."""
    n, k = x.shape
    blocks = -(-k // 128)
    y = torch.zeros(n, blocks * 128, device=x.device)
    y[:, :k] = x
    y = y.view(n, blocks, 128)
    top = y.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    s = torch.ldexp(torch.ones_like(top), (e - torch.where(m <= 0.875, 9, 8)).clamp(min=-126))
    s = torch.where(top > 0, s, torch.ones_like(s))
    return (y / s).to(F8).float().view(n, blocks * 128)[:, :k], s.squeeze(-1)


def _times_scales(codes, s):
    return codes * s.repeat_interleave(128, dim=1)[:, :codes.shape[1]]


# ---- inputs

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    c = case
    host = torch.Generator().manual_seed(seed)
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    s = dict(c)
    if c["op"] == "product":
        size = torch.exp(0.7 * normal(1, c["k"]))  # channels differ in size
        s["x"] = (normal(c["rows"], c["k"]) * size).to(PATH[c["x"]])
        s["b"] = normal(c["n"]) if c["bias"] else None
        w = normal(c["n"], c["k"]) / (size * math.sqrt(c["k"]))
        s["w"], s["w_scale"] = _codes(w)  # laid out once, as a program keeps its weights
        s["w"] = s["w"].to(F8)
        return s
    if c["op"] == "verify":
        rows, V = _rows(c), c["vocab"]
        n, cu = sum(rows), np.cumsum([0] + rows)
        parents = np.zeros(n, np.int64)
        pick = torch.rand(n, generator=host).numpy()
        for b in range(c["seqs"]):
            for i in range(1, rows[b]):
                parents[cu[b] + i] = int(pick[cu[b] + i] * i) if c["tree"] else i - 1
        at = torch.from_numpy(parents + np.repeat(cu[:-1], rows)).to(DEVICE)  # the parent's row in the batch
        logits = 1.5 * normal(n, V)
        peaks = torch.randint(0, V, (n, 8), generator=g, device=DEVICE)
        logits.scatter_(1, peaks, 9.0 + 3.0 * torch.rand(n, 8, generator=g, device=DEVICE))
        s["logits"] = logits.to(PATH[c["dtype"]])
        guess = logits + 0.7 * normal(n, V)  # the draft model's opinion of the same rows
        if c["draft"]:
            s["draft"] = torch.softmax(guess, 1)
            s["tokens"] = torch.multinomial(s["draft"][at], 1, generator=g).view(-1).int()
        else:
            s["draft"] = None
            rank = [sum(parents[cu[b]:j] * 1 == parents[j]) - (1 if parents[j] == 0 else 0) if j > cu[b] else 0
                    for b in range(c["seqs"]) for j in range(cu[b], cu[b + 1])]  # which of its parent's children a row is
            best = torch.topk(guess, min(V, max(rank) + 1), dim=1).indices
            s["tokens"] = best[at, torch.tensor(rank, device=DEVICE) % best.shape[1]].int()
        s["cu"] = _ints(cu.tolist())
        s["parents"] = _ints(parents.tolist()) if c["tree"] else None
        s["temperature"] = torch.tensor([0.0 if c["greedy"] and b % c["greedy"] == 0 else 0.7 + 0.1 * (b % 5) for b in range(c["seqs"])], device=DEVICE)
        s["u"] = torch.rand(n, generator=g, device=DEVICE)
        s["u_last"] = torch.rand(c["seqs"], generator=g, device=DEVICE)
        return s
    if c["op"] == "commit":
        lengths, page = _lengths(c), c["page"]
        each = [-(-(l + c["rows"]) // page) for l in lengths]
        pages = sum(each)
        table = torch.full((c["seqs"], max(each)), -1, dtype=torch.int32)
        order, at = torch.randperm(pages, generator=host).int(), 0
        for b, e in enumerate(each):
            table[b, :e] = order[at:at + e]
            at += e
        s["table"] = table.to(DEVICE)
        shape = (c["layers"], pages, c["heads"], page, c["dim"])
        s["k_pages"], s["v_pages"] = (normal(*shape).to(F8 if c["fmt"] == "e4m3" else torch.bfloat16) if c["fmt"] != "int8" else
                                      torch.randint(-127, 128, shape, generator=g, device=DEVICE, dtype=torch.int8) for _ in range(2))
        s["k_scale"], s["v_scale"] = (torch.rand(shape[:4], generator=g, device=DEVICE).bfloat16() if c["fmt"] != "bf16" else None for _ in range(2))
        paths = _paths(c)
        s["kept"] = _ints([len(p) for p in paths])
        s["path"] = _ints([p + [-1] * (c["rows"] - len(p)) for p in paths])
        s["start"] = _ints(lengths)
        return s
    rows, lengths, page = _rows(c), _lengths(c), c["page"]
    held = [-(-l // page) for l in lengths]
    gone = [int(bool(c["every"]) and i % c["every"] == 0) for i in range(c["seqs"])]
    need = sum(max(0, -(-((0 if e else l) + r) // page) - (0 if e else h)) if r else 0 for r, l, h, e in zip(rows, lengths, held, gone))
    free = int(need * c["spare"]) + 1
    pages = sum(held) + free
    order = torch.randperm(pages, generator=host).int()
    table = torch.full((c["seqs"], max(-(-(max(l, 0) + r) // page) for l, r in zip(lengths, rows)) + 1), -1, dtype=torch.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    head = int(torch.randint(0, pages, (1,), generator=host))
    ring = torch.full((pages,), -1, dtype=torch.int32)
    ring[(head + torch.arange(free)) % pages] = order[at:]
    s["ring"], s["pool"], s["table"] = ring.to(DEVICE), _ints([head, free]), table.to(DEVICE)
    s["held"], s["lengths"], s["new"] = _ints(held), _ints(lengths), _ints(rows)
    s["ended"] = torch.tensor(gone, dtype=torch.uint8, device=DEVICE) if c["every"] else None
    s["room"] = sum(rows) + sum(rows) // 16
    return s


# ---- one pass

def run(state):
    return {"product": _product, "verify": _verify, "commit": _commit, "plan": _plan}[state["op"]](state)


_kept = {}


def _decoder(s):
    """The framework's handle for these heads and this cache, kept as a program keeps it."""
    from paper_2412_11272_b200.binding import Decoder
    fmt = s.get("fmt") or "bf16"
    key = (s.get("heads") or 1, s.get("dim") or 64, "path" if fmt == "bf16" else fmt, s.get("page") or 16)
    if key not in _kept:
        _kept[key] = Decoder(n_head=key[0], d_head=key[1], dtype="bf16", cache_format=key[2], page_size=key[3])
    return _kept[key]


def _product(s):
    if own:
        from paper_2412_11272_b200.binding import ScaledCodes
        d = _decoder(s)
        if "weights" not in s:  # laid out once
            s["weights"] = ScaledCodes.pack(s["w"], s["w_scale"])
        return d.wf_gemm_e4m3(d.wf_quantise_e4m3(s["x"]), s["weights"], bias=s["b"], gelu=s["gelu"], out_dtype=s["out"])
    y = torch.matmul(_times_scales(*_codes(s["x"].float())), _times_scales(s["w"].float(), s["w_scale"]).T)
    if s["b"] is not None:
        y += s["b"]
    if s["gelu"]:
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    return y.to(PATH[s["out"]])


def _softmax(s, row, t):
    """The target's distribution after these rows of the batch, in 64 bits; at temperature 0 all of it on the first largest."""
    x = s["logits"][row].double()
    m, first = x.max(1, keepdim=True)
    first = (x == m).float().argmax(1, keepdim=True)
    p = ((x - m) / torch.where(t > 0, t, 1.0)[:, None]).exp()
    p = p / p.sum(1, keepdim=True)
    return torch.where((t > 0)[:, None], p, torch.zeros_like(p).scatter_(1, first, 1.0))


def _verify(s):
    if own:
        return _decoder(s).wf_draft_verify(s["logits"], s["cu"], s["tokens"], s["u"], s["u_last"], s["rows"], parents=s["parents"], draft=s["draft"],
                                           temperature=s["temperature"])
    B, R, V = s["seqs"], s["rows"], s["vocab"]
    first, count = s["cu"][:-1].long(), (s["cu"][1:] - s["cu"][:-1]).long()
    t, every = s["temperature"].double(), torch.arange(B, device=DEVICE)
    kept = (count > 0).long()
    path = torch.full((B, R), -1, dtype=torch.long, device=DEVICE)
    token = path.clone()
    path[:, 0] = kept - 1
    cur = torch.zeros(B, dtype=torch.long, device=DEVICE)
    last = s["logits"].shape[0] - 1
    p = _softmax(s, first.clamp(max=last), t)
    for i in range(1, R):  # a row's children come after it, in the order in which they are tried
        row = (first + i).clamp(max=last)
        parent = s["parents"][row].long() if s["parents"] is not None else torch.full_like(cur, i - 1)
        tried = (i < count) & (parent == cur)
        x = s["tokens"][row].long()[:, None]
        q = s["draft"][first + cur].double() if s["draft"] is not None else torch.zeros_like(p).scatter_(1, x, 1.0)
        px, qx = p.gather(1, x).squeeze(1), q.gather(1, x).squeeze(1)
        taken = tried & torch.where(t > 0, s["u"][row].double() * qx < px, px > 0)
        rest = (p - q).clamp(min=0.0)
        if s["draft"] is None:
            rest = p.scatter(1, x, 0.0)
        total = rest.sum(1, keepdim=True)
        refused = tried & ~taken & (t > 0) & (total.squeeze(1) > 0)
        p = torch.where(refused[:, None], rest / total.clamp(min=1e-300), p)
        path[every, torch.where(taken, kept, R - 1)] = torch.where(taken, i, path[:, R - 1])
        token[every, torch.where(taken, kept - 1, R - 1)] = torch.where(taken, x.squeeze(1), token[:, R - 1])
        kept += taken
        cur = torch.where(taken, i, cur)
        p = torch.where(taken[:, None], _softmax(s, row, t), p)
    sums = p.cumsum(1)
    drawn = (sums <= s["u_last"].double()[:, None] * sums[:, -1:]).sum(1).clamp(max=V - 1)
    token[every, (kept - 1).clamp(min=0)] = torch.where(count > 0, drawn, -1)
    return kept.int(), token.int(), path.int()


def _commit(s):
    if own:
        d = _decoder(s)
        if "caches" not in s:  # the views of the layers' caches, kept beside them as a program keeps them
            from paper_2412_11272_b200.binding import KvCache
            parts = [s["k_pages"], s["v_pages"]] + ([] if s["fmt"] == "bf16" else [s["k_scale"], s["v_scale"]])
            s["caches"] = [KvCache(*layer) for layer in zip(*parts)]
        lengths = d.wf_draft_commit(s["start"], s["kept"], s["path"], caches=s["caches"], page_table=s["table"])
    else:
        R, page, start = s["rows"], s["page"], s["start"].long()[:, None]
        i = torch.arange(R, device=DEVICE)[None]
        moves = (i < s["kept"][:, None]) & (s["path"] != i)
        seq = torch.arange(s["seqs"], device=DEVICE)[:, None].expand(-1, R)
        to = torch.where(moves, start + i, 0)
        of = torch.where(moves, start + s["path"].long(), 0)
        table = s["table"].long()
        to_page, of_page = table[seq, to // page], table[seq, of // page]
        for x in (s["k_pages"], s["v_pages"]) + (() if s["fmt"] == "bf16" else (s["k_scale"].unsqueeze(-1), s["v_scale"].unsqueeze(-1))):
            x = x.view(torch.uint8) if x.dtype == F8 else x
            # what does not move is written back as it is: each place is named once
            new = x[:, torch.where(moves, of_page, to_page), :, torch.where(moves, of % page, to % page)]
            x[:, to_page[moves], :, (to % page)[moves]] = new[moves]
        lengths = s["start"] + s["kept"]
    out = [lengths, s["k_pages"], s["v_pages"]]
    return out if s["fmt"] == "bf16" else out + [s["k_scale"], s["v_scale"]]


def _plan(s):
    if own:
        d = _decoder(s)
        if "page_pool" not in s:
            from paper_2412_11272_b200.binding import PagePool
            s["page_pool"] = PagePool(s["ring"], s["pool"])
        out = d.wf_page_plan(s["page_pool"], s["table"], s["held"], s["lengths"], s["new"], s["room"], ended=s["ended"])
        return list(out) + [s["table"], s["held"], s["lengths"], s["ring"], s["pool"]]
    B, page, N, stride = s["seqs"], s["page"], s["ring"].numel(), s["table"].shape[1]
    head, free = s["pool"][0].long(), s["pool"][1].long()
    ended = s["ended"].bool() if s["ended"] is not None else torch.zeros(B, dtype=torch.bool, device=DEVICE)
    held, length = s["held"].long(), s["lengths"].long().masked_fill(ended, 0)
    gone = held.masked_fill(~ended, 0)
    held = held.masked_fill(ended, 0)
    want = s["new"].long()
    want = want.masked_fill(length + want > stride * page, 0)
    need = torch.where(want > 0, ((length + want + page - 1) // page - held).clamp(min=0), 0)
    may = (want.cumsum(0) <= s["room"]) & ((need == 0) | (need.cumsum(0) <= free))
    want, need = want * may, need * may
    old = s["table"].clone()
    # pages given back, behind the free ones
    i = torch.arange(N, device=DEVICE)
    behind = gone.cumsum(0)
    seq = torch.searchsorted(behind, i, right=True).clamp(max=B - 1)
    at = (i - (behind - gone)[seq]).clamp(0, stride - 1)
    back = i < behind[-1]
    place = (head + free + i) % N
    s["ring"][place] = torch.where(back, old[seq, at], s["ring"][place])
    # pages handed out, from the front of the ring
    behind = need.cumsum(0)
    seq = torch.searchsorted(behind, i, right=True).clamp(max=B - 1)
    at = held[seq] + i - (behind - need)[seq]
    given = i < behind[-1]
    wide = torch.cat([s["table"], s["table"][:, :1]], 1)  # a column for what is not given
    wide[seq, torch.where(given, at, stride)] = s["ring"][(head + i) % N]
    s["table"].copy_(wide[:, :stride])
    s["pool"][0] = (head + behind[-1]) % N
    s["pool"][1] = free - behind[-1] + gone.sum()
    s["held"].copy_(held + need)
    s["lengths"].copy_(length)
    # rows
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=DEVICE), want.cumsum(0)])
    row = torch.arange(s["room"], device=DEVICE)
    seq = (torch.searchsorted(cu, row, right=True) - 1).clamp(max=B - 1)
    pos = length[seq] + row - cu[seq]
    inside = row < cu[-1]
    slot = s["table"][seq, (pos // page).clamp(max=stride - 1)].long() * page + pos % page
    return [cu.int(), torch.where(inside, seq, -1).int(), torch.where(inside, pos, -1).int(), torch.where(inside, slot, -1),
            s["table"], s["held"], s["lengths"], s["ring"], s["pool"]]


# ---- the definition in 64 bits

def exact(case, seed):
    c = case
    if c["op"] != "product":
        return None  # whole numbers and moved bytes
    s = prepare(case, seed)
    a = _exact_values(s["x"])
    w = s["w"].float().double() * s["w_scale"].double().repeat_interleave(128, dim=1)[:, :c["k"]]
    out = torch.empty(c["rows"], c["n"], dtype=torch.float64, device=DEVICE)
    for i in range(0, c["rows"], 4096):
        y = a[i:i + 4096] @ w.T
        if s["b"] is not None:
            y = y + s["b"].double()
        out[i:i + 4096] = y * torch.special.ndtr(y) if c["gelu"] else y
    return out


def _exact_values(x):
    """What the rows of x are worth as codes, by the definition, in 64 bits, step by step."""
    n, k = x.shape
    out = torch.empty(n, k, dtype=torch.float64, device=x.device)
    for b in range(0, k, 128):
        a = x[:, b:b + 128].double()
        top = a.abs().amax(1, keepdim=True)
        safe = torch.where(top > 0, top, 1.0)
        s = torch.exp2(torch.ceil(torch.log2(safe / 448.0)).clamp(min=-126.0))
        s = torch.where(safe > 448.0 * s, 2.0 * s, torch.where(safe <= 224.0 * s, (0.5 * s).clamp(min=2.0 ** -126), s))  # the logarithm is rounded
        y = a / s
        e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -40))).clamp(min=-6.0)
        step = torch.exp2(e - 3.0)
        out[:, b:b + 128] = torch.where(top > 0, torch.round(y / step) * step * s, 0.0)
    return out
