"""Operators of a forward pass over a cache: rotary positions, keys and values appended to a paged
cache in 8 bits with the rotation on the way, and attention over that cache.

A case is one call (an append is followed by reading back the blocks that it wrote). Where `own` is
false the operators are computed from elementary torch operations; where it is true by the library's
kernels.

The cache: pages of `page` tokens, int8 [pages][heads][page / 16][2][16 dim]: of each 16 tokens and
head a block of keys [16][dim] and one of values [dim][16], and fp32 scales [pages][heads][page / 16][2].
A block's scale is the largest magnitude that was written to it over 127; where a later token of the
block raises it, the earlier codes are rounded again to the new scale.
"""
import math

import torch

own = False

DEV = "cuda"
F32, F64 = torch.float32, torch.float64
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 16
# query heads, kv heads and head dim of mebp_inputs.CONFIGS
HEADS = [(4, 2, 64), (14, 2, 64), (12, 2, 128), (4, 1, 256), (8, 4, 256)]
BLK, Q05, Q15, G1, G4 = HEADS


def _rope(tokens, heads, dim, dtype, **kw):
    c = {"op": "rope", "tokens": tokens, "heads": heads, "dim": dim, "dtype": dtype, "rot": dim, "interleaved": False,
         "backward": False, "gap": 0, "n_pos": 2048, "factor": 1.0, "theta": 1e4, "seqs": 1}
    c.update(kw)
    return c


def _cache(op, shape, dtype, **kw):
    hq, hkv, dim = shape
    c = {"op": op, "hq": hq, "hkv": hkv, "dim": dim, "dtype": dtype, "page": 64, "seqs": 1, "new": 1, "past": 0,
         "ragged": False, "window": 0}
    c.update(kw)
    return c


def listed():
    cases = {
        # the query heads of one decoded token: latency
        "rope-1x14x64-f16": _rope(1, 14, 64, "f16", n_pos=4096),
        # queries of a training batch, 8 sequences of 2048 tokens
        "rope-16384x8x256-bf16": _rope(16384, 8, 256, "bf16", seqs=8),
        # half of each head turns, in pairs of neighbours, at far positions of a scaled context; rows
        # of a matrix that holds the keys and values beside the queries
        "rope-part-1111x12x128-f32": _rope(1111, 12, 128, "f32", rot=64, interleaved=True, gap=512, n_pos=131072,
                                           factor=8.0, theta=1e6),
        # gradients of a batch on their way back to the projections
        "rope-backward-4096x12x128-f32": _rope(4096, 12, 128, "f32", backward=True, n_pos=1024, seqs=4, theta=1e6),
        # one decoded token: its key, value and queries; latency
        "append-1-q05-f16": _cache("append", Q05, "f16", past=1000),
        # a decoding step of a batch of conversations of all ages
        "append-64x1-q15-bf16": _cache("append", Q15, "bf16", seqs=64, past=4000, ragged=True, page=32),
        # prompts of a whole batch
        "append-8x2048-g4-bf16": _cache("append", G4, "bf16", seqs=8, new=2048),
        # one conversation, one token: latency
        "attend-1x4096-q05-f16": _cache("attend", Q05, "f16", past=4095),
        # a decoding step of a batch, lengths from a few tokens to 8192
        "attend-48x8192-g4-bf16": _cache("attend", G4, "bf16", seqs=48, past=8191, ragged=True),
        # one token behind a very long text
        "attend-1x131072-q15-f16": _cache("attend", Q15, "f16", past=131071, page=256),
        # chunks of prompts behind texts of odd lengths, in a sliding window
        "attend-5x333-window-g1-bf16": _cache("attend", G1, "bf16", seqs=5, new=333, past=3001, ragged=True, window=512, page=16),
        # prompts of a whole batch: the products bound it
        "attend-8x2048-g4-f16": _cache("attend", G4, "f16", seqs=8, new=2048),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def draw(rng):
    def log(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))

    op = rng.choice(["rope", "append", "attend", "attend"])
    if op == "rope":
        hq, hkv, dim = rng.choice(HEADS)
        heads = rng.choice([hq, hkv, hq + hkv])
        tokens = min(log(1, 16384), (1 << 25) // (heads * dim))
        dtype = rng.choice(["f32", "f16", "bf16"])
        return _rope(tokens, heads, dim, dtype, rot=rng.choice([dim, dim, dim // 2, dim // 4, 2 * rng.randrange(1, dim // 2 + 1)]),
                     interleaved=rng.random() < 0.4, backward=rng.random() < 0.4, gap=rng.choice([0, 0, 1, 8, 512]),
                     n_pos=log(64, 131072), factor=rng.choice([1.0, 1.0, 8.0, round(rng.uniform(1.5, 32.0), 2)]),
                     theta=rng.choice([1e4, 1e6]), seqs=rng.choice([1, 1, 3, 8]))
    shape = rng.choice(HEADS)
    hq, hkv, dim = shape
    kw = {"page": rng.choice([16, 32, 64, 128, 256]), "ragged": rng.random() < 0.6, "window": 0}
    if op == "append":
        kw["new"] = rng.choice([1, 1, log(1, 4096)])
        kw["seqs"] = max(1, min(log(1, 256), 16384 // kw["new"]))
        kw["past"] = rng.choice([0, log(1, 4096)])
        return _cache(op, shape, rng.choice(["f32", "f16", "bf16"]), **kw)
    # single tokens, a few at once, chunks and whole prompts
    kw["new"] = rng.choice([1, 1, 1, log(2, 16), log(16, 2048)])
    kw["past"] = rng.choice([0, log(1, 8192), log(1, 131072)]) if kw["new"] < 64 else rng.choice([0, log(1, 4096)])
    kw["window"] = rng.choice([0, 0, 512, 1024, log(1, 4096)])
    length = kw["past"] + kw["new"]
    most = min(400_000_000 // (length * 2 * hkv * dim), (1 << 28) // (kw["new"] * length * hq), 16384 // kw["new"])
    kw["seqs"] = max(1, min(log(1, 256), most))
    return _cache(op, shape, rng.choice(["f16", "bf16"]), **kw)


# ------------------------------------------------------------------------------- sizes
def _spread(case, key):
    """A number for each sequence: the case's own, or spread over 0 (a new token: 1) to it."""
    n, most = case["seqs"], case[key]
    if not case["ragged"]:
        return [most] * n
    low = 1 if key == "new" else 0
    return [most if s == n // 2 else low + int((most - low) * ((s * 0.6180339887 + 0.31) % 1.0)) for s in range(n)]


def _pairs(case):
    """Queries times visible keys, and keys that any query of their sequence sees, over the sequences."""
    pairs = seen = 0
    w = case["window"] or 1 << 30
    for new, past in zip(_spread(case, "new"), _spread(case, "past")):
        first, last = past + 1, past + new  # visible keys of the first and last query, without a window
        under = max(0, min(last, w) - past)  # queries whose window is not full
        pairs += under * (first + first + under - 1) // 2 + (new - under) * min(w, last)
        seen += min(past + new, w + new - 1)
    return pairs, seen


# ------------------------------------------------------------------------------- inputs
def _table(n_pos, rot, theta, factor):
    """(cos, sin) of each position and pair, the frequencies of the slower pairs lowered by `factor`
    (by parts: those with under one turn in 8192 positions whole, those with over 4 not)."""
    f = theta ** (-torch.arange(0, rot, 2, dtype=F64, device=DEV) / rot)
    part = ((8192 * f / (2 * math.pi) - 1.0) / 3.0).clamp(0, 1)
    f = f * (part + (1 - part) / factor)
    angle = torch.arange(n_pos, dtype=F64, device=DEV)[:, None] * f
    return torch.stack([torch.cos(angle), torch.sin(angle)], 2).float()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device=DEV) * std

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=DEV)

    st = dict(case)
    if case["op"] == "rope":
        n, h, d = case["tokens"], case["heads"], case["dim"]
        per = -(-n // case["seqs"])
        first = torch.randint(0, max(1, case["n_pos"] - per + 1), (case["seqs"],), generator=gen, device=DEV)
        at = torch.arange(n, device=DEV)
        st["pos"] = ((first[at // per] + at % per) % case["n_pos"]).to(torch.int32)
        st["table"] = _table(case["n_pos"], case["rot"], case["theta"], case["factor"])
        whole = torch.zeros((n, h * d + case["gap"]), dtype=dtype, device=DEV)
        st["x"] = whole[:, :h * d].view(n, h, d)
        st["x"].copy_(normal(n, h, d))
        st["y"] = torch.empty((n, h, d), dtype=dtype, device=DEV)
        return st
    hq, hkv, d, page = case["hq"], case["hkv"], case["dim"], case["page"]
    news, pasts = _spread(case, "new"), _spread(case, "past")
    start = [sum(news[:i]) for i in range(len(news) + 1)]
    n = start[-1]
    cols = max(-(-(a + b) // page) for a, b in zip(news, pasts))
    # a pool somewhat larger than the sequences need, its pages in no order; the last one stays free
    pages = case["seqs"] * cols + case["seqs"] // 8 + 2
    order = torch.randperm(pages - 1, generator=gen, device=DEV)
    st["ptable"] = order[:case["seqs"] * cols].view(case["seqs"], cols).to(torch.int32)
    st["past"], st["start"], st["max_len"] = ints(pasts), ints(start), max(a + b for a, b in zip(news, pasts))
    shape = (pages, hkv, page // BLOCK, 2, BLOCK * d)
    st["pages"] = torch.empty(shape, dtype=torch.int8, device=DEV)
    for p in range(0, pages, 256):
        part = st["pages"][p:p + 256]
        part.copy_(normal(*part.shape, std=36.0).round_().clamp_(-127, 127))
    # values of about 1, some blocks several times as large as others
    st["scales"] = torch.exp(normal(*shape[:4], std=0.3)) / 36.0
    st["q"] = normal(n, hq, d).to(dtype)
    if case["op"] == "append":
        # the projections' outputs side by side: keys and values are rows of one matrix
        kv = (normal(n, 2 * hkv, d) * torch.exp(normal(n, 2 * hkv, 1, std=0.4))).to(dtype)
        st["k"], st["v"] = kv[:, :hkv], kv[:, hkv:]
        st["table"] = _table(st["max_len"], d, 1e6, 1.0)
        st["q_out"] = torch.empty_like(st["q"])
        # what is read back: from each sequence's first block that is written to its end
        first = [p // BLOCK * BLOCK for p in pasts]
        rows = [p + m - f for p, m, f in zip(pasts, news, first)]
        st["first"], st["rows"] = ints(first), ints([sum(rows[:i]) for i in range(len(rows) + 1)])
        st["most"] = max(rows)
        st["k_out"] = torch.empty((sum(rows), hkv, d), dtype=F32, device=DEV)
        st["v_out"] = torch.empty_like(st["k_out"])
        return st
    st["out"] = torch.empty((n, hq, d), dtype=dtype, device=DEV)
    st["lse"] = torch.empty((n, hq), dtype=F32, device=DEV)
    # scratch for the parts of long sequences, which a program keeps beside its outputs
    st["ws"] = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    return st


# ------------------------------------------------------------------------------- plain form
def _turn(x, table, rot, interleaved, back):
    """x [tokens][heads][dim] turned by table [tokens][rot / 2][2], in x's type."""
    c, s = table[:, None, :, 0].to(x.dtype), table[:, None, :, 1].to(x.dtype)
    s = -s if back else s
    part = x[..., :rot]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :rot // 2], part[..., rot // 2:])
    ya, yb = a * c - b * s, b * c + a * s
    y = torch.stack([ya, yb], -1).flatten(-2) if interleaved else torch.cat([ya, yb], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _rows(start, n):
    """The sequence of each of n rows, and its place in it."""
    at = torch.arange(n, device=DEV)
    seq = torch.searchsorted(start[1:].contiguous(), at.to(torch.int32), right=True)
    return seq, at - start[seq]


def _blocks(st, seq, key):
    """The page, the block in it and the place in the block of tokens `key` of sequences `seq`."""
    page = st["ptable"][seq, (key // st["page"]).clamp(0, st["ptable"].shape[1] - 1)].long()
    return page, key % st["page"] // BLOCK, key % BLOCK


def _values(st, seq, key, heads=slice(None)):
    """Keys and values [.., heads, dim] in 32 bits of tokens `key` of sequences `seq`."""
    page, b, t = _blocks(st, seq, key)
    p, h, nb, _, _ = st["pages"].shape
    kc = st["pages"][:, :, :, 0].view(p, h, nb, BLOCK, -1)
    vc = st["pages"][:, :, :, 1].view(p, h, nb, -1, BLOCK)
    scale = st["scales"][page, :, b]
    return kc[page, :, b, t].float() * scale[..., 0, None], vc[page, :, b, :, t].float() * scale[..., 1, None]


def _plain_append(st):
    # rotation, scales and codes in 64 bits: a value next to the border of two codes
    n, d, dtype = st["k"].shape[0], st["dim"], st["q"].dtype
    seq, i = _rows(st["start"], n)
    pos = st["past"][seq] + i
    turn = st["table"][pos]
    st["q_out"].copy_(_turn(st["q"].double(), turn, d, False, False).to(dtype))
    new = torch.stack([_turn(st["k"].double(), turn, d, False, False), st["v"].double()], 2)  # [n][heads][2][dim]
    # the blocks from each sequence's first that is written
    off = st["past"] % BLOCK
    nb = (st["new"] + 2 * BLOCK - 2) // BLOCK
    at = (off[seq] + i).long()
    x = torch.zeros((st["seqs"], nb * BLOCK, st["hkv"], 2, d), dtype=F64, device=DEV)
    x[seq, at] = new
    x = x.view(st["seqs"], nb, BLOCK, st["hkv"], 2, d)
    mine = torch.zeros((st["seqs"], nb * BLOCK), dtype=torch.bool, device=DEV)
    mine[seq, at] = True
    mine = mine.view(st["seqs"], nb, BLOCK)
    first = torch.arange(nb, device=DEV)[None, :] == 0
    block = (st["past"] // BLOCK)[:, None] + torch.arange(nb, device=DEV)
    used = mine.any(2)
    # blocks that nothing is written to go to the page that no sequence has
    s = torch.arange(st["seqs"], device=DEV)[:, None].expand(-1, nb)
    page, b, _ = _blocks(st, s, block * BLOCK)
    page = torch.where(used, page, st["pages"].shape[0] - 1)
    old = torch.where((first & (off[:, None] > 0))[..., None, None], st["scales"][page, :, b], 0.0)  # [s][nb][heads][2]
    scale = torch.maximum(old, (x.abs().amax((2, 5)) / 127).float())
    over = torch.where(scale > 0, scale, 1.0).double()
    codes = torch.round(x / over[:, :, None, :, :, None])
    k_old = st["pages"][page, :, b, 0].view(st["seqs"], nb, st["hkv"], BLOCK, d)
    v_old = st["pages"][page, :, b, 1].view(st["seqs"], nb, st["hkv"], d, BLOCK)
    ratio = old.double() / over
    keep = (first[..., None] & (torch.arange(BLOCK, device=DEV) < off[:, None, None]))
    m, e = mine[:, :, None, :, None], keep[:, :, None, :, None]
    k_new = torch.where(m, codes[..., 0, :].transpose(2, 3),
                        torch.where(e, torch.round(k_old * ratio[..., 0, None, None]), k_old.double()))
    v_new = torch.where(m.transpose(3, 4), codes[..., 1, :].permute(0, 1, 3, 4, 2),
                        torch.where(e.transpose(3, 4), torch.round(v_old * ratio[..., 1, None, None]), v_old.double()))
    both = torch.stack([k_new.flatten(3), v_new.flatten(3)], 3).to(torch.int8)
    st["pages"][page, :, b] = both
    st["scales"][page, :, b] = scale
    seq, i = _rows(st["rows"], st["k_out"].shape[0])
    k, v = _values(st, seq, st["first"][seq] + i)
    st["k_out"].copy_(k)
    st["v_out"].copy_(v)
    return {"k": st["k_out"], "v": st["v_out"], "q": st["q_out"]}


def _plain_attend(st):
    n, hq, d = st["q"].shape
    s, new, most, hkv, w = st["seqs"], st["new"], st["max_len"], st["hkv"], st["window"]
    seq, i = _rows(st["start"], n)
    q = torch.zeros((s, new, hq, d), device=DEV)
    q[seq, i] = st["q"].float()
    seqs, keys = torch.arange(s, device=DEV)[:, None].expand(-1, most), torch.arange(most, device=DEV).expand(s, -1)
    k, v = _values(st, seqs, keys)
    # [s][kv heads][group x new][keys]
    q = q.view(s, new, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(s, hkv, -1, d)
    x = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * d ** -0.5
    at = (st["past"][:, None] + torch.arange(new, device=DEV))[:, :, None]
    seen = keys[:, None] <= at
    seen = seen & (keys[:, None] > at - w) if w else seen
    x = x.view(s, hkv, -1, new, most).masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(s, hkv, -1, most), v.permute(0, 2, 1, 3).contiguous()).view(s, hkv, -1, new, d) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(s, new, hq, d)
    lse = (m + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(s, new, hq)
    return {"out": o[seq, i].to(st["q"].dtype), "lse": lse[seq, i]}


# ------------------------------------------------------------------------------- the calls
def run(st):
    if own:
        from paper_2510_03425_amd import device as D
        if st["op"] == "rope":
            if "rope" not in st:
                st["rope"] = D.Rope(st["table"], st["dim"], st["interleaved"])
            return D.rope_apply(st["rope"], st["x"], st["pos"], st["y"], backward=st["backward"])
        if "cache" not in st:
            st["cache"] = D.KvCache(st["pages"], st["scales"])
            st["batch"] = D.KvBatch(st["start"], st["past"], st["ptable"], st["new"], st["max_len"])
            if st["op"] == "append":
                st["rope"] = D.Rope(st["table"], st["dim"])
                st["back"] = D.KvBatch(st["rows"], st["first"], st["ptable"], st["most"], st["max_len"])
        if st["op"] == "append":
            D.kv_append(st["cache"], st["batch"], st["k"], st["v"], st["rope"], st["q"], st["q_out"])
            D.kv_read(st["cache"], st["back"], st["k_out"], st["v_out"])
            return {"k": st["k_out"], "v": st["v_out"], "q": st["q_out"]}
        D.kv_attention(st["cache"], st["batch"], st["q"], st["out"], st["lse"], window=st["window"], ws=st["ws"])
        return {"out": st["out"], "lse": st["lse"]}
    if st["op"] == "rope":
        return _turn(st["x"].float(), st["table"][st["pos"].long()], st["rot"], st["interleaved"], st["backward"]).to(st["x"].dtype)
    return _plain_append(st) if st["op"] == "append" else _plain_attend(st)


def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"]
        # the table's rows that the positions need, once
        rows = min(case["tokens"], case["n_pos"])
        return {"bytes": 2 * n * case["dim"] * size + case["tokens"] * 4 + rows * case["rot"] * 4, "flops": n * case["rot"] * 3}
    hq, hkv, d, n = case["hq"], case["hkv"], case["dim"], sum(_spread(case, "new"))
    if case["op"] == "append":
        # keys and values in, codes out; queries in and out; the blocks' values in 32 bits
        back = sum(p % BLOCK + m for p, m in zip(_spread(case, "past"), _spread(case, "new")))
        nbytes = n * d * (2 * hkv * (size + 1) + 2 * hq * size) + back * hkv * d * 2 * 5 + n * d * 4
        return {"bytes": nbytes, "flops": n * d * (3 * (hq + hkv) + 2 * 3 * hkv) + back * hkv * d * 2}
    pairs, seen = _pairs(case)
    nbytes = seen * hkv * 2 * (d + 4 / BLOCK) + n * hq * (2 * d * size + 4)
    return {"bytes": int(nbytes), "flops": pairs * hq * (4 * d + 4)}


# ------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        # as products with the matrices of complex numbers
        x, r = st["x"].double(), case["rot"]
        t = st["table"][st["pos"].long()].double()
        z = torch.view_as_complex(t)[:, None, :]
        z = z.conj() if case["backward"] else z
        pick = torch.arange(r, device=DEV).view((r // 2, 2) if case["interleaved"] else (2, r // 2))
        pick = pick if case["interleaved"] else pick.t()
        u = torch.complex(x[..., pick[:, 0]], x[..., pick[:, 1]]) * z
        y = x.clone()
        y[..., pick[:, 0]], y[..., pick[:, 1]] = u.real, u.imag
        return y
    news, pasts, d, hkv = _spread(case, "new"), _spread(case, "past"), case["dim"], case["hkv"]
    group = case["hq"] // hkv
    if case["op"] == "append" and case["seqs"] * case["new"] > 4096:
        return None
    parts = {}

    def keep(**kw):
        for k, v in kw.items():
            parts.setdefault(k, []).append(v)

    row = 0
    for s, (new, past) in enumerate(zip(news, pasts)):
        ids = st["ptable"][s].long()
        # [heads][tokens][dim] of the sequence's pages, in 64 bits
        codes, scale = st["pages"][ids].double(), st["scales"][ids].double()
        scale = scale.permute(1, 0, 2, 3).reshape(hkv, -1, 2)
        codes = codes.permute(1, 0, 2, 3, 4).reshape(hkv, -1, 2, BLOCK * d)
        kc = codes[:, :, 0].reshape(hkv, -1, BLOCK, d)
        vc = codes[:, :, 1].reshape(hkv, -1, d, BLOCK).transpose(2, 3)
        rows = slice(row, row + new)
        row += new
        if case["op"] == "attend":
            k = (kc * scale[:, :, 0, None, None]).reshape(hkv, -1, d)
            v = (vc * scale[:, :, 1, None, None]).reshape(hkv, -1, d)
            lo = max(0, past - case["window"] + 1) if case["window"] else 0
            k, v = k[:, lo:past + new], v[:, lo:past + new]
            i = torch.arange(past, past + new, device=DEV)[:, None]
            j = torch.arange(lo, past + new, device=DEV)[None, :]
            hide = (j > i) | (j <= i - case["window"]) if case["window"] else j > i
            q = st["q"][rows].double().view(new, hkv, group, d)
            o = torch.empty_like(q)
            lse = torch.empty((new, hkv, group), dtype=F64, device=DEV)
            for h in range(hkv):
                for g in range(group):
                    x = (q[:, h, g] @ k[h].t() / math.sqrt(d)).masked_fill(hide, -math.inf)
                    lse[:, h, g] = torch.logsumexp(x, 1)
                    o[:, h, g] = torch.softmax(x, 1) @ v[h]
            keep(out=o.view(new, -1, d), lse=lse.view(new, -1))
            continue
        # complex numbers again for the rotation; then block by block
        z = torch.view_as_complex(st["table"][past:past + new].double())[:, None, :]

        def turned(x):
            u = torch.complex(x[..., :d // 2], x[..., d // 2:]) * z
            return torch.cat([u.real, u.imag], -1)

        keep(q=turned(st["q"][rows].double()))
        first = past // BLOCK
        for name, fresh, c, which in (("k", turned(st["k"][rows].double()), kc, 0), ("v", st["v"][rows].double(), vc, 1)):
            done = []
            for b in range(first, (past + new - 1) // BLOCK + 1):
                lo, hi = max(past, b * BLOCK), min(past + new, b * BLOCK + BLOCK)
                x = fresh[lo - past:hi - past].transpose(0, 1)  # [heads][tokens][dim]
                want = (x.abs().amax((1, 2)) / 127.0).float()
                had = lo - b * BLOCK
                was = scale[:, b, which].float() if had else torch.zeros_like(want)
                new_scale = torch.maximum(was, want).double()[:, None, None]
                codes = torch.cat([torch.round(c[:, b, :had] * (was.double()[:, None, None] / new_scale)), torch.round(x / new_scale)], 1)
                done.append((codes * new_scale).transpose(0, 1))
            keep(**{name: torch.cat(done)})
    whole = {k: torch.cat(v) for k, v in parts.items()}
    return {k: whole[k] for k in (("k", "v", "q") if case["op"] == "append" else ("out", "lse"))}
