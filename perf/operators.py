"""What is measured of the operators around the paged cache and the head.

Four calls, each in its plain form (elementary torch operations in 32 bits) and as a user makes it of the package:

* append: per-head norms of queries and keys, the position rotation, and the append to the paged cache (bf16, or 4-bit),
  with what the appended positions then stand for;
* attend: decode rows over a cache held in 4 bits;
* chunks: causal prompt chunks over such a cache;
* score: log probabilities of given tokens, entropy and the best alternatives.

The 4-bit cache. A pool is [layer][block][KV head] of 16 * D + 128 bytes, D the head width, a block 16 positions:
  K codes [16][D / 2]:  byte i of a position holds dims 2 i (low four bits) and 2 i + 1;
  V codes [D / 2][16]:  byte i of a position holds dims i (low four bits) and i + D / 2;
  K scales [16], V scales [16]:  bf16 pairs (s, m).
Code c stands for m + s c. A row (a position's K or V of one head) is stored with m = bf16(min), s = bf16((max - min) /
15) and c = clamp(round_half_even((x - m) / s), 0, 15), x in float32.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16
HEADS = {"8b": (32, 8, 128), "1b": (32, 8, 64), "gqa8": (16, 2, 128)}   # query heads, KV heads, head width


def _cache(name, op, heads, **kw):
    nh, nkv, hd = HEADS[heads] if isinstance(heads, str) else heads
    c = dict(name=name, op=op, heads=nh, kv_heads=nkv, head_dim=hd, dtype="bf16", kind="int4",
             seqs=1, rows_lo=1, rows_hi=1,     # rows of each sequence in this call, log-spaced
             before_lo=0, before_hi=0)         # positions that it holds already, log-spaced
    c.update(kw)
    return c


def listed():
    return [
        # the next token of one call: a launch's latency
        _cache("append one token", "append", "8b", before_lo=137, before_hi=137),
        # a decode step of 512 running calls, straight from the projection's fp32 sums
        _cache("append decode batch", "append", "8b", dtype="f32", seqs=512, before_lo=256, before_hi=32767),
        # a burst of ragged prompts, prefilled in one step
        _cache("append prompt burst", "append", "8b", seqs=24, rows_lo=64, rows_hi=3001),
        # the same at the narrow heads into a bf16 cache, chunks that start inside a block
        _cache("append bf16 cache", "append", "1b", kind="bf16", dtype="f32", seqs=40, rows_lo=32, rows_hi=1501,
               before_lo=1, before_hi=700),
        # one user's short question
        _cache("attend one call", "attend", "8b", before_lo=136, before_hi=136),
        # the steady state of a full card
        _cache("attend decode batch", "attend", "8b", seqs=384, before_lo=999, before_hi=7999),
        # the tail of a batch: a handful of very long contexts
        _cache("attend long tail", "attend", "8b", dtype="f32", seqs=7, before_lo=11999, before_hi=32000),
        # an expert batch at the narrow heads
        _cache("attend narrow heads", "attend", "1b", dtype="f32", seqs=160, before_lo=63, before_hi=2999),
        # aggregator prompts: long chunks behind what earlier steps cached
        _cache("chunks aggregator", "chunks", "8b", dtype="f32", seqs=2, rows_lo=1501, rows_hi=4096, before_lo=1001,
               before_hi=8000),
        # prompts arriving together, narrow heads
        _cache("chunks prompt burst", "chunks", "1b", seqs=24, rows_lo=64, rows_hi=3001),
        # the next token of one call, a small vocabulary
        dict(name="score one token", op="score", dtype="f32", rows=1, vocab=32000, pad=0, top=5, spread=3.0),
        # a full batch at the large vocabulary
        dict(name="score full batch", op="score", dtype="f32", rows=512, vocab=128256, pad=0, top=20, spread=2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another call of the same ranges: 1 to 512 sequences of 1 to 32k positions, every grouping of heads, both widths
    and types; 1 to 512 rows of logits over vocabularies of 32 to 160k, odd ones and padded rows among them."""
    while True:
        op = rng.choice(["append", "attend", "attend", "chunks", "score"])
        dtype = rng.choice(["bf16", "f32"])
        if op == "score":
            vocab = rng.choice([_log(rng, 32, 160000), 128256, 32000])
            c = dict(op=op, dtype=dtype, rows=_log(rng, 1, 512), vocab=vocab, pad=rng.choice([0, 0, 1, 8, 61]),
                     top=min(vocab, rng.choice([0, 1, 5, 20, rng.randint(2, 32)])), spread=round(rng.uniform(0.5, 6.0), 2))
            if work(c)["bytes"] <= 5.2e8:
                return c
            continue
        hd = rng.choice([64, 128])
        nkv, gq = rng.choice([(2, 8), (4, 8), (8, 4), (8, 4), (1, 4), (3, 2), (8, 2), (8, 1), (16, 1)])
        rows = sorted(_log(rng, 1, 4096) for _ in range(2)) if op == "chunks" or (op == "append" and rng.random() < 0.6) else [1, 1]
        before = sorted(_log(rng, 1, 32768) - 1 for _ in range(2))
        c = _cache("", op, (nkv * gq, nkv, hd), dtype=dtype, kind=rng.choice(["int4", "int4", "bf16"]) if op == "append" else "int4",
                   seqs=_log(rng, 1, 512), rows_lo=rows[0], rows_hi=rows[1], before_lo=before[0], before_hi=before[1])
        del c["name"]
        n, before = _lengths(c)
        total, longest = int(n.sum()), int((n + before).max())
        w = work(c)
        if total > 20000 or (n + before).sum() > 1.4e6 or w["bytes"] > 1.4e9 or w["flops"] > 4.5e11:
            continue
        if op != "append" and len(n) * longest * nkv * hd * 8 > 2.6e10:
            continue
        if op == "chunks" and len(n) * nkv * gq * int(n.max()) * longest * 4 > 1.2e10:
            continue
        return c


# ------------------------------------------------------------------ the sequences of a case

def _lengths(c):
    """(rows of this call, positions before them) of every sequence: fixed quantiles in a fixed order."""
    def spaced(lo, hi, key):
        q = (np.arange(c["seqs"]) + 0.5) / c["seqs"]
        v = np.rint(np.exp(np.log(lo + 1.0) + q * (np.log(hi + 1.0) - np.log(lo + 1.0)))).astype(np.int64) - 1
        return np.random.default_rng([c["seqs"], lo, hi, key]).permutation(v)
    return spaced(c["rows_lo"], c["rows_hi"], 1), spaced(c["before_lo"], c["before_hi"], 2)


def _pairs(c):
    n, before = _lengths(c)
    return float((n * before).sum() + (n * (n + 1) // 2).sum())


def work(c):
    """append: qkv in; q, the cache rows and the values that they stand for out. attend and chunks: the cached rows of
    every sequence once, q in, the answer out, and two products per visible (row, key). score: the logits once."""
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "score":
        return {"bytes": c["rows"] * (c["vocab"] * e + 12.0 + 8.0 * c["top"]), "flops": 4.0 * c["rows"] * c["vocab"]}
    nh, nkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    n, before = _lengths(c)
    rows, row = float(n.sum()), 2.0 * nkv * (hd / 2 + 4 if c["kind"] == "int4" else 2 * hd)
    if c["op"] == "append":
        return {"bytes": rows * ((2 * nh + 2 * nkv) * hd * e + row + 4 * nkv * hd), "flops": 10.0 * rows * (nh + 2 * nkv) * hd}
    return {"bytes": float((n + before).sum()) * row + 2 * rows * nh * hd * e, "flops": 4.0 * nh * hd * _pairs(c)}


# ------------------------------------------------------------------ inputs

def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _ints(v):
    return torch.as_tensor(np.ascontiguousarray(v), dtype=torch.int32, device="cuda")


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rnd = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    if c["op"] == "score":
        R, V = c["rows"], c["vocab"]
        x = (rnd(R, V + c["pad"]) * c["spread"]).to(_dtype(c))
        tok = torch.randint(0, V, (R,), device="cuda", generator=g, dtype=torch.int32)
        tok[::2] = x[::2, :V].float().argmax(1).int()            # as a sampler does: the likeliest, or another one
        return {"case": c, "logits": x[:, :V], "tokens": tok}

    nh, nkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    n, before = _lengths(c)
    T, longest = int(n.sum()), int((n + before).max())
    need = (n + before + BLOCK - 1) // BLOCK
    order = np.random.default_rng([int(seed), 3]).permutation(int(need.sum()))
    tables = np.full((c["seqs"], int(need.max())), -1)           # -1: blocks that a sequence does not have
    tables[np.arange(int(need.max()))[None] < need[:, None]] = order
    first = np.repeat(np.cumsum(n) - n, n)
    seq = np.repeat(np.arange(c["seqs"]), n)
    s = {"case": c, "blocks": len(order), "longest": longest, "tables": _ints(tables), "row_seq": _ints(seq),
         "row_pos": _ints(before[seq] + np.arange(T) - first)}
    if c["op"] == "append":
        a = torch.arange(longest, device="cuda").double()[:, None] * 10000.0 ** (-2.0 * torch.arange(hd // 2, device="cuda").double() / hd)
        s["rope"] = torch.stack([a.cos(), a.sin()], -1).float()  # [position][pair] of (cos, sin)
        s["q_gain"], s["k_gain"] = (1 + 0.2 * rnd(2, hd)).to(torch.bfloat16)
        s["qkv"] = (rnd(T, (nh + 2 * nkv) * hd) * torch.exp(0.5 * rnd(T, 1))).to(_dtype(c))
        size = 16 * hd + 128 if c["kind"] == "int4" else 4 * BLOCK * hd
        s["pool"] = torch.zeros(len(order) * nkv * size, dtype=torch.uint8, device="cuda")
        return s
    # a filled cache: codes of rows that are spread about their middle
    pool = torch.empty(len(order) * nkv, 16 * hd + 128, dtype=torch.uint8, device="cuda")
    for part in pool.split(1 << 15):
        code = lambda: (rnd(len(part), 16 * hd) * 2.7 + 7.5).round().clamp(0, 15).to(torch.uint8)  # noqa: E731
        part[:, :16 * hd] = code() | code() << 4
        sc = 0.2 * torch.exp(0.3 * rnd(len(part), 32, 1))
        part[:, 16 * hd:] = torch.cat([sc, 0.1 * rnd(len(part), 32, 1) - 7.5 * sc], -1).to(torch.bfloat16).view(torch.uint8).view(len(part), 128)
    s["pool"] = pool.view(-1)
    s["q"] = (2 * rnd(T, nh, hd)).to(_dtype(c))
    s["scale"] = 1.0 / math.sqrt(hd)
    if c["op"] == "attend":
        s["row_ctx"] = s["row_pos"] + 1
    else:
        s["chunk_start"] = _ints(np.concatenate([[0], np.cumsum(n)]))
        s["chunk_ctx"] = _ints(n + before)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    return {"append": _plain_append, "attend": _plain_attend, "chunks": _plain_chunks, "score": _plain_score}[s["case"]["op"]](s)


def _run_own(s):
    from paper_2606_03014_amd import ops
    c = s["case"]
    if c["op"] == "score":
        return ops.score_tokens(s["logits"], s["tokens"], top_k=c["top"])
    if "cache" not in s:                                         # the handle on the pool, which a program keeps
        s["cache"] = ops.PagedKV(c["kind"], 1, s["blocks"], c["heads"], c["kv_heads"], c["head_dim"], pool=s["pool"])
    if c["op"] == "append":
        q = s["cache"].append(0, s["qkv"], s["row_seq"], s["row_pos"], s["tables"], rope=s["rope"], q_gain=s["q_gain"],
                              k_gain=s["k_gain"], eps=1e-5)
        return (q, *s["cache"].read(0, s["row_seq"], s["row_pos"], s["tables"]))
    if c["op"] == "attend":
        return s["cache"].attend(0, s["q"], s["row_seq"], s["row_ctx"], s["tables"], s["longest"], s["scale"])
    return s["cache"].attend_chunks(0, s["q"], s["chunk_start"], s["chunk_ctx"], s["tables"], s["longest"], s["scale"])


def _norm_rotate(x, gain, cs):
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gain
    a, b = y.chunk(2, -1)
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _four_bit(x):
    """What the 4-bit rows of x (float32) stand for; in 64 bits, where a quotient lies next to the border of two codes."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    m, sc = lo.bfloat16().double(), ((hi - lo) / 15).bfloat16().double()
    code = ((x.double() - m) / torch.where(sc == 0, 1.0, sc)).round().clamp(0, 15)
    return m + sc * torch.where(sc == 0, 0.0, code)


def _plain_append(s):
    c = s["case"]
    nh, nkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    x = s["qkv"].float().view(-1, nh + 2 * nkv, hd)
    cs = s["rope"][s["row_pos"].long()]
    q = _norm_rotate(x[:, :nh], s["q_gain"].float(), cs)
    k = _norm_rotate(x[:, nh:nh + nkv].double(), s["k_gain"].double(), cs.double()).float()   # next to borders again
    v = x[:, nh + nkv:]
    if c["kind"] == "int4":
        k, v = _four_bit(k), _four_bit(v)
    return q.to(s["qkv"].dtype), k.bfloat16(), v.bfloat16()


def _values(s, tables):
    """K and V that the blocks of `tables` stand for, [sequence][KV head][position][dim]."""
    c = s["case"]
    nkv, hd = c["kv_heads"], c["head_dim"]
    b = s["pool"].view(s["blocks"], nkv, -1)[tables.clamp(min=0).long()].transpose(1, 2)   # [seq][head][block][bytes]
    at = 8 * hd
    k = b[..., :at].reshape(*b.shape[:3], BLOCK, hd // 2)
    v = b[..., at:2 * at].reshape(*b.shape[:3], hd // 2, BLOCK).transpose(3, 4)
    sc = b[..., 2 * at:].contiguous().view(torch.bfloat16).view(*b.shape[:3], 2, BLOCK, 2).float()
    k = torch.stack([k & 15, k >> 4], -1).flatten(4).float() * sc[..., 0, :, :1] + sc[..., 0, :, 1:]
    v = torch.cat([v & 15, v >> 4], -1).float() * sc[..., 1, :, :1] + sc[..., 1, :, 1:]
    return k.flatten(2, 3), v.flatten(2, 3)


def _attention(s, q, k, v, sees):
    """q [seq][KV head][query][dim]; sees: which keys a query sees, [seq][1][query][key]."""
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"]).masked_fill_(~sees, -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    return torch.matmul(p, v) / p.sum(-1, keepdim=True)


def _plain_attend(s):
    c = s["case"]
    k, v = _values(s, s["tables"])
    q = s["q"].float().view(c["seqs"], c["kv_heads"], -1, c["head_dim"])          # row i is sequence i's
    sees = torch.arange(k.shape[2], device="cuda")[None, None, None] < s["row_ctx"].view(-1, 1, 1, 1)
    return _attention(s, q, k, v, sees).reshape(s["q"].shape).to(s["q"].dtype)


def _plain_chunks(s):
    c = s["case"]
    nkv, gq, hd = c["kv_heads"], c["heads"] // c["kv_heads"], c["head_dim"]
    k, v = _values(s, s["tables"])
    seq = s["row_seq"].long()
    at = torch.arange(len(seq), device="cuda") - s["chunk_start"].long()[seq]     # a row's place in its chunk
    most = c["rows_hi"]
    q = torch.zeros(c["seqs"], nkv, gq, most, hd, device="cuda")
    q[seq, :, :, at] = s["q"].float().view(-1, nkv, gq, hd)
    pos = torch.zeros(c["seqs"], most, dtype=torch.int64, device="cuda")          # a padding row sees the first key
    pos[seq, at] = s["row_pos"].long()
    sees = (torch.arange(k.shape[2], device="cuda") <= pos[..., None]).repeat(1, gq, 1)[:, None]
    o = _attention(s, q.view(c["seqs"], nkv, gq * most, hd), k, v, sees).view(c["seqs"], nkv, gq, most, hd)
    return o[seq, :, :, at].reshape(s["q"].shape).to(s["q"].dtype)


def _plain_score(s):
    x = s["logits"].float()
    tok = s["tokens"].long()[:, None]
    top, ids = torch.sort(x, dim=1, descending=True, stable=True)
    x = x - top[:, :1]
    e = x.exp()
    total = e.sum(1, keepdim=True)
    norm = total.log()
    k = s["case"]["top"]
    return ((x.gather(1, tok) - norm)[:, 0], (norm - (e * x).sum(1, keepdim=True) / total)[:, 0],
            ids[:, :k].int().contiguous(), top[:, :k] - top[:, :1] - norm)


# ------------------------------------------------------------------ the definition in 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "score":
        x = s["logits"].double()
        lp = x - torch.logsumexp(x, 1, keepdim=True)
        r = torch.arange(c["rows"], device="cuda")
        order = torch.argsort(x, dim=1, descending=True, stable=True)[:, :c["top"]]
        return lp[r, s["tokens"].long()], -(lp.exp() * lp).sum(1), order.int(), lp.gather(1, order)
    nh, nkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    n, before = _lengths(c)
    if c["op"] == "append":
        return _exact_append(c, s)
    out = torch.empty(int(n.sum()), nh, hd, dtype=torch.float64, device="cuda")
    at = 0
    for b in range(c["seqs"]):
        L, m = int(n[b] + before[b]), int(n[b])
        pages = s["pool"].view(-1, nkv, 16 * hd + 128)[s["tables"][b, :(L + 15) // 16].long()]
        for h in range(nkv):
            page = pages[:, h]
            pair = page[:, 16 * hd:].contiguous().view(torch.bfloat16).double().view(-1, 2, 16, 2)
            kc = page[:, :8 * hd].reshape(-1, hd // 2)
            k = torch.empty(len(kc), hd, dtype=torch.float64, device="cuda")
            k[:, 0::2], k[:, 1::2] = (kc % 16).double(), (kc // 16).double()
            k = pair[:, 0, :, 1].reshape(-1, 1) + pair[:, 0, :, 0].reshape(-1, 1) * k
            vc = page[:, 8 * hd:16 * hd].reshape(-1, hd // 2, 16).permute(0, 2, 1).reshape(-1, hd // 2)
            v = torch.empty_like(k)
            v[:, :hd // 2], v[:, hd // 2:] = (vc % 16).double(), (vc // 16).double()
            v = pair[:, 1, :, 1].reshape(-1, 1) + pair[:, 1, :, 0].reshape(-1, 1) * v
            k, v = k[:L], v[:L]
            late = torch.arange(L, device="cuda")[None] > torch.arange(L - m, L, device="cuda")[:, None]
            for j in range(h * nh // nkv, (h + 1) * nh // nkv):
                w = (s["q"][at:at + m, j].double() @ k.t() * s["scale"]).masked_fill(late, -math.inf)
                out[at:at + m, j] = torch.softmax(w, 1) @ v
        at += m
    return out


def _exact_append(c, s):
    nh, nkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    x = s["qkv"].double().view(-1, nh + 2 * nkv, hd)
    cs = torch.view_as_complex(s["rope"].double())[s["row_pos"].long()]

    def turn(y, gain):
        y = y / (y.pow(2).sum(-1, keepdim=True) / hd + 1e-5).sqrt() * gain.double()
        z = torch.complex(y[..., :hd // 2], y[..., hd // 2:]) * cs[:, None]
        return torch.cat([z.real, z.imag], -1)

    def stored(x):
        x = x.float()                                            # what is cached is the float32 value
        if c["kind"] != "int4":
            return x.double()
        lo = x.min(-1, keepdim=True).values
        step = ((x.max(-1, keepdim=True).values - lo) / 15).to(torch.bfloat16).double()
        base = lo.to(torch.bfloat16).double()
        j = torch.floor((x.double() - base) / step)
        off = (x.double() - base) / step - j
        up = (off > 0.5) | ((off == 0.5) & (j % 2 == 1))
        return base + step * (j + up).clamp(0, 15)

    return turn(x[:, :nh], s["q_gain"]), stored(turn(x[:, nh:nh + nkv], s["k_gain"])), stored(x[:, nh + nkv:])
