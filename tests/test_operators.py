"""The cache and head operators (paper_2606_03014_amd/ops.py) against plain 64-bit implementations, and their refusals.

Tolerances. u = 2^-24 is half a step of float32, 2^-8 of bf16.
* append: cached rows are compared for equality, since the definition fixes every rounding. q: a norm of D terms and a
  rotation are fewer than 32 roundings of a row: 32 u of the row's largest value, and 2^-8 of the value in bf16.
* attention. A score is off by at most A * 2^-15 with A = max over keys of |scale| sum |q||k| (a split-bf16 q is 2^-17
  off; 128 products of codes offset by 16 add at most 200 u * 31 / 15). A probability is then off by twice that
  relatively, and the products with V and their sums by 2^-15: |out| is off by at most Vmax (2 A + 1) 2^-15; in bf16, 2^-8 of
  the value more, and 2^-12 of each probability, whose V-row spans 15 steps: 2^-11 Vmax. Those roundings are independent, so over all elements the 2-norm is far smaller: for scores with a
  standard deviation of up to 2 the relative 2-norm is at most 2 * 2^-18 (scores) + 2^-18 (probabilities) + sums below
  2^-18: 2^-16 (bf16: 2^-8 / sqrt(3) of the answer and 2^-12 of a probability more, at most 2^-8).
* scores: sums of n positive terms in partial sums of at most n / 256 + 16: 2^-17 for 128k tokens; the terms' exponents
  are |d| u off: 1e-5 + 4 u |logprob| (entropy: 1e-5 (1 + H)).
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2606_03014_amd import moa as M

F, B = torch.float32, torch.bfloat16
gpu = pytest.mark.gpu


# ------------------------------------------------------------------ plain forms, 64 bits, on the CPU

def q4(x):
    """(values, codes, scale, min) of the 4-bit rows of x (float32) along its last axis."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    m, s = lo.to(B), ((hi - lo) * torch.tensor(1 / 15, dtype=F)).to(B)
    bad = ~(x.isfinite().all(-1, keepdim=True) & (hi - lo).isfinite() & m.isfinite())
    s = torch.where(bad, torch.tensor(math.nan, dtype=B), s)
    m = torch.where(bad, torch.tensor(0.0, dtype=B), m)
    ok = s > 0
    c = ((x.double() - m.double()) / torch.where(ok, s.double(), 1.0)).round().clamp(0, 15)
    c = torch.where(ok, c, 0.0)
    return m.double() + s.double() * c, c.to(torch.uint8), s, m


def turn(x, gain, eps, rope, pos):
    x = x.double()
    if gain is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + float(np.float32(eps))).sqrt() * gain.double()
    if rope is not None:
        cos, sin = rope.double()[pos.long()][:, None].unbind(-1)
        a, b = x.chunk(2, -1)
        x = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return x


def cells(k, v, fill):
    """Pool bytes of an int4 cell from 4-bit rows [n <= 16, D] of K and V (codes, s, m); unused slots hold `fill` codes
    and NaN scales."""
    D = k[0].shape[1]
    n = len(k[0])
    out = np.full(16 * D + 128, fill, np.uint8)
    kc, vc = out[:8 * D].reshape(16, D // 2), out[8 * D:16 * D].reshape(D // 2, 16)
    kc[:n] = (k[0][:, 0::2] | k[0][:, 1::2] << 4).numpy()
    vc[:, :n] = (v[0][:, :D // 2] | v[0][:, D // 2:] << 4).t().numpy()
    sc = torch.full((2, 16, 2), math.nan, dtype=B)
    for i, r in enumerate((k, v)):
        sc[i, :n, 0], sc[i, :n, 1] = r[1].flatten(), r[2].flatten()
    out[16 * D:] = sc.view(torch.uint8).numpy().reshape(-1)
    return out


def attention(q, k, v, scale):
    """q [n_h, D] against k, v [keys, n_kv, D], all float64; no keys: zeros. Also A of the tolerance."""
    n_h, g = len(q), len(q) // k.shape[1]
    if not len(k):
        return torch.zeros_like(q), 0.0
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    s = torch.einsum("hd,khd->hk", q, k) * scale
    A = float((torch.einsum("hd,khd->hk", q.abs(), k.abs()) * abs(scale)).max())
    return torch.einsum("hk,khd->hd", torch.softmax(s, -1), v), A


class Pool:
    """An int4 pool of given sequences' random rows, blocks in a random order, everything else NaN scales."""

    def __init__(self, ops, lens, n_kv, gq, D, seed, layers=1, layer=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.need = [-(-n // 16) for n in lens]
        n_blocks = sum(self.need) + 3
        order = torch.randperm(n_blocks, generator=g).tolist()
        raw = np.full((layers, n_blocks, n_kv, 16 * D + 128), 0xA7, np.uint8)
        raw[..., 16 * D:] = torch.full((64,), math.nan, dtype=B).view(torch.uint8).numpy()
        width = max(max(self.need), 1) + 2
        tab = np.full((len(lens), width), -1, np.int32)
        self.k, self.v = [], []
        for i, n in enumerate(lens):
            x = torch.randn(2, n, n_kv, D, generator=g) * spread * torch.exp(0.5 * torch.randn(2, n, n_kv, 1, generator=g))
            kq, vq = q4(x[0]), q4(x[1])
            self.k.append(kq[0])
            self.v.append(vq[0])
            for b in range(self.need[i]):
                blk = tab[i, b] = order.pop()
                sl = slice(16 * b, min(n, 16 * b + 16))
                for h in range(n_kv):
                    raw[layer, blk, h] = cells([t[sl, h] for t in kq[1:]], [t[sl, h] for t in vq[1:]], 0xA7)
        tab[tab < 0] = -7 if seed % 2 else 2 ** 30        # never followed
        self.tables = torch.from_numpy(tab).cuda()
        self.kv = ops.PagedKV("int4", layers, n_blocks, n_kv * gq, n_kv, D,
                              pool=torch.from_numpy(raw.reshape(-1)).cuda())


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


def check_out(got, want, A, vmax, dtype, what=""):
    got, want = got.double().cpu(), want.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    tol = vmax * (2 * A + 1) * 2.0 ** -15 + (2.0 ** -8 * want.abs() + 2.0 ** -11 * vmax if dtype == B else 0)
    worst = float(((got - want).abs() - tol).max()) if got.numel() else -1
    assert worst <= 0, f"{what}: {worst} past the tolerance"
    rel = float((got - want).norm() / want.norm().clamp(min=1e-30))
    print(f"{what}: relative 2-norm {rel:.2e}", flush=True)
    return rel


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "GPU tests need the MI355X"
    from paper_2606_03014_amd import ops
    return ops


# ------------------------------------------------------------------ refusals (CPU: nothing is launched)

A1 = 1 << 20                                    # an aligned address that nothing may follow
KV = dict(kind=2, n_layers=2, num_blocks=9, n_heads=8, n_kv_heads=2, head_dim=128)
APPEND = dict(cfg=KV, kv=A1, layer=1, qkv=A1, type=1, stride=12 * 128, rows=0, row_seq=A1, row_pos=A1, tables=A1, n_seqs=3,
              table_len=4, rope=A1, rope_len=64, q_gain=A1, k_gain=A1, gain_type=1, eps=1e-5, q=A1, stream=None)
READ = dict(cfg=KV, kv=A1, layer=0, rows=0, row_seq=A1, row_pos=A1, tables=A1, n_seqs=3, table_len=4, k=A1, v=A1, stream=None)
ROWS = dict(cfg=KV, kv=A1, layer=0, q=A1, type=0, stride=1024, rows=0, row_seq=A1, row_ctx=A1, tables=A1, n_seqs=3,
            table_len=4, max_ctx=64, scale=0.1, out=A1, ws=A1, ws_bytes=1 << 40, stream=None)
CHUNKS = dict(ROWS)
SCORE = dict(logits=A1, type=0, stride=100, rows=0, vocab=100, tokens=A1, logprob=A1, entropy=A1, top=5, ids=A1, lps=A1, ws=A1,
             ws_bytes=1 << 40, stream=None)
SHARED = [("cfg", dict(KV, kind=3)), ("cfg", dict(KV, kind=-1)), ("cfg", dict(KV, n_layers=0)), ("cfg", dict(KV, num_blocks=0)),
          ("cfg", dict(KV, n_heads=0)), ("cfg", dict(KV, n_kv_heads=3)), ("cfg", dict(KV, n_heads=6)),
          ("cfg", dict(KV, n_heads=32)), ("cfg", dict(KV, head_dim=96)), ("cfg", None), ("kv", None), ("kv", A1 + 8),
          ("layer", -1), ("layer", 2), ("rows", -1), ("tables", None), ("tables", A1 + 2), ("n_seqs", 0), ("table_len", 0)]
ATTEND = SHARED + [("cfg", dict(KV, kind=1)), ("cfg", dict(KV, kind=0)), ("type", 2), ("max_ctx", 0), ("max_ctx", 65), ("scale", math.nan),
                   ("scale", math.inf), ("q", None), ("q", A1 + 2), ("out", None), ("out", A1 + 8), ("stride", 1023),
                   ("row_seq", None), ("row_ctx", None), ("row_ctx", A1 + 1), ("ws", A1 + 16)]
REFUSED = {
    "moa_kv_append": (APPEND, SHARED + [("type", 2), ("qkv", None), ("qkv", A1 + 1), ("stride", 12 * 128 - 1), ("row_seq", None),
                                        ("row_pos", None), ("q_gain", None), ("k_gain", None), ("gain_type", 2), ("eps", -1.0),
                                        ("eps", math.nan), ("q", None), ("q", A1 + 4), ("rope_len", 0), ("rope", A1 + 8)]),
    "moa_kv_read": (READ, SHARED + [("row_seq", None), ("row_pos", None), ("k", None), ("v", None), ("v", A1 + 2)]),
    "moa_kv_attend": (ROWS, ATTEND),
    "moa_kv_attend_chunks": (CHUNKS, ATTEND),
    "moa_score_tokens": (SCORE, [("type", 2), ("rows", -1), ("vocab", 0), ("vocab", 101), ("logits", None), ("logits", A1 + 2), ("tokens", None),
                                 ("logprob", None), ("entropy", None), ("top", -1), ("top", 33), ("ids", None), ("lps", None), ("ws", A1 + 1)]),
}


def _c(name, args):
    a = [C.byref(M.moa_kv_cfg(**v)) if isinstance(v, dict) else v for v in args.values()]
    return getattr(M.lib(), name)(*a)


@pytest.mark.parametrize("name", sorted(REFUSED))
def test_arguments_are_refused(name):
    base, wrong = REFUSED[name]
    assert _c(name, base) == M.MOA_OK            # no rows: valid, and nothing to do
    for key, v in wrong:
        if key == "ws" and not _workspace(name, dict(base, rows=1)):
            continue                             # such a call needs none
        got = _c(name, dict(base, rows=v if key == "rows" else 1, **({} if key == "rows" else {key: v})))
        assert got == M.MOA_EINVAL, (key, v, got)


def _workspace(name, a):
    n = C.c_size_t()
    if name == "moa_score_tokens":
        code = M.lib().moa_score_tokens_bytes(a["rows"], a["vocab"], a["top"], C.byref(n))
    elif name == "moa_kv_attend":
        code = M.lib().moa_kv_attend_bytes(C.byref(M.moa_kv_cfg(**a["cfg"])), a["rows"], a["max_ctx"], C.byref(n))
    elif name == "moa_kv_attend_chunks":
        code = M.lib().moa_kv_attend_chunks_bytes(C.byref(M.moa_kv_cfg(**a["cfg"])), a["rows"], a["n_seqs"], a["max_ctx"], C.byref(n))
    else:
        return 0
    assert code == M.MOA_OK
    return n.value


@pytest.mark.parametrize("name,a", [("moa_kv_attend", dict(ROWS, rows=1, table_len=4096, max_ctx=65536)),
                                    ("moa_kv_attend_chunks", dict(CHUNKS, rows=2, n_seqs=1, table_len=4096, max_ctx=65536)),
                                    ("moa_score_tokens", dict(SCORE, rows=1, vocab=128256, stride=128256))])
def test_a_short_workspace_is_refused(name, a):
    need = _workspace(name, a)
    if not need:
        pytest.skip("needs none")
    assert _c(name, dict(a, ws_bytes=need - 1)) == M.MOA_ENOMEM
    assert _c(name, dict(a, ws=None)) == M.MOA_ENOMEM


def test_pool_sizes():
    n = C.c_size_t()
    for kind, cell in ((0, 2 * 16 * 128 * 4), (1, 2 * 16 * 128 * 2), (2, 16 * 128 + 128)):
        assert M.lib().moa_kv_bytes(C.byref(M.moa_kv_cfg(**dict(KV, kind=kind))), C.byref(n)) == M.MOA_OK
        assert n.value == 2 * 9 * 2 * cell
    big = M.moa_kv_cfg(2, 80, 4000000, 64, 8, 128)
    assert M.lib().moa_kv_bytes(C.byref(big), C.byref(n)) == M.MOA_OK and n.value == 80 * 4000000 * 8 * 2176
    assert M.lib().moa_kv_bytes(C.byref(M.moa_kv_cfg(**dict(KV, head_dim=80))), C.byref(n)) == M.MOA_EINVAL
    assert M.lib().moa_kv_bytes(C.byref(big), None) == M.MOA_EINVAL


def test_the_torch_layer_refuses_cpu_tensors():
    from paper_2606_03014_amd import ops
    with pytest.raises(ValueError):
        ops.PagedKV("int4", 1, 2, 4, 1, 64, pool=torch.zeros(2 * (16 * 64 + 128), dtype=torch.uint8))
    with pytest.raises(ValueError):
        ops.PagedKV("int8", 1, 2, 4, 1, 64)
    with pytest.raises(M.MoaError):
        ops.PagedKV("int4", 1, 2, 4, 1, 96, pool=torch.zeros(1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        ops.score_tokens(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32))


@gpu
def test_the_torch_layer_refuses_wrong_tensors(ops):
    kv = ops.PagedKV("int4", 1, 4, 4, 1, 64)
    tab, z = i32([[0, 1], [2, 3]]), i32([0, 1])
    q = torch.zeros(2, 4, 64, device="cuda")
    for bad in (q.double(), q.cpu(), q[:, :3], q.transpose(1, 2)):
        with pytest.raises((ValueError, M.MoaError)):
            kv.attend(0, bad, z, z, tab, 32)
    for seq in (z.long(), z[:1], z.cpu(), i32([0, 0, 1, 1])[::2]):
        with pytest.raises(ValueError):
            kv.attend(0, q, seq, z, tab, 32)
    for t in (tab.t(), tab[0], tab.long()):
        with pytest.raises(ValueError):
            kv.attend(0, q, z, z, t, 32)
    with pytest.raises(M.MoaError):
        kv.attend(0, q, z, z, tab, 33)
    with pytest.raises(ValueError):
        kv.attend(0, q, z, z, tab, 32, out=torch.zeros(2, 4, 64, device="cuda", dtype=B))
    with pytest.raises(ValueError):
        kv.append(0, torch.zeros(2, 6 * 64, device="cuda"), z, z, tab, q_gain=torch.ones(64, device="cuda"))
    with pytest.raises(M.MoaError):
        ops.PagedKV("bf16", 1, 4, 4, 1, 64).attend(0, q, z, z, tab, 32)
    with pytest.raises(ValueError):
        ops.score_tokens(torch.zeros(2, 8, device="cuda"), z, top_k=9)


@pytest.mark.parametrize("name", sorted(REFUSED))
def test_sizes_past_the_grids_are_refused(name):
    base = dict(REFUSED[name][0])
    wrong = [dict(rows=(1 << 20) + 1)]
    if name == "moa_score_tokens":
        wrong += [dict(rows=1, vocab=(1 << 30) + 1, stride=1 << 31)]
    else:
        wrong += [dict(rows=1, table_len=(1 << 26) + 1), dict(rows=1, n_seqs=(1 << 20) + 1)]
    if "max_ctx" in base:
        wide = dict(KV, n_heads=512, n_kv_heads=512)
        wrong += [dict(cfg=wide, stride=512 * 128, rows=1 << 20, n_seqs=1 << 20), dict(rows=1, table_len=1 << 26, max_ctx=(1 << 30) + 1)]
    for w in wrong:
        assert _c(name, dict(base, **w)) == M.MOA_EINVAL, w


def test_sizes_past_64_bits_are_refused():
    n = C.c_size_t()
    top = (1 << 31) - 1
    assert M.lib().moa_kv_bytes(C.byref(M.moa_kv_cfg(2, top, top, 4096, 4096, 128)), C.byref(n)) == M.MOA_EINVAL
    cfg = C.byref(M.moa_kv_cfg(**KV))
    assert M.lib().moa_kv_attend_bytes(cfg, 1, top, C.byref(n)) == M.MOA_EINVAL
    assert M.lib().moa_kv_attend_chunks_bytes(cfg, 1, 1, top, C.byref(n)) == M.MOA_EINVAL
    assert M.lib().moa_kv_attend_chunks_bytes(cfg, 1, top, 64, C.byref(n)) == M.MOA_EINVAL
    assert M.lib().moa_score_tokens_bytes(1, top, 5, C.byref(n)) == M.MOA_EINVAL


# ------------------------------------------------------------------ append and read

def rows_of(lens, before, seed=0):
    """(row_seq, row_pos) of lens[i] rows behind before[i] positions of each sequence, in sequence order."""
    seq = np.repeat(np.arange(len(lens)), lens)
    pos = np.concatenate([np.arange(b, b + n) for n, b in zip(lens, before)])
    return seq, pos


@gpu
@pytest.mark.parametrize("kind", ["f32", "bf16", "int4"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("norm,rope,pad", [(True, True, 0), (False, True, 4), (True, False, 3), (False, False, 1)])
def test_append_caches_what_read_returns(ops, kind, hd, dtype, norm, rope, pad):
    nh, nkv, layers, layer = 6, 3, 3, 1
    lens, before = [1, 40, 0, 17, 1, 33], [0, 5, 3, 16, 47, 0]
    seq, pos = rows_of(lens, before)
    T = len(seq)
    g = torch.Generator().manual_seed(hd + pad)
    perm = torch.randperm(T, generator=g).numpy()        # rows of a step stand in any order
    seq, pos = seq[perm], pos[perm].copy()
    x = (torch.randn(T, (nh + 2 * nkv) * hd + pad, generator=g) * torch.exp(torch.randn(T, 1, generator=g))).to(dtype)
    wide = x.cuda()
    x = x[:, :(nh + 2 * nkv) * hd].view(T, nh + 2 * nkv, hd)
    n_blocks = 30
    tables = torch.randperm(n_blocks, generator=g)[:24].view(6, 4).int()
    tab = ops.rope_table(64, hd) if rope else None
    gains = (1 + 0.3 * torch.randn(2, hd, generator=g)).to(B if hd == 64 else F)
    kv = ops.PagedKV(kind, layers, n_blocks, nh, nkv, hd)
    kv.pool.fill_(0x5B)
    kw = dict(rope=tab, eps=1e-5, **(dict(q_gain=gains[0].cuda(), k_gain=gains[1].cuda()) if norm else {}))
    q = kv.append(layer, wide[:, :(nh + 2 * nkv) * hd], i32(seq), i32(pos), tables.cuda(), **kw)
    k, v = kv.read(layer, i32(seq), i32(pos), tables.cuda())
    p = torch.as_tensor(pos)
    cpu_tab = tab.cpu() if rope else None
    want_q = turn(x[:, :nh], gains[0] if norm else None, 1e-5, cpu_tab, p)
    err = (q.double().cpu() - want_q).abs()
    tol = 32 * 2.0 ** -24 * want_q.abs().amax(-1, keepdim=True) + (2.0 ** -8 * want_q.abs() if dtype == B else 0)
    assert (err <= tol).all(), float((err - tol).max())
    wk = turn(x[:, nh:nh + nkv], gains[1] if norm else None, 1e-5, cpu_tab, p)
    wv = x[:, nh + nkv:].double()
    if kind == "int4":
        wk, wv = (q4(t)[0].to(torch.float32).to(B).double() for t in (wk, wv))
        assert torch.equal(k.double().cpu(), wk) and torch.equal(v.double().cpu(), wv)
    else:
        tol = 32 * 2.0 ** -24 * wk.abs().amax(-1, keepdim=True) + (2.0 ** -8 * wk.abs() if kind == "bf16" else 0)
        assert ((k.double().cpu() - wk).abs() <= tol).all()
        assert torch.equal(v.double().cpu(), wv if kind == "f32" else x[:, nh + nkv:].to(B).double())
    # nothing else is touched: other layers, other slots
    raw = kv.pool.cpu().view(layers, n_blocks, nkv, -1)
    assert (raw[0] == 0x5B).all() and (raw[2] == 0x5B).all()
    used = np.zeros((n_blocks, 16), bool)
    used[tables.numpy()[seq, pos // 16], pos % 16] = True
    cell = raw[layer].permute(0, 1, 2)
    free = torch.from_numpy(~used)
    if kind == "int4":
        kc = cell[..., :8 * hd].reshape(n_blocks, nkv, 16, hd // 2).permute(0, 2, 1, 3)[free]
        vc = cell[..., 8 * hd:16 * hd].reshape(n_blocks, nkv, hd // 2, 16).permute(0, 3, 1, 2)[free]
        sc = cell[..., 16 * hd:].reshape(n_blocks, nkv, 2, 16, 4).permute(0, 3, 1, 2, 4)[free]
        assert all((t == 0x5B).all() for t in (kc, vc, sc))
    else:
        assert (cell.reshape(n_blocks, nkv, 2, 16, -1).permute(0, 3, 1, 2, 4)[free] == 0x5B).all()


@gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_rows_that_are_hard_to_quantise(ops, hd):
    """Constant rows, single outliers, ties, tiny and huge values, infinities and NaN."""
    x = torch.zeros(12, 3, hd)
    g = torch.Generator().manual_seed(1)
    x[0] = 0.0
    x[1] = -3.25
    x[2, :, hd // 2] = 1e4
    x[3] = torch.arange(hd).float() % 16 / 2                     # multiples of half a step
    x[4] = (torch.arange(hd).float() % 31) * 0.5                 # every code and every border
    x[5] = torch.randn(3, hd, generator=g) * 1e-38
    x[6] = torch.randn(3, hd, generator=g) * 1e37
    x[7] = torch.randn(3, hd, generator=g)
    x[7, 0, 5], x[7, 1, 6], x[7, 2, 7] = math.inf, -math.inf, math.nan
    x[8] = torch.randn(3, hd, generator=g) * 1e-45
    x[9, :, 0], x[9, :, 1] = 3e38, -3e38                         # a range past float32
    x[10] = torch.randn(3, hd, generator=g) + 1000
    x[11, :, ::2] = -0.0
    kv = ops.PagedKV("int4", 1, 2, 1, 1, hd)
    seq, pos, tab = i32([0] * 12), i32(range(12)), i32([[1, 0]])
    kv.append(0, x.view(12, -1).cuda(), seq, pos, tab)
    k, v = kv.read(0, seq, pos, tab)
    for got, want in ((k, q4(x[:, 1])[0]), (v, q4(x[:, 2])[0])):
        want = want.float().to(B)
        got = got[:, 0].cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())
        assert got[7].isnan().all() and got[9].isnan().all()


@gpu
@pytest.mark.parametrize("rows", [3, 512])
def test_scales_next_to_a_border(ops, rows):
    """Ranges whose 15th part lies between two bf16 values, where one bit of it decides."""
    g = torch.Generator().manual_seed(2)
    step = (torch.randint(128, 256, (rows,), generator=g) + 0.5) * 2.0 ** torch.randint(-9, -5, (rows,), generator=g).double()
    hi = (step * 15).float()
    for k in range(3):                                           # the nearest floats as well
        x = torch.rand(rows, 3, 64, generator=g) * hi[:, None, None]
        x[:, :, 5], x[:, :, 9] = 0.0, hi[:, None]
        kv = ops.PagedKV("int4", 1, -(-rows // 16), 1, 1, 64)
        tab = i32([range(-(-rows // 16))])
        kv.append(0, x.flatten(1).cuda(), i32([0] * rows), i32(range(rows)), tab)
        s = q4(x)[2][..., 0].view(torch.int16)
        got = kv.pool.cpu().view(-1, 64 * 16 + 128)[:, 1024:].contiguous().view(torch.int16).view(-1, 2, 16, 2)[..., 0]
        got = got.transpose(0, 1).reshape(2, -1)[:, :rows]
        assert torch.equal(got[0], s[:, 1]) and torch.equal(got[1], s[:, 2])
        hi = torch.nextafter(hi, torch.full_like(hi, math.inf))


@gpu
@pytest.mark.parametrize("hd,rows", [(64, 1), (128, 1), (64, 16), (128, 16)])
def test_codes_next_to_a_border(ops, hd, rows):
    """Values 2^-20 to 2^-29 of a step below and above the border of two codes, and on it (m = -2.75, s = 1.1015625)."""
    kv = ops.PagedKV("int4", 1, 1, 1, 1, hd)
    x = torch.zeros(rows, 3, hd, dtype=torch.float64)
    i = torch.arange(hd, dtype=torch.float64)
    for r in range(rows):
        near = -2.75 + ((i % 14) + 0.5) * 1.1015625
        near[2::14] *= 1 + (torch.arange(len(near[2::14])) - 2) * 2.0 ** (-12 - r % 10)     # 2.5 steps from m: next to 0, fine steps
        near[0], near[-1] = -2.75, 13.75
        x[r, 1:] = near
    x = x.float().flatten(1)
    kv.append(0, x.cuda(), i32([0] * rows), i32(range(rows)), i32([[0]]))
    raw = kv.pool.cpu().numpy()
    c, s, m = q4(x.view(rows, 3, hd)[:, 2])[1:]
    assert float(s[0]) == 1.1015625 and float(m[0]) == -2.75 and len(c[0].unique()) > 8
    vc = raw[8 * hd:16 * hd].reshape(hd // 2, 16)[:, :rows].T
    kc = raw[:8 * hd].reshape(16, hd // 2)[:rows]
    for r in range(rows):
        assert np.concatenate([vc[r] & 15, vc[r] >> 4]).tolist() == c[r].tolist(), r
        assert np.stack([kc[r] & 15, kc[r] >> 4], 1).reshape(-1).tolist() == c[r].tolist(), r


@gpu
@pytest.mark.parametrize("kind", ["bf16", "int4"])
def test_rows_out_of_range_are_skipped(ops, kind):
    hd, nh, nkv = 64, 2, 1
    kv = ops.PagedKV(kind, 1, 4, nh, nkv, hd)
    x = torch.randn(9, 4 * hd, device="cuda")
    tab = i32([[0, 1], [2, 99], [-1, 3]])
    seq = i32([0, 0, 0, 1, 1, 2, 3, -1, 2])
    pos = i32([0, -1, 32, 15, 16, 0, 0, 0, 31])                  # fine, padding, past the table, fine, block 99, block -1, no sequence, no sequence, fine
    before = kv.pool.clone()
    rope = ops.rope_table(32, hd)
    q = kv.append(0, x, seq, pos, tab, rope=rope)
    k, v = kv.read(0, seq, pos, tab)
    ok = [0, 3, 8]
    for i in range(9):
        assert bool((v[i] != 0).any()) == (i in ok)
    want = turn(x[:, :2 * hd].cpu().view(9, 2, hd), None, 0, rope.cpu(), pos.cpu().clamp(0, 31))
    written = [0, 3, 4, 5, 6, 7, 8]
    assert ((q.double().cpu() - want)[written].abs() < 1e-5).all()
    changed = (kv.pool != before).view(4, -1).any(1).tolist()
    assert changed == [True, False, True, True]


# ------------------------------------------------------------------ attention, decode rows

CTX = [1, 15, 16, 17, 63, 64, 65, 127, 128, 130, 255, 511, 512, 513, 700, 1100, 2049]


@gpu
@pytest.mark.parametrize("gq,n_kv", [(1, 3), (2, 1), (4, 2), (8, 1)])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [F, B])
def test_decode_rows(ops, gq, n_kv, hd, dtype):
    p = Pool(ops, CTX, n_kv, gq, hd, seed=gq + hd, layers=2, layer=1)
    n_h = n_kv * gq
    g = torch.Generator().manual_seed(5)
    # every sequence whole, the longest again at shorter contexts, empty rows and rows without a sequence
    seq = list(range(len(CTX))) + [16] * 6 + [3, 2, -1, 99]
    ctx = CTX + [1, 16, 40, 64, 1000, 2048] + [0, -5, 7, 7]
    wide = torch.randn(len(seq), 2 * n_h * hd, generator=g).to(dtype).cuda()
    q = wide[:, 1:1 + n_h * hd].unflatten(1, (n_h, hd))          # rows of a wider matrix, off any alignment
    out = p.kv.attend(1, q, i32(seq), i32(ctx), p.tables, 2049)
    want, As, vm = [], 0.0, 0.0
    for r, (b, n) in enumerate(zip(seq, ctx)):
        n = max(n, 0) if 0 <= b < len(CTX) else 0
        o, A = attention(q[r].double().cpu(), p.k[b % 17][:n], p.v[b % 17][:n], hd ** -0.5)
        want.append(o)
        As, vm = max(As, A), max(vm, float(p.v[b % 17].abs().max()))
    want = torch.stack(want)
    rel = check_out(out, want, As, vm, dtype, f"rows gq {gq} hd {hd} {dtype}")
    assert rel <= (2.0 ** -16 if dtype == F else 2.0 ** -8)
    assert (out[-4:] == 0).all()
    # a call of the same sizes gives a row the same bits, wherever it stands and whatever the others are
    assert torch.equal(p.kv.attend(1, q, i32(seq), i32(ctx), p.tables, 2049), out)
    back = torch.arange(len(seq) - 1, -1, -1)
    assert torch.equal(p.kv.attend(1, q[back.cuda()], i32(seq)[back.cuda()], i32(ctx)[back.cuda()], p.tables, 2049)[back.cuda()], out)
    # alone, and bounded by the whole table
    alone = p.kv.attend(1, q[16:17], i32([16]), i32([2049]), p.tables, 16 * p.tables.shape[1])
    check_out(alone, want[16:17], As, vm, dtype, "alone")
    short = p.kv.attend(1, q, i32(seq), i32(ctx), p.tables, 100)
    ref, _ = attention(q[16].double().cpu(), p.k[16][:100], p.v[16][:100], hd ** -0.5)
    assert (short[16].double().cpu() - ref).abs().max() <= vm * (2 * As + 1) * 2.0 ** -15 + (2.0 ** -7 if dtype == B else 0)


@gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_decode_rows_with_sharp_scores(ops, hd):
    """Scores hundreds apart, one key far above the others, all keys equal: the running maximum moves late, early, never."""
    p = Pool(ops, [900, 900], 1, 4, hd, seed=3, spread=4.0)
    q = torch.randn(5, 4, hd, generator=torch.Generator().manual_seed(2))
    q[1] *= 30
    q[2] = p.k[0][870, 0].float() * 2
    q[3] = p.k[0][2, 0].float() * 2
    q[4] = 0
    got = p.kv.attend(0, q.cuda(), i32([0] * 5), i32([900] * 5), p.tables, 900)
    for r in range(5):
        want, A = attention(q[r].double(), p.k[0], p.v[0], hd ** -0.5)
        check_out(got[r], want, A, float(p.v[0].abs().max()), F, f"sharp row {r}")


@gpu
@pytest.mark.parametrize("q_size,scale", [(1e-42, 0.125), (1e-30, 1e-20), (1.0, 1e-44), (1.0, 0.0), (1.0, -0.125), (1e30, 1e-30)])
def test_units_of_tiny_queries_and_scales(ops, q_size, scale):
    """Subnormal queries, scales that leave no unit in float32, none and a negative one."""
    p = Pool(ops, [100], 1, 2, 64, seed=9)
    q = torch.randn(3, 2, 64, generator=torch.Generator().manual_seed(5)) * q_size
    vm = float(p.v[0].abs().max())
    for out, seen in ((p.kv.attend(0, q.cuda(), i32([0, 0, 0]), i32([98, 99, 100]), p.tables, 100, scale=scale), (98, 99, 100)),
                      (p.kv.attend_chunks(0, q.cuda(), i32([0, 3]), i32([100]), p.tables, 100, scale=scale), (98, 99, 100))):
        for r, n in enumerate(seen):
            want, A = attention(q[r].double(), p.k[0][:n], p.v[0][:n], scale)
            check_out(out[r], want, A, vm, F, f"q {q_size} scale {scale} row {r}")


@gpu
def test_chunk_starts_that_do_not_ascend_stay_inside(ops):
    p = Pool(ops, [60, 60, 60], 1, 4, 64, seed=9)
    whole = torch.full((200, 4, 64), 2.5, device="cuda")
    q = torch.randn(70, 4, 64, generator=torch.Generator().manual_seed(5)).cuda()
    for starts in ([0, 50, 20, 70], [60, 0, 65, 3], [70, 70, -5, 300]):
        p.kv.attend_chunks(0, q, i32(starts), i32([60, 60, 60]), p.tables, 60, out=whole[60:130])
    assert (whole[:60] == 2.5).all() and (whole[130:] == 2.5).all()


@gpu
def test_a_nan_row_reaches_only_those_that_see_it(ops):
    hd = 64
    p = Pool(ops, [200, 200], 1, 2, hd, seed=8)
    x = torch.zeros(1, 4 * hd)
    x[0, 2 * hd] = math.nan                                      # its keys
    p.kv.append(0, x.cuda(), i32([1]), i32([150]), p.tables)
    q = torch.randn(3, 2, hd).cuda()
    out = p.kv.attend(0, q, i32([0, 1, 1]), i32([200, 150, 151]), p.tables, 200)
    assert torch.isfinite(out[:2]).all() and out[2].isnan().all()


# ------------------------------------------------------------------ attention, chunks

def chunk_want(p, q, lens, ctx, hd):
    want, As, at = torch.zeros(q.shape, dtype=torch.float64), 0.0, 0
    for i, (n, c) in enumerate(zip(lens, ctx)):
        for j in range(n):
            keys = max(c - n + j + 1, 0)
            want[at + j], A = attention(q[at + j].double().cpu(), p.k[i][:keys], p.v[i][:keys], hd ** -0.5)
            As = max(As, A)
        at += n
    return want, As


@gpu
@pytest.mark.parametrize("gq,n_kv", [(1, 2), (2, 1), (4, 2), (8, 1)])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [F, B])
def test_chunks(ops, gq, n_kv, hd, dtype):
    lens = [1, 5, 0, 33, 130, 16, 2, 64, 31]
    ctx = [1, 5, 40, 33, 131, 700, 1030, 65, 95]
    p = Pool(ops, ctx, n_kv, gq, hd, seed=gq + hd + 1)
    n_h, T = n_kv * gq, sum(lens)
    wide = torch.randn(T + 7, (n_h + 1) * hd, generator=torch.Generator().manual_seed(6)).to(dtype).cuda()
    q = wide[:, hd:].unflatten(1, (n_h, hd))
    start = i32(np.concatenate([[0], np.cumsum(lens)]))
    out = torch.full((T + 7, n_h, hd), 7.5, dtype=dtype, device="cuda")
    p.kv.attend_chunks(0, q, start, i32(ctx), p.tables, max(ctx), out=out)
    assert (out[T:] == 7.5).all()                                # rows behind the last chunk
    want, A = chunk_want(p, q[:T], lens, ctx, hd)
    vm = max(float(v.abs().max()) for v in p.v)
    rel = check_out(out[:T], want, A, vm, dtype, f"chunks gq {gq} hd {hd} {dtype}")
    assert rel <= (2.0 ** -16 if dtype == F else 2.0 ** -8)


@gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_chunks_before_the_first_position_and_sharp_ones(ops, hd):
    """Rows at negative positions see nothing; scores hundreds apart; a chunk that starts past row 0."""
    p = Pool(ops, [20, 300], 1, 4, hd, seed=4, spread=4.0)
    q = torch.randn(200, 4, hd, generator=torch.Generator().manual_seed(3)) * 5
    out = torch.full((200, 4, hd), -1.0, device="cuda")
    p.kv.attend_chunks(0, q.cuda(), i32([10, 40, 190]), i32([20, 300]), p.tables, 300, out=out)
    assert (out[:10] == -1).all() and (out[190:] == -1).all() and (out[10:20] == 0).all()
    want, A = chunk_want(p, q[10:190], [30, 150], [20, 300], hd)
    check_out(out[10:190], want, A, max(float(v.abs().max()) for v in p.v), F, f"sharp chunks {hd}")


@gpu
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("hd", [64, 128])
def test_a_nan_row_reaches_only_later_rows_of_a_chunk(ops, hd, dtype):
    p = Pool(ops, [150, 70], 2, 2, hd, seed=9)
    for col in (4, 6):                                           # keys of head 0, values of head 0
        x = torch.zeros(1, 8 * hd)
        x[0, col * hd + 3] = math.nan
        p.kv.append(0, x.cuda(), i32([0]), i32([90 + col]), p.tables)      # the head's other rows stand for 0
    q = torch.randn(220, 4, hd, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    out = p.kv.attend_chunks(0, q, i32([0, 150, 220]), i32([150, 70]), p.tables, 150)
    assert torch.isfinite(out[150:]).all() and torch.isfinite(out[:94]).all() and torch.isfinite(out[:, 2:]).all()
    assert out[94:150, :2].isnan().all()


@gpu
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("hd,gq,spread", [(64, 4, 1.0), (128, 2, 3.0), (64, 1, 4.0), (128, 8, 1.0)])
def test_chunk_bits_do_not_hang_on_the_cuts(ops, hd, gq, spread, dtype):
    """One prompt whole, and cut at any row, in calls without key splits: the same bits, also where references move."""
    n = 400
    p = Pool(ops, [n], 1, gq, hd, seed=12, spread=spread)
    q = (torch.randn(n, gq, hd, generator=torch.Generator().manual_seed(4)) * spread).to(dtype).cuda()
    whole = p.kv.attend_chunks(0, q, i32([0, n]), i32([n]), p.tables, n)
    for cuts in ([0, 150, n], [0, 1, 18, 83, 311, n]):
        for a, b in zip(cuts, cuts[1:]):
            part = p.kv.attend_chunks(0, q[a:b], i32([0, b - a]), i32([b]), p.tables, n)
            assert torch.equal(part, whole[a:b]), (a, b)


@gpu
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("hd,gq", [(64, 4), (128, 2)])
def test_few_rows_behind_long_contexts(ops, hd, gq, dtype):
    """Grids that are split over the keys: chunks whose first rows see none of the later splits, an empty one."""
    lens, ctx = [3, 0, 40, 1], [2900, 5, 41, 513]
    p = Pool(ops, ctx, 1, gq, hd, seed=5)
    q = torch.randn(44, gq, hd, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    out = torch.full_like(q, 3.0)
    out = p.kv.attend_chunks(0, q, i32([0, 3, 3, 43, 44]), i32(ctx), p.tables, 16 * p.tables.shape[1], out=out)
    want, A = chunk_want(p, q, lens, ctx, hd)
    rel = check_out(out, want, A, max(float(v.abs().max()) for v in p.v if len(v)), dtype, f"long {hd} {dtype}")
    assert rel <= (2.0 ** -16 if dtype == F else 2.0 ** -8)


@gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_decode_rows_in_long_splits(ops, hd):
    """Enough rows for splits of 2,048 keys: rows that end on, before and behind one."""
    n = [2047, 2048, 2049, 4096, 4500, 64, 1]
    p = Pool(ops, n, 1, 1, hd, seed=6)
    seq = [i % 7 for i in range(300)]
    q = torch.randn(300, 1, hd, generator=torch.Generator().manual_seed(4))
    out = p.kv.attend(0, q.cuda(), i32(seq), i32([n[i] for i in seq]), p.tables, 4500).cpu()
    want, A = zip(*(attention(q[r].double(), p.k[b], p.v[b], hd ** -0.5) for r, b in enumerate(seq)))
    assert check_out(out, torch.stack(want), max(A), max(float(v.abs().max()) for v in p.v), F, "long splits") <= 2.0 ** -16


# ------------------------------------------------------------------ scores

def score_want(x, tok, k):
    x = x.double().cpu()
    d = x - x.amax(1, keepdim=True)                              # first: a norm of -1e30 + 3.7 has lost the 3.7 in 64 bits too
    lp = d - d.exp().sum(1, keepdim=True).log()
    p = lp.exp()
    H = -torch.where(p > 0, p * lp, 0.0).sum(1)
    ids = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k]
    return lp.gather(1, tok.long().cpu()[:, None])[:, 0], H, ids.int(), lp.gather(1, ids)


def check_score(got, want):
    lp, H, ids, tops = (t.cpu() for t in got)
    assert torch.equal(ids, want[2])
    assert ((lp.double() - want[0]).abs() <= 1e-5 + 2.0 ** -22 * want[0].abs()).all()
    assert ((H.double() - want[1]).abs() <= 1e-5 * (1 + want[1])).all()
    assert ((tops.double() - want[3]).abs() <= 1e-5 + 2.0 ** -22 * want[3].abs()).all()


@gpu
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("R,V,k,pad", [(1, 1, 1, 0), (3, 2, 2, 1), (2, 31, 5, 0), (5, 33, 32, 3), (4, 255, 1, 0), (7, 1000, 20, 8),
                                       (1, 4097, 32, 0), (300, 129, 3, 7), (2, 32000, 0, 1), (9, 50257, 20, 0), (1, 128256, 20, 0),
                                       (33, 128256, 5, 5)])
def test_scores(ops, dtype, R, V, k, pad):
    g = torch.Generator().manual_seed(V + R)
    x = (torch.randn(R, V + pad, generator=g) * 3).to(dtype).cuda()[:, :V]
    tok = torch.randint(0, V, (R,), generator=g, dtype=torch.int32).cuda()
    check_score(ops.score_tokens(x, tok, top_k=k), score_want(x, tok, k))


@gpu
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("V", [40, 5000, 70000])
def test_scores_of_equal_masked_and_sharp_logits(ops, dtype, V):
    g = torch.Generator().manual_seed(V)
    x = torch.randn(8, V, generator=g)
    x[0] = 1.5                                                   # all equal: ids 0, 1, 2 ..
    x[1, :] = -math.inf
    x[1, 5:9] = 2.0                                              # four possible tokens of many
    x[2, V - 1] = 90.0                                           # all of the mass on the last token
    x[3] = torch.randint(0, 3, (V,), generator=g).float()        # ties everywhere
    x[4] = torch.finfo(dtype).min                                # masked with the lowest value
    x[4, 7] = 0.0
    x[5] = x[5] * 1e4
    x[6, ::2] = -math.inf
    x[7] = -x[7].abs() - 1e30
    x = x.to(dtype).cuda()
    tok = i32([3, 6, V - 1, 1, 7, 0, 1, 2])
    got, want = ops.score_tokens(x, tok, top_k=20), score_want(x, tok, 20)
    check_score([t[[0, 2, 3, 4, 5, 6, 7]] for t in got], [t[[0, 2, 3, 4, 5, 6, 7]] for t in want])
    # a row with fewer possible tokens than alternatives: impossible ones follow by id, at -inf
    assert torch.equal(got[2][1].cpu(), want[2][1]) and torch.allclose(got[0][1].cpu().double(), want[0][1])
    assert abs(float(got[1][1]) - math.log(4)) < 1e-5
    assert (got[3][1][4:] == -math.inf).all() and torch.allclose(got[3][1][:4].cpu(), torch.full((4,), -math.log(4)))
    # an impossible token
    assert float(ops.score_tokens(x[6:7], i32([0]))[0]) == -math.inf


@gpu
@pytest.mark.parametrize("V", [50, 9000])
def test_rows_without_probabilities_and_tokens_outside(ops, V):
    x = torch.randn(5, V, generator=torch.Generator().manual_seed(1))
    x[0] = -math.inf
    x[1, 3] = math.nan
    x[2, 4] = math.inf
    tok = i32([0, 1, 2, -1, V])
    lp, H, ids, tops = ops.score_tokens(x.cuda(), tok, top_k=6)
    assert lp.isnan().all() and H[:3].isnan().all() and tops[:3].isnan().all()
    assert torch.isfinite(H[3:]).all() and torch.isfinite(tops[3:]).all()
    assert ids[0].tolist() == [0, 1, 2, 3, 4, 5] and int(ids[2, 0]) == 4
    rest = x[1].clone()
    rest[3] = -math.inf                                          # NaN comes last
    assert torch.equal(ids[1].cpu(), torch.sort(rest, descending=True, stable=True)[1][:6].int())


@gpu
@pytest.mark.parametrize("V", [300, 70000])
def test_alternatives_of_rows_of_nan(ops, V):
    """NaN everywhere, beside impossible tokens, and in all but three of the 64 groups that set the bar of a row's first run."""
    x = torch.randn(4, V, generator=torch.Generator().manual_seed(5))
    x[0] = math.nan
    x[1] = math.nan
    x[1, 2::9] = -math.inf
    e = torch.arange(V)
    x[2, (e < 16384) & (e // 4 % 64 >= 3)] = math.nan
    x[3, 1:] = math.nan
    lp, H, ids, tops = ops.score_tokens(x.cuda(), i32([0, 1, 2, 3]), top_k=20)
    assert lp.isnan().all() and H.isnan().all() and tops.isnan().all()
    for r in range(4):
        v = x[r].numpy()
        want = np.lexsort((np.arange(V), -np.nan_to_num(v, nan=0.0, neginf=-np.inf), np.isnan(v)))[:20]
        assert ids[r].tolist() == want.tolist(), r
    one = ops.score_tokens(x.cuda(), i32([0, 1, 2, 3]), top_k=1)[2][:, 0].tolist()
    assert one == ids[:, 0].tolist()


# ------------------------------------------------------------------ together, streams and graphs

class Session:
    """Two layers' attention of three calls over one int4 cache: prompts in two chunks, then decode steps, as a decoder
    makes them (random projections' outputs instead of a model's)."""

    def __init__(self, ops, hd=64, nkv=2, gq=4, seed=0):
        self.ops, self.hd, self.nkv, self.nh = ops, hd, nkv, nkv * gq
        self.kv = ops.PagedKV("int4", 2, 40, self.nh, nkv, hd)
        self.g = torch.Generator().manual_seed(seed)
        self.tables = torch.randperm(40, generator=self.g)[:36].view(3, 12).int().cuda()
        self.rope = ops.rope_table(192, hd)
        self.gains = (1 + 0.2 * torch.randn(2, hd, generator=self.g)).cuda()
        self.seen = [torch.zeros(2, 2, 0, nkv, hd, dtype=torch.float64) for _ in range(3)]   # [layer][K|V][pos]

    def step(self, lens, dtype, chunks):
        before = [s.shape[2] for s in self.seen]
        seq, pos = rows_of(lens, before)
        x = torch.randn(2, len(seq), (self.nh + 2 * self.nkv) * self.hd, generator=self.g).to(dtype)
        got = []
        for layer in range(2):
            q = self.kv.append(layer, x[layer].cuda(), i32(seq), i32(pos), self.tables, rope=self.rope,
                               q_gain=self.gains[0], k_gain=self.gains[1])
            if chunks:
                o = self.kv.attend_chunks(layer, q, i32(np.concatenate([[0], np.cumsum(lens)])),
                                          i32([b + n for b, n in zip(before, lens)]), self.tables, 192)
            else:
                o = self.kv.attend(layer, q, i32(seq), i32(pos + 1), self.tables, 192)
            got.append((q, o))
        p = torch.as_tensor(pos)
        for layer in range(2):
            h = x[layer].view(len(seq), -1, self.hd)
            k = q4(turn(h[:, self.nh:self.nh + self.nkv], self.gains[1].cpu(), 1e-5, self.rope.cpu(), p))[0]
            v = q4(h[:, self.nh + self.nkv:])[0]
            q, o = got[layer]
            want = torch.empty(len(seq), self.nh, self.hd, dtype=torch.float64)
            A = 0.0
            for i in range(3):
                mine = torch.as_tensor(seq == i)
                old = self.seen[i][layer]
                K, V = torch.cat([old[0][:before[i]], k[mine]]), torch.cat([old[1][:before[i]], v[mine]])
                if layer == 0:
                    grown = torch.zeros(2, 2, len(K), self.nkv, self.hd, dtype=torch.float64)
                    grown[:, :, :before[i]] = self.seen[i]
                    self.seen[i] = grown
                self.seen[i][layer, 0], self.seen[i][layer, 1] = K, V
                for r in torch.nonzero(mine)[:, 0].tolist():
                    n = int(pos[r]) + 1
                    want[r], a = attention(q[r].double().cpu(), K[:n], V[:n], self.hd ** -0.5)
                    A = max(A, a)
            check_out(o, want, A, float(v.abs().max().clamp(min=4)), dtype, f"layer {layer} rows {lens}")


@gpu
@pytest.mark.parametrize("hd,gq,dtype", [(64, 4, F), (128, 8, B)])
def test_prompts_then_decode_then_scores(ops, hd, gq, dtype):
    s = Session(ops, hd=hd, gq=gq)
    s.step([70, 3, 33], dtype, True)
    s.step([30, 64, 0], dtype, True)
    for _ in range(3):
        s.step([1, 1, 1], dtype, False)
    s.step([1, 0, 1], dtype, False)
    logits = torch.randn(3, 4096, generator=s.g).cuda()
    tok = logits.argmax(1).int()
    lp, H, ids, tops = ops.score_tokens(logits, tok, top_k=3)
    assert torch.equal(ids[:, 0], tok) and torch.equal(lp, tops[:, 0])


@gpu
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("kind", ["f32", "bf16", "int4"])
def test_operands_of_any_alignment_give_the_same_bits(ops, dtype, kind):
    """Views that begin one element behind a 16-byte boundary, with odd strides, against contiguous copies."""
    hd, nkv, nh, T = 64, 2, 4, 40
    g = torch.Generator().manual_seed(8)

    def views(*shape):
        x = torch.randn(shape[0], math.prod(shape[1:]) + 3, generator=g).to(dtype).cuda()
        v = x[:, 1:-2]
        assert v.data_ptr() % 16
        return v, v.contiguous()

    x, gains = views(T, (nh + 2 * nkv) * hd), [views(1, hd) for _ in range(2)]
    seq, pos, tab, rope = i32([0] * T), i32(range(T)), i32([[2, 0, 1]]), ops.rope_table(T, hd)
    got = []
    for i in range(2):
        kv = ops.PagedKV(kind, 1, 3, nh, nkv, hd)
        got.append((kv.append(0, x[i], seq, pos, tab, rope=rope, q_gain=gains[0][i][0], k_gain=gains[1][i][0]), kv.pool))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    if kind != "int4":
        return
    q, c = views(T, nh * hd), i32([T])
    outs = [(kv.attend(0, q[i].unflatten(1, (nh, hd)), seq, i32(range(1, T + 1)), tab, T),
             kv.attend_chunks(0, q[i].unflatten(1, (nh, hd)), i32([0, T]), c, tab, T)) for i in range(2)]
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    v = views(3, 40001)
    scores = [ops.score_tokens(v[i], i32([1, 2, 3]), top_k=9) for i in range(2)]
    assert torch.equal(scores[0][2], scores[1][2])               # (sums run over other pieces: not their bits)
    check_score(scores[0], score_want(v[1], i32([1, 2, 3]), 9))


@gpu
def test_calls_on_another_stream(ops):
    p = Pool(ops, [700, 90], 2, 4, 128, seed=2)
    q = torch.randn(2, 8, 128).cuda()
    seq, ctx = i32([0, 1]), i32([700, 90])
    want = p.kv.attend(0, q, seq, ctx, p.tables, 700)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = [p.kv.attend(0, q, seq, ctx, p.tables, 700) for _ in range(8)]
        x = torch.randn(4, 50000, device="cuda")
        scores = ops.score_tokens(x, i32([1, 2, 3, 4]), top_k=4)
    here = [p.kv.attend(0, q, seq, ctx, p.tables, 700) for _ in range(8)]      # beside them
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs + here)
    check_score(scores, score_want(x, i32([1, 2, 3, 4]), 4))


@gpu
def test_a_captured_step_replays_with_new_inputs(ops):
    """Two decode steps captured into graphs of their own, replayed in turn and beside eager work, with contexts that grow."""
    hd, nkv, gq, V = 128, 2, 4, 20000
    nh = nkv * gq
    pools = [Pool(ops, [600, 40, 1], nkv, gq, hd, seed=s) for s in (11, 12)]
    rope = ops.rope_table(640, hd)
    sets = []
    for p in pools:
        s = dict(x=torch.randn(3, (nh + 2 * nkv) * hd, device="cuda"), seq=i32([0, 1, 2]), pos=i32([600, 40, 1]),
                 ctx=i32([601, 41, 2]), logits=torch.randn(3, V, device="cuda"), tok=i32([5, 6, 7]))

        def go(p=p, s=s):
            q = p.kv.append(0, s["x"], s["seq"], s["pos"], p.tables, rope=rope)
            return (q, p.kv.attend(0, q, s["seq"], s["ctx"], p.tables, 640), *ops.score_tokens(s["logits"], s["tok"], top_k=5))

        sets.append((p, s, go))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _, _, go in sets:
            go()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _, _, go in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(go())
        graphs.append(g)
    for rep in range(4):
        for (p, s, go), g, o in zip(sets, graphs, outs):
            s["x"].normal_()
            s["logits"].normal_()
            s["pos"].copy_(i32([600 + rep, 40 + rep, 1 + rep]))
            s["ctx"].copy_(s["pos"] + 1)
            keep = p.kv.pool.clone()
            want = go()
            after = p.kv.pool.clone()
            p.kv.pool.copy_(keep)
            for t in o:
                t.fill_(0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(p.kv.pool, after)
            assert all(torch.equal(a, b) for a, b in zip(o, want)), rep


@gpu
def test_offsets_past_32_bits(ops):
    """A pool of more than 4 GiB: the last blocks of the last layer."""
    hd, nkv, gq = 128, 8, 1
    layers, blocks = 2, 130000                                   # 4.5 GB
    kv = ops.PagedKV("int4", layers, blocks, nkv * gq, nkv, hd)
    tab = i32([[blocks - 1, blocks - 2], [0, 1]])
    x = torch.randn(64, 3 * nkv * hd, generator=torch.Generator().manual_seed(1)).cuda()
    seq, pos = i32([0] * 32 + [1] * 32), i32(list(range(32)) * 2)
    x[32:] = x[:32]
    q = kv.append(1, x, seq, pos, tab)
    k, v = kv.read(1, seq, pos, tab)
    assert torch.equal(k[:32], k[32:]) and torch.equal(v[:32], v[32:]) and bool((v != 0).any())
    out = kv.attend(1, q, seq, pos + 1, tab, 32)
    assert torch.equal(out[:32], out[32:])
    ref, A = attention(q[31].double().cpu(), q4(x[:32].cpu().view(32, 3, nkv, hd)[:, 1])[0], q4(x[:32].cpu().view(32, 3, nkv, hd)[:, 2])[0], hd ** -0.5)
    check_out(out[31], ref, A, 5.0, F, "last block")
    start, ctx = i32([0, 32, 64]), i32([32, 32])
    ch = kv.attend_chunks(1, q, start, ctx, tab, 32)
    assert torch.equal(ch[:32], ch[32:])
    check_out(ch[31], ref, A, 5.0, F, "last block, chunk")


@gpu
def test_no_rows(ops):
    kv = ops.PagedKV("int4", 1, 4, 4, 1, 64)
    tab, none = i32([[0, 1]]), i32([])
    assert kv.append(0, torch.zeros(0, 6 * 64, device="cuda"), none, none, tab).shape == (0, 4, 64)
    assert kv.read(0, none, none, tab)[0].shape == (0, 1, 64)
    assert kv.attend(0, torch.zeros(0, 4, 64, device="cuda"), none, none, tab, 16).shape == (0, 4, 64)
    assert kv.attend_chunks(0, torch.zeros(0, 4, 64, device="cuda"), i32([0, 0]), i32([0]), tab, 16).shape == (0, 4, 64)
    assert ops.score_tokens(torch.zeros(0, 50, device="cuda"), none, top_k=3)[2].shape == (0, 3)
