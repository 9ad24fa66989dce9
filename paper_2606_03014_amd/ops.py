"""The cache and head operators on torch tensors: the C ABI's moa_kv_* and moa_score_tokens.

Tensors live on one GPU; the work goes to torch's current stream of that GPU, results and workspaces come from torch's
allocator, and nothing waits, so the calls can be captured into a graph. Arguments that do not fit are refused before
anything is launched, with ValueError (tensors) or MoaError (sizes that the library refuses); index tensors are read on
the GPU (include/moa.h says what an entry that is out of range does). These are operators of inference: no gradient
passes through them. There is no fallback: without the built library or a GPU the calls raise.
"""
import ctypes as C
import math

import torch

from . import moa as M

KINDS = {"f32": M.MOA_KV_F32, "bf16": M.MOA_KV_BF16, "int4": M.MOA_KV_INT4}
_TYPES = {torch.float32: M.MOA_F32, torch.bfloat16: M.MOA_BF16}


def rope_table(n, head_dim, theta=10000.0, device="cuda"):
    """[n, head_dim / 2, 2] float32 (cos, sin) of position * theta^(-2 i / head_dim), computed in 64 bits."""
    i = torch.arange(head_dim // 2, dtype=torch.float64, device=device)
    a = torch.arange(n, dtype=torch.float64, device=device)[:, None] * theta ** (-2.0 * i / head_dim)
    return torch.stack([a.cos(), a.sin()], -1).float()


def _need(ok, what):
    if not ok:
        raise ValueError(what)


_raw_stream = torch._C._cuda_getCurrentRawStream      # torch.cuda.current_stream() without the Stream object
_F = {}


def _call(name, device, *args):
    """The library call on `device`, on torch's current stream of it."""
    f = _F.get(name)
    if f is None:
        f = _F[name] = getattr(M.lib(), name)
    i = device.index
    if torch._C._cuda_getDevice() == i:
        code = f(*args, _raw_stream(i))
    else:
        with torch.cuda.device(device):
            code = f(*args, _raw_stream(i))
    if code != M.MOA_OK:
        raise M.MoaError(code, name)


def _rows(t, name, width, device):
    """A matrix of rows of `width` elements each with a row stride of its own: (type, stride)."""
    typ = _TYPES.get(t.dtype)
    if typ is None or t.device != device:
        raise ValueError(f"{name}: a float32 or bfloat16 tensor on {device}")
    n = t.shape[0] if t.dim() >= 2 else -1
    if n < 0 or t.numel() != n * width or (n == 0 and math.prod(t.shape[1:]) != width):
        raise ValueError(f"{name}: rows of {width} elements")
    if t.is_contiguous():
        return typ, width
    inner = 1
    for k, s in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if k != 1 and s != inner:
            raise ValueError(f"{name}: the elements of a row must be contiguous")
        inner *= k
    return typ, t.stride(0) if n > 1 else width


def _ints(t, name, n, device):
    if t.dtype != torch.int32 or t.device != device or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous int32 on {device}")
    return t.data_ptr()


class PagedKV:
    """A paged pool of K and V, 16 positions a block, for n_layers layers of n_kv_heads heads.

    kind: "f32", "bf16" or "int4" (include/moa.h has the layouts). pool: a contiguous uint8 tensor of nbytes() bytes
    that the caller keeps, or None for a new one (zeros). Position p of sequence b lies in block tables[b, p // 16];
    tables is an int32 [sequences, blocks] tensor whose rows may be longer than a sequence needs."""

    def __init__(self, kind, n_layers, num_blocks, n_heads, n_kv_heads, head_dim, pool=None, device="cuda"):
        _need(kind in KINDS, f"kind must be one of {sorted(KINDS)}")
        self.kind, self.cfg = kind, M.moa_kv_cfg(KINDS[kind], n_layers, num_blocks, n_heads, n_kv_heads, head_dim)
        self._ref = C.byref(self.cfg)
        n = C.c_size_t()
        M.check(M.lib().moa_kv_bytes(self._ref, C.byref(n)), "moa_kv_bytes")
        self._bytes = n.value
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        if pool is None:
            pool = torch.zeros(n.value, dtype=torch.uint8, device=device)
        _need(pool.is_cuda, "pool: a GPU tensor")
        _need(pool.dtype == torch.uint8 and pool.is_contiguous() and pool.numel() == n.value,
              f"pool: {n.value} contiguous bytes")
        self.pool, self.device, self._at = pool, pool.device, pool.data_ptr()

    def nbytes(self):
        return self._bytes

    def _tables(self, tables):
        if (tables.dtype != torch.int32 or tables.device != self.device or tables.dim() != 2 or
                not tables.is_contiguous() or tables.numel() == 0):
            raise ValueError(f"tables: a contiguous int32 matrix on {self.device}")
        n, width = tables.shape
        return tables.data_ptr(), n, width

    def append(self, layer, qkv, row_seq, row_pos, tables, rope=None, q_gain=None, k_gain=None, eps=1e-5):
        """Norm (with gains), rotate (with a rope_table()) and cache rows of [queries | keys | values]; returns the
        queries, [rows, n_heads, head_dim] of qkv's type. Row r is position row_pos[r] of sequence row_seq[r]; a
        negative position is padding, and its row of the result is left unset. See moa_kv_append."""
        hd, T, dev = self.head_dim, qkv.shape[0], self.device
        typ, stride = _rows(qkv, "qkv", (self.n_heads + 2 * self.n_kv_heads) * hd, dev)
        tab, n_seqs, table_len = self._tables(tables)
        rope_len, gain_type = 0, 0
        if rope is not None:
            _need(rope.dtype == torch.float32 and rope.device == dev and rope.is_contiguous() and
                  rope.shape[1:] == (hd // 2, 2), f"rope: contiguous float32 [positions, {hd // 2}, 2]")
            rope_len = rope.shape[0]
        _need((q_gain is None) == (k_gain is None), "q_gain and k_gain go together")
        if q_gain is not None:
            for g in (q_gain, k_gain):
                _need(g.shape == (hd,) and g.dtype == q_gain.dtype and g.dtype in _TYPES and g.device == dev and
                      g.stride(0) == 1, f"gains: {hd} contiguous float32 or bfloat16 values")
            gain_type = _TYPES[q_gain.dtype]
        q = torch.empty(T, self.n_heads, hd, dtype=qkv.dtype, device=dev)
        _call("moa_kv_append", dev, self._ref, self._at, layer, qkv.data_ptr(), typ, stride, T,
              _ints(row_seq, "row_seq", T, dev), _ints(row_pos, "row_pos", T, dev), tab, n_seqs, table_len,
              rope.data_ptr() if rope is not None else None, rope_len,
              q_gain.data_ptr() if q_gain is not None else None, k_gain.data_ptr() if k_gain is not None else None,
              gain_type, eps, q.data_ptr())
        return q

    def read(self, layer, row_seq, row_pos, tables):
        """(k, v), each [rows, n_kv_heads, head_dim], of cached positions: float32 from an f32 pool, else bfloat16.
        See moa_kv_read."""
        T, dev = row_pos.shape[0], self.device
        tab, n_seqs, table_len = self._tables(tables)
        dt = torch.float32 if self.kind == "f32" else torch.bfloat16
        k = torch.empty(T, self.n_kv_heads, self.head_dim, dtype=dt, device=dev)
        v = torch.empty_like(k)
        _call("moa_kv_read", dev, self._ref, self._at, layer, T, _ints(row_seq, "row_seq", T, dev),
              _ints(row_pos, "row_pos", T, dev), tab, n_seqs, table_len, k.data_ptr(), v.data_ptr())
        return k, v

    def _out(self, out, q):
        if out is None:
            return torch.empty(q.shape[0], self.n_heads, self.head_dim, dtype=q.dtype, device=self.device)
        _need(out.shape == (q.shape[0], self.n_heads, self.head_dim) and out.dtype == q.dtype and
              out.device == self.device and out.is_contiguous(), "out: contiguous, of q's shape and type")
        return out

    def _workspace(self, name, *args):
        n = C.c_size_t()
        M.check(getattr(M.lib(), name)(self._ref, *args, C.byref(n)), name)
        n = n.value
        return torch.empty(n, dtype=torch.uint8, device=self.device) if n else None, n

    def attend(self, layer, q, row_seq, row_ctx, tables, max_ctx, scale=None, out=None):
        """Decode rows over an int4 pool: row r of q ([rows, n_heads, head_dim]) sees the first row_ctx[r] positions
        (at most max_ctx, which the host knows) of sequence row_seq[r]. scale: 1 / sqrt(head_dim) by default. Returns
        rows of q's shape and type. See moa_kv_attend."""
        T, dev = q.shape[0], self.device
        typ, stride = _rows(q, "q", self.n_heads * self.head_dim, dev)
        tab, n_seqs, table_len = self._tables(tables)
        out = self._out(out, q)
        ws, n = self._workspace("moa_kv_attend_bytes", T, max_ctx)
        _call("moa_kv_attend", dev, self._ref, self._at, layer, q.data_ptr(), typ, stride, T,
              _ints(row_seq, "row_seq", T, dev), _ints(row_ctx, "row_ctx", T, dev), tab, n_seqs, table_len, max_ctx,
              self.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), ws.data_ptr() if n else None, n)
        return out

    def attend_chunks(self, layer, q, chunk_start, chunk_ctx, tables, max_ctx, scale=None, out=None):
        """Causal prompt chunks over an int4 pool: rows [chunk_start[i], chunk_start[i + 1]) of q end at position
        chunk_ctx[i] - 1 of sequence i of tables (their K and V are appended before). Rows in no chunk keep what
        `out` held. See moa_kv_attend_chunks."""
        T, dev = q.shape[0], self.device
        typ, stride = _rows(q, "q", self.n_heads * self.head_dim, dev)
        tab, n, table_len = self._tables(tables)
        out = self._out(out, q)
        ws, nb = self._workspace("moa_kv_attend_chunks_bytes", T, n, max_ctx)
        _call("moa_kv_attend_chunks", dev, self._ref, self._at, layer, q.data_ptr(), typ, stride, T,
              _ints(chunk_start, "chunk_start", n + 1, dev), _ints(chunk_ctx, "chunk_ctx", n, dev), tab, n, table_len,
              max_ctx, self.head_dim ** -0.5 if scale is None else scale, out.data_ptr(),
              ws.data_ptr() if nb else None, nb)
        return out


def score_tokens(logits, tokens, top_k=0):
    """(logprob, entropy, top_ids, top_logprobs) of rows of logits ([rows, vocab], float32 or bfloat16, any row stride)
    and one given token each: float32 [rows], [rows], int32 and float32 [rows, top_k]. See moa_score_tokens."""
    _need(logits.is_cuda and logits.dim() == 2, "logits: a matrix on a GPU")
    dev, (R, V) = logits.device, logits.shape
    typ, stride = _rows(logits, "logits", V, dev)
    _need(V > 0 and 0 <= top_k <= min(V, M.MOA_MAX_TOP), f"top_k: 0 to {M.MOA_MAX_TOP}, at most the vocabulary")
    tok = _ints(tokens, "tokens", R, dev)
    lp = torch.empty(R, dtype=torch.float32, device=dev)
    entropy = torch.empty_like(lp)
    ids = torch.empty(R, top_k, dtype=torch.int32, device=dev)
    lps = torch.empty(R, top_k, dtype=torch.float32, device=dev)
    n = C.c_size_t()
    M.check(M.lib().moa_score_tokens_bytes(R, V, top_k, C.byref(n)), "moa_score_tokens_bytes")
    n = n.value
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _call("moa_score_tokens", dev, logits.data_ptr(), typ, stride, R, V, tok, lp.data_ptr(), entropy.data_ptr(), top_k,
          ids.data_ptr() if top_k else None, lps.data_ptr() if top_k else None,
          ws.data_ptr() if n else None, n)
    return lp, entropy, ids, lps
