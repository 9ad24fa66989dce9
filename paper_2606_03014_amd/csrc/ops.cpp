// C ABI of the operators on the caller's own tensors: argument checks, then the
// launch. See include/moa.h for the contract.
#include "moa.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "kernels.h"

using namespace moa;

static_assert((int)MOA_KV_F32 == (int)KV_F32 && (int)MOA_KV_BF16 == (int)KV_BF16 && (int)MOA_KV_INT4 == (int)KV_INT4,
              "pool kinds");
static_assert((int)MOA_MAX_TOP == kMaxTop, "alternatives");

namespace {

bool valid_kv(const moa_kv_cfg* c) {
  if (!c || c->kind < MOA_KV_F32 || c->kind > MOA_KV_INT4) return false;
  if (c->n_layers < 1 || c->num_blocks < 1 || c->n_heads < 1 || c->n_kv_heads < 1) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->n_heads % c->n_kv_heads) return false;
  const int gq = c->n_heads / c->n_kv_heads;
  // a row's heads are one grid dimension, and their elements an int
  if ((gq != 1 && gq != 2 && gq != 4 && gq != 8) || c->n_heads > 4096) return false;
  const double bytes = (double)c->n_layers * c->num_blocks * c->n_kv_heads * kv_cell_bytes(c->kind, c->head_dim);
  return bytes < 0x1p60;                         // no size or offset overflows
}

// Counts of rows and sequences, table entries and tokens: grids and positions fit 32 bits.
constexpr int32_t kMaxRows = 1 << 20, kMaxTable = 1 << 26, kMaxVocab = 1 << 30;

size_t pool_bytes(const moa_kv_cfg* c) {
  return (size_t)c->n_layers * c->num_blocks * c->n_kv_heads * kv_cell_bytes(c->kind, c->head_dim);
}

bool valid_type(int32_t t) { return t == MOA_F32 || t == MOA_BF16; }
bool aligned(const void* p, size_t a) { return p && (uintptr_t)p % a == 0; }

// The pool, the layer, the rows and their tables of one call.
bool valid_call(const moa_kv_cfg* c, const void* kv, int32_t layer, int32_t n_rows, const int32_t* tables,
                int32_t n_seqs, int32_t table_len) {
  return valid_kv(c) && aligned(kv, 16) && layer >= 0 && layer < c->n_layers && n_rows >= 0 && n_rows <= kMaxRows &&
         aligned(tables, 4) && n_seqs >= 1 && n_seqs <= kMaxRows && table_len >= 1 && table_len <= kMaxTable;
}

KvPlace place_of(const moa_kv_cfg* c, const int32_t* row_seq, const int32_t* tables, int32_t n_seqs, int32_t table_len) {
  return {tables, row_seq, table_len, n_seqs, table_len, c->num_blocks};
}

moa_status status_of(hipError_t err, const char* what) {
  if (err == hipSuccess) return MOA_OK;
  std::fprintf(stderr, "moa: HIP error in %s: %s\n", what, hipGetErrorString(err));
  return MOA_EHIP;
}

moa_status check_attend(const moa_kv_cfg* c, const void* kv, int32_t layer, const void* q, int32_t type,
                        int64_t q_stride, int32_t n_rows, const int32_t* tables, int32_t n_seqs, int32_t table_len,
                        int32_t max_ctx, float scale, void* out) {
  if (!valid_call(c, kv, layer, n_rows, tables, n_seqs, table_len) || c->kind != MOA_KV_INT4 || !valid_type(type))
    return MOA_EINVAL;
  const size_t el = type == MOA_BF16 ? 2 : 4;
  if (max_ctx < 1 || max_ctx > 16ll * table_len || !std::isfinite(scale)) return MOA_EINVAL;
  if (n_rows > 0 && (!aligned(q, el) || !aligned(out, 16) || q_stride < (int64_t)c->n_heads * c->head_dim)) return MOA_EINVAL;
  return MOA_OK;
}

Attend4Args attend_args(const moa_kv_cfg* c, const void* kv, int32_t layer, const void* q, int32_t type,
                        int64_t q_stride, int32_t n_rows, const int32_t* tables, int32_t n_seqs, int32_t table_len,
                        int32_t max_ctx, float scale, void* out) {
  Attend4Args a{};
  a.q = q;
  a.q_stride = (size_t)q_stride;
  a.q_bf16 = type == MOA_BF16;
  a.out = out;
  a.out_type = type == MOA_BF16 ? OUT_BF16 : OUT_F32;
  a.kv = kv;
  a.layer = layer;
  a.num_blocks = c->num_blocks;
  a.n_h = c->n_heads;
  a.n_kv = c->n_kv_heads;
  a.hd = c->head_dim;
  a.scale = scale;
  a.tables = tables;
  a.T = n_rows;
  a.n_seqs = n_seqs;
  a.table_len = table_len;
  a.max_ctx = max_ctx;
  return a;
}

// MOA_OK when the workspace holds `need` bytes.
moa_status check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need == 0) return MOA_OK;
  if (workspace && (uintptr_t)workspace % 256) return MOA_EINVAL;
  return workspace && bytes >= need ? MOA_OK : MOA_ENOMEM;
}

}  // namespace

extern "C" {

moa_status moa_kv_bytes(const moa_kv_cfg* c, size_t* bytes) {
  if (!valid_kv(c) || !bytes) return MOA_EINVAL;
  *bytes = pool_bytes(c);
  return MOA_OK;
}

moa_status moa_kv_append(const moa_kv_cfg* c, void* kv, int32_t layer, const void* qkv, int32_t type,
                         int64_t qkv_stride, int32_t n_rows, const int32_t* row_seq, const int32_t* row_pos,
                         const int32_t* tables, int32_t n_seqs, int32_t table_len, const float* rope,
                         int32_t rope_len, const void* q_gain, const void* k_gain, int32_t gain_type, float eps,
                         void* q, void* hip_stream) {
  if (!valid_call(c, kv, layer, n_rows, tables, n_seqs, table_len) || !valid_type(type)) return MOA_EINVAL;
  if (!q_gain != !k_gain || (rope && (rope_len < 1 || !aligned(rope, 16)))) return MOA_EINVAL;
  if (q_gain && (!valid_type(gain_type) || !(eps >= 0.f) || !std::isfinite(eps))) return MOA_EINVAL;
  if (q_gain && (!aligned(q_gain, gain_type == MOA_BF16 ? 2 : 4) || !aligned(k_gain, gain_type == MOA_BF16 ? 2 : 4)))
    return MOA_EINVAL;
  if (n_rows == 0) return MOA_OK;
  const int64_t width = (int64_t)(c->n_heads + 2 * c->n_kv_heads) * c->head_dim;
  if (!aligned(qkv, type == MOA_BF16 ? 2 : 4) || qkv_stride < width || !aligned(q, 16)) return MOA_EINVAL;
  if (!aligned(row_seq, 4) || !aligned(row_pos, 4)) return MOA_EINVAL;
  AppendArgs a{};
  a.x = qkv;
  a.stride = (size_t)qkv_stride;
  a.nsplit = 1;
  a.row_pos = row_pos;
  a.place = place_of(c, row_seq, tables, n_seqs, table_len);
  a.rope = (const float2*)rope;
  a.rope_len = rope_len;
  a.q_gain.p[0] = q_gain;
  a.k_gain.p[0] = k_gain;
  a.gain_bf16 = gain_type == MOA_BF16;
  a.eps = eps;
  a.q = q;
  a.kv = kv;
  a.layer = layer;
  a.n_h = c->n_heads;
  a.n_kv = c->n_kv_heads;
  a.hd = c->head_dim;
  a.T = n_rows;
  return status_of(launch_kv_append((hipStream_t)hip_stream, type == MOA_BF16, c->kind, a), "moa_kv_append");
}

moa_status moa_kv_read(const moa_kv_cfg* c, const void* kv, int32_t layer, int32_t n_rows, const int32_t* row_seq,
                       const int32_t* row_pos, const int32_t* tables, int32_t n_seqs, int32_t table_len, void* k,
                       void* v, void* hip_stream) {
  if (!valid_call(c, kv, layer, n_rows, tables, n_seqs, table_len)) return MOA_EINVAL;
  if (n_rows == 0) return MOA_OK;
  if (!aligned(row_seq, 4) || !aligned(row_pos, 4) || !aligned(k, 16) || !aligned(v, 16)) return MOA_EINVAL;
  return status_of(launch_kv_read((hipStream_t)hip_stream, c->kind, kv, layer, c->n_kv_heads, c->head_dim, n_rows,
                                  row_pos, 0, place_of(c, row_seq, tables, n_seqs, table_len), k, v), "moa_kv_read");
}

moa_status moa_kv_attend_bytes(const moa_kv_cfg* c, int32_t n_rows, int32_t max_ctx, size_t* bytes) {
  if (!valid_kv(c) || c->kind != MOA_KV_INT4 || n_rows < 0 || n_rows > kMaxRows || max_ctx < 1 || max_ctx > 16 * kMaxTable || !bytes)
    return MOA_EINVAL;
  if (!attend4_rows_fits(c->n_kv_heads, n_rows, max_ctx)) return MOA_EINVAL;
  *bytes = attend4_rows_bytes(c->n_heads, c->n_kv_heads, c->head_dim, n_rows, max_ctx);
  return MOA_OK;
}

moa_status moa_kv_attend(const moa_kv_cfg* c, const void* kv, int32_t layer, const void* q, int32_t type,
                         int64_t q_stride, int32_t n_rows, const int32_t* row_seq, const int32_t* row_ctx,
                         const int32_t* tables, int32_t n_seqs, int32_t table_len, int32_t max_ctx, float scale,
                         void* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  moa_status st = check_attend(c, kv, layer, q, type, q_stride, n_rows, tables, n_seqs, table_len, max_ctx, scale, out);
  if (st != MOA_OK) return st;
  if (n_rows == 0) return MOA_OK;
  if (!aligned(row_seq, 4) || !aligned(row_ctx, 4)) return MOA_EINVAL;
  size_t need = 0;
  st = moa_kv_attend_bytes(c, n_rows, max_ctx, &need);
  if (st == MOA_OK) st = check_workspace(workspace, workspace_bytes, need);
  if (st != MOA_OK) return st;
  Attend4Args a = attend_args(c, kv, layer, q, type, q_stride, n_rows, tables, n_seqs, table_len, max_ctx, scale, out);
  a.row_seq = row_seq;
  a.row_ctx = row_ctx;
  return status_of(launch_attend4_rows((hipStream_t)hip_stream, a, workspace), "moa_kv_attend");
}

moa_status moa_kv_attend_chunks_bytes(const moa_kv_cfg* c, int32_t n_rows, int32_t n_chunks, int32_t max_ctx,
                                      size_t* bytes) {
  if (!valid_kv(c) || c->kind != MOA_KV_INT4 || n_rows < 0 || n_rows > kMaxRows || n_chunks < 1 || n_chunks > kMaxRows ||
      max_ctx < 1 || max_ctx > 16 * kMaxTable || !bytes)
    return MOA_EINVAL;
  const Chunks4Size z{c->n_heads, c->n_kv_heads, c->head_dim, n_rows, n_chunks, max_ctx};
  if (!attend4_chunks_fits(z)) return MOA_EINVAL;
  *bytes = attend4_chunks_bytes(z);
  return MOA_OK;
}

moa_status moa_kv_attend_chunks(const moa_kv_cfg* c, const void* kv, int32_t layer, const void* q, int32_t type,
                                int64_t q_stride, int32_t n_rows, const int32_t* chunk_start,
                                const int32_t* chunk_ctx, const int32_t* tables, int32_t n_chunks,
                                int32_t table_len, int32_t max_ctx, float scale, void* out, void* workspace,
                                size_t workspace_bytes, void* hip_stream) {
  moa_status st = check_attend(c, kv, layer, q, type, q_stride, n_rows, tables, n_chunks, table_len, max_ctx, scale, out);
  if (st != MOA_OK) return st;
  if (n_rows == 0) return MOA_OK;
  if (!aligned(chunk_start, 4) || !aligned(chunk_ctx, 4)) return MOA_EINVAL;
  size_t need = 0;
  st = moa_kv_attend_chunks_bytes(c, n_rows, n_chunks, max_ctx, &need);
  if (st == MOA_OK) st = check_workspace(workspace, workspace_bytes, need);
  if (st != MOA_OK) return st;
  Attend4Args a = attend_args(c, kv, layer, q, type, q_stride, n_rows, tables, n_chunks, table_len, max_ctx, scale, out);
  a.chunk_start = chunk_start;
  a.chunk_ctx = chunk_ctx;
  return status_of(launch_attend4_chunks((hipStream_t)hip_stream, a, workspace), "moa_kv_attend_chunks");
}

moa_status moa_score_tokens_bytes(int32_t n_rows, int32_t vocab, int32_t top_k, size_t* bytes) {
  if (n_rows < 0 || n_rows > kMaxRows || vocab < 1 || vocab > kMaxVocab || top_k < 0 || top_k > MOA_MAX_TOP || top_k > vocab || !bytes) return MOA_EINVAL;
  *bytes = score_bytes(n_rows, vocab, top_k);
  return MOA_OK;
}

moa_status moa_score_tokens(const void* logits, int32_t type, int64_t stride, int32_t n_rows, int32_t vocab,
                            const int32_t* tokens, float* logprob, float* entropy, int32_t top_k, int32_t* top_ids,
                            float* top_logprobs, void* workspace, size_t workspace_bytes, void* hip_stream) {
  size_t need = 0;
  const moa_status st = moa_score_tokens_bytes(n_rows, vocab, top_k, &need);
  if (st != MOA_OK) return st;
  if (!valid_type(type) || stride < vocab) return MOA_EINVAL;
  if (n_rows == 0) return MOA_OK;
  if (!aligned(logits, type == MOA_BF16 ? 2 : 4) || !aligned(tokens, 4) || !aligned(logprob, 4) || !aligned(entropy, 4))
    return MOA_EINVAL;
  if (top_k > 0 && (!aligned(top_ids, 4) || !aligned(top_logprobs, 4))) return MOA_EINVAL;
  const moa_status ws = check_workspace(workspace, workspace_bytes, need);
  if (ws != MOA_OK) return ws;
  ScoreArgs a{};
  a.logits = logits;
  a.bf16 = type == MOA_BF16;
  a.stride = (size_t)stride;
  a.rows = n_rows;
  a.vocab = vocab;
  a.top = top_k;
  a.tokens = tokens;
  a.logprob = logprob;
  a.entropy = entropy;
  a.top_ids = top_ids;
  a.top_logprobs = top_logprobs;
  return status_of(launch_score((hipStream_t)hip_stream, a, workspace), "moa_score_tokens");
}

}  // extern "C"
