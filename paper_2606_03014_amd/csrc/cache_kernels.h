// Kernels around the paged cache for callers' own pools and for engines with
// 4-bit K/V or per-head norms: append, read-back, and attention over 4-bit
// cells. Part of kernels.hip (its helpers are above).

// The cell of (layer, block, KV head).
__device__ __forceinline__ unsigned char* kv_cell(const void* kv, int kind, int hd, int layer, int num_blocks, int block,
                                                  int n_kv, int head) {
  return (unsigned char*)kv + (((size_t)layer * num_blocks + block) * n_kv + head) * kv_cell_bytes(kind, hd);
}
// The block of a position of sequence `key`, -1 if anything is out of range.
__device__ __forceinline__ int kv_block(const KvPlace& p, int key, int pos) {
  if ((unsigned)key >= (unsigned)p.n_keys || pos < 0 || (pos >> 4) >= p.table_len) return -1;
  const int b = p.tables[(size_t)key * p.mul + (pos >> 4)];
  return (unsigned)b < (unsigned)p.num_blocks ? b : -1;
}

// The row of workgroup b of T, for 4-bit cells: the 16 rows of a block share V's lines, a byte each, and
// an XCD's L2 joins only what its own workgroups touch. Every eighth workgroup goes to one XCD, so it
// gets 16 neighbours of each 128 rows (18,432 rows appended at 8 KV heads of 128: 137 us against 148, 2,048
// rows 18.8 against 20.3; read back 27 against 30.8).
__device__ __forceinline__ int row_of(int b, int T) {
  return (b | 127) < T ? (b & ~127) + (b & 7) * 16 + ((b >> 3) & 15) : b;
}

// A cross-lane move of a double: its two words.
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
  const unsigned lo = (unsigned)__builtin_amdgcn_mov_dpp((int)(unsigned)u, CTRL, 0xF, 0xF, true);
  const unsigned hi = (unsigned)__builtin_amdgcn_mov_dpp((int)(unsigned)(u >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, ((unsigned long long)hi << 32) | lo);
}
// Combine over the LP lanes (4, 8 or 16) that hold one row of a head; all get the result.
template <int LP, typename T, typename F>
__device__ __forceinline__ T over_row(T v, F f) {
  v = f(v, dpp<0xB1>(v));
  v = f(v, dpp<0x4E>(v));
  if constexpr (LP >= 8) v = f(v, dpp<0x141>(v));
  if constexpr (LP == 16) v = f(v, dpp<0x128>(v));
  return v;
}

// One 4-bit row from hd / N lanes, lane l holding dims N / 2 l .. + N / 2 and the
// same + hd / 2: its scale word and the lane's N codes.
// The quotient is that of 64-bit division (a product with the reciprocal, and one step
// that takes its residual in): exact where it lies on the border of two codes, as bf16
// values often do, and on the right side of it otherwise. Rounded to 24 bits it made a
// tie, and the other code, of one float32 value in a million.
template <int HD, int N>
__device__ __forceinline__ unsigned quantise(const float x[N], int c[N]) {
  constexpr int LP = HD / N;
  // NaN goes through these, so one test finds NaN, infinities and ranges past float32
  auto least = [](float a, float b) { return __builtin_elementwise_minimum(a, b); };
  auto most = [](float a, float b) { return __builtin_elementwise_maximum(a, b); };
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) { lo = least(lo, x[i]); hi = most(hi, x[i]); }
  lo = over_row<LP>(lo, least);
  hi = over_row<LP>(hi, most);
  unsigned word = pack_bf16((hi - lo) * (1.f / 15.f), lo);   // a product: a division is ten instructions, and no better a step
  if (!(hi - lo < INFINITY) || !(fabsf(__uint_as_float(word & 0xffff0000u)) < INFINITY)) word = 0x7fc0u;
  const float sf = __uint_as_float(word << 16);
  const bool some = sf > 0.f;                            // else all codes are 0, for NaN too
  const double md = __uint_as_float(word & 0xffff0000u), sd = some ? (double)sf : 1.0;
  double inv = __builtin_amdgcn_rcp(sd);                 // 2^-24; after the step 2^-48, which the residual squares
  inv = fma(inv, fma(-sd, inv, 1.0), inv);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double d = (double)x[i] - md, u = d * inv, q = fma(fma(-sd, u, d), inv, u);
    c[i] = some ? (int)__builtin_rint(fmin(fmax(q, 0.0), 15.0)) : 0;
  }
  return word;
}

template <bool BF>
__device__ __forceinline__ float load_el(const void* p, size_t i) {
  return BF ? bf2f(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}

// N consecutive elements as float32; vec: 16-byte loads (8 for four bf16) may be used.
template <int N>
__device__ __forceinline__ void load_run(const void* p, size_t at, bool bf16, bool vec, float* v) {
  if (vec && bf16 && N % 8 != 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x2_t x = *(const u32x2_t*)((const uint16_t*)p + at + i);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        v[i + 2 * k] = __uint_as_float(x[k] << 16);
        v[i + 2 * k + 1] = __uint_as_float(x[k] & 0xffff0000u);
      }
    }
  } else if (vec && bf16) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      const u32x4 x = *(const u32x4*)((const uint16_t*)p + at + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[i + 2 * k] = __uint_as_float(x[k] << 16);
        v[i + 2 * k + 1] = __uint_as_float(x[k] & 0xffff0000u);
      }
    }
  } else if (vec) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const f32x4_t x = *(const f32x4_t*)((const float*)p + at + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[i + k] = x[k];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = bf16 ? load_el<true>(p, at + i) : load_el<false>(p, at + i);
  }
}

// Four consecutive values as float32 or bf16.
__device__ __forceinline__ void store4(void* p, bool bf16, size_t at, const float* x) {
  if (bf16) *(uint2*)((uint16_t*)p + at) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  else *(float4*)((float*)p + at) = make_float4(x[0], x[1], x[2], x[3]);
}
// Lane l's part of a row of hd values, both halves.
template <int HD, int N>
__device__ __forceinline__ void store_part(void* p, bool bf16, size_t at, int l, const float x[N]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const size_t o = at + h * (HD / 2) + N / 2 * l;
    const float* y = x + h * (N / 2);
    if constexpr (N == 16) {
      if (bf16) {
        *(u32x4*)((uint16_t*)p + o) = u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
        continue;
      }
    }
#pragma unroll
    for (int i = 0; i < N / 2; i += 4) store4(p, bf16, o + i, y + i);
  }
}

// Store a row held as for quantise() (lane l) as K (v = false) or V of a cell's slot.
template <int HD, int KIND, int N>
__device__ __forceinline__ void store_row(unsigned char* cell, int slot, bool v, const float x[N], int l) {
  if constexpr (KIND == KV_INT4) {
    int c[N];
    const unsigned sc = quantise<HD, N>(x, c);
    if (v) {
      unsigned char* p = cell + 8 * HD + N / 2 * l * 16 + slot;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) p[i * 16] = (unsigned char)(c[i] | (c[i + N / 2] << 4));
    } else {
      unsigned char* p = cell + slot * (HD / 2) + N / 4 * l;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        unsigned word = 0;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) word |= (unsigned)c[h * (N / 2) + i] << (4 * i);
        if constexpr (N == 16) *(unsigned*)(p + h * (HD / 4)) = word;
        else *(uint16_t*)(p + h * (HD / 4)) = (uint16_t)word;
      }
    }
    if (l == 0) ((unsigned*)(cell + 16 * HD))[(v ? 16 : 0) + slot] = sc;
  } else {
    store_part<HD, N>(cell, KIND == KV_BF16, (size_t)((v ? kBlock : 0) + slot) * HD, l, x);
  }
}

// ------------------------------ per-head norms, rotation and append in one pass
// hd / N lanes hold one head of one row, each both halves of N / 2 rotation pairs, so
// the norm's sum, the row's range and its codes stay within a row of 16 lanes; N = 8
// values a lane in float32 and 16 in bf16 are 16-byte loads. Rows of codes take 8 in bf16 too:
// in 64 bits 16 need 80 registers, and fewer waves hide less (142 against 131 us for 18,348 rows).
// Keys of a 4-bit cache are computed in 64 bits: their codes are then
// those of the float32 value, whatever the order of the norm's sum (one bit of the
// float32 value can move the row's bf16 minimum, and with it every code).
// Bound by bytes, and in 4-bit pools by the arithmetic in 64 bits and V's single bytes. 32 + 2 * 8 heads: 15,347
// float32 rows (64 wide) into a bf16 pool 68 us, 5.0 TB/s; 18,348 bf16 rows (128 wide) into a 4-bit one
// 131 us, 3.0 TB/s (their queries alone 72, 4.2 TB/s); 512 float32 rows 7.3 us. A wave for each run of
// rows of one block, V in words, was slower (18,432 rows 157 against 130 us, 8,192 66 against 54).

// Lane l's dims of a head of row t.
template <bool XBF, int HD, int N>
__device__ __forceinline__ void load_head(const AppendArgs& a, bool aligned, int t, int head, int l, float x[N]) {
  const size_t at = (size_t)t * a.stride + (size_t)head * HD + N / 2 * l;
  if (XBF) {
    load_run<N / 2>(a.x, at, true, aligned, x);
    load_run<N / 2>(a.x, at + HD / 2, true, aligned, x + N / 2);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 0.f;
    for (int s = 0; s < a.nsplit; ++s) {
      float y[N];
      load_run<N / 2>(a.x, at + (size_t)s * a.split_stride, false, aligned, y);
      load_run<N / 2>(a.x, at + (size_t)s * a.split_stride + HD / 2, false, aligned, y + N / 2);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += y[i];
    }
  }
}

// Lane l's dims of a gain, and its rotation's (cos, sin) at a position.
template <int HD, int N>
__device__ __forceinline__ void load_gain(const AppendArgs& a, const ModelPtrs& gains, int t, int l, float g[N]) {
  const void* p = pick(gains, a.row_model ? a.row_model[t] : 0);
  load_run<N / 2>(p, N / 2 * l, a.gain_bf16, a.gain_vec, g);
  load_run<N / 2>(p, N / 2 * l + HD / 2, a.gain_bf16, a.gain_vec, g + N / 2);
}
template <int HD, int N>
__device__ __forceinline__ void load_turn(const AppendArgs& a, int pos, int l, float c[N]) {
  load_run<N>(a.rope, ((size_t)pos * (HD / 2) + N / 2 * l) * 2, false, true, c);
}

// Norm (with gain g) and rotation by c, in type T.
template <typename T, int HD, int N, bool NORM>
__device__ __forceinline__ void norm_rotate(const AppendArgs& a, const float g[N], const float c[N], float x[N]) {
  constexpr int H = N / 2;
  T y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = (T)x[i];
  if constexpr (NORM) {
    T ss = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) ss += y[i] * y[i];
    ss = over_row<HD / N>(ss, [](T u, T w) { return u + w; });
    const T mean = ss / (T)HD + (T)a.eps;
    T inv;
    if constexpr (sizeof(T) == 8) {                  // two Newton steps: 2^-50
      inv = __builtin_amdgcn_rsq(mean);
      inv *= 1.5 - 0.5 * mean * inv * inv;
      inv *= 1.5 - 0.5 * mean * inv * inv;
    } else {
      inv = rsqrtf(mean);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] *= inv * (T)g[i];
  }
  if (a.rope) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      if constexpr (sizeof(T) == 8) {
        const T u = y[i], w = y[i + H];
        y[i] = u * c[2 * i] - w * c[2 * i + 1];
        y[i + H] = w * c[2 * i] + u * c[2 * i + 1];
      } else {
        const float2 r = rotate((float)y[i], (float)y[i + H], make_float2(c[2 * i], c[2 * i + 1]));
        y[i] = r.x;
        y[i + H] = r.y;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = (float)y[i];
}

// Values a lane: of a query head (and of any head into f32 and bf16 cells), and of a key's or value's row of codes.
constexpr int append_q_vals(bool xbf) { return xbf ? 16 : 8; }
constexpr int append_kv_vals(bool xbf, int kind) { return kind == KV_INT4 ? 8 : append_q_vals(xbf); }

// A workgroup is as many heads of one row as its threads hold, of queries or of keys and values:
// its position and block are scalars.
template <bool XBF, int KIND, int HD, bool NORM>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a, bool aligned) {
  const int t = KIND == KV_INT4 ? row_of(blockIdx.x, a.T) : blockIdx.x;
  {
    constexpr int N = append_q_vals(XBF), LP = HD / N, HW = 256 / LP;
    const int l = threadIdx.x % LP, head = blockIdx.y * HW + threadIdx.x / LP;
    if (blockIdx.y * HW < a.n_h) {
      if (head >= a.n_h) return;
      float x[N], g[N], c[N];
      load_head<XBF, HD, N>(a, aligned, t, head, l, x);
      if (NORM) load_gain<HD, N>(a, a.q_gain, t, l, g);
      const int pos = a.row_pos[t];
      if (pos < 0 || (a.rope && pos >= a.rope_len)) return;
      if (a.rope) load_turn<HD, N>(a, pos, l, c);
      norm_rotate<float, HD, N, NORM>(a, g, c, x);
      store_part<HD, N>(a.q, XBF, ((size_t)t * a.n_h + head) * HD, l, x);
      return;
    }
  }
  constexpr int N = append_kv_vals(XBF, KIND), LP = HD / N, HW = 256 / LP, QW = 256 * append_q_vals(XBF) / HD;
  const int l = threadIdx.x % LP, kv = (blockIdx.y - (a.n_h + QW - 1) / QW) * HW + threadIdx.x / LP;
  if (kv >= 2 * a.n_kv) return;
  const bool is_v = kv >= a.n_kv;
  float x[N], g[N], c[N];
  load_head<XBF, HD, N>(a, aligned, t, a.n_h + kv, l, x);
  if (NORM && !is_v) load_gain<HD, N>(a, a.k_gain, t, l, g);
  const int pos = a.row_pos[t];
  if (pos < 0 || (a.rope && pos >= a.rope_len)) return;
  if (!is_v) {
    if (a.rope) load_turn<HD, N>(a, pos, l, c);
    using T = std::conditional_t<KIND == KV_INT4, double, float>;
    norm_rotate<T, HD, N, NORM>(a, g, c, x);
  }
  const int block = kv_block(a.place, a.place.key[t], pos);
  if (block < 0) return;
  store_row<HD, KIND, N>(kv_cell(a.kv, KIND, HD, a.layer, a.place.num_blocks, block, a.n_kv, is_v ? kv - a.n_kv : kv), pos & 15, is_v, x, l);
}

// ------------------------------------------------- what cached positions hold
// hd / 8 lanes a row. Bound by bytes and, in 4-bit cells, by V's single bytes: 18,348 rows of 8 heads of 128 27 us (95 MB).
template <int KIND, int HD>
__global__ __launch_bounds__(256) void k_kv_read(const void* __restrict__ kv, int layer, int n_kv, int T,
                                                 const int* __restrict__ row_pos, int pos0, KvPlace place,
                                                 void* __restrict__ kout, void* __restrict__ vout) {
  constexpr int LP = HD / 8;
  const int t = KIND == KV_INT4 ? row_of(blockIdx.x, T) : blockIdx.x, l = threadIdx.x % LP;
  const int kh = blockIdx.y * (256 / LP) + threadIdx.x / LP;
  if (kh >= n_kv) return;
  const int pos = row_pos ? row_pos[t] : pos0 + t, block = kv_block(place, place.key ? place.key[t] : 0, pos), slot = pos & 15;
  const size_t o = ((size_t)t * n_kv + kh) * HD;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    float x[8] = {};
    if (block >= 0) {
      const unsigned char* cell = kv_cell(kv, KIND, HD, layer, place.num_blocks, block, n_kv, kh);
      if constexpr (KIND == KV_INT4) {
        const unsigned sc = ((const unsigned*)(cell + 16 * HD))[16 * v + slot];
        const float s = __uint_as_float(sc << 16), m = __uint_as_float(sc & 0xffff0000u);
        int c[8];
        if (v) {
          const unsigned char* p = cell + 8 * HD + 4 * l * 16 + slot;
#pragma unroll
          for (int i = 0; i < 4; ++i) { c[i] = p[i * 16] & 15; c[i + 4] = p[i * 16] >> 4; }
        } else {
          const uint16_t* p = (const uint16_t*)(cell + slot * (HD / 2) + 2 * l);
#pragma unroll
          for (int i = 0; i < 8; ++i) c[i] = (p[(i >> 2) * (HD / 8)] >> (4 * (i & 3))) & 15;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(s, (float)c[i], m);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[i] = load_el<KIND == KV_BF16>(cell, (v * kBlock + slot) * HD + 4 * l + (i & 3) + (i >> 2) * (HD / 2));
      }
    }
    store_part<HD, 8>(v ? vout : kout, KIND != KV_F32, o, l, x);
  }
}

// ---------------------------- decode attention over 4-bit cells (16x16x32 MFMA)
// One workgroup is a row, a KV head and one split of its keys; its four waves take
// every fourth tile of 64 keys (four blocks) and join at the end.
//
// A code reaches the matrix cores as it is: its four bits, moved to bits 4 to 7 of a
// half, are the float16 2^-20 c (subnormal, and exact), so seven integer instructions
// unpack eight codes, and scales and minima are applied after the products, per key:
//   q . k = s_k sum(c q) + m_k sum(q),   sum p v = sum (p s_v) c + sum p m_v.
// q, scaled to a power of two below 2^13, and p s_v enter as pairs of float16 (hi + lo, 22
// bits): the head's hi part is column h of an operand and its lo part column h + 8, so
// the pair costs no product. The code bits lie as high in the half as a mask without
// a shift for one pair in four allows: at bits 0 to 3 the products lose four more bits
// in the matrix cores (3.6e-6 of the sum against 6.8e-8, measured).
//
// S^T = K Q^T: row r of score tile n is block r / 4, slot 4 n + r % 4 of the 64 keys, so a
// lane (col, q = lane / 16) ends with the scores of slots 0 to 15 of block q, which are
// the k-slots that O^T = V^T P^T wants from it: no probability crosses lanes. V's cells
// are laid out for that product (16 slots of a dim side by side): nothing is transposed.
//
// The softmax's reference M is kept so that p s_v stays below 2^13 (float16 holds it) and is
// moved, with everything that was summed, only when a product passes that; p alone
// may be as large as 2^98 then (tiny scales), which float32 sums hold.
//
// Bound by reading the cells, non-temporal, once: 384 rows of 1,000 to 8,000 keys, 32 heads of 128 over 8 KV
// heads, bf16, 265 us, 5.3 TB/s; 7 float32 rows of 12,000 to 32,000 keys 41 us (3.8 TB/s: the join, the
// start and the grid's tail); 160 of 64 to 3,000 at heads of 64 34 us. Three waves a SIMD hold a tile of keys and
// one of values in registers; four spill (450 us), and double buffers gain nothing over non-temporal single ones.
constexpr int kSplit4Max = 2048;
constexpr unsigned kCodeMask = 0x00F000F0u;
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));

struct Partial4 { float *acc, *ml; };              // [slot][n_h][hd] sums; [slot][n_h] (M, l)

// (a, b) -> two float16 in one word, round to nearest even: a truncated lo part would
// put a bias of 2^-23 on every probability, and the codes, which are all positive, and
// the minima nearly cancel in the answer (6e-6 of it over 900 equal probabilities).
__device__ __forceinline__ unsigned pack_f16(float a, float b) {
  return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2_t){a, b}, f16x2_t));
}
// For a head whose largest |q| is mx: the power of two, with scale's sign, that brings q just below
// 2^13, and a score's unit after it in powers of two (f > 0). The exponent stops at 2^-100,
// so that the factor of subnormal queries stays finite; a scale that leaves no unit is 0.
__device__ __forceinline__ void q_units(float mx, float scale, float& up, float& f) {
  int e = 0;
  if (mx > 0.f && mx < INFINITY) (void)frexpf(mx, &e);
  e = max(e, -100);
  f = ldexpf(fabsf(scale) * 1.4426950408889634f, e - 13);
  const bool some = f > 0.f;
  up = some ? copysignf(ldexpf(1.f, 13 - e), scale) : 0.f;
  f = some ? f : 1.f;
}
// Over a column of four lanes 16 apart.
__device__ __forceinline__ float max_column(float v) {
  v = fmaxf(v, swz_xor16(v));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_column(float v) {
  v += swz_xor16(v);
  return v + __shfl_xor(v, 32, 64);
}
// Two codes, at bits 0 to 3 of each half after the shift, as float16 c - 8.
__device__ __forceinline__ unsigned centred(unsigned w) {
  const f16x2_t x = __builtin_bit_cast(f16x2_t, (w & 0x03C003C0u) | 0x4C004C00u);   // 16 + c
  return __builtin_bit_cast(unsigned, x - (f16x2_t){(_Float16)24, (_Float16)24});
}
// Eight codes of a word as float16, in the order 0 4 1 5 2 6 3 7: 2^-20 c; or 2^-24 c and,
// for odd ones, 2^-20 c (two instructions fewer).
__device__ __forceinline__ u32x4 codes_mixed(unsigned w) {
  const unsigned v = w >> 8;
  return u32x4{w & 0x000F000Fu, w & kCodeMask, v & 0x000F000Fu, v & kCodeMask};
}
__device__ __forceinline__ u32x4 codes_f16(unsigned w) {
  return u32x4{(w << 4) & kCodeMask, w & kCodeMask, (w >> 4) & kCodeMask, (w >> 8) & kCodeMask};
}

template <int HD, bool ITEMS, bool FINE>
__global__ __launch_bounds__(256, 3) void k_attend4_rows(Attend4Args a, const AttnItem* __restrict__ items, int split,
                                                         Partial4 part, bool q_vec) {
  constexpr int CELL = (int)kv_cell_bytes(KV_INT4, HD);
  constexpr int W = HD / 32;                       // words of a key's row per lane; 16-dim tiles of half a head
  __shared__ __align__(16) float ssc[4][2][4][36]; // wave: K and V (s, m) of 4 blocks of 16 keys, blocks 36 words apart
  __shared__ float sml[4][2][8];
  __shared__ __align__(16) float so[4][8][HD + 4];
  __shared__ unsigned sid[kSplit4Max / kBlock];       // the split's blocks
  __shared__ __align__(16) unsigned sq[W][69][4];  // the queries' fragments (lane + lane / 16: other banks)
  __shared__ float sqf[2][8];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4, gq = a.n_h / a.n_kv, kvh = blockIdx.x % a.n_kv;
  const int item = blockIdx.x / a.n_kv;            // heads fastest, then rows: every XCD gets its part of each split
  int row, k0, k1, slot, last;                     // last: the last table entry that may be read
  const int* tab;
  if constexpr (ITEMS) {
    const AttnItem it = items[item];
    row = it.row; k0 = it.k0; k1 = it.k1; slot = it.slot;
    tab = a.tables + it.bt_off - (it.k0 >> 4);
    last = (k1 - 1) >> 4;
  } else {
    row = item % a.T;
    k0 = item / a.T * split;
    const int seq = a.row_seq[row];
    const bool known = (unsigned)seq < (unsigned)a.n_seqs;
    tab = a.tables + (known ? (size_t)seq * a.table_len : 0);
    last = a.table_len - 1;
    const int ctx = known ? min(a.row_ctx[row], a.max_ctx) : 0;
    k1 = min(ctx, k0 + split);
    slot = ctx > split ? item : -1;
  }
  const int t0 = (k0 >> 6) + w, b0 = k0 >> 4;
  // Block ids lie in LDS, those of the first tile beside them in registers: an address
  // then never waits for a global load, which (vector loads complete in order) would
  // wait for every tile in flight too; and no id waits for the context's length.
  auto id_of = [&](int b) { return min((unsigned)tab[min(b, last)], (unsigned)a.num_blocks - 1u); };
  const unsigned kid = id_of(4 * t0 + (col >> 2)), vid = id_of(4 * t0 + quad);
  for (int i = threadIdx.x; i < split / kBlock; i += 256) sid[i] = id_of(b0 + i);
  if (!ITEMS && k0 >= k1) {
    if (k0 > 0) return;
    for (int i = threadIdx.x; i < gq * HD; i += 256) {       // a row without keys
      const size_t o = ((size_t)row * a.n_h + kvh * gq) * HD + i;
      if (a.out_type == OUT_F32) ((float*)a.out)[o] = 0.f;
      else ((uint16_t*)a.out)[o] = 0;
    }
    return;
  }
  const unsigned char* pool = (const unsigned char*)a.kv + ((size_t)a.layer * a.num_blocks * a.n_kv + kvh) * CELL;
  const size_t stride = (size_t)a.n_kv * CELL;
  // A tile's keys (and scales) and values are reloaded for the next tile as soon as they are
  // used: keys while the softmax and P V run, values while the next scores do.
  unsigned kw[4][W], ks, vs;
  u32x4 vw[W];
  auto load_k = [&](unsigned kb, unsigned vb) {
    const unsigned char* kp = pool + kb * stride + (lane & 3) * (HD / 2) + quad * (HD / 8);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      if constexpr (W == 4) {
        const u32x4 y = __builtin_nontemporal_load((const u32x4*)(kp + n * 2 * HD));
#pragma unroll
        for (int j = 0; j < 4; ++j) kw[n][j] = y[j];
      } else {
        const u32x2_t y = __builtin_nontemporal_load((const u32x2_t*)(kp + n * 2 * HD));
        kw[n][0] = y[0]; kw[n][1] = y[1];
      }
    }
    // this lane's key: slot col of block quad
    const unsigned* sp = (const unsigned*)(pool + vb * stride + 16 * HD) + col;
    ks = __builtin_nontemporal_load(sp);
    vs = __builtin_nontemporal_load(sp + 16);
  };
  auto load_v = [&](unsigned vb) {
    const unsigned char* vp = pool + vb * stride + 8 * HD + col * 16;
#pragma unroll
    for (int i = 0; i < W; ++i) vw[i] = __builtin_nontemporal_load((const u32x4*)(vp + i * 256));
  };
  load_k(kid, vid);
  load_v(vid);

  // B operand of the scores, made once by all threads: lane (col, quad) of step j holds head
  // col % 8's part col / 8 of dims 8 (W quad + j) .. + 8, in the order of the codes.
  {
    constexpr int TH = HD / 4;                     // threads a head: four dims each
    const int h = threadIdx.x / TH, d = (threadIdx.x % TH) * 4;
    if (h < 8) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      if (h < gq) load_run<4>(a.q, (size_t)row * a.q_stride + (size_t)(kvh * gq + h) * HD + d, a.q_bf16, q_vec, v);
      float mx = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
      mx = max16(mx);
      if constexpr (TH == 32) mx = fmaxf(mx, swz_xor16(mx));
      float up, f;
      q_units(mx, a.scale, up, f);
      float sum = 0.f;
      uint16_t* hi = (uint16_t*)sq[(d >> 3) % W][17 * ((d >> 3) / W) + h] + ((d >> 2) & 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = v[i] * up;
        const _Float16 g = (_Float16)x, r = FINE ? (_Float16)(x - (float)g) : (_Float16)0;
        sum += (float)g + (float)r;
        // codes of K that are not shifted stand at bits 4 to 7, 16 times as large
        hi[2 * i] = __builtin_bit_cast(uint16_t, !FINE && (i & 1) ? (_Float16)(g * (_Float16)0.0625f) : g);
        hi[2 * i + 64] = __builtin_bit_cast(uint16_t, r);
      }
      sum = sum16(sum);
      if constexpr (TH == 32) sum += swz_xor16(sum);
      if (threadIdx.x % TH == 0) {
        sqf[0][h] = sum;
        sqf[1][h] = f;
      }
    }
  }
  __syncthreads();
  u32x4 qf[W];
#pragma unroll
  for (int j = 0; j < W; ++j) qf[j] = *(const u32x4*)sq[j][lane + quad];
  const float Q = sqf[0][col & 7], f = sqf[1][col & 7];  // sum of the head's q; a score's unit in powers of two
  const unsigned part2 = col >= 8 ? 0xffffffffu : 0u;

  f32x4_t acc[2 * W];
#pragma unroll
  for (int i = 0; i < 2 * W; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float M = -INFINITY, l = 0.f, mv = 0.f;
  for (int t = t0; t * 64 < k1; t += 4) {
    const int nb = min(4 * (t + 4) - b0, split / kBlock - 4);      // past the split: any tile
    if (64 * t + lane >= k1) ks = vs = 0;          // whatever lies behind the last key
    *(float2*)&ssc[w][0][quad][2 * col] = make_float2(__uint_as_float(ks << 16) * (FINE ? 0x1p20f : 0x1p24f), __uint_as_float(ks & 0xffff0000u));
    *(float2*)&ssc[w][1][quad][2 * col] = make_float2(__uint_as_float(vs << 16), fmaf(__uint_as_float(vs << 16), FINE ? 8.f : 0.f, __uint_as_float(vs & 0xffff0000u)));
    wave_lds_fence();

    f32x4_t d[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      d[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < W; ++j)
        d[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, FINE ? codes_f16(kw[n][j]) : codes_mixed(kw[n][j])),
                                                   __builtin_bit_cast(f16x8_t, qf[j]), d[n], 0, 0, 0);
    }
    load_k(sid[nb + (col >> 2)], sid[nb + quad]);
    float s[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float2 sm = *(const float2*)&ssc[w][0][quad][2 * e];
      // without a lo part, columns past 7 are not used
      const float x = FINE ? d[e >> 2][e & 3] + dpp<0x128>(d[e >> 2][e & 3]) : d[e >> 2][e & 3];
      s[e] = fmaf(sm.x, x, sm.y * Q);
    }
    if (64 * t + 64 > k1) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (64 * t + 16 * quad + e >= k1) s[e] = -INFINITY;
    }
    float pv[16], ts, tm, pm;
    auto probabilities = [&] {
      ts = tm = pm = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[e], f, -M));
        const float2 sm = *(const float2*)&ssc[w][1][quad][2 * e];
        pv[e] = p * sm.x;
        ts += p;
        tm = fmaf(p, sm.y, tm);
        pm = fmaxf(pm, pv[e]);
      }
    };
    const bool first = __any(M == -INFINITY);
    if (!first) probabilities();
    if (first || !__all(pm <= 8192.f && ts < INFINITY)) {
      float u = -INFINITY, big = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        u = fmaxf(u, s[e]);
        big = fmaxf(big, ssc[w][1][quad][2 * e]);
      }
      u = fmaf(max_column(u), f, fmaxf(__builtin_amdgcn_logf(max_column(big)), -90.f));
      u = fmaxf(u - 8.f, M);
      const float alpha = __builtin_amdgcn_exp2f(M - u);
      M = u;
      l *= alpha;
      mv *= alpha;
#pragma unroll
      for (int i = 0; i < 2 * W; ++i) acc[i] *= alpha;
      probabilities();
    }
    l += ts;
    mv += tm;
    // P^T: k-slots 0 to 7 of step h are slots 8 h + 0 2 1 3 4 6 5 7 of block quad
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 pf;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 8 * h + 4 * (i >> 1) + (i & 1);
        if constexpr (FINE) {
          const f16x2_t hi = __builtin_bit_cast(f16x2_t, pack_f16(pv[e], pv[e + 2]) & part2);
          pf[i] = pack_f16(pv[e] - (float)hi[0], pv[e + 2] - (float)hi[1]);
        } else {
          pf[i] = pack_f16(pv[e], pv[e + 2]) & ~part2;
        }
      }
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const unsigned x = vw[i][2 * h], y = vw[i][2 * h + 1];
        u32x4 lo, hi;
        if constexpr (FINE) {
          lo = u32x4{centred(x << 6), centred(x >> 2), centred(y << 6), centred(y >> 2)};
          hi = u32x4{centred(x << 2), centred(x >> 6), centred(y << 2), centred(y >> 6)};
        } else {
          lo = u32x4{(x << 4) & kCodeMask, (x >> 4) & kCodeMask, (y << 4) & kCodeMask, (y >> 4) & kCodeMask};
          hi = u32x4{x & kCodeMask, (x >> 8) & kCodeMask, y & kCodeMask, (y >> 8) & kCodeMask};
        }
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, lo), __builtin_bit_cast(f16x8_t, pf), acc[i], 0, 0, 0);
        acc[W + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, hi), __builtin_bit_cast(f16x8_t, pf), acc[W + i], 0, 0, 0);
      }
    }
    load_v(sid[nb + quad]);
    wave_lds_fence();
  }

  // join the lanes of a head, then the waves
  l = sum_column(l);
  mv = sum_column(mv);
  if (quad == 0 && col < 8) { sml[w][0][col] = M; sml[w][1][col] = l; }
#pragma unroll
  for (int i = 0; i < 2 * W; ++i) {
    f32x4_t o;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = fmaf(acc[i][k] + dpp<0x128>(acc[i][k]), FINE ? 1.f : 0x1p20f, mv);
    if (col < gq) *(f32x4_t*)&so[w][col][16 * i + 4 * quad] = o;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < gq * HD; i += 256) {
    const int h = i / HD, d = i % HD;
    float Mt = sml[0][0][h];
#pragma unroll
    for (int k = 1; k < 4; ++k) Mt = fmaxf(Mt, sml[k][0][h]);
    float lt = 0.f, ot = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float x = __builtin_amdgcn_exp2f(sml[k][0][h] - Mt);       // a wave without keys: 0
      lt = fmaf(sml[k][1][h], x, lt);
      ot = fmaf(so[k][h][d], x, ot);
    }
    const int head = kvh * gq + h;
    if (slot >= 0) {
      const size_t o = (size_t)slot * a.n_h + head;
      part.acc[o * HD + d] = ot;
      if (d == 0) { part.ml[2 * o] = Mt; part.ml[2 * o + 1] = lt; }
    } else {
      const size_t o = ((size_t)row * a.n_h + head) * HD + d;
      const float r = ot / lt;
      if (a.out_type == OUT_F32) ((float*)a.out)[o] = r;
      else if (a.out_type == OUT_BF16) ((uint16_t*)a.out)[o] = f2bf(r);
      else store_split((uint16_t*)a.out, a.out_lo, o, r);
    }
  }
}

// The join of a row's splits, in their order: a workgroup a row and KV head, four dims a thread.
template <int HD>
__global__ __launch_bounds__(256) void k_attend4_join(Attend4Args a, int split, Partial4 part) {
  const int row = blockIdx.x, gq = a.n_h / a.n_kv;
  const int seq = a.row_seq[row];
  const int ctx = (unsigned)seq < (unsigned)a.n_seqs ? min(a.row_ctx[row], a.max_ctx) : 0;
  const int h = blockIdx.y * gq + threadIdx.x / (HD / 4), d = threadIdx.x % (HD / 4) * 4;
  if (ctx <= split || threadIdx.x >= gq * (HD / 4)) return;
  const int n = (ctx + split - 1) / split;
  float M = -INFINITY, l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const size_t b = ((size_t)s * a.T + row) * a.n_h + h;
    const float2 ml = *(const float2*)(part.ml + 2 * b);
    const f32x4_t as = *(const f32x4_t*)(part.acc + b * HD + d);
    const float mn = fmaxf(M, ml.x), x = __builtin_amdgcn_exp2f(M - mn), y = __builtin_amdgcn_exp2f(ml.x - mn);
    l = l * x + ml.y * y;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = o[k] * x + as[k] * y;
    M = mn;
  }
  const size_t at = ((size_t)row * a.n_h + h) * HD + d;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] /= l;
  if (a.out_type == OUT_F32) *(f32x4_t*)((float*)a.out + at) = o;
  else *(uint2*)((uint16_t*)a.out + at) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
}

// ------------------------- causal chunk attention over 4-bit cells (32x32x16 MFMA)
// One workgroup is 128 queries of one chunk and KV head: 128 / gq positions of its gq query
// heads, side by side, so short chunks fill the tile too; a wave has 32 of them.
// Tiles of 64 keys are unpacked once for the four waves: each thread brings 16 bytes of K
// codes and 16 of V, a tile ahead of its unpacking and two ahead of their use, and
// writes them as float16 codes (as in k_attend4_rows) to LDS in the order of the MFMA
// operands, where V's [dim][slot] cells need no transposing. Two LDS buffers each. S^T = K Q^T:
// row 8 a + 4 h + i of a 32-key score tile is block a / 2, slot 8 h + 4 (a % 2) + i, so lane half h ends with
// slots 8 h .. + 8 of both blocks, the k-slots of O^T = V^T P^T. Scales, minima, the reference M and float16 pairs as in k_attend4_rows;
// in bf16 calls q is one exact float16 and P one float16, half the products.
// Bound by the matrix cores and the VALU in turn. Float32, 32 heads of 128 over 8 KV heads, two chunks of
// 1,501 to 4,096 rows behind 1,001 to 8,000 keys: 817 us, 508 TFLOP/s of useful products (twice that issued);
// bf16, heads of 64, 24 prompts of 64 to 3,001 rows: 254 to 274 us, 420 to 450 TFLOP/s. Before a subtile's softmax ran
// beside the next one's products: 873 and 369 us.
struct Chunk { int row0, nq, pos0; const int* tab; };

// The block of 128 / gq rows that workgroup slot b stands for: chunk i has the slots
// start_i / PB + i and on, which never meet the next chunk's. nq = 0: none.
__device__ __forceinline__ Chunk find_chunk(const Attend4Args& a, int b, int PB) {
  int n = 0;
  for (int i0 = 0; i0 < a.n_seqs; i0 += 256) {
    const int i = i0 + threadIdx.x;
    n += __syncthreads_count(i < a.n_seqs && a.chunk_start[min(i, a.n_seqs)] / PB + i <= b);
  }
  Chunk c{0, 0, 0, nullptr};
  const int i = n - 1;
  if (i < 0) return c;
  const int s0 = max(a.chunk_start[i], 0), s1 = min(a.chunk_start[i + 1], a.T);
  const int r0 = s0 + (b - (s0 / PB + i)) * PB;
  c.row0 = r0;
  c.nq = r0 < s0 ? 0 : max(min(PB, s1 - r0), 0);   // r0 < s0: the starts do not ascend
  c.pos0 = min(a.chunk_ctx[i], a.max_ctx) - (s1 - r0);
  c.tab = a.tables + (size_t)i * a.table_len;
  return c;
}

__device__ __forceinline__ void store_out4(const Attend4Args& a, size_t at, f32x4_t o) {
  if (a.out_type == OUT_F32) {
    *(f32x4_t*)((float*)a.out + at) = o;
  } else if (a.out_type == OUT_BF16) {
    *(uint2*)((uint16_t*)a.out + at) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
  } else {
    unsigned h0, h1, l0, l1;
    split_pair(o[0], o[1], h0, l0);
    split_pair(o[2], o[3], h1, l1);
    *(uint2*)((uint16_t*)a.out + at) = make_uint2(h0, h1);
    *(uint2*)((uint16_t*)a.out + a.out_lo + at) = make_uint2(l0, l1);
  }
}

// Waves a SIMD: three of bf16 calls at heads of 64 (305 -> 274 us for the burst above); float32 ones spill
// (560 -> 630 us for two long chunks), and 128 dims need the registers of two.
constexpr int chunks4_waves(int hd, bool fine) { return hd == 64 && !fine ? 3 : 2; }

template <int HD, bool ITEMS, bool FINE>
__global__ __launch_bounds__(256, chunks4_waves(HD, FINE)) void k_attend4_chunks(Attend4Args a, const PrefillItem* __restrict__ items, int nslots,
                                                           int split, Partial4 part, bool q_vec) {
  constexpr int CELL = (int)kv_cell_bytes(KV_INT4, HD);
  constexpr int DS = HD / 16, DT = HD / 32;        // 16-dim steps of the scores, 32-dim tiles of the answer
  constexpr int W = HD / 32;                       // words of a key's row per wave
  constexpr int KB = 64 * HD * 2;                  // bytes of a tile's K (and V) as float16
  extern __shared__ __align__(1024) unsigned char lds[];
  float* ssc = (float*)(lds + 4 * KB);             // (s, m) of 64 keys, K then V: three buffers, filled two tiles ahead
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hf = lane >> 5, gq = a.n_h / a.n_kv, kvh = blockIdx.x % a.n_kv;
  const int item = blockIdx.x / a.n_kv, PB = 128 / gq;
  const int sp = item / nslots, b = nslots - 1 - (item - sp * nslots);    // late positions, long ones, first
  Chunk c;
  if constexpr (ITEMS) {
    const PrefillItem it = items[b];
    c = Chunk{it.row0, it.nq, it.pos0, a.tables + it.bt_off};
  } else {
    c = find_chunk(a, b, PB);
  }
  if (c.nq == 0) return;
  const int kmax = c.pos0 + c.nq;                  // keys [0, kmax)
  const int k0 = sp * split, k1 = min(kmax, k0 + split);
  // this lane's query (those past nq repeat the last row's and are never stored)
  const int slot = min(32 * w + c32, c.nq * gq - 1), r = slot / gq, h = kvh * gq + slot - r * gq;
  const bool mine = 32 * w + c32 < c.nq * gq;
  const int qpos = c.pos0 + r;
  const size_t orow = (size_t)(c.row0 + r) * a.n_h + h;
  const size_t prow = ((size_t)sp * a.T + c.row0 + r) * a.n_h + h;
  if (k0 >= k1) {                                  // no key of this split, or none at all
    if (part.ml) {
      if (mine && hf == 0) *(float2*)(part.ml + 2 * prow) = make_float2(-INFINITY, 0.f);
    } else if (mine) {
      for (int d = 4 * hf; d < HD; d += 8) store_out4(a, orow * HD + d, f32x4_t{0.f, 0.f, 0.f, 0.f});
    }
    return;
  }
  const unsigned char* pool = (const unsigned char*)a.kv + ((size_t)a.layer * a.num_blocks * a.n_kv + kvh) * CELL;
  const size_t stride = (size_t)a.n_kv * CELL;
  const int last = (kmax - 1) >> 4;
  auto id_of = [&](int x) { return min((unsigned)c.tab[min(x, last)], (unsigned)a.num_blocks - 1u); };

  // staging: thread (w, lane) brings words W w .. of key `lane`'s row, and the 16 slots of dim `lane` (and
  // + HD / 2) of block w; threads below 128 one scale word (K of keys 0 .. 63, then V)
  const int vb = HD == 128 ? w : threadIdx.x >> 5, vd = HD == 128 ? lane : lane & 31;
  const bool has_v = HD == 128 || w < 2;
  unsigned kid, vid, kw[W], ks;
  u32x4 vw;
  // row of the score tile that key `lane` takes
  const int krow = 8 * (2 * ((lane >> 4) & 1) + ((lane >> 2) & 1)) + 4 * ((lane >> 3) & 1) + (lane & 3);
  auto load_k = [&](int t) {                       // the ids that it needs came a tile before
    const unsigned char* cell = pool + kid * stride;
    if constexpr (W == 4) {
      const u32x4 x = *(const u32x4*)(cell + (lane & 15) * (HD / 2) + w * 16);
      kw[0] = x[0]; kw[1] = x[1]; kw[2] = x[2]; kw[3] = x[3];
    } else {
      const u32x2_t x = *(const u32x2_t*)(cell + (lane & 15) * (HD / 2) + w * 8);
      kw[0] = x[0]; kw[1] = x[1];
    }
    // scale words of key `lane`: K's by wave 0, V's (of the same tile) by wave 1
    if (w < 2) {
      ks = *(const unsigned*)(cell + 16 * HD + 64 * w + 4 * (lane & 15));
      if (64 * t + lane >= kmax) ks = 0;           // whatever lies behind the last key
    }
    kid = id_of(4 * (t + 1) + (lane >> 4));
  };
  auto load_v = [&](int t) {
    if (has_v) vw = *(const u32x4*)(pool + vid * stride + 8 * HD + vd * 16);
    vid = id_of(4 * (t + 1) + min(vb, 3));
  };
  auto unpack_k = [&](int t) __attribute__((always_inline)) {
    unsigned char* kb = lds + (t & 1) * KB + (((lane >> 5) * DS + (W * w >> 1)) * 64 + krow) * 16;
#pragma unroll
    for (int j = 0; j < W; ++j)                    // word W w + j: half j % 2 of step (W w + j) / 2
      *(u32x4*)(kb + (j >> 1) * 1024 + (j & 1) * 512) = codes_f16(kw[j]);
    if (w < 2) {
      const float s = __uint_as_float(ks << 16), m = __uint_as_float(ks & 0xffff0000u);
      *(float2*)&ssc[((t % 3 * 2 + w) * 64 + lane) * 2] = w == 0 ? make_float2(s * 0x1p20f, m) : make_float2(s, FINE && s == s ? fmaf(s, 8.f, m) : m);
    }
  };
  auto unpack_v = [&](int t) __attribute__((always_inline)) {
    unsigned char* f = lds + 2 * KB + (t & 1) * KB + ((vb * DT + (vd >> 5)) * 64 + (vd & 31)) * 16;
    if (has_v) {
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        const unsigned x = vw[2 * o], y = vw[2 * o + 1];
        u32x4 lo, hi;
        if constexpr (FINE) {
          lo = u32x4{centred(x << 6), centred(x >> 2), centred(y << 6), centred(y >> 2)};
          hi = u32x4{centred(x << 2), centred(x >> 6), centred(y << 2), centred(y >> 6)};
        } else {
          lo = u32x4{(x << 4) & kCodeMask, (x >> 4) & kCodeMask, (y << 4) & kCodeMask, (y >> 4) & kCodeMask};
          hi = u32x4{x & kCodeMask, (x >> 8) & kCodeMask, y & kCodeMask, (y >> 8) & kCodeMask};
        }
        *(u32x4*)(f + o * 512) = lo;
        *(u32x4*)(f + o * 512 + DT / 2 * 1024) = hi;
      }
    }
  };
  const int ta = k0 >> 6, tb = (k1 + 63) >> 6;     // tiles
  kid = id_of(4 * ta + (lane >> 4));
  vid = id_of(4 * ta + min(vb, 3));
  load_k(ta);
  load_v(ta);

  // B operand of the scores: query `slot`, dims 16 s + 8 hf .. + 8 in the order of codes_f16
  u32x4 qh[DS], ql[FINE ? DS : 1];
  float Q, f;
  {
    float v[DS][8], mx = 0.f;
    const size_t qo = (size_t)(c.row0 + r) * a.q_stride + (size_t)h * HD + 8 * hf;
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      load_run<8>(a.q, qo + 16 * s, a.q_bf16, q_vec, v[s]);
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(v[s][i]));
    }
    mx = max_halves(mx);
    float up;
    q_units(mx, a.scale, up, f);
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < DS; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = v[s][i] * up, y = v[s][i + 4] * up;
        qh[s][i] = pack_f16(x, y);
        const f16x2_t g = __builtin_bit_cast(f16x2_t, (unsigned)qh[s][i]);
        sum += (float)g[0] + (float)g[1];
        if constexpr (FINE) {
          ql[s][i] = pack_f16(x - (float)g[0], y - (float)g[1]);
          const f16x2_t k = __builtin_bit_cast(f16x2_t, (unsigned)ql[s][i]);
          sum += (float)k[0] + (float)k[1];
        }
      }
    Q = add_halves(sum);
  }

  f32x16_t O[DT], S, N;                            // the answer, a subtile's scores, the next one's products
#pragma unroll
  for (int d = 0; d < DT; ++d) O[d] = f32x16_t{};
  float M = -INFINITY, l = 0.f, mv = 0.f;
  const int first_pos = c.pos0 + min(32 * w, c.nq * gq - 1) / gq;
  auto product = [&](const unsigned char* kf, int s) __attribute__((always_inline)) {
    const f16x8_t x = __builtin_bit_cast(f16x8_t, *(const u32x4*)(kf + (s * 64 + lane) * 16));
    N = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, __builtin_bit_cast(f16x8_t, qh[s]), s ? N : f32x16_t{}, 0, 0, 0);
    if constexpr (FINE) N = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, __builtin_bit_cast(f16x8_t, ql[s]), N, 0, 0, 0);
  };
  // Subtile k of tile t: its softmax beside the products of the next subtile (at kf), a
  // share of each at a time, so that one wave keeps both the matrix cores and the VALU; then P V.
  auto stage = [&](int t, int k, const unsigned char* kf) __attribute__((always_inline)) {
    // element e: key 64 t + 32 k + 16 (e / 8) + 8 hf + e % 8
    const float* kc = ssc + (t % 3 * 128 + 32 * k + 8 * hf) * 2;
    const float* vc = kc + 128;
    const bool masked = 64 * t + 32 * k + 31 > first_pos;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float2 sm = *(const float2*)(kc + (16 * (e >> 3) + (e & 7)) * 2);
      S[e] = fmaf(sm.x, S[e], sm.y * Q);
    }
    if (masked) {
      const int see = qpos - (64 * t + 32 * k + 8 * hf);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (16 * (e >> 3) + (e & 7) > see) S[e] = -INFINITY;
    }
    float pv[16], ts = 0.f, tm = 0.f, pm = 0.f;
    auto probability = [&](int e, float base) __attribute__((always_inline)) {
      const float p = __builtin_amdgcn_exp2f(fmaf(S[e], f, -base));
      const float2 sm = *(const float2*)(vc + (16 * (e >> 3) + (e & 7)) * 2);
      pv[e] = p * sm.x;
      ts += p;
      tm = fmaf(p, sm.y, tm);
      pm = fmaxf(pm, pv[e]);
    };
    const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      product(kf, s);
#pragma unroll
      for (int e = 16 * s / DS; e < 16 * (s + 1) / DS; ++e) probability(e, base);
      __builtin_amdgcn_sched_barrier(0);
    }
    // a query's reference moves at the first keys that it meets, or past 2^13: by its own scores alone,
    // so that its bits do not hang on the rows beside it
    const int fine = __all(pm <= 8192.f && ts < INFINITY) & !__any(M == -INFINITY);
    if (!fine) {
      float u = -INFINITY, big = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        u = fmaxf(u, S[e]);
        big = fmaxf(big, S[e] == -INFINITY ? 0.f : vc[(16 * (e >> 3) + (e & 7)) * 2]);   // of the keys that it sees
      }
      u = fmaf(max_halves(u), f, fmaxf(__builtin_amdgcn_logf(max_halves(big)), -90.f));
      const bool stays = max_halves(pm) <= 8192.f && add_halves(ts) < INFINITY && M != -INFINITY;
      u = stays ? M : fmaxf(u - 4.f, M);               // 2^9 from there to the next move, 2^-28 of the largest p s kept
      const float alpha = M == u ? 1.f : __builtin_amdgcn_exp2f(M - u);
      M = u;
      l *= alpha;
      mv *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d) O[d] *= alpha;
      ts = tm = pm = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) probability(e, M == -INFINITY ? 0.f : M);
    }
    if (masked) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (S[e] == -INFINITY) pv[e] = 0.f;        // also where the unseen row stands for NaN
    }
    l += ts;
    mv += tm;
    const unsigned char* vf = lds + 2 * KB + (t & 1) * KB + 2 * k * DT * 1024 + lane * 16;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 ph, pl;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 8 * u + 4 * (i >> 1) + (i & 1);
        ph[i] = pack_f16(pv[e], pv[e + 2]);
        if constexpr (FINE) {
          const f16x2_t g = __builtin_bit_cast(f16x2_t, (unsigned)ph[i]);
          pl[i] = pack_f16(pv[e] - (float)g[0], pv[e + 2] - (float)g[1]);
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f16x8_t x = __builtin_bit_cast(f16x8_t, *(const u32x4*)(vf + (u * DT + d) * 1024));
        O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, __builtin_bit_cast(f16x8_t, ph), O[d], 0, 0, 0);
        if constexpr (FINE) O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, __builtin_bit_cast(f16x8_t, pl), O[d], 0, 0, 0);
      }
    }
    S = N;
  };
  unpack_k(ta);
  unpack_v(ta);
  load_k(ta + 1);
  unpack_k(ta + 1);
  load_k(ta + 2);
  load_v(ta + 1);
  __syncthreads();
#pragma unroll
  for (int s = 0; s < DS; ++s) product(lds + (ta & 1) * KB, s);
  S = N;
  for (int t = ta; t < tb; ++t) {
    stage(t, 0, lds + (t & 1) * KB + DS * 1024);
    __syncthreads();                               // K of tile t has been read
    unpack_k(t + 2);
    load_k(t + 3);
    unpack_v(t + 1);
    load_v(t + 2);
    stage(t, 1, lds + ((t + 1) & 1) * KB);       // (behind the last tile: finite codes, never used)
    __syncthreads();
  }

  l = add_halves(l);
  mv = add_halves(mv);
  if (!mine) return;
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;       // a query at a negative position: 0
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      f32x4_t o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = fmaf(O[d][e + i], FINE ? 1.f : 0x1p20f, mv);
      const int dim = 32 * d + 2 * e + 4 * hf;
      if (part.ml) {
        *(f32x4_t*)(part.acc + prow * HD + dim) = o;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= inv;
        store_out4(a, orow * HD + dim, o);
      }
    }
  if (part.ml && hf == 0) *(float2*)(part.ml + 2 * prow) = make_float2(M, l);
}

// The join of a chunk's splits, in their order: hd / 4 threads a row and head, workgroups of 1,024 / hd of
// a block's 128 (all of them in one workgroup took 16 rows one after the other, each a chain of loads).
template <int HD>
__global__ __launch_bounds__(256) void k_attend4_chunks_join(Attend4Args a, int nsplit, Partial4 part) {
  const int gq = a.n_h / a.n_kv, PB = 128 / gq;
  const Chunk c = find_chunk(a, blockIdx.x, PB);
  constexpr int TR = HD / 4;
  const int i = blockIdx.z * (256 / TR) + threadIdx.x / TR, d = threadIdx.x % TR * 4;
  if (i >= c.nq * gq) return;
  const size_t row = (size_t)(c.row0 + i / gq) * a.n_h + blockIdx.y * gq + i % gq;
  float M = -INFINITY, l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < nsplit; ++s) {
    const size_t b = (size_t)s * a.T * a.n_h + row;
    const float2 ml = *(const float2*)(part.ml + 2 * b);
    const f32x4_t as = *(const f32x4_t*)(part.acc + b * HD + d);
    const bool some = ml.x != -INFINITY;               // else nothing was seen in this split, and nothing written
    const float mn = fmaxf(M, ml.x), x = M == mn ? 1.f : __builtin_amdgcn_exp2f(M - mn);
    const float y = some ? __builtin_amdgcn_exp2f(ml.x - mn) : 0.f;
    l = l * x + (some ? ml.y * y : 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = o[k] * x + (some ? as[k] * y : 0.f);
    M = mn;
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] *= inv;
  store_out4(a, row * HD + d, o);
}

// =============================================================== launchers

constexpr long long kMaxGrid = (1ll << 24) - 1;    // workgroups of 256 in a grid: its threads are counted in 32 bits

hipError_t launch_kv_append(hipStream_t st, bool x_bf16, int kind, const AppendArgs& args) {
  if (args.T <= 0) return hipSuccess;
  AppendArgs a = args;
  a.gain_vec = true;
  for (int i = 0; i < kMaxModels; ++i)
    a.gain_vec = a.gain_vec && (uintptr_t)a.q_gain.p[i] % 16 == 0 && (uintptr_t)a.k_gain.p[i] % 16 == 0;
  const size_t el = x_bf16 ? 8 : 4;                  // elements per 16 bytes
  const bool aligned = a.stride % el == 0 && a.split_stride % el == 0 && (uintptr_t)a.x % 16 == 0;
  const int qw = 256 * append_q_vals(x_bf16) / a.hd, kw = 256 * append_kv_vals(x_bf16, kind) / a.hd;   // heads per workgroup
  const dim3 grid(a.T, (a.n_h + qw - 1) / qw + (2 * a.n_kv + kw - 1) / kw), blk(256);
  const bool norm = a.q_gain.p[0] != nullptr;
  auto go = [&](auto bf, auto hd, auto k) {
    constexpr bool B = decltype(bf)::value;
    constexpr int D = decltype(hd)::value, K = decltype(k)::value;
    if (norm) klaunch(k_kv_append<B, K, D, true>, grid, blk, st, a, aligned);
    else klaunch(k_kv_append<B, K, D, false>, grid, blk, st, a, aligned);
    return hipGetLastError();
  };
  auto by_kind = [&](auto bf, auto hd) {
    if (kind == KV_F32) return go(bf, hd, std::integral_constant<int, KV_F32>{});
    if (kind == KV_BF16) return go(bf, hd, std::integral_constant<int, KV_BF16>{});
    return go(bf, hd, std::integral_constant<int, KV_INT4>{});
  };
  auto by_hd = [&](auto bf) {
    return a.hd == 64 ? by_kind(bf, std::integral_constant<int, 64>{}) : by_kind(bf, std::integral_constant<int, 128>{});
  };
  if (a.hd != 64 && a.hd != 128) return hipErrorInvalidValue;
  return x_bf16 ? by_hd(std::true_type{}) : by_hd(std::false_type{});
}

hipError_t launch_kv_read(hipStream_t st, int kind, const void* kv, int layer, int n_kv, int hd, int T,
                          const int* row_pos, int pos0, const KvPlace& place, void* k, void* v) {
  if (T <= 0) return hipSuccess;
  if (hd != 64 && hd != 128) return hipErrorInvalidValue;
  const int heads = 2048 / hd;                       // per workgroup
  const dim3 grid(T, (n_kv + heads - 1) / heads), blk(256);
  auto go = [&](auto kern) { klaunch(kern, grid, blk, st, kv, layer, n_kv, T, row_pos, pos0, place, k, v); };
  if (kind == KV_F32) hd == 64 ? go(k_kv_read<KV_F32, 64>) : go(k_kv_read<KV_F32, 128>);
  else if (kind == KV_BF16) hd == 64 ? go(k_kv_read<KV_BF16, 64>) : go(k_kv_read<KV_BF16, 128>);
  else hd == 64 ? go(k_kv_read<KV_INT4, 64>) : go(k_kv_read<KV_INT4, 128>);
  return hipGetLastError();
}

// Keys per split: the longest of 2,048, 1,024 and 512 that gives every CU a workgroup. us at
// 8 KV heads of 128, splits of 512, 1,024, 2,048: 256 rows of 4,000 keys 271, 223, 196; 16 of
// 8,000 37.2, 32.5, 29.9; 16 of 2,000 14.0, 14.0, 15.9; 1 of 32,000 20.8, 17.4, 19.4; 1 of 4,000 10.9,
// 12.5, 18.2; 256 keys: 10.5 there, but 20.0 where 512 take 14.9 (4 of 8,000).
static int split4(int n_kv, int T, int max_ctx) {
  int s = kSplit4Max;
  while (s > 512 && (long long)T * n_kv * ((max_ctx + s - 1) / s) < 256) s /= 2;
  return s;
}
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

bool attend4_rows_fits(int n_kv, int T, int max_ctx) {
  const int s = split4(n_kv, T, max_ctx);
  return (long long)T * ((max_ctx + s - 1) / s) * n_kv <= kMaxGrid;
}

size_t attend4_rows_bytes(int n_h, int n_kv, int hd, int T, int max_ctx) {
  const int s = split4(n_kv, T, max_ctx), n = (max_ctx + s - 1) / s;
  const size_t slots = n > 1 ? (size_t)T * n : 0;
  return up256(slots * n_h * hd * 4) + slots * n_h * 8;
}

hipError_t launch_attend4_rows(hipStream_t st, const Attend4Args& a, void* workspace) {
  if (a.T <= 0) return hipSuccess;
  const int s = split4(a.n_kv, a.T, a.max_ctx), n = (a.max_ctx + s - 1) / s;
  if ((a.hd != 64 && a.hd != 128) || a.n_h / a.n_kv > 8 || (long long)a.T * n * a.n_kv > kMaxGrid) return hipErrorInvalidValue;
  Partial4 part{(float*)workspace, (float*)((char*)workspace + up256((size_t)a.T * n * a.n_h * a.hd * 4))};
  const dim3 grid((unsigned)(a.T * n * a.n_kv)), blk(256);
  const bool vec = a.q_stride % (a.q_bf16 ? 8 : 4) == 0 && (uintptr_t)a.q % 16 == 0;
  auto go = [&](auto kern) { klaunch(kern, grid, blk, st, a, (const AttnItem*)nullptr, s, part, vec); };
  if (a.hd == 64) a.q_bf16 ? go(k_attend4_rows<64, false, false>) : go(k_attend4_rows<64, false, true>);
  else a.q_bf16 ? go(k_attend4_rows<128, false, false>) : go(k_attend4_rows<128, false, true>);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || n == 1) return err;
  if (a.hd == 64) klaunch(k_attend4_join<64>, dim3(a.T, a.n_kv), blk, st, a, s, part);
  else klaunch(k_attend4_join<128>, dim3(a.T, a.n_kv), blk, st, a, s, part);
  return hipGetLastError();
}

// Workgroup slots and key splits of a chunk call: splits (of whole tiles, at least 256 keys)
// only where the blocks of rows make fewer workgroups than run at once, two or three a CU. us with a target of
// 256, 512, 1,024 (bf16, 8 KV heads of 128, 4 query heads each): 128 rows behind 32,000 keys 192, 136, 149; 512 behind
// 8,000 161, 119, 133; 2,048 behind 4,096 154, 154, 184; rows of 300, 40 and 900 behind 12,000 467, 445, 391. At
// least 256, 512, 1,024 keys: 17 rows behind 8,000 31, 35, 50; 128 55, 55, 67. Heads of 64, targets of 512 and
// 768: 128 rows behind 32,000 102, 91; 1,024 behind 16,000 278, 244; 2,048 behind 4,096 116, 120.
static void plan_chunks4(const Chunks4Size& z, bool bf16, int& nslots, int& split, int& nsplit) {
  nslots = z.T / (128 / (z.n_h / z.n_kv)) + z.n_chunks;
  const long long wgs = (long long)nslots * z.n_kv, target = 256 * chunks4_waves(z.hd, !bf16);
  nsplit = (int)std::max(1ll, std::min((target + wgs - 1) / wgs, (long long)z.max_ctx / 256));
  split = ((z.max_ctx + nsplit - 1) / nsplit + 63) / 64 * 64;
  nsplit = (z.max_ctx + split - 1) / split;
}

bool attend4_chunks_fits(const Chunks4Size& z) {
  int nslots, split, n;
  plan_chunks4(z, true, nslots, split, n);               // (the type with the most splits)
  return (long long)nslots * n * z.n_kv <= kMaxGrid;
}

size_t attend4_chunks_bytes(const Chunks4Size& z) {
  int nslots, split, n;
  plan_chunks4(z, true, nslots, split, n);
  return n > 1 ? up256((size_t)n * z.T * z.n_h * z.hd * 4) + (size_t)n * z.T * z.n_h * 8 : 0;
}

static unsigned chunks4_lds(int hd) { return 4u * 64u * (unsigned)hd * 2u + 3u * 1024u; }
static hipError_t chunks4_attributes() {
  static std::atomic<unsigned long long> done{0};    // devices whose instantiations have the attribute
  int dev = 0;
  const hipError_t err = hipGetDevice(&dev);
  if (err != hipSuccess) return err;
  const unsigned long long bit = 1ull << (dev & 63);
  if (done.load() & bit) return hipSuccess;
  for (const void* f : {(const void*)k_attend4_chunks<64, false, false>, (const void*)k_attend4_chunks<64, false, true>,
                        (const void*)k_attend4_chunks<64, true, true>, (const void*)k_attend4_chunks<128, false, false>,
                        (const void*)k_attend4_chunks<128, false, true>, (const void*)k_attend4_chunks<128, true, true>}) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)chunks4_lds(128));
    if (e != hipSuccess) return e;
  }
  done.fetch_or(bit);
  return hipSuccess;
}

hipError_t launch_attend4_chunks(hipStream_t st, const Attend4Args& a, void* workspace) {
  if (a.T <= 0) return hipSuccess;
  int nslots, split, n;
  plan_chunks4({a.n_h, a.n_kv, a.hd, a.T, a.n_seqs, a.max_ctx}, a.q_bf16, nslots, split, n);
  if ((a.hd != 64 && a.hd != 128) || a.n_h / a.n_kv > 8 || (long long)nslots * n * a.n_kv > kMaxGrid) return hipErrorInvalidValue;
  Partial4 part{nullptr, nullptr};
  if (n > 1) part = {(float*)workspace, (float*)((char*)workspace + up256((size_t)n * a.T * a.n_h * a.hd * 4))};
  const unsigned shm = chunks4_lds(a.hd);
  const bool vec = a.q_stride % (a.q_bf16 ? 8 : 4) == 0 && (uintptr_t)a.q % 16 == 0;
  const hipError_t attr = chunks4_attributes();
  if (attr != hipSuccess) return attr;
  const dim3 grid((unsigned)(nslots * n * a.n_kv)), blk(256);
  auto go = [&](auto kern) { klaunch_shm(kern, grid, blk, shm, st, a, (const PrefillItem*)nullptr, nslots, split, part, vec); };
  if (a.hd == 64) a.q_bf16 ? go(k_attend4_chunks<64, false, false>) : go(k_attend4_chunks<64, false, true>);
  else a.q_bf16 ? go(k_attend4_chunks<128, false, false>) : go(k_attend4_chunks<128, false, true>);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || n == 1) return err;
  if (a.hd == 64) klaunch(k_attend4_chunks_join<64>, dim3(nslots, a.n_kv, 8), blk, st, a, n, part);
  else klaunch(k_attend4_chunks_join<128>, dim3(nslots, a.n_kv, 16), blk, st, a, n, part);
  return hipGetLastError();
}

hipError_t launch_attend4_items(hipStream_t st, const Attend4Args& a, const AttnItem* items, int nitems, int split,
                                float* pacc, float* pml) {
  if (nitems <= 0) return hipSuccess;
  if ((a.hd != 64 && a.hd != 128) || a.n_h / a.n_kv > 8 || a.q_bf16 || split > kSplit4Max || (long long)nitems * a.n_kv > kMaxGrid)
    return hipErrorInvalidValue;
  const dim3 grid((unsigned)nitems * a.n_kv), blk(256);
  const Partial4 part{pacc, pml};
  if (a.hd == 64) klaunch(k_attend4_rows<64, true, true>, grid, blk, st, a, items, split, part, true);
  else klaunch(k_attend4_rows<128, true, true>, grid, blk, st, a, items, split, part, true);
  return hipGetLastError();
}

hipError_t launch_attend4_prefill(hipStream_t st, const Attend4Args& a, const PrefillItem* items, int nitems) {
  if (nitems <= 0) return hipSuccess;
  if ((a.hd != 64 && a.hd != 128) || a.n_h / a.n_kv > 8 || a.q_bf16 || (long long)nitems * a.n_kv > kMaxGrid)
    return hipErrorInvalidValue;
  const hipError_t e = chunks4_attributes();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)nitems * a.n_kv), blk(256);
  const Partial4 none{nullptr, nullptr};
  const int whole = 1 << 30;                         // keys per split: all
  if (a.hd == 64) klaunch_shm(k_attend4_chunks<64, true, true>, grid, blk, chunks4_lds(64), st, a, items, nitems, whole, none, true);
  else klaunch_shm(k_attend4_chunks<128, true, true>, grid, blk, chunks4_lds(128), st, a, items, nitems, whole, none, true);
  return hipGetLastError();
}

// Injected history into 4-bit cells: hd / 8 lanes a row, as for quantise(); values are rounded to
// bf16 first, as the bf16 cache would hold them.
template <int HD>
__global__ __launch_bounds__(256) void k_kv4_scatter(const uint16_t* __restrict__ src, void* __restrict__ kv,
                                                     const int* __restrict__ blocks, int p0, int layer, int kv_sel, int NB, int n_kv) {
  constexpr int LP = HD / 8;
  const int t = blockIdx.x, l = threadIdx.x % LP, h = blockIdx.y * (256 / LP) + threadIdx.x / LP, p = p0 + t;
  if (h >= n_kv) return;
  const uint16_t* s = src + ((size_t)t * n_kv + h) * HD + 4 * l;
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = bf2f(s[(i & 3) + (i >> 2) * (HD / 2)]);
  store_row<HD, KV_INT4, 8>(kv_cell(kv, KV_INT4, HD, layer, NB, blocks[p >> 4], n_kv, h), p & 15, kv_sel != 0, x, l);
}

// The values of k_kv_fill: a workgroup per (KV block, layer).
template <int HD>
__global__ __launch_bounds__(256) void k_kv4_fill(void* __restrict__ kv, const int* __restrict__ bt_store,
                                                  const FillReq* __restrict__ reqs, int nreqs, int NB, int n_kv) {
  constexpr int LP = HD / 8;
  const int item = blockIdx.x, layer = blockIdx.y, l = threadIdx.x % LP;
  int lo = 0, hi = nreqs - 1;                        // the last entry with item0 <= item
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (reqs[mid].item0 <= item) lo = mid;
    else hi = mid - 1;
  }
  const FillReq rq = reqs[lo];
  const int b = item - rq.item0, block = bt_store[rq.bt_off + b];
  const uint32_t tg = rq.tag * 0x9e3779b9u;
  for (int row = threadIdx.x / LP; row < n_kv * 2 * kBlock; row += 256 / LP) {
    const int head = row / (2 * kBlock), kv_sel = (row / kBlock) & 1, slot = row & (kBlock - 1), p = b * kBlock + slot;
    if (p >= rq.ctx) continue;
    const uint32_t hp = tg ^ mix32(((uint32_t)(layer * 2 + kv_sel) << 24) ^ (uint32_t)p);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int rem = head * HD + 4 * l + (i & 3) + (i >> 2) * (HD / 2);
      const uint32_t u = mix32(hp ^ (uint32_t)(rem * 0x85ebca6bu));
      x[i] = bf2f(f2bf((float)(int)(u >> 8) * (1.0f / 8388608.0f) - 1.0f));
    }
    store_row<HD, KV_INT4, 8>(kv_cell(kv, KV_INT4, HD, layer, NB, block, n_kv, head), slot, kv_sel != 0, x, l);
  }
}

hipError_t launch_kv4_scatter(hipStream_t st, const void* src, void* kv, const int* blocks, int p0, int n, int layer,
                              int kv_sel, int num_blocks, int n_kv, int hd) {
  if (n <= 0) return hipSuccess;
  if (hd != 64 && hd != 128) return hipErrorInvalidValue;
  const int heads = 2048 / hd;                       // per workgroup
  const dim3 grid(n, (n_kv + heads - 1) / heads), blk(256);
  if (hd == 64) klaunch(k_kv4_scatter<64>, grid, blk, st, (const uint16_t*)src, kv, blocks, p0, layer, kv_sel, num_blocks, n_kv);
  else klaunch(k_kv4_scatter<128>, grid, blk, st, (const uint16_t*)src, kv, blocks, p0, layer, kv_sel, num_blocks, n_kv);
  return hipGetLastError();
}

hipError_t launch_kv4_fill(hipStream_t st, void* kv, const int* bt_store, const FillReq* reqs, int nreqs, int nitems,
                           int n_layers, int num_blocks, int n_kv, int hd) {
  if (nitems <= 0) return hipSuccess;
  if (nreqs < 1 || (hd != 64 && hd != 128) || n_layers > 65535) return hipErrorInvalidValue;
  const dim3 grid(nitems, n_layers), blk(256);
  if (hd == 64) klaunch(k_kv4_fill<64>, grid, blk, st, kv, bt_store, reqs, nreqs, num_blocks, n_kv);
  else klaunch(k_kv4_fill<128>, grid, blk, st, kv, bt_store, reqs, nreqs, num_blocks, n_kv);
  return hipGetLastError();
}
