// Kernels around the paged cache for callers' own pools and for engines with
// 4-bit K/V or per-head norms: append, read-back, and attention over 4-bit
// cells. Part of kernels.hip (its helpers are above).

// The cell of (layer, block, KV head).
__device__ __forceinline__ unsigned char* kv_cell(const void* kv, int kind, int hd, int layer, int num_blocks, int block,
                                                  int n_kv, int head) {
  return (unsigned char*)kv + (((size_t)layer * num_blocks + block) * n_kv + head) * kv_cell_bytes(kind, hd);
}
// The block of a row's position, -1 if anything is out of range.
__device__ __forceinline__ int kv_block(const KvPlace& p, int row, int pos) {
  const int key = p.key[row];
  if ((unsigned)key >= (unsigned)p.n_keys || pos < 0 || (pos >> 4) >= p.table_len) return -1;
  const int b = p.tables[(size_t)key * p.mul + (pos >> 4)];
  return (unsigned)b < (unsigned)p.num_blocks ? b : -1;
}

// A cross-lane move of a double: its two words.
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
  const unsigned lo = (unsigned)__builtin_amdgcn_mov_dpp((int)(unsigned)u, CTRL, 0xF, 0xF, true);
  const unsigned hi = (unsigned)__builtin_amdgcn_mov_dpp((int)(unsigned)(u >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, ((unsigned long long)hi << 32) | lo);
}
// Combine over the LP lanes (8 or 16) that hold one row of a head; all get the result.
template <int LP, typename T, typename F>
__device__ __forceinline__ T over_row(T v, F f) {
  v = f(v, dpp<0xB1>(v));
  v = f(v, dpp<0x4E>(v));
  v = f(v, dpp<0x141>(v));
  if constexpr (LP == 16) v = f(v, dpp<0x128>(v));
  return v;
}

// One 4-bit row from LP = hd / 8 lanes, lane l holding dims 4 l .. 4 l + 3 and the
// same + hd / 2: its scale word and the lane's eight codes.
// The quotient is formed in 64 bits from the exact difference and rounded to 24
// before the rounding to a code, so a quotient that lies on the border of two codes
// (bf16 values often do) is a tie here too, and goes to the even code.
template <int LP>
__device__ __forceinline__ unsigned quantise(const float x[8], int c[8]) {
  float lo = x[0], hi = x[0];
  bool fine = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    fine = fine && fabsf(x[i]) < INFINITY;
  }
  lo = over_row<LP>(lo, [](float a, float b) { return fminf(a, b); });
  hi = over_row<LP>(hi, [](float a, float b) { return fmaxf(a, b); });
  const float ok = over_row<LP>(fine ? 1.f : 0.f, [](float a, float b) { return fminf(a, b); });
  uint16_t m = f2bf(lo), s = f2bf((hi - lo) / 15.f);
  if (ok == 0.f || !(hi - lo < INFINITY) || !(fabsf(bf2f(m)) < INFINITY)) { s = 0x7fc0; m = 0; }
  const float sf = bf2f(s);
  const double md = bf2f(m), inv = sf > 0.f ? 1.0 / (double)sf : 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = sf > 0.f ? (int)fminf(fmaxf(rintf((float)(((double)x[i] - md) * inv)), 0.f), 15.f) : 0;
  return (unsigned)s | ((unsigned)m << 16);
}

template <bool BF>
__device__ __forceinline__ float load_el(const void* p, size_t i) {
  return BF ? bf2f(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}

// Store a row held as for quantise() (lane l of LP) as K (v = false) or V of a cell's slot.
template <int HD, int KIND>
__device__ __forceinline__ void store_row(unsigned char* cell, int slot, bool v, const float x[8], int l) {
  if constexpr (KIND == KV_INT4) {
    int c[8];
    const unsigned sc = quantise<HD / 8>(x, c);
    if (v) {
      unsigned char* p = cell + 8 * HD + 4 * l * 16 + slot;
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i * 16] = (unsigned char)(c[i] | (c[i + 4] << 4));
    } else {
      uint16_t* p = (uint16_t*)(cell + slot * (HD / 2) + 2 * l);
      p[0] = (uint16_t)(c[0] | (c[1] << 4) | (c[2] << 8) | (c[3] << 12));
      p[HD / 8] = (uint16_t)(c[4] | (c[5] << 4) | (c[6] << 8) | (c[7] << 12));
    }
    if (l == 0) ((unsigned*)(cell + 16 * HD))[(v ? 16 : 0) + slot] = sc;
  } else if constexpr (KIND == KV_BF16) {
    uint16_t* p = (uint16_t*)cell + ((v ? kBlock : 0) + slot) * HD + 4 * l;
    *(uint2*)p = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    *(uint2*)(p + HD / 2) = make_uint2(pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  } else {
    float* p = (float*)cell + ((v ? kBlock : 0) + slot) * HD + 4 * l;
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + HD / 2) = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// ------------------------------ per-head norms, rotation and append in one pass
// hd / 8 lanes hold one head of one row, each both halves of four rotation pairs, so
// the norm's sum, the row's range and its codes stay within a row of 16 lanes.
// Keys of a 4-bit cache are computed in 64 bits: their codes are then
// those of the float32 value, whatever the order of the norm's sum (one bit of the
// float32 value can move the row's bf16 minimum, and with it every code).
template <bool XBF, int KIND, int HD, bool NORM>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a, bool aligned) {
  constexpr int LP = HD / 8;
  const int H = a.n_h + 2 * a.n_kv;
  const long long item = ((long long)blockIdx.x * 256 + threadIdx.x) / LP;
  const int l = threadIdx.x % LP;
  const bool live = item < (long long)a.T * H;     // lanes of a row agree; the others' results are dropped
  const int t = live ? (int)(item / H) : 0, head = live ? (int)(item % H) : 0;
  const int pos = a.row_pos[t];
  if (!live || pos < 0 || (a.rope && pos >= a.rope_len)) return;
  float x[8];
  const size_t at = (size_t)t * a.stride + (size_t)head * HD + 4 * l;
  if (XBF) {
    const uint16_t* p = (const uint16_t*)a.x + at;
    if (aligned) {
      const uint2 u = *(const uint2*)p, w = *(const uint2*)(p + HD / 2);
      x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
      x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
      x[4] = __uint_as_float(w.x << 16); x[5] = __uint_as_float(w.x & 0xffff0000u);
      x[6] = __uint_as_float(w.y << 16); x[7] = __uint_as_float(w.y & 0xffff0000u);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = bf2f(p[(i & 3) + (i >> 2) * (HD / 2)]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    for (int s = 0; s < a.nsplit; ++s) {
      const float* p = (const float*)a.x + (size_t)s * a.split_stride + at;
      if (aligned) {
        const float4 u = *(const float4*)p, w = *(const float4*)(p + HD / 2);
        x[0] += u.x; x[1] += u.y; x[2] += u.z; x[3] += u.w;
        x[4] += w.x; x[5] += w.y; x[6] += w.z; x[7] += w.w;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += p[(i & 3) + (i >> 2) * (HD / 2)];
      }
    }
  }
  const bool is_q = head < a.n_h, is_v = head >= a.n_h + a.n_kv;
  auto norm_rotate = [&](auto one) {
    using T = decltype(one);
    T y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (T)x[i];
    if constexpr (NORM) {
      const void* g = pick(is_q ? a.q_gain : a.k_gain, a.row_model ? a.row_model[t] : 0);
      T ss = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += y[i] * y[i];
      ss = over_row<LP>(ss, [](T u, T w) { return u + w; });
      const T mean = ss / (T)HD + (T)a.eps;
      const T inv = sizeof(T) == 8 ? (T)(1.0 / sqrt((double)mean)) : (T)rsqrtf((float)mean);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = 4 * l + (i & 3) + (i >> 2) * (HD / 2);
        y[i] *= inv * (T)(a.gain_bf16 ? load_el<true>(g, d) : load_el<false>(g, d));
      }
    }
    if (a.rope) {
      const float4* cs = (const float4*)(a.rope + (size_t)pos * (HD / 2) + 4 * l);
      const float4 c01 = cs[0], c23 = cs[1];
      const float c[8] = {c01.x, c01.y, c01.z, c01.w, c23.x, c23.y, c23.z, c23.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 8) {
          const T u = y[i], w = y[i + 4];
          y[i] = u * c[2 * i] - w * c[2 * i + 1];
          y[i + 4] = w * c[2 * i] + u * c[2 * i + 1];
        } else {
          const float2 r = rotate((float)y[i], (float)y[i + 4], make_float2(c[2 * i], c[2 * i + 1]));
          y[i] = r.x;
          y[i + 4] = r.y;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)y[i];
  };
  if (is_q) {
    norm_rotate(0.f);
    const size_t o = ((size_t)t * a.n_h + head) * HD + 4 * l;
    if (XBF) {
      *(uint2*)((uint16_t*)a.q + o) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
      *(uint2*)((uint16_t*)a.q + o + HD / 2) = make_uint2(pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    } else {
      *(float4*)((float*)a.q + o) = make_float4(x[0], x[1], x[2], x[3]);
      *(float4*)((float*)a.q + o + HD / 2) = make_float4(x[4], x[5], x[6], x[7]);
    }
    return;
  }
  if (!is_v) {
    if constexpr (KIND == KV_INT4) norm_rotate(0.0);
    else norm_rotate(0.f);
  }
  const int block = kv_block(a.place, t, pos);
  if (block < 0) return;
  const int kh = (head - a.n_h) % a.n_kv;
  store_row<HD, KIND>(kv_cell(a.kv, KIND, HD, a.layer, a.place.num_blocks, block, a.n_kv, kh), pos & 15, is_v, x, l);
}

// ------------------------------------------------- what cached positions hold
template <int KIND, int HD>
__global__ __launch_bounds__(256) void k_kv_read(const void* __restrict__ kv, int layer, int n_kv, int T,
                                                 const int* __restrict__ row_pos, KvPlace place, void* __restrict__ kout,
                                                 void* __restrict__ vout) {
  constexpr int LP = HD / 8;
  const long long item = ((long long)blockIdx.x * 256 + threadIdx.x) / LP;
  if (item >= (long long)T * n_kv) return;
  const int l = threadIdx.x % LP, t = (int)(item / n_kv), kh = (int)(item % n_kv);
  const int pos = row_pos[t], block = kv_block(place, t, pos), slot = pos & 15;
  const size_t o = (size_t)item * HD + 4 * l;
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
    void* out = v ? vout : kout;
    if constexpr (KIND == KV_F32) {
      *(float4*)((float*)out + o) = make_float4(x[0], x[1], x[2], x[3]);
      *(float4*)((float*)out + o + HD / 2) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
      *(uint2*)((uint16_t*)out + o) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
      *(uint2*)((uint16_t*)out + o + HD / 2) = make_uint2(pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
  }
}

// ------------------------------------------- attention over 4-bit cells, one wave
// a row and query head: key after key, lane l holding dims l (and l + 64).
template <int HD>
__global__ __launch_bounds__(64) void k_attend4(Attend4Args a) {
  constexpr int N = HD / 64;
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  int seq, ctx;
  if (a.chunk_start) {
    seq = -1;
    for (int i = 0; i < a.n_seqs; ++i)
      if (t >= a.chunk_start[i] && t < a.chunk_start[i + 1]) seq = i;
    if (seq < 0) return;
    ctx = min(a.chunk_ctx[seq], a.max_ctx) - (a.chunk_start[seq + 1] - 1 - t);
  } else {
    seq = a.row_seq[t];
    ctx = (unsigned)seq < (unsigned)a.n_seqs ? min(a.row_ctx[t], a.max_ctx) : 0;
  }
  const int kh = h / (a.n_h / a.n_kv);
  float q[N], o[N], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const size_t at = (size_t)t * a.q_stride + (size_t)h * HD + lane + 64 * i;
    q[i] = (a.q_bf16 ? load_el<true>(a.q, at) : load_el<false>(a.q, at)) * a.scale;
    o[i] = 0.f;
  }
  for (int j = 0; j < ctx; ++j) {
    const unsigned b = min((unsigned)a.tables[(size_t)seq * a.table_len + (j >> 4)], (unsigned)a.num_blocks - 1);
    const unsigned char* cell = kv_cell(a.kv, KV_INT4, HD, a.layer, a.num_blocks, (int)b, a.n_kv, kh);
    const int slot = j & 15;
    const unsigned ks = ((const unsigned*)(cell + 16 * HD))[slot], vs = ((const unsigned*)(cell + 16 * HD))[16 + slot];
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int d = lane + 64 * i, c = (cell[slot * (HD / 2) + (d >> 1)] >> (4 * (d & 1))) & 15;
      dot = fmaf(q[i], fmaf(__uint_as_float(ks << 16), (float)c, __uint_as_float(ks & 0xffff0000u)), dot);
    }
    dot = wave_sum(dot);
    const float mn = fmaxf(m, dot), alpha = __expf(m - mn), p = __expf(dot - mn);
    m = mn;
    l = l * alpha + p;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int d = lane + 64 * i, half = d / (HD / 2);
      const int c = (cell[8 * HD + (d - half * (HD / 2)) * 16 + slot] >> (4 * half)) & 15;
      o[i] = o[i] * alpha + p * fmaf(__uint_as_float(vs << 16), (float)c, __uint_as_float(vs & 0xffff0000u));
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const size_t at = ((size_t)t * a.n_h + h) * HD + lane + 64 * i;
    const float r = ctx > 0 ? o[i] / l : 0.f;
    if (a.out_type == OUT_F32) ((float*)a.out)[at] = r;
    else if (a.out_type == OUT_BF16) ((uint16_t*)a.out)[at] = f2bf(r);
    else store_split((uint16_t*)a.out, a.out_lo, at, r);
  }
}

// =============================================================== launchers

hipError_t launch_kv_append(hipStream_t st, bool x_bf16, int kind, const AppendArgs& a) {
  if (a.T <= 0) return hipSuccess;
  const bool aligned = a.stride % 4 == 0 && a.split_stride % 4 == 0 && (uintptr_t)a.x % (x_bf16 ? 8 : 16) == 0;
  const long long lanes = (long long)a.T * (a.n_h + 2 * a.n_kv) * (a.hd / 8);
  const dim3 grid((unsigned)((lanes + 255) / 256)), blk(256);
  auto go = [&](auto bf, auto hd, auto k) {
    constexpr bool B = decltype(bf)::value;
    constexpr int D = decltype(hd)::value, K = decltype(k)::value;
    if (a.q_gain.p[0]) klaunch(k_kv_append<B, K, D, true>, grid, blk, st, a, aligned);
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
                          const int* row_pos, const KvPlace& place, void* k, void* v) {
  if (T <= 0) return hipSuccess;
  if (hd != 64 && hd != 128) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(((long long)T * n_kv * (hd / 8) + 255) / 256)), blk(256);
  auto go = [&](auto kern) { klaunch(kern, grid, blk, st, kv, layer, n_kv, T, row_pos, place, k, v); };
  if (kind == KV_F32) hd == 64 ? go(k_kv_read<KV_F32, 64>) : go(k_kv_read<KV_F32, 128>);
  else if (kind == KV_BF16) hd == 64 ? go(k_kv_read<KV_BF16, 64>) : go(k_kv_read<KV_BF16, 128>);
  else hd == 64 ? go(k_kv_read<KV_INT4, 64>) : go(k_kv_read<KV_INT4, 128>);
  return hipGetLastError();
}

size_t attend4_rows_bytes(int, int, int, int) { return 0; }
size_t attend4_chunks_bytes(int, int, int, int, int, int) { return 0; }

static hipError_t attend4(hipStream_t st, const Attend4Args& a) {
  if (a.T <= 0) return hipSuccess;
  const dim3 grid(a.T, a.n_h), blk(64);
  if (a.hd == 64) klaunch(k_attend4<64>, grid, blk, st, a);
  else if (a.hd == 128) klaunch(k_attend4<128>, grid, blk, st, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}
hipError_t launch_attend4_rows(hipStream_t st, const Attend4Args& a, void*) { return attend4(st, a); }
hipError_t launch_attend4_chunks(hipStream_t st, const Attend4Args& a, void*) { return attend4(st, a); }
