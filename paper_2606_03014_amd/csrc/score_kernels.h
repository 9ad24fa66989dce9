// Log probabilities of given tokens, entropies and the likeliest alternatives.
// Part of kernels.hip (its helpers are above).

// A logit's place in the order of alternatives: larger first, NaN last.
__device__ __forceinline__ bool before(float a, int ia, float b, int ib) {
  const bool na = a != a, nb = b != b;
  if (na != nb) return nb;
  return a > b || ((a == b || na) && ia < ib);
}

// One pass over a row by one workgroup of 1,024 threads, 16 logits a thread at a time, the
// next 16 in flight. Bound by reading the logits.
//  * Every thread keeps its own maximum m, sum of e^(x - m) and sum of e^(x - m) (x - m); they
//    are joined once at the end.
//  * Alternatives: of the first 16,384 logits, 64 groups of threads give their maxima; the
//    k-th largest of those is no larger than the row's k-th logit. Logits from there up go to a
//    list in LDS (about as many as a normal row's k largest twice over), which is cut back to
//    its k largest, raising the bar, after 2, 4, 8 .. steps. Its order is that of (logit, id)
//    however the threads came to it.
//  * Rows where that list would not hold them (thousands of equal logits) or that hold NaN
//    beside too few possible tokens search for one alternative after the other.
// Rows of any alignment are read in 16-byte pieces from the last 16-byte boundary on (such
// a piece is inside the row's pages); what lies outside the row counts as -inf.
constexpr int kScoreList = 1024;

template <bool BF>
__global__ __launch_bounds__(1024) void k_score(ScoreArgs a) {
  constexpr int E = BF ? 8 : 4, NV = 16 / E;       // logits per 16 bytes, pieces per thread and step
  __shared__ float lv[2][kScoreList];
  __shared__ int li[2][kScoreList];
  __shared__ __align__(16) float sg[64];
  __shared__ float sm[3][16];
  __shared__ int cnt;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6, V = a.vocab, k = a.top;
  const uintptr_t row = (uintptr_t)a.logits + (size_t)r * a.stride * (BF ? 2 : 4);
  const int mis = (int)(row & 15) / (BF ? 2 : 4);  // logits of the first piece that lie before the row
  const u32x4* pieces = (const u32x4*)(row & ~(uintptr_t)15);
  const int np = (mis + V + E - 1) / E, steps = (np + NV * 1024 - 1) / (NV * 1024);
  const float ninf = -INFINITY;
  auto at = [&](int i) { return load_el<BF>((const void*)row, i); };
  u32x4 raw[NV];
  auto load = [&](int c) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int p = (c * NV + j) * 1024 + tid;
      const unsigned none = BF ? 0xFF80FF80u : 0xFF800000u;
      u32x4 x = {none, none, none, none};
      if (p < np) {
        x = __builtin_nontemporal_load(pieces + p);
        const int e0 = p * E - mis;
        if (e0 < 0 || e0 + E > V) {
#pragma unroll
          for (int i = 0; i < E; ++i)
            if (e0 + i < 0 || e0 + i >= V) {
              if constexpr (BF) x[i >> 1] = (i & 1) ? (x[i >> 1] & 0xffffu) | 0xFF800000u : (x[i >> 1] & 0xffff0000u) | 0xFF80u;
              else x[i] = none;
            }
        }
      }
      raw[j] = x;
    }
  };
  float m = ninf, sum = 0.f, mom = 0.f, bar = INFINITY;
  int cur = 0;
  bool over = false;                               // the list did not hold a step's candidates
  // rank of entry i of the list
  auto rank_of = [&](int n, int i) {
    const float v = lv[cur][i];
    const int id = li[cur][i];
    int rk = 0;
    for (int j = 0; j < n; ++j) rk += before(lv[cur][j], li[cur][j], v, id);
    return rk;
  };
  if (tid == 0) cnt = 0;
  load(0);
  for (int c = 0; c < steps; ++c) {
    float x[16];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (BF) {
          x[j * 8 + 2 * i] = __uint_as_float(raw[j][i] << 16);
          x[j * 8 + 2 * i + 1] = __uint_as_float(raw[j][i] & 0xffff0000u);
        } else {
          x[j * 4 + i] = __uint_as_float(raw[j][i]);
        }
      }
    if (c + 1 < steps) load(c + 1);
    float cm = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) cm = fmaxf(cm, x[i]);
    if (cm > m) {
      const float d = m == ninf ? 0.f : fmaxf(m - cm, -1e30f), al = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
      mom = al * fmaf(d, sum, mom);
      sum *= al;
      m = cm;
    }
    const float ref = m == ninf ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float d = x[i] - ref, e = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
      sum += e;
      mom = fmaf(e, fmaxf(d, -1e30f), mom);        // an impossible token, or one masked with the lowest value, adds 0
    }
    if (k > 0) {
      if (c == 0) {
        const float g = max16(cm);
        if ((tid & 15) == 0) sg[tid >> 4] = g;
        __syncthreads();
        const float v = sg[lane];
        int rk = 0;
#pragma unroll
        for (int j = 0; j < 64; ++j) rk += sg[j] > v || (sg[j] == v && j < lane);
        const unsigned long long who = __ballot(rk == k - 1);
        bar = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), who ? __builtin_ctzll(who) : 0));
      }
      if (!over && cm >= bar && cm > ninf) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (x[i] >= bar && x[i] > ninf) {
            const int n = atomicAdd(&cnt, 1);
            if (n < kScoreList) {
              lv[cur][n] = x[i];
              li[cur][n] = ((c * NV + i / E) * 1024 + tid) * E + i % E - mis;
            }
          }
      }
      if (c + 1 < steps && c > 0 && (c & (c + 1)) == 0) {    // after 2, 4, 8 .. steps
        __syncthreads();
        const int n = cnt;
        over = over || n > kScoreList;
        if (!over && n > k) {
          if (tid < n) {
            const int rk = rank_of(n, tid);
            if (rk < k) { lv[cur ^ 1][rk] = lv[cur][tid]; li[cur ^ 1][rk] = li[cur][tid]; }
          }
          cur ^= 1;
          __syncthreads();
          bar = lv[cur][k - 1];
          if (tid == 0) cnt = k;
        }
        __syncthreads();
      }
    }
  }
  // join the threads
  {
    float mw = max16(m);
    mw = fmaxf(mw, swz_xor16(mw));
    mw = fmaxf(mw, __shfl_xor(mw, 32, 64));
    const float d = m == ninf ? 0.f : fmaxf(m - mw, -1e30f), al = m == ninf ? 1.f : __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
    mom = wave_sum(al * fmaf(d, sum, mom));
    sum = wave_sum(sum * al);
    if (lane == 0) { sm[0][w] = mw; sm[1][w] = sum; sm[2][w] = mom; }
  }
  __syncthreads();
  m = sm[0][0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m = fmaxf(m, sm[0][i]);
  sum = mom = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float d = sm[0][i] == ninf ? 0.f : fmaxf(sm[0][i] - m, -1e30f), al = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
    mom += al * fmaf(d, sm[1][i], sm[2][i]);
    sum = fmaf(sm[1][i], al, sum);
  }
  const bool bad = sum != sum || !(fabsf(m) < INFINITY);     // NaN, +inf, or nothing above -inf
  const float nan = __uint_as_float(0x7fc00000u), norm = bad ? nan : logf(sum);
  if (tid == 0) {
    const int tok = a.tokens[r];
    a.logprob[r] = (unsigned)tok < (unsigned)V ? at(tok) - m - norm : nan;
    a.entropy[r] = norm - mom / sum;
  }
  if (k == 0) return;
  int* ids = a.top_ids + (size_t)r * k;
  float* tops = a.top_logprobs + (size_t)r * k;
  const int n = cnt;                               // every append came before the join's barrier
  if (!over && n <= kScoreList && (n >= k || sum == sum || m == ninf)) {
    if (tid < n) {
      const int rk = rank_of(n, tid);
      if (rk < k) {
        ids[rk] = li[cur][tid];
        tops[rk] = bad ? nan : lv[cur][tid] - m - norm;
      }
    }
    if (n < k && w == 0) {                         // fewer possible tokens: impossible ones by id (64 ids hold enough)
      const bool no = lane < V && at(min(lane, V - 1)) == ninf;
      const unsigned long long all = __ballot(no);
      const int rk = n + __popcll(all & ((1ull << lane) - 1));
      if (no && rk < k) {
        ids[rk] = lane;
        tops[rk] = bad ? nan : ninf;
      }
    }
    return;
  }
  float last = INFINITY;
  int last_id = -1;
  for (int q = 0; q < k; ++q) {
    float best = nan;
    int id = INT_MAX;
    for (int i = tid; i < V; i += 1024) {
      const float x = at(i);
      if (before(last, last_id, x, i) && before(x, i, best, id)) { best = x; id = i; }
    }
    __syncthreads();
    lv[0][tid] = best;
    li[0][tid] = id;
    for (int s = 512; s > 0; s >>= 1) {
      __syncthreads();
      if (tid < s && before(lv[0][tid + s], li[0][tid + s], lv[0][tid], li[0][tid])) { lv[0][tid] = lv[0][tid + s]; li[0][tid] = li[0][tid + s]; }
    }
    __syncthreads();
    last = lv[0][0];
    last_id = li[0][0];
    if (tid == 0) {
      ids[q] = last_id;
      tops[q] = bad ? nan : last - m - norm;
    }
  }
}

size_t score_bytes(int, int, int) { return 0; }

hipError_t launch_score(hipStream_t st, const ScoreArgs& a, void*) {
  if (a.rows <= 0) return hipSuccess;
  if (a.bf16) klaunch(k_score<true>, dim3(a.rows), dim3(1024), st, a);
  else klaunch(k_score<false>, dim3(a.rows), dim3(1024), st, a);
  return hipGetLastError();
}
