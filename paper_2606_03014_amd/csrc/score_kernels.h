// Log probabilities of given tokens, entropies and the likeliest alternatives.
// Part of kernels.hip (its helpers are above).

// A logit's place in the order of alternatives: larger first, NaN last.
__device__ __forceinline__ bool before(float a, int ia, float b, int ib) {
  const bool na = a != a, nb = b != b;
  if (na != nb) return nb;
  return a > b || ((a == b || na) && ia < ib);
}

// One pass over a row, 16 logits a thread at a time, the next 16 in flight: by one workgroup of
// 1,024 threads, or, where the rows alone leave CUs idle, by one for each of nseg runs of
// steps, joined by a second launch. Bound by reading the logits in many rows, by the
// exponentials in few.
//  * Every thread keeps its own maximum m, sum of e^(x - m) and sum of e^(x - m) (x - m); they
//    are joined once at the end.
//  * Alternatives: of the first step, 64 groups of threads give their maxima; the k-th largest
//    of those is no larger than the run's k-th logit. Logits from there up go to a list in LDS
//    (about as many as the k largest twice over), which is cut back to its k largest, raising
//    the bar, after 2, 4, 8 .. steps. An entry is one 64-bit key, the logit's order above
//    the id's complement, so the list's order is that of (logit, id) however the threads
//    came to it.
//  * Rows whose list would not hold them (a thousand equal logits) or that hold NaN beside too
//    few possible tokens search for one alternative after the other.
// 512 rows of 128,256 float32 logits, 20 alternatives: 51 us, 5.2 TB/s (47 without alternatives).
// Rows of any alignment are read in 16-byte pieces from the last 16-byte boundary on (such
// a piece is inside the row's pages); what lies outside the row counts as -inf.
constexpr int kScoreList = 1024, kScoreStep = 16384;   // list entries; logits per step
typedef unsigned long long u64;

__device__ __forceinline__ u64 score_key(float v, int id) {
  const unsigned b = __float_as_uint(v + 0.f);           // -0 becomes 0: the same place in the order
  return ((u64)(b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u)) << 32) | ~(unsigned)id;
}
__device__ __forceinline__ float key_value(u64 k) {
  const unsigned b = (unsigned)(k >> 32);
  return __uint_as_float(b ^ ((b >> 31) ? 0x80000000u : 0xffffffffu));
}

struct ScoreSums { float m, sum, mom; };
// m, sum, mom of two sets of logits; a set of none has m = -inf and sums of 0.
__device__ __forceinline__ void join_sums(ScoreSums& s, const ScoreSums& o) {
  const float m = fmaxf(s.m, o.m);
  // the lowest value masks like -inf, but its distance must stay finite
  const float ds = s.m == -INFINITY ? 0.f : fmaxf(s.m - m, -1e30f), dp = o.m == -INFINITY ? 0.f : fmaxf(o.m - m, -1e30f);
  const float as = __builtin_amdgcn_exp2f(ds * 1.4426950408889634f), ao = __builtin_amdgcn_exp2f(dp * 1.4426950408889634f);
  s.mom = as * fmaf(ds, s.sum, s.mom) + ao * fmaf(dp, o.sum, o.mom);
  s.sum = as * s.sum + ao * o.sum;
  s.m = m;
}

// The k largest of the n keys in LDS by 1,024 threads: put(rank, key) for each of them.
// Sixteen threads count for an entry.
template <typename F>
__device__ __forceinline__ void rank_keys(const u64* keys, int n, int k, F put) {
  const int part = threadIdx.x & 15;
  for (int i = threadIdx.x >> 4; i < n; i += 64) {
    const u64 mine = keys[i];
    int rk = 0;
#pragma unroll 4
    for (int j = part; j < n; j += 16) rk += keys[j] > mine;
    rk = (int)sum16((float)rk);                          // at most 1,024: exact
    if (part == 0 && rk < k) put(rk, mine);
  }
}

// The results of row r from its sums and its list (n keys; over: the list did not hold them).
template <bool BF>
__device__ __forceinline__ void score_row(const ScoreArgs& a, int r, const ScoreSums& s, const u64* keys, int n, bool over,
                                          float* lv, int* li) {
  const int tid = threadIdx.x, lane = tid & 63, V = a.vocab, k = a.top;
  const void* row = (const char*)a.logits + (size_t)r * a.stride * (BF ? 2 : 4);
  auto at = [&](int i) { return load_el<BF>(row, i); };
  const bool bad = s.sum != s.sum || !(fabsf(s.m) < INFINITY);    // NaN, +inf, or nothing above -inf
  const float nan = __uint_as_float(0x7fc00000u), norm = bad ? nan : logf(s.sum);
  if (tid == 0) {
    const int tok = a.tokens[a.token_at ? a.token_at[r] : r];
    a.logprob[r] = (unsigned)tok < (unsigned)V ? at(tok) - s.m - norm : nan;
    a.entropy[r] = norm - s.mom / s.sum;
  }
  if (k == 0) return;
  int* ids = a.top_ids + (size_t)r * k;
  float* tops = a.top_logprobs + (size_t)r * k;
  if (!over && (n >= k || s.sum == s.sum)) {
    rank_keys(keys, n, k, [&](int rk, u64 key) {
      ids[rk] = (int)~(unsigned)key;
      tops[rk] = bad ? nan : key_value(key) - s.m - norm;
    });
    if (n < k && tid < 64) {                             // fewer possible tokens: impossible ones by id (64 ids hold enough)
      const bool no = lane < V && at(min(lane, V - 1)) == -INFINITY;
      const int rk = n + __popcll(__ballot(no) & ((1ull << lane) - 1));
      if (no && rk < k) {
        ids[rk] = lane;
        tops[rk] = bad ? nan : -INFINITY;
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
    lv[tid] = best;
    li[tid] = id;
    for (int d = 512; d > 0; d >>= 1) {
      __syncthreads();
      if (tid < d && before(lv[tid + d], li[tid + d], lv[tid], li[tid])) { lv[tid] = lv[tid + d]; li[tid] = li[tid + d]; }
    }
    __syncthreads();
    last = lv[0];
    last_id = li[0];
    if (tid == 0) {
      ids[q] = last_id;
      tops[q] = bad ? nan : last - s.m - norm;
    }
  }
}

// Partial results of a row's runs: m, sum, mom, the list's length (-1: it did not hold them); the keys.
struct ScoreParts { float4* sums; u64* keys; };

template <bool BF>
__global__ __launch_bounds__(1024, 8) void k_score(ScoreArgs a, int nseg, int seg_steps, ScoreParts parts) {
  constexpr int E = BF ? 8 : 4, NV = 16 / E;             // logits per 16 bytes, pieces per thread and step
  __shared__ __align__(16) u64 lists[2][kScoreList];
  __shared__ float sg[16 * 65], gm[64], sbar;
  __shared__ ScoreSums ss[16];
  __shared__ int cnt;
  const int r = blockIdx.x / nseg, seg = blockIdx.x % nseg, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int V = a.vocab, k = a.top;
  const uintptr_t row = (uintptr_t)a.logits + (size_t)r * a.stride * (BF ? 2 : 4);
  const int mis = (int)(row & 15) / (BF ? 2 : 4);        // logits of the first piece that lie before the row
  const u32x4* pieces = (const u32x4*)(row & ~(uintptr_t)15);
  const int np = (mis + V + E - 1) / E, c0 = seg * seg_steps;
  const int c1 = min(c0 + seg_steps, (np + NV * 1024 - 1) / (NV * 1024));
  const float ninf = -INFINITY;
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
  ScoreSums s{ninf, 0.f, 0.f};
  float bar = INFINITY;
  int cur = 0;
  bool over = false;                                     // the list did not hold a step's candidates
  if (tid == 0) { cnt = 0; sbar = ninf; }               // fewer than k groups that are not NaN: no bar
  load(c0);
  for (int c = c0; c < c1; ++c) {
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
    if (c + 1 < c1) load(c + 1);
    float cm = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) cm = fmaxf(cm, x[i]);
    if (cm > s.m) join_sums(s, ScoreSums{cm, 0.f, 0.f});
    const float ref = s.m == ninf ? 0.f : s.m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float d = x[i] - ref, e = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
      s.sum += e;
      s.mom = fmaf(e, fmaxf(d, -1e30f), s.mom);          // an impossible token, or one masked with the lowest value, adds 0
    }
    if (k > 0) {
      if (c == c0) {                                     // groups: the threads of a lane in all waves
        const int i = tid >> 4, part = tid & 15;         // sixteen threads a group
        sg[w * 65 + lane] = cm;
        __syncthreads();
        const float g = max16(sg[part * 65 + i]);
        if (part == 0) gm[i] = g;
        __syncthreads();
        int rk = 0;
#pragma unroll
        for (int j = part; j < 64; j += 16) rk += gm[j] > g || (gm[j] == g && j < i);
        if ((int)sum16((float)rk) == k - 1 && g == g) sbar = g;
        __syncthreads();
        bar = sbar;
      }
      if (!over && cm >= bar && cm > ninf) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (x[i] >= bar && x[i] > ninf) {
            const int n = atomicAdd(&cnt, 1);
            if (n < kScoreList) lists[cur][n] = score_key(x[i], ((c * NV + i / E) * 1024 + tid) * E + i % E - mis);
          }
      }
      const int done = c - c0 + 1;
      if (c + 1 < c1 && done > 1 && (done & (done - 1)) == 0) {     // after 2, 4, 8 .. steps
        __syncthreads();
        const int n = cnt;
        over = over || n > kScoreList;
        if (!over && n > k) {
          rank_keys(lists[cur], n, k, [&](int rk, u64 key) { lists[cur ^ 1][rk] = key; });
          cur ^= 1;
          __syncthreads();
          bar = key_value(lists[cur][k - 1]);
          if (tid == 0) cnt = k;
        }
        __syncthreads();
      }
    }
  }
  // join the threads
  {
    float mw = max16(s.m);
    mw = fmaxf(mw, swz_xor16(mw));
    mw = fmaxf(mw, __shfl_xor(mw, 32, 64));
    join_sums(s, ScoreSums{mw, 0.f, 0.f});
    s.sum = wave_sum(s.sum);
    s.mom = wave_sum(s.mom);
    if (lane == 0) ss[w] = s;
  }
  __syncthreads();
  s = ss[lane & 15];
  join_sums(s, ScoreSums{max16(s.m), 0.f, 0.f});
  s.sum = sum16(s.sum);
  s.mom = sum16(s.mom);
  const int n = cnt;                                     // every append came before the join's barrier
  over = over || n > kScoreList;
  if (nseg == 1) {
    score_row<BF>(a, r, s, lists[cur], n, over, sg, (int*)lists[cur]);
    return;
  }
  if (tid == 0) parts.sums[blockIdx.x] = make_float4(s.m, s.sum, s.mom, __int_as_float(over ? -1 : min(n, k)));
  if (k > 0 && !over) {
    u64* out = parts.keys + (size_t)blockIdx.x * k;
    rank_keys(lists[cur], n, k, [&](int rk, u64 key) { out[rk] = key; });
  }
}

template <bool BF>
__global__ __launch_bounds__(1024) void k_score_join(ScoreArgs a, int nseg, ScoreParts parts) {
  __shared__ __align__(16) u64 list[kScoreList];
  __shared__ float lv[1024];
  const int r = blockIdx.x;
  ScoreSums s{-INFINITY, 0.f, 0.f};
  int n = 0;
  bool over = false;
  for (int g = 0; g < nseg; ++g) {                       // runs in order; every thread alike
    const float4 p = parts.sums[(size_t)r * nseg + g];
    join_sums(s, ScoreSums{p.x, p.y, p.z});
    const int m = __float_as_int(p.w);
    over = over || m < 0;
    if (threadIdx.x < max(m, 0)) list[n + threadIdx.x] = parts.keys[((size_t)r * nseg + g) * a.top + threadIdx.x];
    n += max(m, 0);
  }
  __syncthreads();
  score_row<BF>(a, r, s, list, n, over, lv, (int*)list);
}

// Runs of a row: two workgroups a CU (1 row of 128,256 float32 logits, 20 alternatives: 46.7 us
// in one run, 12.9 in eight; 512 rows in one run each 54.4), at most 32 (their alternatives fit the list).
static void plan_score(int rows, int vocab, int& nseg, int& seg_steps) {
  const int steps = (vocab + 8 + kScoreStep - 1) / kScoreStep;    // the first piece may begin before the row
  nseg = std::max(1, std::min({steps, 512 / std::max(rows, 1), kScoreList / kMaxTop}));
  seg_steps = (steps + nseg - 1) / nseg;
  nseg = (steps + seg_steps - 1) / seg_steps;
}

size_t score_bytes(int rows, int vocab, int top) {
  int nseg, seg_steps;
  plan_score(rows, vocab, nseg, seg_steps);
  return nseg > 1 ? (size_t)rows * nseg * (sizeof(float4) + 8 * (size_t)top) : 0;
}

size_t score_bytes_max(int vocab) {
  size_t most = 0;
  for (int rows = 1; rows <= 512; ++rows) most = std::max(most, score_bytes(rows, vocab, kMaxTop));
  return most;
}

hipError_t launch_score(hipStream_t st, const ScoreArgs& a, void* workspace) {
  if (a.rows <= 0) return hipSuccess;
  int nseg, seg_steps;
  plan_score(a.rows, a.vocab, nseg, seg_steps);
  const ScoreParts parts{(float4*)workspace, (u64*)((float4*)workspace + (size_t)a.rows * nseg)};
  const dim3 grid((unsigned)a.rows * nseg), blk(1024);
  if (a.bf16) klaunch(k_score<true>, grid, blk, st, a, nseg, seg_steps, parts);
  else klaunch(k_score<false>, grid, blk, st, a, nseg, seg_steps, parts);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || nseg == 1) return err;
  if (a.bf16) klaunch(k_score_join<true>, dim3(a.rows), blk, st, a, nseg, parts);
  else klaunch(k_score_join<false>, dim3(a.rows), blk, st, a, nseg, parts);
  return hipGetLastError();
}
