// Log probabilities of given tokens, entropies and the likeliest alternatives.
// Part of kernels.hip (its helpers are above).

// A logit's place in the order of alternatives: larger first, NaN last.
__device__ __forceinline__ bool before(float a, int ia, float b, int ib) {
  const bool na = a != a, nb = b != b;
  if (na != nb) return nb;
  return a > b || ((a == b || na) && ia < ib);
}

// One workgroup a row: the maximum, the sums, then the alternatives one pass each.
template <bool BF>
__global__ __launch_bounds__(256) void k_score(ScoreArgs a) {
  __shared__ float sf[256];
  __shared__ int si[256];
  const int r = blockIdx.x, tid = threadIdx.x;
  const size_t base = (size_t)r * a.stride;
  auto at = [&](int i) { return load_el<BF>(a.logits, base + i); };
  auto reduce = [&](float v, auto f) {
    sf[tid] = v;
    for (int n = 128; n > 0; n >>= 1) {
      __syncthreads();
      if (tid < n) sf[tid] = f(sf[tid], sf[tid + n]);
    }
    __syncthreads();
    const float x = sf[0];
    __syncthreads();
    return x;
  };
  float mx = -INFINITY;
  bool bad = false;
  for (int i = tid; i < a.vocab; i += 256) {
    const float x = at(i);
    mx = fmaxf(mx, x);
    bad = bad || x != x;
  }
  mx = reduce(mx, [](float u, float v) { return fmaxf(u, v); });
  bad = reduce(bad ? 1.f : 0.f, [](float u, float v) { return fmaxf(u, v); }) > 0.f || !(fabsf(mx) < INFINITY);
  float sum = 0.f, mom = 0.f;
  if (!bad)
    for (int i = tid; i < a.vocab; i += 256) {
      const float d = at(i) - mx;
      if (d > -INFINITY) {
        const float e = expf(d);
        sum += e;
        mom = fmaf(e, d, mom);
      }
    }
  auto add = [](float u, float v) { return u + v; };
  sum = reduce(sum, add);
  mom = reduce(mom, add);
  const float nan = __uint_as_float(0x7fc00000u), norm = bad ? nan : logf(sum);
  if (tid == 0) {
    const int tok = a.tokens[r];
    a.logprob[r] = (unsigned)tok < (unsigned)a.vocab ? at(tok) - mx - norm : nan;
    a.entropy[r] = norm - mom / sum;
  }
  float last = INFINITY;
  int last_id = -1;
  for (int k = 0; k < a.top; ++k) {
    float best = nan;
    int id = INT_MAX;
    for (int i = tid; i < a.vocab; i += 256) {
      const float x = at(i);
      if (before(last, last_id, x, i) && before(x, i, best, id)) { best = x; id = i; }
    }
    sf[tid] = best;
    si[tid] = id;
    for (int n = 128; n > 0; n >>= 1) {
      __syncthreads();
      if (tid < n && before(sf[tid + n], si[tid + n], sf[tid], si[tid])) { sf[tid] = sf[tid + n]; si[tid] = si[tid + n]; }
    }
    __syncthreads();
    last = sf[0];
    last_id = si[0];
    __syncthreads();
    if (tid == 0) {
      a.top_ids[(size_t)r * a.top + k] = last_id;
      a.top_logprobs[(size_t)r * a.top + k] = bad ? nan : last - mx - norm;
    }
  }
}

size_t score_bytes(int, int, int) { return 0; }

hipError_t launch_score(hipStream_t st, const ScoreArgs& a, void*) {
  if (a.rows <= 0) return hipSuccess;
  if (a.bf16) klaunch(k_score<true>, dim3(a.rows), dim3(256), st, a);
  else klaunch(k_score<false>, dim3(a.rows), dim3(256), st, a);
  return hipGetLastError();
}
