// The next token of every row of logits, from given uniform numbers.  With l_max the row's largest logit and T its temperature,
//   w_i = exp((l_i - l_max) / T)            (NaN and -inf weigh nothing; with infinite logits those alone weigh, 1 each)
// and the tokens in the order (logit descending, index ascending):
//   top-k   the first k                      top-p   the shortest beginning whose w sum to at least p times those of the first k
//   min-p   those with w >= p_min            (w of the best is 1)
// Each keeps a beginning of the same order, so what is kept is the shortest of the three.  The token is the lowest kept index
// t with  sum of the kept w_i, i <= t,  > u W,  W the sum of all kept.
//
// Weights are 64-bit integers, w 2^kFraction rounded: sums of integers do not depend on their order, so the workgroup may add
// them as it likes (histograms by atomics, prefix sums in any tree) and every call gives the same token.
#include "common.h"

namespace earn {

typedef unsigned long long u64;
constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / kWave;
constexpr int kBins = 2048;            // of (l_max - l) / T in steps of 1/64; the last one holds everything from 31.98 on
constexpr int kBinsPerUnit = 64;
constexpr int kFraction = 44;          // exp(-31.98) 2^44 < 1/2: the last bin's weights are all zero
constexpr int kListMax = 2048;

struct SampleParams {
  const void* logits; long long row_stride;
  int vocab;
  const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p; const float* uniform;
  int32_t* token; float* logprob; int32_t* n_kept;
};

// a float as an integer of the same order (no NaN; zeros of either sign equal)
__device__ __forceinline__ unsigned order_key(float x) {
  const unsigned b = __float_as_uint(x == 0.f ? 0.f : x);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

template <typename T>
struct Row {
  const T* p;
  int n;
  __device__ __forceinline__ float at(int i) const {
    float x;
    if constexpr (sizeof(T) == 2) x = bf16_bits_to_f32(((const unsigned short*)p)[i]);
    else x = ((const float*)p)[i];
    return x == x ? x : -INFINITY;
  }
};

// Weights of a row.
struct Weights {
  float best;         // the largest logit
  float bins;         // bins per unit of logit
  double scale;       // log2(e) / T
  bool infinite;      // best is +inf
  __device__ __forceinline__ double real(float l) const {
    if (l == best) return 1.0;
    if (infinite || l == -INFINITY) return 0.0;
    return exp2(((double)l - (double)best) * scale);
  }
  __device__ __forceinline__ u64 of(float l) const { return (u64)(real(l) * (double)(1ull << kFraction) + 0.5); }
  // monotone in l: rounding keeps the order of differences and products
  __device__ __forceinline__ int bin(float l) const {
    return l == best ? 0 : (int)fminf((best - l) * bins, (float)(kBins - 1));
  }
};

struct SampleSmem {
  u64 mass[kBins];
  int count[kBins];
  u64 list_w[kListMax];
  u64 list_key[kListMax];        // (order key, ~index): larger is earlier in the order
  u64 wave_mass[kSampleWaves];
  int wave_count[kSampleWaves];
  float wave_best[kSampleWaves];
  int wave_at[kSampleWaves];
  int n_list, bin, found_count;
  u64 before_mass, limit, found_mass;
  int before_count;
};

__device__ __forceinline__ u64 wave_sum(u64 x) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) x += __shfl_xor(x, o, kWave);
  return x;
}
__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) x += __shfl_xor(x, o, kWave);
  return x;
}
template <typename X>
__device__ __forceinline__ X wave_scan(X x, int lane) {   // inclusive
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const X y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  return x;
}

// A beginning of the order: everything whose (key, ~index) is at least `limit`; `count` entries that weigh `mass`.
struct Beginning { u64 limit, mass; int count; };

// Does an entry end the beginning that is looked for?  By count: it is the k-th.  By mass: it is the one that reaches the target.
struct Target {
  bool by_mass;
  int k;
  u64 mass;
  __device__ __forceinline__ bool hit(int before, u64 mass_before, int n, u64 w) const {
    return by_mass ? mass_before < mass && mass_before + w >= mass : before < k && before + n >= k;
  }
};

// The beginning that `target` ends, from the histogram; called by all threads.  There is one: k is at most the number of
// entries, the mass at most that of all.
template <typename T>
__device__ Beginning find_beginning(const Row<T>& row, const Weights& wt, const Target& target, SampleSmem& sm) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  // the bin that the target ends in
  static_assert(kBins == 2 * kSampleThreads);
  const int c0 = sm.count[2 * tid], c1 = sm.count[2 * tid + 1];
  const u64 m0 = sm.mass[2 * tid], m1 = sm.mass[2 * tid + 1];
  const int cs = wave_scan(c0 + c1, lane);
  const u64 ms = wave_scan(m0 + m1, lane);
  __syncthreads();
  if (lane == kWave - 1) { sm.wave_count[wave] = cs; sm.wave_mass[wave] = ms; }
  if (tid == 0) { sm.n_list = 0; sm.bin = kBins - 1; }
  __syncthreads();
  int cb = cs - c0 - c1;
  u64 mb = ms - m0 - m1;
  for (int i = 0; i < wave; ++i) { cb += sm.wave_count[i]; mb += sm.wave_mass[i]; }
  if (target.hit(cb, mb, c0, m0)) { sm.bin = 2 * tid; sm.before_count = cb; sm.before_mass = mb; }
  if (target.hit(cb + c0, mb + m0, c1, m1)) { sm.bin = 2 * tid + 1; sm.before_count = cb + c0; sm.before_mass = mb + m0; }
  __syncthreads();
  const int bin = sm.bin;
  int before = sm.before_count;
  u64 mass_before = sm.before_mass;
  if (sm.count[bin] <= kListMax) {
    for (int i = tid; i < row.n; i += kSampleThreads) {
      const float l = row.at(i);
      if (l > -INFINITY && wt.bin(l) == bin) {
        const int at = atomicAdd(&sm.n_list, 1);
        sm.list_w[at] = wt.of(l);
        sm.list_key[at] = (u64)order_key(l) << 32 | (unsigned)~i;
      }
    }
    __syncthreads();
    const int n = sm.n_list;
    for (int a = tid; a < n; a += kSampleThreads) {
      const u64 key = sm.list_key[a];
      int cnt = before;
      u64 mass = mass_before;
      for (int b = 0; b < n; ++b) {
        const bool first = sm.list_key[b] > key;
        cnt += first ? 1 : 0;
        mass += first ? sm.list_w[b] : 0;
      }
      if (target.hit(cnt, mass, 1, sm.list_w[a])) { sm.limit = key; sm.found_count = cnt + 1; sm.found_mass = mass + sm.list_w[a]; }
    }
    __syncthreads();
    return Beginning{sm.limit, sm.found_mass, sm.found_count};
  }
  // Too many for the list (mostly equal logits): the last key, bit by bit, then its equals in order of their index.
  auto reach = [&](unsigned key, int& cnt, u64& mass) {   // entries of the bin whose key is at least `key`
    int c = 0;
    u64 m = 0;
    for (int i = tid; i < row.n; i += kSampleThreads) {
      const float l = row.at(i);
      if (l > -INFINITY && wt.bin(l) == bin && order_key(l) >= key) { ++c; m += wt.of(l); }
    }
    c = wave_sum(c);
    m = wave_sum(m);
    __syncthreads();
    if (lane == 0) { sm.wave_count[wave] = c; sm.wave_mass[wave] = m; }
    __syncthreads();
    cnt = before;
    mass = mass_before;
    for (int i = 0; i < kSampleWaves; ++i) { cnt += sm.wave_count[i]; mass += sm.wave_mass[i]; }
  };
  unsigned t = 0;
  int cnt;
  u64 mass;
  for (int bit = 31; bit >= 0; --bit) {
    const unsigned with = t | 1u << bit;
    reach(with, cnt, mass);
    if (target.by_mass ? mass >= target.mass : cnt >= target.k) t = with;
  }
  reach(t + 1, cnt, mass);                        // what comes before the equals (t is a finite float's key)
  const u64 each = wt.of(key_value(t));
  // the r-th equal one is the last
  const int r = target.by_mass ? (int)((target.mass - mass + each - 1) / each) : target.k - cnt;
  const int per = ((row.n + kSampleWaves - 1) / kSampleWaves + kWave - 1) / kWave * kWave;
  const int begin = min(row.n, wave * per), end = min(row.n, begin + per);
  int mine = 0;
  for (int i = begin; i < end; i += kWave) mine += __popcll(__ballot(i + lane < end && order_key(row.at(min(i + lane, end - 1))) == t));
  __syncthreads();
  if (lane == 0) sm.wave_count[wave] = mine;
  __syncthreads();
  int at = 0;
  for (int i = 0; i < wave; ++i) at += sm.wave_count[i];
  for (int i = begin; i < end && at < r; i += kWave) {
    const unsigned long long m = __ballot(i + lane < end && order_key(row.at(min(i + lane, end - 1))) == t);
    if ((m >> lane & 1) && at + __popcll(m & ((1ull << lane) - 1)) == r - 1) sm.limit = (u64)t << 32 | (unsigned)~(i + lane);
    at += __popcll(m);
  }
  __syncthreads();
  return Beginning{sm.limit, mass + (u64)r * each, cnt + r};
}

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleParams p) {
  __shared__ SampleSmem sm;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, r = blockIdx.x;
  const Row<T> row{(const T*)p.logits + (long long)r * p.row_stride, p.vocab};
  const float temperature = p.temperature ? p.temperature[r] : 1.f;
  const int top_k = p.top_k ? p.top_k[r] : 0;
  const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f;
  float u = p.uniform[r];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  // the best entry, and how many there are
  float best = -INFINITY;
  int at = 0x7fffffff, n_finite = 0;
  for (int i = tid; i < p.vocab; i += kSampleThreads) {
    const float l = row.at(i);
    n_finite += l > -INFINITY;
    if (l > best) { best = l; at = i; }
  }
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const float b2 = __shfl_xor(best, o, kWave);
    const int a2 = __shfl_xor(at, o, kWave);
    if (b2 > best || (b2 == best && a2 < at)) { best = b2; at = a2; }
  }
  n_finite = wave_sum(n_finite);
  if (lane == 0) { sm.wave_best[wave] = best; sm.wave_at[wave] = at; sm.wave_count[wave] = n_finite; }
  __syncthreads();
  best = sm.wave_best[0]; at = sm.wave_at[0]; n_finite = sm.wave_count[0];
  for (int i = 1; i < kSampleWaves; ++i) {
    const float b2 = sm.wave_best[i];
    if (b2 > best || (b2 == best && sm.wave_at[i] < at)) { best = b2; at = sm.wave_at[i]; }
    n_finite += sm.wave_count[i];
  }
  __syncthreads();
  auto finish = [&](int token, float logprob, int count) {
    p.token[r] = token;
    if (p.logprob) p.logprob[r] = logprob;
    if (p.n_kept) p.n_kept[r] = count;
  };
  if (best == -INFINITY) { if (tid == 0) finish(-1, -INFINITY, 0); return; }
  if (!(temperature > 0.f) || top_k == 1 || !(top_p > 0.f)) { if (tid == 0) finish(at, 0.f, 1); return; }

  Weights wt;
  wt.best = best;
  wt.infinite = best == INFINITY;
  wt.scale = 1.4426950408889634074 / (double)temperature;
  wt.bins = fminf((float)kBinsPerUnit / temperature, 3e38f);
  const bool by_count = top_k > 0 && top_k < n_finite, by_mass = top_p < 1.f;
  Beginning kept{0, 0, n_finite};
  if (by_count || by_mass) {
    for (int i = tid; i < kBins; i += kSampleThreads) { sm.mass[i] = 0; sm.count[i] = 0; }
    __syncthreads();
    u64 all = 0;
    for (int i = tid; i < p.vocab; i += kSampleThreads) {
      const float l = row.at(i);
      if (l > -INFINITY) {
        const u64 w = wt.of(l);
        const int b = wt.bin(l);
        atomicAdd(&sm.count[b], 1);
        if (w) atomicAdd(&sm.mass[b], w);
        all += w;
      }
    }
    all = wave_sum(all);
    if (lane == 0) sm.wave_mass[wave] = all;
    __syncthreads();
    all = 0;
    for (int i = 0; i < kSampleWaves; ++i) all += sm.wave_mass[i];
    __syncthreads();
    kept.mass = all;
    if (by_count) kept = find_beginning(row, wt, Target{false, top_k, 0}, sm);
    if (by_mass) {
      const double target = ceil((double)top_p * (double)kept.mass);
      const u64 need = min(max((u64)target, (u64)1), kept.mass);
      const Beginning b = find_beginning(row, wt, Target{true, 0, need}, sm);
      if (b.limit > kept.limit) kept = b;
    }
  }
  const double least = min_p > 0.f ? (double)fminf(min_p, 1.f) : 0.0;
  // the kept weights of each wave's run of the row
  auto weight = [&](int i, bool& in) {
    const float l = row.at(i);
    in = l > -INFINITY && ((u64)order_key(l) << 32 | (unsigned)~i) >= kept.limit && !(wt.infinite && l != best);
    if (in && least > 0.0) in = wt.real(l) >= least;
    return in ? wt.of(l) : (u64)0;
  };
  const int per = ((p.vocab + kSampleWaves - 1) / kSampleWaves + kWave - 1) / kWave * kWave;
  const int begin = min(p.vocab, wave * per), end = min(p.vocab, begin + per);
  u64 mine = 0;
  int count = 0;
  for (int i = begin + lane; i < end; i += kWave) {
    bool in;
    mine += weight(i, in);
    count += in;
  }
  mine = wave_sum(mine);
  count = wave_sum(count);
  if (lane == 0) { sm.wave_mass[wave] = mine; sm.wave_count[wave] = count; }
  __syncthreads();
  u64 total = 0, before = 0;
  count = 0;
  for (int i = 0; i < kSampleWaves; ++i) {
    if (i < wave) before += sm.wave_mass[i];
    total += sm.wave_mass[i];
    count += sm.wave_count[i];
  }
  // the lowest index whose sum exceeds u W: the sum reaches floor(u W) + 1, at most W
  const u64 reach = min((u64)((double)u * (double)total) + 1, total);
  if (before < reach && before + mine >= reach) {
    for (int i = begin; i < end; i += kWave) {
      bool in = false;
      const u64 w = i + lane < end ? weight(i + lane, in) : 0;
      const u64 sum = before + wave_scan(w, lane);
      const unsigned long long hit = __ballot(sum >= reach);
      if (hit) {
        if (lane == __ffsll((long long)hit) - 1) {
          const float l = row.at(i + lane);
          const double z = l == best ? 0.0 : ((double)l - (double)best) / (double)temperature;
          finish(i + lane, (float)(z - log((double)total * (1.0 / (double)(1ull << kFraction)))), count);
        }
        break;
      }
      before = __shfl(sum, kWave - 1, kWave);
    }
  }
}

int launch_sample(const void* logits, int dtype, int64_t row_stride, int rows, int vocab, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, const float* uniform, int32_t* token,
                  float* logprob, int32_t* n_kept, hipStream_t stream) {
  const SampleParams p{logits, row_stride, vocab, temperature, top_k, top_p, min_p, uniform, token, logprob, n_kept};
  if (dtype == EARN_F32) hipLaunchKernelGGL(sample_kernel<float>, dim3(rows), dim3(kSampleThreads), 0, stream, p);
  else hipLaunchKernelGGL(sample_kernel<__bf16>, dim3(rows), dim3(kSampleThreads), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return EARN_OK;
  set_error("earn_sample: launch failed: %s", hipGetErrorString(e));
  return EARN_ERR_HIP;
}

}  // namespace earn
