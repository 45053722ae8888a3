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
//
// One workgroup a row.  A wave has a run of the row, 16 bytes a lane and unit, and the row stays in registers (UNITS units; 0:
// any number, read again in every pass).  Passes: the largest logit; a histogram over (l_max - l) / T; the few entries of the bin in
// which a beginning ends, ranked among each other; the kept weights' sums by wave, then by unit of the wave that u W falls to.
#include "common.h"

namespace earn {

typedef unsigned long long u64;
constexpr int kBins = 2048;            // of (l_max - l) / T in steps of 1/64; the last one holds everything from 31.98 on
constexpr int kBinsPerUnit = 64;
constexpr int kFraction = 44;          // exp(-31.98) 2^44 < 1/2: the last bin's weights are all zero
constexpr int kListMax = 1024;
constexpr int kExpSteps = 128;         // of the table of powers of two

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

template <int WAVES>
struct SampleSmem {
  u64 mass[kBins];
  int count[kBins];
  u64 list_w[kListMax];
  u64 list_key[kListMax];        // (order key, ~index): larger is earlier in the order
  double power[kExpSteps];       // 2^(i / kExpSteps)
  u64 wave_mass[WAVES];
  int wave_count[WAVES];
  float wave_best[WAVES];
  int wave_at[WAVES];
  int n_list, bin, found_count, found_index, hit_wave;
  float found_value;
  u64 before_mass, found_mass, hit_before, hit_total;
  int before_count;
};

template <typename X>
__device__ __forceinline__ X wave_sum(X x) {
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

// Weights of a row.  exp((l - best) / T) = 2^(n / 128) exp(r ln 2 / 128) with n whole and |r| <= 1/2: a table and the exponential series
// to the fourth power, whose next term is below 2^-49.
struct Weights {
  float best;         // the largest logit
  float bins;         // bins per unit of logit
  double scale;       // 128 log2(e) / T
  const double* power;
  __device__ __forceinline__ double real(float l) const {
    const double t = fmax(((double)l - (double)best) * scale, -1100.0 * kExpSteps);
    const double shifted = t + 0x1.8p52, r = t - (shifted - 0x1.8p52);
    const int n = (int)(unsigned)__double_as_longlong(shifted);
    constexpr double c = 0.69314718055994530942 / kExpSteps;
    const double e = __builtin_fma(r, __builtin_fma(r, __builtin_fma(r, __builtin_fma(r, c * c * c * c / 24, c * c * c / 6), c * c / 2), c), 1.0);
    return __builtin_amdgcn_ldexp(power[n & (kExpSteps - 1)] * e, n >> 7);
  }
  static __device__ __forceinline__ u64 whole(double w) {   // w 2^kFraction, rounded; w <= 1
    return (u64)__double_as_longlong(__builtin_fma(w, (double)(1ull << kFraction), 0x1p52)) & 0xfffffffffffffull;
  }
  __device__ __forceinline__ u64 of(float l) const { return whole(real(l)); }
  // monotone in l: rounding keeps the order of differences and products
  __device__ __forceinline__ int bin(float l) const { return (int)fminf((best - l) * bins, (float)(kBins - 1)); }
};

// 16 bytes at the alignment of an element
typedef unsigned int u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));

// The wave's run of the row: unit i, element e of lane is entry begin + (64 i + lane) E + e; -inf past the end and for NaN.
template <typename T, int UNITS, int WAVES>
struct Run {
  static constexpr int E = 16 / sizeof(T);
  const T* row;
  int vocab, begin, n_units, lane;
  bool infinite;                 // the best is +inf: those entries count as 0, all others as -inf
  u32x4 held[UNITS > 0 ? UNITS : 1];
  __device__ __forceinline__ u32x4 load(int i) const {
    const int at = begin + (kWave * i + lane) * E;
    u32x4 x;
    if (at + E <= vocab) {
      if constexpr (sizeof(T) == 4) x = *(const u32x4_at4*)(row + at);
      else x = *(const u32x4_at2*)(row + at);
    }
    else {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (sizeof(T) == 4) x[w] = at + w < vocab ? ((const unsigned*)row)[min(at + w, vocab - 1)] : 0xff800000u;
        else {
          const unsigned short* h = (const unsigned short*)row;
          const unsigned lo = at + 2 * w < vocab ? h[min(at + 2 * w, vocab - 1)] : 0xff80u, hi = at + 2 * w + 1 < vocab ? h[min(at + 2 * w + 1, vocab - 1)] : 0xff80u;
          x[w] = lo | hi << 16;
        }
      }
    }
    return x;
  }
  __device__ __forceinline__ void init(const T* row_, int vocab_, int wave, int lane_) {
    row = row_; vocab = vocab_; lane = lane_; infinite = false;
    const int per = ((vocab + WAVES - 1) / WAVES + kWave * E - 1) / (kWave * E);   // units of a wave
    begin = min(vocab, wave * per * (kWave * E));
    n_units = min(per, (vocab - begin + kWave * E - 1) / (kWave * E));
    if constexpr (UNITS > 0) {
#pragma unroll
      for (int i = 0; i < UNITS; ++i)
        if (i < n_units) held[i] = load(i);
    }
  }
  __device__ __forceinline__ float element(const u32x4& x, int e) const {
    float l;
    if constexpr (sizeof(T) == 4) l = __uint_as_float(x[e]);
    else l = e & 1 ? bf16_hi(x[e / 2]) : bf16_lo(x[e / 2]);
    if (infinite) return l == INFINITY ? 0.f : -INFINITY;
    return fmaxf(l, -INFINITY);
  }
  __device__ __forceinline__ int index(int i, int e) const { return begin + (kWave * i + lane) * E + e; }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {       // f(entry, logit)
    if constexpr (UNITS > 0) {
#pragma unroll
      for (int i = 0; i < UNITS; ++i)
        if (i < n_units) {
          u32x4 x = held[i];
          int at = index(i, 0);
          asm volatile("" : "+v"(x), "+v"(at));   // opaque: what one pass works out of them is not kept, in registers that there are not, for the next
#pragma unroll
          for (int e = 0; e < E; ++e) f(at + e, element(x, e));
        }
    } else {
      for (int i = 0; i < n_units; ++i) {
        const u32x4 x = load(i);
#pragma unroll
        for (int e = 0; e < E; ++e) f(index(i, e), element(x, e));
      }
    }
  }
};

// A beginning of the order: what comes before the logit `value`, and its equals up to entry `index`; `count` entries that weigh `mass`.
struct Beginning {
  float value;
  int index;
  u64 mass;
  int count;
  __device__ __forceinline__ bool has(int i, float l) const { return l > value || (l == value && i <= index); }
};

// Does an entry end the beginning that is looked for?  By count: it is the k-th.  By mass: it is the one that reaches the target.
struct Target {
  bool by_mass;
  int k;
  u64 mass;
  __device__ __forceinline__ bool hit(int before, u64 mass_before, int n, u64 w) const {
    return by_mass ? mass_before < mass && mass_before + w >= mass : before < k && before + n >= k;
  }
};

// The beginning that `target` ends, from the histogram; called by all threads.  There is one: k is at most the number of entries,
// the mass at most that of all.
template <typename R, int WAVES>
__device__ __forceinline__ Beginning find_beginning(const R& run, const Weights& wt, const Target target, SampleSmem<WAVES>& sm) {
  constexpr int THREADS = kWave * WAVES, PER = kBins / THREADS;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  // the bin that the target ends in
  int cs = 0;
  u64 ms = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) { cs += sm.count[PER * tid + i]; ms += sm.mass[PER * tid + i]; }
  const int cs_in = wave_scan(cs, lane);
  const u64 ms_in = wave_scan(ms, lane);
  __syncthreads();
  if (lane == kWave - 1) { sm.wave_count[wave] = cs_in; sm.wave_mass[wave] = ms_in; }
  if (tid == 0) sm.n_list = 0;
  __syncthreads();
  int cb = cs_in - cs;
  u64 mb = ms_in - ms;
  for (int i = 0; i < wave; ++i) { cb += sm.wave_count[i]; mb += sm.wave_mass[i]; }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = sm.count[PER * tid + i];
    const u64 m = sm.mass[PER * tid + i];
    if (target.hit(cb, mb, c, m)) { sm.bin = PER * tid + i; sm.before_count = cb; sm.before_mass = mb; }
    cb += c;
    mb += m;
  }
  __syncthreads();
  const int bin = sm.bin, before = sm.before_count;
  const u64 mass_before = sm.before_mass;
  if (sm.count[bin] <= kListMax) {
    run.each([&](int i, float l) {
      if (l > -INFINITY && wt.bin(l) == bin) {
        const int at = atomicAdd(&sm.n_list, 1);
        sm.list_w[at] = wt.of(l);
        sm.list_key[at] = (u64)order_key(l) << 32 | (unsigned)~i;
      }
    });
    __syncthreads();
    const int n = sm.n_list;
    for (int a = tid; a < n; a += THREADS) {
      const u64 key = sm.list_key[a];
      int cnt = before;
      u64 mass = mass_before;
      for (int b = 0; b < n; ++b) {
        const bool first = sm.list_key[b] > key;
        cnt += first ? 1 : 0;
        mass += first ? sm.list_w[b] : 0;
      }
      if (target.hit(cnt, mass, 1, sm.list_w[a])) {
        sm.found_value = key_value((unsigned)(key >> 32));
        sm.found_index = (int)~(unsigned)key;
        sm.found_count = cnt + 1;
        sm.found_mass = mass + sm.list_w[a];
      }
    }
    __syncthreads();
    return Beginning{sm.found_value, sm.found_index, sm.found_mass, sm.found_count};
  }
  // Too many for the list (mostly equal logits): the last key, bit by bit, then its equals in order of their index.
  auto reach = [&](unsigned key, int& cnt, u64& mass) {   // entries of the bin whose key is at least `key`
    int c = 0;
    u64 m = 0;
    run.each([&](int, float l) {
      if (l > -INFINITY && wt.bin(l) == bin && order_key(l) >= key) { ++c; m += wt.of(l); }
    });
    c = wave_sum(c);
    m = wave_sum(m);
    __syncthreads();
    if (lane == 0) { sm.wave_count[wave] = c; sm.wave_mass[wave] = m; }
    __syncthreads();
    cnt = before;
    mass = mass_before;
    for (int i = 0; i < WAVES; ++i) { cnt += sm.wave_count[i]; mass += sm.wave_mass[i]; }
  };
  unsigned t = 0;
  int cnt;
  u64 mass;
#pragma unroll 1
  for (int bit = 31; bit >= 0; --bit) {
    const unsigned with = t | 1u << bit;
    reach(with, cnt, mass);
    if (target.by_mass ? mass >= target.mass : cnt >= target.k) t = with;
  }
  reach(t + 1, cnt, mass);                        // what comes before the equals (t is a finite float's key)
  const float value = key_value(t);
  const u64 each_mass = wt.of(value);
  // the r-th equal one is the last
  const int r = target.by_mass ? (int)((target.mass - mass + each_mass - 1) / each_mass) : target.k - cnt;
  int mine = 0;
  run.each([&](int, float l) { mine += l == value ? 1 : 0; });
  mine = wave_sum(mine);
  __syncthreads();
  if (lane == 0) sm.wave_count[wave] = mine;
  __syncthreads();
  int at = 0;
  for (int i = 0; i < wave; ++i) at += sm.wave_count[i];
  if (at < r && at + mine >= r) {                 // the wave that holds it
    for (int i = 0; i < run.n_units; ++i) {
      const u32x4 x = run.load(i);
      int here = 0;
#pragma unroll
      for (int e = 0; e < R::E; ++e) here += run.element(x, e) == value ? 1 : 0;
      const int upto = at + wave_scan(here, lane);
      int own = upto - here;
#pragma unroll
      for (int e = 0; e < R::E; ++e)
        if (run.element(x, e) == value && ++own == r) sm.found_index = run.index(i, e);
      at = __shfl(upto, kWave - 1, kWave);
    }
  }
  __syncthreads();
  return Beginning{value, sm.found_index, mass + (u64)r * each_mass, cnt + r};
}

template <typename T, int UNITS, int WAVES>
__global__ __launch_bounds__(kWave * WAVES) void sample_kernel(SampleParams p) {
  constexpr int THREADS = kWave * WAVES;
  __shared__ SampleSmem<WAVES> sm;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), r = blockIdx.x;
  Run<T, UNITS, WAVES> run;
  run.init((const T*)p.logits + (long long)r * p.row_stride, p.vocab, wave, lane);
  const float temperature = p.temperature ? p.temperature[r] : 1.f;
  const int top_k = p.top_k ? p.top_k[r] : 0;
  const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f;
  float u = p.uniform[r];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  for (int i = tid; i < kExpSteps; i += THREADS) sm.power[i] = exp2((double)i / kExpSteps);
  for (int i = tid; i < kBins; i += THREADS) { sm.mass[i] = 0; sm.count[i] = 0; }
  float best = -INFINITY;
  run.each([&](int, float l) { best = fmaxf(best, l); });
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) best = fmaxf(best, __shfl_xor(best, o, kWave));
  if (lane == 0) sm.wave_best[wave] = best;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) best = fmaxf(best, sm.wave_best[i]);
  auto finish = [&](int token, float logprob, int count) {
    p.token[r] = token;
    if (p.logprob) p.logprob[r] = logprob;
    if (p.n_kept) p.n_kept[r] = count;
  };
  if (best == -INFINITY) { if (tid == 0) finish(-1, -INFINITY, 0); return; }
  if (!(temperature > 0.f) || top_k == 1 || !(top_p > 0.f)) {   // the first of the best
    int at = 0x7fffffff;
    run.each([&](int i, float l) { at = l == best ? min(at, i) : at; });
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) at = min(at, __shfl_xor(at, o, kWave));
    if (lane == 0) sm.wave_at[wave] = at;
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < WAVES; ++i) at = min(at, sm.wave_at[i]);
      finish(at, 0.f, 1);
    }
    return;
  }
  if (best == INFINITY) { run.infinite = true; best = 0.f; }

  Weights wt;
  wt.best = best;
  wt.scale = kExpSteps * 1.4426950408889634074 / (double)temperature;
  wt.bins = fminf((float)kBinsPerUnit / temperature, 3e38f);
  wt.power = sm.power;
  const bool by_mass = top_p < 1.f;
  Beginning kept{-INFINITY, -1, 0, 0};
  if (top_k > 0 || by_mass) {
    u64 all = 0;
    int n_finite = 0;
    run.each([&](int, float l) {
      if (l > -INFINITY) {
        const int b = wt.bin(l);
        atomicAdd(&sm.count[b], 1);
        ++n_finite;
        if (by_mass && b < kBins - 1) {
          const u64 w = wt.of(l);
          atomicAdd(&sm.mass[b], w);
          all += w;
        }
      }
    });
    all = wave_sum(all);
    n_finite = wave_sum(n_finite);
    if (lane == 0) { sm.wave_mass[wave] = all; sm.wave_count[wave] = n_finite; }
    __syncthreads();
    all = 0;
    n_finite = 0;
    for (int i = 0; i < WAVES; ++i) { all += sm.wave_mass[i]; n_finite += sm.wave_count[i]; }
    kept.mass = all;
#pragma unroll 1
    for (int which = top_k > 0 && top_k < n_finite ? 0 : 1; which < (by_mass ? 2 : 1); ++which) {
      const double least_mass = ceil((double)top_p * (double)kept.mass);
      const Target target{which == 1, top_k, which == 1 ? min(max((u64)least_mass, (u64)1), kept.mass) : 0};
      const Beginning b = find_beginning<Run<T, UNITS, WAVES>, WAVES>(run, wt, target, sm);
      if (which == 0 || b.value > kept.value || (b.value == kept.value && b.index < kept.index)) kept = b;
    }
  }
  const double least = min_p > 0.f ? (double)fminf(min_p, 1.f) : 0.0;
  auto weight = [&](int i, float l, bool& in) {
    in = kept.has(i, l);
    u64 w = 0;
    if (in) {
      const double x = wt.real(l);
      in = x >= least;
      w = in ? Weights::whole(x) : 0;
    }
    return w;
  };
  // the kept weights of each wave's run
  u64 mine = 0;
  int count = 0;
  run.each([&](int i, float l) {
    bool in;
    mine += weight(i, l, in);
    count += in ? 1 : 0;
  });
  mine = wave_sum(mine);
  count = wave_sum(count);
  __syncthreads();
  if (lane == 0) { sm.wave_mass[wave] = mine; sm.wave_count[wave] = count; }
  __syncthreads();
  u64 total = 0, before = 0;
  count = 0;
  for (int i = 0; i < WAVES; ++i) {
    if (i < wave) before += sm.wave_mass[i];
    total += sm.wave_mass[i];
    count += sm.wave_count[i];
  }
  // the lowest index whose sum exceeds u W: the sum reaches floor(u W) + 1, at most W
  const u64 reach = min((u64)((double)u * (double)total) + 1, total);
  if (before < reach && before + mine >= reach) {
    for (int i = 0; i < run.n_units; ++i) {
      const u32x4 x = run.load(i);
      u64 w[Run<T, UNITS, WAVES>::E], sum = 0;
#pragma unroll
      for (int e = 0; e < run.E; ++e) {
        bool in;
        w[e] = weight(run.index(i, e), run.element(x, e), in);
        sum += w[e];
      }
      const u64 upto = before + wave_scan(sum, lane);
      const unsigned long long hit = __ballot(upto >= reach);
      if (hit) {
        if (lane == __ffsll((long long)hit) - 1) {
          u64 at = upto - sum;
          bool done = false;
#pragma unroll
          for (int e = 0; e < run.E; ++e) {
            at += w[e];
            if (!done && at >= reach) {
              const float l = run.element(x, e);
              const double z = l == best ? 0.0 : ((double)l - (double)best) / (double)temperature;
              finish(run.index(i, e), (float)(z - log((double)total * (1.0 / (double)(1ull << kFraction)))), count);
              done = true;
            }
          }
        }
        break;
      }
      before = __shfl(upto, kWave - 1, kWave);
    }
  }
}

template <typename T>
static void launch_sample_t(const SampleParams& p, int rows, hipStream_t stream) {
  constexpr int E = 16 / sizeof(T), small = 4 * 4 * kWave * E, middle = 16 * 8 * kWave * E, large = 16 * 16 * kWave * E;
  if (p.vocab <= small) hipLaunchKernelGGL((sample_kernel<T, 4, 4>), dim3(rows), dim3(4 * kWave), 0, stream, p);
  else if (p.vocab <= middle) hipLaunchKernelGGL((sample_kernel<T, 8, 16>), dim3(rows), dim3(16 * kWave), 0, stream, p);
  else if (p.vocab <= large) hipLaunchKernelGGL((sample_kernel<T, 16, 16>), dim3(rows), dim3(16 * kWave), 0, stream, p);
  else hipLaunchKernelGGL((sample_kernel<T, 0, 16>), dim3(rows), dim3(16 * kWave), 0, stream, p);
}

int launch_sample(const void* logits, int dtype, int64_t row_stride, int rows, int vocab, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, const float* uniform, int32_t* token,
                  float* logprob, int32_t* n_kept, hipStream_t stream) {
  const SampleParams p{logits, row_stride, vocab, temperature, top_k, top_p, min_p, uniform, token, logprob, n_kept};
  if (dtype == EARN_F32) launch_sample_t<float>(p, rows, stream);
  else launch_sample_t<__bf16>(p, rows, stream);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return EARN_OK;
  set_error("earn_sample: launch failed: %s", hipGetErrorString(e));
  return EARN_ERR_HIP;
}

}  // namespace earn
