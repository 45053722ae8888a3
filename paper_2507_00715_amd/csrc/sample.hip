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
// One workgroup a row.  A wave has a run of the row, 16 bytes a lane and unit, which every pass reads again from the caches, four
// units at a time (held in registers, with the passes unrolled over them, a row of 32000 took as long: the code, 120 KB, came from
// memory instead).  What bounds a row is how many vector instructions its entries take on their one CU, so the passes over all
// entries are few and short:
//   - the largest logit;
//   - top-k up to kSmallK: the largest entries of every 16 bytes (of longer rows, of some of them together) stay in LDS; a histogram of
//     them over (l_max - l) / T gives a border that at least k entries reach, and few more: those are listed, and the rest happens in the
//     list;
//   - else top-k: a histogram of all entries; top-p: one of their weights; the entries of the bin in which a beginning ends are
//     ranked among each other, or found bit by bit where they are more than the list holds;
//   - the kept weights' sums by wave (gathered 64 at a time before their exponentials are taken, where few of the entries are kept;
//     with top-p in the same pass that lists the bin's), then by unit of the wave that u W falls to, all waves together.
#include <type_traits>

#include "common.h"

namespace earn {

typedef unsigned long long u64;
constexpr int kBins = 2048;            // of (l_max - l) / T in steps of 1/64; the last one holds everything from 31.98 on
constexpr int kBinsPerUnit = 64;
constexpr int kFraction = 44;          // exp(-31.98) 2^44 < 1/2: the last bin's weights are all zero
constexpr int kListMax = 1024;
constexpr int kSmallK = 512;           // largest top-k that is worked out in the list
constexpr int kGroups = 16384;         // groups of entries whose largest are kept in LDS
constexpr int kExpBits = 9, kExpSteps = 1 << kExpBits;   // of the table of powers of two

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
  u64 sorted[kSmallK];
  float group_best[WAVES > 4 ? kGroups : 4 * 4 * kWave];   // a lane's 16 bytes of one unit, or of the next 2, 4, ... units of longer rows
  int by_index[kSmallK];
  double power[kExpSteps];
  float queue[WAVES][2 * kWave];
  u64 wave_mass[WAVES];
  int wave_count[WAVES];
  float wave_best[WAVES];
  int wave_at[WAVES];
  int n_list, n_groups, bin, found_index, before_count;
  float found_value;
  u64 before_mass, kept_mass[WAVES];
  int kept_count[WAVES];
};

// Sums over a wave without trips through LDS: inclusive prefix sums inside rows of 16 lanes, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 x) {
  return (u64)(unsigned)moved<CTRL, ROWS>((int)(x >> 32)) << 32 | (unsigned)moved<CTRL, ROWS>((int)x);
}
template <typename X>
__device__ __forceinline__ X wave_scan(X x) {   // inclusive; all lanes
  x += moved<0x111, 0xf>(x);   // row_shr 1, 2, 4, 8
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);   // lane 15 of rows 0 and 2 to the rows behind them
  x += moved<0x143, 0xc>(x);   // lane 31 to the second half
  return x;
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, kWave - 1); }
__device__ __forceinline__ u64 last_lane(u64 x) { return (u64)(unsigned)last_lane((int)(x >> 32)) << 32 | (unsigned)last_lane((int)x); }
template <typename X>
__device__ __forceinline__ X wave_sum(X x) { return last_lane(wave_scan(x)); }

// Weights of a row, as doubles times 2^kFraction.  exp((l - best) / T) = 2^(n / 512) exp(r ln 2 / 512) with n whole and |r| <= 1/2: a
// table and the exponential series to the third power, whose next term is below 2^-46.
struct Weights {
  float best, half;   // the largest logit, half of it
  float bins;         // bins per half a unit of logit
  double scale;       // kExpSteps log2(e) / T
  double c1, c2, c3;  // of the series, in scalar registers
  const double* power;   // 2^(i / kExpSteps), times 2^kFraction
  __device__ __forceinline__ void init(float best_, float temperature, const double* power_) {
    best = best_;
    half = 0.5f * best_;
    bins = fminf(2.f * (float)kBinsPerUnit / temperature, 3e38f);
    scale = kExpSteps * 1.4426950408889634074 / (double)temperature;
    power = power_;
    constexpr double c = 0.69314718055994530942 / kExpSteps;
    c1 = c; c2 = c * c / 2; c3 = c * c * c / 6;
    asm("" : "+s"(c1), "+s"(c2), "+s"(c3));
  }
  __device__ __forceinline__ double real(float l) const {
    const double t = fmax(((double)l - (double)best) * scale, -1100.0 * kExpSteps);
    const double shifted = t + 0x1.8p52, r = t - (shifted - 0x1.8p52);
    const int n = (int)(unsigned)__double_as_longlong(shifted);
    const double e = __builtin_fma(r, __builtin_fma(r, __builtin_fma(r, c3, c2), c1), 1.0);
    return __builtin_amdgcn_ldexp(power[n & (kExpSteps - 1)] * e, n >> kExpBits);
  }
  static __device__ __forceinline__ u64 whole(double w) {   // rounded; w <= 2^kFraction
    return (u64)__double_as_longlong(w + 0x1p52) & 0xfffffffffffffull;
  }
  __device__ __forceinline__ u64 of(float l) const { return whole(real(l)); }
  // monotone in l: rounding keeps the order of differences and products.  (Halves: the difference of two logits may overflow.)
  __device__ __forceinline__ int bin(float l) const { return (int)fminf(__builtin_fmaf(l, -0.5f, half) * bins, (float)(kBins - 1)); }
};

// 16 bytes at the alignment of an element
typedef unsigned int u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));

// The wave's run of the row: unit i, element e of lane is entry begin + (64 i + lane) E + e; -inf past the end.
// (NaN fails every comparison below and falls into the last bin, where it is taken for none of the entries looked for.)
template <typename T, int WAVES>
struct Run {
  static constexpr int E = 16 / sizeof(T);
  const T* row;
  int vocab, units, begin, n_units, lane;   // units: of a wave's run, of the last ones fewer
  __device__ __forceinline__ u32x4 load(int i) const { return load_at(index(i, 0)); }
  __device__ __forceinline__ u32x4 load_whole(int at) const {
    if constexpr (sizeof(T) == 4) return *(const u32x4_at4*)((const char*)row + (unsigned)at * 4u);
    else return *(const u32x4_at2*)((const char*)row + (unsigned)at * 2u);
  }
  __device__ __forceinline__ u32x4 load_at(int at) const {
    u32x4 x;
    if (at + E <= vocab) x = load_whole(at);
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
    row = row_; vocab = vocab_; lane = lane_;
    units = ((vocab + WAVES - 1) / WAVES + kWave * E - 1) / (kWave * E);
    begin = min(vocab, wave * units * (kWave * E));
    n_units = min(units, (vocab - begin + kWave * E - 1) / (kWave * E));
  }
  __device__ __forceinline__ static float element(const u32x4& x, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(x[e]);
    else return e & 1 ? bf16_hi(x[e / 2]) : bf16_lo(x[e / 2]);
  }
  __device__ __forceinline__ int index(int i, int e) const { return begin + (kWave * i + lane) * E + e; }
  template <typename F>
  __device__ __forceinline__ void each_unit(F f) const {  // f(first entry, unit)
    constexpr int TOGETHER = 4;
    int i = 0;
#pragma unroll 1
    for (; i + TOGETHER <= n_units && begin + kWave * E * (i + TOGETHER) <= vocab; i += TOGETHER) {   // whole units
      const int at = index(i, 0);
      u32x4 x[TOGETHER];
#pragma unroll
      for (int k = 0; k < TOGETHER; ++k) x[k] = load_whole(at + kWave * E * k);
#pragma unroll
      for (int k = 0; k < TOGETHER; ++k) f(at + kWave * E * k, x[k]);
    }
#pragma unroll 1
    for (; i < n_units; ++i) f(index(i, 0), load(i));
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {       // f(entry, logit)
    each_unit([&](int at, const u32x4& x) {
#pragma unroll
      for (int e = 0; e < E; ++e) f(at + e, element(x, e));
    });
  }
};

// A beginning of the order: what comes before the logit `value`, and its equals up to entry `index`.
struct Beginning {
  float value;
  int index;
  __device__ __forceinline__ bool has(int i, float l) const { return l > value || (l == value && i <= index); }
};

// The bin in which the k-th entry lies (by sm.count), or in which the weights reach `share` (at most 1) of their sum (by sm.mass; that
// weight to `target`), and what the bins before it hold in sm; kBins: none.  Called by all threads.
template <bool BY_MASS, int WAVES>
__device__ __forceinline__ int find_bin(SampleSmem<WAVES>& sm, int k, double share, u64& target_mass) {
  constexpr int THREADS = kWave * WAVES, PER = kBins / THREADS;
  typedef typename std::conditional<BY_MASS, u64, int>::type Sum;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  __syncthreads();
  Sum own[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if constexpr (BY_MASS) own[i] = sm.mass[PER * tid + i]; else own[i] = sm.count[PER * tid + i];
    sum += own[i];
  }
  const Sum upto = wave_scan(sum);
  if (lane == kWave - 1) { if constexpr (BY_MASS) sm.wave_mass[wave] = upto; else sm.wave_count[wave] = upto; }
  if (tid == 0) { sm.bin = kBins; sm.n_list = sm.n_groups = 0; }
  __syncthreads();
  Sum before = upto - sum, all = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    Sum w;
    if constexpr (BY_MASS) w = sm.wave_mass[i]; else w = sm.wave_count[i];
    before += i < wave ? w : 0;
    all += w;
  }
  Sum target;
  if constexpr (BY_MASS) target = target_mass = min(max((u64)ceil(share * (double)all), (u64)1), all); else target = k;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < target && before + own[i] >= target) {
      sm.bin = PER * tid + i;
      if constexpr (BY_MASS) sm.before_mass = before; else sm.before_count = before;
    }
    before += own[i];
  }
  __syncthreads();
  return sm.bin;
}

// The index of the r-th entry (1, 2, ...) that equals `value`, in sm.found_index; there is one.  Called by all threads.
template <typename R, int WAVES>
__device__ __forceinline__ void find_equal(const R& run, float value, int r, SampleSmem<WAVES>& sm) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
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
      const int upto = at + wave_scan(here);
      int own = upto - here;
#pragma unroll
      for (int e = 0; e < R::E; ++e)
        if (run.element(x, e) == value && ++own == r) sm.found_index = run.index(i, e);
      at = last_lane(upto);
    }
  }
  __syncthreads();
}

// The beginning that the k-th entry ends, or the first entry at which the weights reach `mass`, of those in `within`, where the bin that
// it ends in, T / 64 wide, holds too many for the list: equal logits, flat rows, and large vocabularies at ordinary temperatures.  The last
// key, bit by bit, 33 passes over the row, then its equals in order of their index.  131072 normal logits, top-p 0.9: 731 us where their
// deviation is half of T, 74 where it is 2.5 T and the list holds them; 40000 equal ones 239-270 us.
// Called by all threads.
template <bool BY_MASS, typename R, int WAVES>
__device__ __forceinline__ Beginning find_bit_by_bit(const R& run, const Weights& wt, const Beginning& within, int bin, int before, u64 mass_before, int k,
                                                    u64 mass, SampleSmem<WAVES>& sm) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  auto reach = [&](unsigned key, int& cnt, u64& sum) {   // entries of the bin whose key is at least `key`
    int c = 0;
    u64 m = 0;
    run.each([&](int i, float l) {
      if (l > -INFINITY && wt.bin(l) == bin && order_key(l) >= key && within.has(i, l)) { ++c; m += BY_MASS ? wt.of(l) : 0; }
    });
    c = wave_sum(c);
    m = wave_sum(m);
    __syncthreads();
    if (lane == 0) { sm.wave_count[wave] = c; sm.wave_mass[wave] = m; }
    __syncthreads();
    cnt = before;
    sum = mass_before;
    for (int i = 0; i < WAVES; ++i) { cnt += sm.wave_count[i]; sum += sm.wave_mass[i]; }
  };
  unsigned t = 0;
  int cnt;
  u64 sum;
#pragma unroll 1
  for (int bit = 31; bit >= -1; --bit) {          // the last round: what comes before the equals (t is a finite float's key)
    const unsigned with = bit >= 0 ? t | 1u << bit : t + 1;
    reach(with, cnt, sum);
    if (bit >= 0 && (BY_MASS ? sum >= mass : cnt >= k)) t = with;
  }
  const float value = key_value(t);
  const u64 each_mass = BY_MASS ? wt.of(value) : 0;
  // the r-th equal one is the last
  const int r = BY_MASS ? (int)((mass - sum + each_mass - 1) / each_mass) : k - cnt;
  find_equal(run, value, r, sm);
  return Beginning{value, sm.found_index};
}

// Sum over the workgroup, in every thread.
template <int WAVES>
__device__ __forceinline__ u64 block_sum(u64 x, SampleSmem<WAVES>& sm) {
  x = wave_sum(x);
  __syncthreads();
  if (threadIdx.x % kWave == 0) sm.wave_mass[threadIdx.x / kWave] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) x += sm.wave_mass[i];
  return x;
}

// What the threads need of the row's parameters to finish it.
struct Draw { double u, temperature; float top_p; double least; int top_k; };   // least: min-p's weight, times 2^kFraction
// u W falls to the first sum that reaches this
__device__ __forceinline__ u64 reach_of(double u, u64 total) { return min((u64)(u * (double)total) + 1, total); }
__device__ __forceinline__ float logprob_of(float l, float best, double temperature, u64 total) {
  const double z = l == best ? 0.0 : ((double)l - (double)best) / temperature;
  return (float)(z - log((double)total * (1.0 / (double)(1ull << kFraction))));
}

// Inclusive prefix sums over the workgroup's threads, on top of `base`; base then is the sum of all.
template <int WAVES>
__device__ __forceinline__ u64 block_scan(u64 x, u64& base, SampleSmem<WAVES>& sm) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  x = wave_scan(x);
  __syncthreads();
  if (lane == kWave - 1) sm.wave_mass[wave] = x;
  __syncthreads();
  x += base;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    const u64 m = sm.wave_mass[i];
    x += i < wave ? m : 0;
    base += m;
  }
  return x;
}

// Top-k with the rest in the list: its n entries hold the first k.  They are put in order by counting who comes before whom (four
// threads an entry), summed up in that order for top-p, then in the order of their indices for the draw.
template <int WAVES>
__device__ __forceinline__ void draw_from_list(const SampleParams& p, const Weights& wt, const Draw& d, int n, SampleSmem<WAVES>& sm) {
  constexpr int THREADS = kWave * WAVES;
  const int tid = threadIdx.x, part = tid % 4, r = blockIdx.x, k = d.top_k;
  auto quad = [](int x) { x += __shfl_xor(x, 1, kWave); return x + __shfl_xor(x, 2, kWave); };
#pragma unroll 1
  for (int a0 = 0; a0 < n; a0 += THREADS / 4) {
    const int a = a0 + tid / 4;
    const u64 key = a < n ? sm.list_key[a] : 0;
    int rank = 0;
#pragma unroll 4
    for (int b = part; b < n; b += 4) rank += sm.list_key[b] > key ? 1 : 0;
    rank = quad(rank);
    if (part == 0 && a < n && rank < k) sm.sorted[rank] = key;
  }
  __syncthreads();
  // in order: what of the first k top-p and min-p keep
  u64 first_k = 0, total = 0;
  constexpr int ROUNDS = (kSmallK + THREADS - 1) / THREADS;
  u64 w[ROUNDS], upto[ROUNDS];
#pragma unroll
  for (int s = 0; s < ROUNDS; ++s) {
    const int i = s * THREADS + tid;
    w[s] = i < k ? wt.of(key_value((unsigned)(sm.sorted[i] >> 32))) : 0;
    upto[s] = s * THREADS < k ? block_scan(w[s], first_k, sm) : 0;
  }
  const u64 need = d.top_p < 1.f ? min(max((u64)ceil((double)d.top_p * (double)first_k), (u64)1), first_k) : ~0ull;
  int m = 0;
#pragma unroll
  for (int s = 0; s < ROUNDS; ++s) {
    const int i = s * THREADS + tid;
    const bool keep = i < k && upto[s] - w[s] < need && wt.real(key_value((unsigned)(sm.sorted[i] >> 32))) >= d.least;
    m += keep ? 1 : 0;
    if (i < k) sm.list_w[i] = w[s];
  }
  m = (int)block_sum((u64)m, sm);                 // the first m
  // by index
#pragma unroll 1
  for (int a0 = 0; a0 < m; a0 += THREADS / 4) {
    const int a = a0 + tid / 4;
    const unsigned index = a < m ? ~(unsigned)sm.sorted[a] : 0;
    int rank = 0;
#pragma unroll 4
    for (int b = part; b < m; b += 4) rank += ~(unsigned)sm.sorted[b] < index ? 1 : 0;
    rank = quad(rank);
    if (part == 0 && a < m) sm.by_index[rank] = a;
  }
  __syncthreads();
  int at[ROUNDS];
#pragma unroll
  for (int s = 0; s < ROUNDS; ++s) {
    const int i = s * THREADS + tid;
    at[s] = i < m ? sm.by_index[i] : 0;
    w[s] = i < m ? sm.list_w[at[s]] : 0;
    upto[s] = s * THREADS < m ? block_scan(w[s], total, sm) : 0;
  }
  const u64 reach = reach_of(d.u, total);
#pragma unroll
  for (int s = 0; s < ROUNDS; ++s) {
    if (s * THREADS + tid >= m || !(upto[s] - w[s] < reach && upto[s] >= reach)) continue;
    const u64 key = sm.sorted[at[s]];
    p.token[r] = (int)~(unsigned)key;
    if (p.logprob) p.logprob[r] = logprob_of(key_value((unsigned)(key >> 32)), wt.best, d.temperature, total);
    if (p.n_kept) p.n_kept[r] = m;
  }
}

template <typename T, int WAVES>
__global__ __launch_bounds__(kWave * WAVES) void sample_kernel(SampleParams p) {
  constexpr int THREADS = kWave * WAVES;
  __shared__ SampleSmem<WAVES> sm;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), r = blockIdx.x;
  Run<T, WAVES> run;
  run.init((const T*)p.logits + (long long)r * p.row_stride, p.vocab, wave, lane);
  const float temperature = p.temperature ? p.temperature[r] : 1.f;
  const int top_k = p.top_k ? p.top_k[r] : 0;
  const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f;
  float u = p.uniform[r];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  for (int i = tid; i < kExpSteps; i += THREADS) sm.power[i] = exp2((double)i / kExpSteps + kFraction);
  for (int i = tid; i < kBins; i += THREADS) { sm.mass[i] = 0; sm.count[i] = 0; }
  typedef Run<T, WAVES> R;
  int shift = 0;                                  // 2^shift units a group
  while ((run.units + (1 << shift) - 1) >> shift > (int)(sizeof(sm.group_best) / sizeof(float)) / THREADS) ++shift;
  // (with fewer groups than 4 k, the border lies so deep that the list holds most of the row: 935 tokens, k = 115, 21 us for 10)
  const bool few = top_k > 1 && top_k <= kSmallK && (long long)4 * top_k * (R::E << shift) <= p.vocab;
  float* group_best = sm.group_best + wave * ((run.units + (1 << shift) - 1) >> shift) * kWave + lane;
  float best = -INFINITY;
  if (few) {                                      // the groups' largest stay: a thread reads what it wrote
    run.each_unit([&](int at, const u32x4& x) {
      const int i = (at - run.begin) / (kWave * R::E);
      float most = i & ((1 << shift) - 1) ? group_best[(i >> shift) * kWave] : -INFINITY;
#pragma unroll
      for (int e = 0; e < R::E; ++e) { const float l = run.element(x, e); most = l > most ? l : most; }
      group_best[(i >> shift) * kWave] = most;
      best = fmaxf(best, most);
    });
  } else run.each([&](int, float l) { best = l > best ? l : best; });
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
  if (best == INFINITY) {                         // the infinite ones alone, at equal weights: the first of them by index
    int n = 0;
    run.each([&](int, float l) { n += l == INFINITY ? 1 : 0; });
    u64 m = block_sum((u64)n, sm);
    if (top_k > 0 && (u64)top_k < m) m = (u64)top_k;
    if (top_p < 1.f) m = min(max((u64)ceil((double)top_p * (double)m), (u64)1), m);
    find_equal(run, INFINITY, (int)reach_of((double)u, m), sm);
    if (tid == 0) finish(sm.found_index, (float)-log((double)m), (int)m);
    return;
  }

  Weights wt;
  wt.init(best, temperature, sm.power);
  const Draw d{(double)u, (double)temperature, top_p, min_p > 0.f ? (double)fminf(min_p, 1.f) * (double)(1ull << kFraction) : 0.0, top_k};
  Beginning kept{-INFINITY, -1};
  u64 unused;
  auto list_key = [&](int i, float l) {
    const int at = atomicAdd(&sm.n_list, 1);
    if (at < kListMax) sm.list_key[at] = (u64)order_key(l) << 32 | (unsigned)~i;
  };
  bool limited = false;
  if (top_k > 0) {
    if (few) {
      const int groups = (run.n_units + (1 << shift) - 1) >> shift;
#pragma unroll 4
      for (int i = 0; i < groups; ++i) {
        const float most = group_best[i * kWave];
        if (most > -INFINITY) atomicAdd(&sm.count[wt.bin(most)], 1);
      }
      const int bin = find_bin<false>(sm, top_k, 0.0, unused);
      if (bin < kBins - 1) {
        // the groups that reach it, then their entries, a unit a thread: one trip to memory for all of them
        int* reaching = (int*)sm.list_w;
#pragma unroll 4
        for (int i = 0; i < groups; ++i)
          if (wt.bin(group_best[i * kWave]) <= bin) {
            const int at = atomicAdd(&sm.n_groups, 1);
            if (at < 2 * kListMax) reaching[at] = run.index(i << shift, 0);
          }
        __syncthreads();
        const int n_groups = sm.n_groups;
        if (n_groups <= 2 * kListMax) {
          for (int g = tid; g < n_groups << shift; g += THREADS) {
            const int at = reaching[g >> shift] + (g & ((1 << shift) - 1)) * (kWave * R::E);   // (the last group's may lie behind the row, or be the next wave's)
            if ((g & ((1 << shift) - 1)) && at / (run.units * (kWave * R::E)) != reaching[g >> shift] / (run.units * (kWave * R::E))) continue;
            const u32x4 x = run.load_at(at);
#pragma unroll
            for (int e = 0; e < R::E; ++e) {
              const float l = run.element(x, e);
              if (wt.bin(l) <= bin) list_key(at + e, l);
            }
          }
        } else if (tid == 0) sm.n_list = kListMax + 1;
        __syncthreads();
        const int n = sm.n_list;
        if (n <= kListMax) { draw_from_list(p, wt, d, n, sm); return; }
      }
      // too few groups, too many equal entries, or far ones: all entries count
      __syncthreads();
      for (int i = tid; i < kBins; i += THREADS) sm.count[i] = 0;
      __syncthreads();
    }
    int n_finite = 0;
    run.each([&](int, float l) {
      if (l > -INFINITY) { atomicAdd(&sm.count[wt.bin(l)], 1); ++n_finite; }
    });
    limited = block_sum((u64)n_finite, sm) > (u64)top_k;
    if (limited) {
      const int bin = find_bin<false>(sm, top_k, 0.0, unused), before = sm.before_count;
      run.each([&](int i, float l) { if (l > -INFINITY && wt.bin(l) == bin) list_key(i, l); });
      __syncthreads();
      const int n = sm.n_list;
      if (n <= kListMax) {
        for (int a = tid; a < n; a += THREADS) {
          const u64 key = sm.list_key[a];
          int rank = before;
          for (int b = 0; b < n; ++b) rank += sm.list_key[b] > key ? 1 : 0;
          if (rank == top_k - 1) { sm.found_value = key_value((unsigned)(key >> 32)); sm.found_index = (int)~(unsigned)key; }
        }
        __syncthreads();
        kept = Beginning{sm.found_value, sm.found_index};
      } else kept = find_bit_by_bit<false>(run, wt, kept, bin, before, 0, top_k, 0, sm);
    }
  }
  // the kept weights of each wave's run
  auto weight = [&](float l, bool& in) {          // of an entry of the beginning
    const double x = wt.real(l);
    in = x >= d.least;
    return in ? Weights::whole(x) : (u64)0;
  };
  u64 mine = 0;
  int count = 0, waiting = 0;
  float* queue = sm.queue[wave];
  auto take = [&](int n) {                        // the first n <= 64 of the queue
    bool in;
    const u64 w = weight(queue[lane], in);
    if (lane < n) { mine += w; count += in ? 1 : 0; }
  };
  // few entries of many, as a rule: gathered before their weights are worked out
  auto gather = [&](bool has, float l) {
    const unsigned long long who = __ballot(has);
    if (who == 0) return;
    if (has) queue[waiting + __popcll(who & ((1ull << lane) - 1))] = l;
    asm volatile("" ::: "memory");                // the wave's LDS operations complete in order: only the compiler has to keep theirs
    waiting += __popcll(who);
    if (waiting >= kWave) {
      take(kWave);
      const float rest = queue[kWave + lane];
      asm volatile("" ::: "memory");
      queue[lane] = rest;
      asm volatile("" ::: "memory");
      waiting -= kWave;
    }
  };
  bool summed = false;
  if (top_p < 1.f) {
    auto add_mass = [&](float l, int b) { atomicAdd(&sm.mass[b], wt.of(l)); };
    if (limited) run.each([&](int i, float l) {
      const int b = wt.bin(l);
      if (b < kBins - 1 && kept.has(i, l)) add_mass(l, b);
    });
    else run.each([&](int, float l) {
      const int b = wt.bin(l);
      if (b < kBins - 1) add_mass(l, b);
    });
    u64 need;
    const int bin = find_bin<true>(sm, 0, (double)top_p, need);
    const u64 before = sm.before_mass;
    if (tid < WAVES) { sm.kept_mass[tid] = 0; sm.kept_count[tid] = 0; }
    run.each([&](int i, float l) {
      const int b = wt.bin(l);
      const bool in = !limited || kept.has(i, l);
      if (in && b == bin) list_key(i, l);
      gather(in && b < bin, l);
    });
    __syncthreads();
    const int n = sm.n_list;
    if (n <= kListMax) {
      summed = true;
      for (int a = tid; a < n; a += THREADS) sm.list_w[a] = wt.of(key_value((unsigned)(sm.list_key[a] >> 32)));
      __syncthreads();
      for (int a = tid; a < n; a += THREADS) {
        const u64 key = sm.list_key[a], own = sm.list_w[a];
        u64 weighed = before;
        for (int b = 0; b < n; ++b) weighed += sm.list_key[b] > key ? sm.list_w[b] : 0;
        if (weighed >= need) continue;            // behind the beginning
        const float l = key_value((unsigned)(key >> 32));
        const int i = (int)~(unsigned)key, holder = i / (run.units * (kWave * R::E));
        bool in;
        const u64 w = weight(l, in);
        if (in) { atomicAdd(&sm.kept_mass[holder], w); atomicAdd(&sm.kept_count[holder], 1); }
        if (weighed + own >= need) { sm.found_value = l; sm.found_index = i; }
      }
      __syncthreads();
      kept = Beginning{sm.found_value, sm.found_index};
      if (waiting > 0) take(waiting);
      mine += lane == 0 ? sm.kept_mass[wave] : 0;
      count += lane == 0 ? sm.kept_count[wave] : 0;
    } else {
      kept = find_bit_by_bit<true>(run, wt, kept, bin, 0, before, 0, need, sm);
      mine = 0;
      count = waiting = 0;
    }
    limited = true;
  }
  // min-p alone keeps few entries too: those in bins up to its own border's, rounding included, are looked at
  // (19 rows of 109963 tokens: 31 us for 38)
  const int last_bin = d.least > 0.0 ? (int)fmin(-log(d.least * (1.0 / (double)(1ull << kFraction))) * kBinsPerUnit + 2.0, (double)kBins) : kBins;
  if (!summed && (limited || last_bin < kBins - 1)) {
    run.each([&](int i, float l) { gather(kept.has(i, l) && wt.bin(l) <= last_bin, l); });
    if (waiting > 0) take(waiting);
  } else if (!summed) {
    run.each([&](int, float l) {
      if (l > -INFINITY) {
        bool in;
        mine += weight(l, in);
        count += in ? 1 : 0;
      }
    });
  }
  mine = wave_sum(mine);
  count = wave_sum(count);
  __syncthreads();
  if (lane == 0) { sm.wave_mass[wave] = mine; sm.wave_count[wave] = count; }
  __syncthreads();
  u64 total = 0;
  count = 0;
  for (int i = 0; i < WAVES; ++i) { total += sm.wave_mass[i]; count += sm.wave_count[i]; }
  const u64 reach = reach_of(d.u, total);
  u64 before = 0;
  int hit = 0;                                    // the wave whose run holds the token
  while (before + sm.wave_mass[hit] < reach) before += sm.wave_mass[hit++];
  const int first = hit * run.units * (kWave * R::E);
  for (int i0 = 0; i0 < run.units; i0 += WAVES) {  // its units, one a wave
    const int at = first + (kWave * (i0 + wave) + lane) * R::E;
    u64 w[R::E], sum = 0;
    u32x4 x = u32x4{0u, 0u, 0u, 0u};
    if (i0 + wave < run.units) {
      x = run.load_at(at);
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        const float l = run.element(x, e);
        bool in = false;
        w[e] = at + e < p.vocab && kept.has(at + e, l) ? weight(l, in) : 0;
        sum += w[e];
      }
    }
    const u64 upto = wave_scan(sum);
    __syncthreads();
    if (lane == kWave - 1) sm.wave_mass[wave] = upto;
    __syncthreads();
    u64 mine_before = before;
    for (int i = 0; i < WAVES; ++i) {
      if (i < wave) mine_before += sm.wave_mass[i];
      before += sm.wave_mass[i];
    }
    u64 so_far = mine_before + upto - sum;
    if (so_far < reach && so_far + sum >= reach) {   // one lane of one wave
      bool done = false;
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        so_far += w[e];
        if (!done && so_far >= reach) {
          finish(at + e, logprob_of(run.element(x, e), best, d.temperature, total), count);
          done = true;
        }
      }
    }
    if (before >= reach) break;
  }
}

template <typename T>
static void launch_sample_t(const SampleParams& p, int rows, hipStream_t stream) {
  if (p.vocab <= 4 * 4 * kWave * 16 / (int)sizeof(T)) hipLaunchKernelGGL((sample_kernel<T, 4>), dim3(rows), dim3(4 * kWave), 0, stream, p);
  else hipLaunchKernelGGL((sample_kernel<T, 16>), dim3(rows), dim3(16 * kWave), 0, stream, p);
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
