// Caches in pages: a stream's rows lie in pages of `page_size` rows, [n_pages, Hkv, page_size, d], that a table names in the
// order of its rows.  A (page, kv head) is contiguous, so that the rows a workgroup reads for one kv head are.
//   paged_store_kernel   rows of a prefill to their pages
//   paged_decode_kernel  one new token per stream: append, then attention over the pages (paper Section 2.2, Eq. 4)
//   paged_join_kernel    joins the splits of long caches; running sums of the weights every row received
//   evict_select_kernel, evict_move_kernel  the rows of largest sums, to fresh pages
// No value of a table or a length reaches past the pools: a page number outside them names no page (its rows are not
// attended, stored to it is nothing).
#include <type_traits>

#include "common.h"
#include "decode_pieces.h"

namespace earn {

// Pools and tables, as all kernels here take them.
struct Pages {
  void* k; void* v;            // [n_pages, hkv, page_size, d]
  const int32_t* table;        // [streams, max_pages]
  int max_pages, n_pages, page_size, hkv;
  FastDiv by_page;             // row -> page of the stream
};
// The stream's page that holds row r, -1: none.  (r < max_pages * page_size)
__device__ __forceinline__ int page_of_row(const Pages& pg, int u, int r, int& in_page) {
  const int at = (int)pg.by_page.div((unsigned)r);
  in_page = r - at * pg.page_size;
  const int page = pg.table[(long long)u * pg.max_pages + at];
  return (unsigned)page < (unsigned)pg.n_pages ? page : -1;
}
// Element offset of row `in_page` of kv head c in a pool.
template <int D>
__device__ __forceinline__ long long row_offset(const Pages& pg, int page, int c, int in_page) {
  return (((long long)page * pg.hkv + c) * pg.page_size + in_page) * D;
}
__device__ __forceinline__ int capacity_of(const Pages& pg) {   // rows that a table's pages hold
  return (int)min((long long)pg.max_pages * pg.page_size, 0x7fffff00ll);
}

// ------------------------------------------------------------------------------------------------------------------
// store: a copy, four times 16 bytes of a K and a V row per thread, all asked for before the places are looked up.  256 prompts of
// 64-1024 rows, 2 heads of 128 (180 MB read and written): 40 us, 4.5 TB/s, of 35 that a large copy takes.  (One unit a thread 48; a
// search for every unit's sequence instead of one a workgroup 45.)
// ------------------------------------------------------------------------------------------------------------------
constexpr int kStoreUnits = 4;
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_store_kernel(const u32x4* __restrict__ k, const u32x4* __restrict__ v, Pages pg,
                                                          const int32_t* __restrict__ cu, const int32_t* __restrict__ start,
                                                          int batch, int total, FastDiv by_heads) {
  constexpr int UPR = D * (int)sizeof(T) / 16;   // 16-byte units of a row
  constexpr int STEP = 256 / UPR;                // rows (token, kv head) of 256 units
  const int unit = threadIdx.x % UPR;
  const long long row0 = (long long)blockIdx.x * (STEP * kStoreUnits) + threadIdx.x / UPR, rows = (long long)total * pg.hkv;
  u32x4 x[kStoreUnits], y[kStoreUnits];
  long long to[kStoreUnits];
#pragma unroll
  for (int i = 0; i < kStoreUnits; ++i) {
    const long long row = row0 + i * STEP;
    to[i] = -1;
    if (row >= rows) continue;
    x[i] = __builtin_nontemporal_load(k + row * UPR + unit);
    y[i] = __builtin_nontemporal_load(v + row * UPR + unit);
  }
  // the sequence of the workgroup's first token, looked up once; later ones are the same or follow it
  auto token_of = [&](long long row) { return rows < 0x7fffffff ? (int)by_heads.div((unsigned)row) : (int)(row / pg.hkv); };
  int s = find_seq(cu, batch, token_of((long long)blockIdx.x * (STEP * kStoreUnits)));
#pragma unroll
  for (int i = 0; i < kStoreUnits; ++i) {
    const long long row = row0 + i * STEP;
    if (row >= rows) continue;
    const int token = token_of(row), c = (int)(row - (long long)token * pg.hkv);
    while (s + 1 < batch && cu[s + 1] <= token) ++s;
    int b0, n;
    clamped_bounds(cu, s, total, total, b0, n);
    if (token < b0 || token >= b0 + n) continue;   // behind the last sequence
    const long long r = (long long)(token - b0) + (start ? start[s] : 0);
    if (r < 0 || r >= capacity_of(pg)) continue;
    int in_page;
    const int page = page_of_row(pg, s, (int)r, in_page);
    if (page >= 0) to[i] = row_offset<D>(pg, page, c, in_page) * (long long)sizeof(T) / 16 + unit;
  }
#pragma unroll
  for (int i = 0; i < kStoreUnits; ++i) {
    if (to[i] < 0) continue;
    ((u32x4*)pg.k)[to[i]] = x[i];
    ((u32x4*)pg.v)[to[i]] = y[i];
  }
}

// ------------------------------------------------------------------------------------------------------------------
// decode
// ------------------------------------------------------------------------------------------------------------------
// The vector form (fp32): a row is spread over d / 8 lanes, a wave takes whole rows, every lane keeps softmax states of up to 8 query
// heads over its share of them (larger groups: a workgroup each for 8 heads, which read the rows again: 16 streams of 8000 rows, heads of
// 128, 8 / 1 49 us, 16 / 1 81).  Bound by HBM, with the vector ALU near it: 8 streams of 16384 rows, 32 / 8 heads of 128 (1.07 GB), 217 us, 4.95
// TB/s; one of 32768 (268 MB) 63.
constexpr int kPagedThreads = 256, kPagedWaves = kPagedThreads / kWave;
constexpr int kPagedMaxChunk = 2048;   // rows of a split: its page numbers lie in LDS

// What stands among the scores for a row that is not there, and weighs 0 whatever the others are.  A signalling NaN, which no sum or product
// gives: a score that is -inf, or NaN, is a row's own.
constexpr unsigned kNoRow = 0x7fa00000u;

struct PagedParams {
  Pages pg;
  const void* q; const void* k_new; const void* v_new; const int32_t* q_pos; const int32_t* cache_len;
  const float* w_in; float* w_out;       // [streams, hkv, w_cap]
  void* out;
  float* part_o; float* part_ml;         // [streams, hq, n_splits, d], [.., 2]
  float* scores;                         // [streams, hq, score_stride], base-2 exponents; kNoRow: a row without a page
  int hq, hkv, w_cap, max_len, n_splits, chunk, score_stride, join_rows;
  float scale_log2;
  RopeTable rope;
  HeadMap heads;
};

// rows of stream u before this step, -1: an idle stream
__device__ __forceinline__ int length_of(const int32_t* cache_len, int u, int max_len, const Pages& pg) {
  const int n = cache_len[u];
  return n < 0 ? -1 : min(min(n, max_len), capacity_of(pg));
}

// The sums of rows [j0, j1) of a (stream, kv head), by the whole workgroup: old sums and the first head's scores are asked for
// before `states` gives the heads' (reference, 1 / sum) in LDS, and waits for all threads.
constexpr int kWeightRows = 4 * kPagedThreads;   // of one round of kPagedThreads
template <int THREADS, typename States>
__device__ __forceinline__ void add_weights(const PagedParams& p, int u, int c, int n, int j0, int j1, const f32x2* state, States states) {
  const int gq = p.hq / p.hkv, tid = threadIdx.x;
  const unsigned* scores = (const unsigned*)p.scores + ((long long)u * p.hq + c * gq) * p.score_stride;
  const long long to = ((long long)u * p.hkv + c) * p.w_cap;
  bool first = true;
  for (int jb = j0; jb < j1; jb += 4 * THREADS) {
    float w[4], old[4];
    unsigned s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = jb + i * THREADS + tid;
      w[i] = 0.f;
      old[i] = j < j1 && j < n && p.w_in ? p.w_in[to + j] : 0.f;
      s[i] = j < j1 ? scores[j] : kNoRow;
    }
    if (first) { states(); first = false; }
    for (int a = 0; a < gq; ++a) {
      if (a > 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = jb + i * THREADS + tid;
          s[i] = j < j1 ? scores[(long long)a * p.score_stride + j] : kNoRow;
        }
      }
      const f32x2 st = state[a];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] += s[i] == kNoRow ? 0.f : __builtin_amdgcn_exp2f(__uint_as_float(s[i]) - st[0]) * st[1];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = jb + i * THREADS + tid;
      if (j < j1) p.w_out[to + j] = old[i] + w[i];
    }
  }
}

// One head's 8 elements of a workgroup's result: a split's state, or the output.
template <typename T, int D>
__device__ __forceinline__ void finish_group(const PagedParams& p, long long first_head, int slot_head, int z, int e, float m, float l, float* x) {
  if (p.part_o) {
    const long long slot = (first_head + slot_head) * p.n_splits + z;
    *(f32x4*)(p.part_o + slot * D + e) = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4*)(p.part_o + slot * D + e + 4) = f32x4{x[4], x[5], x[6], x[7]};
    if (e == 0) *(f32x2*)(p.part_ml + slot * 2) = f32x2{m, l};
  } else {
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= inv;
    Row8<T>::store((T*)p.out + (first_head + head_of_slot(p.heads, slot_head)) * D + e, x);
  }
}

template <typename T, int D, int GQ>
__global__ __launch_bounds__(kPagedThreads) void paged_decode_kernel(PagedParams p) {
  constexpr int LPK = D / 8, KPW = kWave / LPK;      // lanes per row, rows per wave instruction
  constexpr int NP = GQ >= 8 ? 2 : Row8<T>::kRowsInFlight;
  constexpr int STEP = kPagedWaves * KPW;
  __shared__ int pages[kPagedMaxChunk + 2];
  __shared__ float merge[kPagedWaves][GQ][LPK][10];
  __shared__ f32x2 states[GQ];
  const int gq = p.hq / p.hkv, parts = (gq + GQ - 1) / GQ;
  const int z = blockIdx.z, c = blockIdx.x / parts, u = blockIdx.y, a0 = (int)(blockIdx.x % parts) * GQ;
  const int na = min(gq - a0, GQ);                   // query heads of this workgroup
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, sub = lane % LPK, kk = lane / LPK;
  const int n = length_of(p.cache_len, u, p.max_len, p.pg);
  if (n < 0) {                                       // idle: zeros
    if (z == 0)
      for (int i = tid; i < na * LPK; i += kPagedThreads) {
        const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        Row8<T>::store((T*)p.out + ((long long)u * p.hq + head_of_slot(p.heads, c * gq + a0 + i / LPK)) * D + i % LPK * 8, zero);
      }
    return;
  }
  const int j_begin = z * p.chunk, j_end = min(n + 1, j_begin + p.chunk);
  if (j_begin >= j_end) return;
  const bool has_new = j_end == n + 1;
  const int page0 = (int)p.pg.by_page.div((unsigned)j_begin);
  {
    const int last = (int)p.pg.by_page.div((unsigned)max(j_begin, min(j_end, n) - 1));
    for (int i = page0 + tid; i <= min(last, p.pg.max_pages - 1); i += kPagedThreads) {
      const int page = p.pg.table[(long long)u * p.pg.max_pages + i];
      pages[i - page0] = (unsigned)page < (unsigned)p.pg.n_pages ? page : -1;
    }
  }
  // queries and the new key, rotated
  float cs[8], sn[8];
  const float pos = (float)p.q_pos[u];
  const int e0 = (sub * 8) % (D / 2);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = 1.f; sn[i] = 0.f;
    if (p.rope.enabled) sincos_turns_precise(rope_turns(pos, p.rope.hi[e0 + i], p.rope.lo[e0 + i]), &sn[i], &cs[i]);
  }
  const bool upper = sub * 8 >= D / 2;
  auto rotate = [&](float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float other = __shfl_xor(x[i], LPK / 2, kWave);
      x[i] = upper ? __builtin_fmaf(x[i], cs[i], other * sn[i]) : __builtin_fmaf(x[i], cs[i], -(other * sn[i]));
    }
  };
  float qv[GQ][8], kn[8], vn[8];
#pragma unroll
  for (int a = 0; a < GQ; ++a) {
#pragma unroll
    for (int i = 0; i < 8; ++i) qv[a][i] = 0.f;
    if (a < na) {
      Row8<T>::load((const T*)p.q + ((long long)u * p.hq + head_of_slot(p.heads, c * gq + a0 + a)) * D + sub * 8, qv[a]);
      rotate(qv[a]);
#pragma unroll
      for (int i = 0; i < 8; ++i) qv[a][i] *= p.scale_log2;
    }
  }
  Row8<T>::load((const T*)p.k_new + ((long long)u * p.hkv + c) * D + sub * 8, kn);
  Row8<T>::load((const T*)p.v_new + ((long long)u * p.hkv + c) * D + sub * 8, vn);
  rotate(kn);
#pragma unroll
  for (int i = 0; i < 8; ++i) kn[i] = Row8<T>::round(kn[i]);
  __syncthreads();
  const T* K = (const T*)p.pg.k + sub * 8;
  const T* V = (const T*)p.pg.v + sub * 8;
  if (has_new && a0 == 0 && wave == 0 && kk == 0 && n < capacity_of(p.pg)) {   // cache append
    int in_page;
    const int page = page_of_row(p.pg, u, n, in_page);
    if (page >= 0) {
      const long long to = row_offset<D>(p.pg, page, c, in_page) + sub * 8;
      Row8<T>::store((T*)p.pg.k + to, kn);
      Row8<T>::store((T*)p.pg.v + to, vn);
    }
  }
  float mx[GQ], ls[GQ], o[GQ][8];
#pragma unroll
  for (int a = 0; a < GQ; ++a) {
    mx[a] = -INFINITY; ls[a] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[a][i] = 0.f;
  }
  for (int jb = j_begin + wave * KPW; jb < j_end; jb += NP * STEP) {
    typename Row8<T>::Raw kr[NP], vr[NP];
    bool there[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int j = jb + i * STEP + kk;
      kr[i] = typename Row8<T>::Raw{}; vr[i] = typename Row8<T>::Raw{};
      there[i] = j == n && j < j_end;
      if (j < n && j < j_end) {
        const int at = (int)p.pg.by_page.div((unsigned)j), page = pages[at - page0];
        if (page >= 0) {
          const long long from = row_offset<D>(p.pg, page, c, j - at * p.pg.page_size);
          kr[i] = Row8<T>::load_raw(K + from);
          vr[i] = Row8<T>::load_raw(V + from);
          there[i] = true;
        }
      }
    }
    float sc[NP][GQ];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int j = jb + i * STEP + kk;
      float kx[8];
      Row8<T>::unpack(kr[i], kx);
      if (j == n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) kx[e] = kn[e];
      }
#pragma unroll
      for (int a = 0; a < GQ; ++a) {
        float d = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) d = __builtin_fmaf(qv[a][e], kx[e], d);
        d = group_sum<LPK>(d);
        sc[i][a] = there[i] ? d : -INFINITY;
        if (p.scores && sub == 0 && a < na && j < j_end)
          ((unsigned*)p.scores)[((long long)u * p.hq + c * gq + a0 + a) * p.score_stride + j] = there[i] ? __float_as_uint(d) : kNoRow;
      }
    }
#pragma unroll
    for (int a = 0; a < GQ; ++a) {
      float mn = mx[a];
#pragma unroll
      for (int i = 0; i < NP; ++i) mn = fmaxf(mn, sc[i][a]);
      const float corr = mx[a] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx[a] - mn);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        sc[i][a] = sc[i][a] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sc[i][a] - mn);
        sum += sc[i][a];
      }
      ls[a] = ls[a] * corr + sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[a][e] *= corr;
      mx[a] = mn;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      float vx[8];
      Row8<T>::unpack(vr[i], vx);
      if (jb + i * STEP + kk == n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) vx[e] = vn[e];
      }
#pragma unroll
      for (int a = 0; a < GQ; ++a)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[a][e] = __builtin_fmaf(sc[i][a], vx[e], o[a][e]);
    }
  }
#pragma unroll
  for (int a = 0; a < GQ; ++a) {
#pragma unroll
    for (int off = LPK; off < kWave; off <<= 1) {
      const float m2 = __shfl_xor(mx[a], off, kWave), l2 = __shfl_xor(ls[a], off, kWave);
      float o2[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o2[i] = __shfl_xor(o[a][i], off, kWave);
      merge_state<8>(mx[a], ls[a], o[a], m2, l2, o2);
    }
  }
  if (kk == 0) {
#pragma unroll
    for (int a = 0; a < GQ; ++a) {
      merge[wave][a][sub][0] = mx[a];
      merge[wave][a][sub][1] = ls[a];
#pragma unroll
      for (int i = 0; i < 8; ++i) merge[wave][a][sub][2 + i] = o[a][i];
    }
  }
  __syncthreads();
  for (int i = tid; i < na * LPK; i += kPagedThreads) {
    const int a = i / LPK, sb = i % LPK;
    float m = merge[0][a][sb][0], l = merge[0][a][sb][1], x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = merge[0][a][sb][2 + e];
#pragma unroll
    for (int w = 1; w < kPagedWaves; ++w) merge_state<8>(m, l, x, merge[w][a][sb][0], merge[w][a][sb][1], &merge[w][a][sb][2]);
    finish_group<T, D>(p, (long long)u * p.hq, c * gq + a0 + a, z, sb * 8, m, l, x);
    if (sb == 0) states[a] = f32x2{m, 1.f / l};
  }
  if (p.scores && !p.part_o) add_weights<kPagedThreads>(p, u, c, n, 0, min(n + 1, p.w_cap), states, [] { __syncthreads(); });
}

// bf16: the same on the matrix cores.  Per block of 32 rows a wave computes
//   S^T = K Q^T     (16 keys x up to 16 query heads)
//   O^T += V^T P^T  (the layout of two S^T tiles is this product's operand)
// with queries and weights as sums of three bf16 operands each, 24 significant bits, as in the short decode kernels.  Keys, then
// values pass through one swizzled LDS tile of the wave's own: they leave memory whole lines at a time, as they lie there (key
// fragments straight from memory touch half lines, which loads that leave nothing in the caches then fetch twice).  While a
// block is worked on, the next one's rows are on their way: each half is asked for as soon as this block's is in LDS.
// Bound by HBM: 16 streams of 8192-32768 rows, 32 / 8 heads of 128 (1.28 GB), 218 us with the joining launch, 5.9 TB/s; loads of the same addresses and
// nothing else take 188.  (The vector form 292; key fragments straight from memory, three waves a SIMD instead of two, 225.)
// 16 consecutive rows have a chunk at different places: a fragment's reads meet no bank twice
template <int D>
__device__ __forceinline__ int key_swz(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
template <int D, int QR, bool STREAMED, int WAVES>
__global__ __launch_bounds__(kWave * WAVES, D == 64 ? 3 : 2) void paged_decode_mfma_kernel(PagedParams p) {
  constexpr int THREADS = kWave * WAVES, KS = D / 32, DB = D / 16, UPR = D / 8, BLK = 32, NV = BLK * UPR / kWave;
  union Tile { __bf16 v[BLK * D]; float o[QR][D + 4]; };
  __shared__ Tile tile[WAVES];
  __shared__ f32x2 ml[WAVES][QR], states[QR];
  __shared__ __align__(16) __bf16 rot[3][QR + 1][D + 8];   // queries in three terms; row QR of the first: the new key as stored
  __shared__ int pages[kPagedMaxChunk + 2];
  const int gq = p.hq / p.hkv, parts = (gq + QR - 1) / QR;
  const int z = blockIdx.z, c = blockIdx.x / parts, u = blockIdx.y, a0 = (int)(blockIdx.x % parts) * QR;
  const int na = min(gq - a0, QR);
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int r16 = lane & 15, quad = lane >> 4;
  const int n = length_of(p.cache_len, u, p.max_len, p.pg);
  const int j_begin = z * p.chunk, j_end = min(n + 1, j_begin + p.chunk);
  if (n < 0) {                                       // idle: zeros
    if (z == 0)
      for (int i = tid; i < na * UPR; i += THREADS) {
        const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        Row8<__bf16>::store((__bf16*)p.out + ((long long)u * p.hq + head_of_slot(p.heads, c * gq + a0 + i / UPR)) * D + i % UPR * 8, zero);
      }
    return;
  }
  if (j_begin >= j_end) return;
  const int page0 = (int)p.pg.by_page.div((unsigned)j_begin);
  {
    const int last = (int)p.pg.by_page.div((unsigned)max(j_begin, min(j_end, n) - 1));
    for (int i = page0 + tid; i <= last; i += THREADS) {   // (a table that is full has no page for row n)
      const int page = i < p.pg.max_pages ? p.pg.table[(long long)u * p.pg.max_pages + i] : -1;
      pages[i - page0] = (unsigned)page < (unsigned)p.pg.n_pages ? page : -1;
    }
  }
  const __bf16* new_k = (const __bf16*)p.k_new + ((long long)u * p.hkv + c) * D;
  const __bf16* new_v = (const __bf16*)p.v_new + ((long long)u * p.hkv + c) * D;
  // queries and the new key: 4 rotary pairs of a row per item
  {
    const float pos = (float)p.q_pos[u];
    for (int item = tid; item < (na + 1) * (D / 8); item += THREADS) {
      const int row = item / (D / 8), e = item % (D / 8) * 4;
      const bool key = row == na;
      const __bf16* src = (key ? new_k : (const __bf16*)p.q + ((long long)u * p.hq + head_of_slot(p.heads, c * gq + a0 + row)) * D) + e;
      const u32x2 lo = *(const u32x2*)src, hi = *(const u32x2*)(src + D / 2);
      const float scale = key ? 1.f : p.scale_log2;
      float y[2][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float sn = 0.f, cs = 1.f;
        if (p.rope.enabled) sincos_turns_precise(rope_turns(pos, p.rope.hi[e + j], p.rope.lo[e + j]), &sn, &cs);
        const float a = j & 1 ? bf16_hi(lo[j / 2]) : bf16_lo(lo[j / 2]), b = j & 1 ? bf16_hi(hi[j / 2]) : bf16_lo(hi[j / 2]);
        y[0][j] = __builtin_fmaf(a, cs, -(b * sn)) * scale;
        y[1][j] = __builtin_fmaf(b, cs, a * sn) * scale;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        unsigned w0[3], w1[3];
        split_pair(y[h][0], y[h][1], w0);
        split_pair(y[h][2], y[h][3], w1);
        if (key) *(u32x2*)&rot[0][QR][e + h * (D / 2)] = u32x2{w0[0], w1[0]};   // the first term: rounded as stored
        else {
#pragma unroll
          for (int i = 0; i < 3; ++i) *(u32x2*)&rot[i][row][e + h * (D / 2)] = u32x2{w0[i], w1[i]};
        }
      }
    }
  }
  __syncthreads();
  if (j_end == n + 1 && a0 == 0 && n < capacity_of(p.pg)) {   // cache append
    int in_page;
    const int page = page_of_row(p.pg, u, n, in_page);
    if (page >= 0 && tid < 2 * UPR) {
      const long long to = row_offset<D>(p.pg, page, c, in_page) + tid % UPR * 8;
      if (tid < UPR) *(u32x4*)((__bf16*)p.pg.k + to) = *(const u32x4*)&rot[0][QR][tid * 8];
      else *(u32x4*)((__bf16*)p.pg.v + to) = *(const u32x4*)(new_v + tid % UPR * 8);
    }
  }
  const int n_blocks = (j_end - j_begin + BLK - 1) / BLK;
  // A block as it lies in memory: unit lane + 64 i of its rows, 16 bytes each.  Every unit is loaded, those of rows that are not
  // there from some row that is in the pool.  Returns which rows are there.
  // Whole blocks over pages of a multiple of 8 rows: 8 rows lie in one page, one behind the other, and a wave looks their pages up
  // once (one row at a time, a block took 590 vector instructions; 280 now: 100 streams of 3000 rows, 32 heads over 8, pages of 8,
  // 132 us for 155).
  constexpr int RPI = kWave / UPR;                    // rows of 64 units
  const bool by_eight = p.pg.page_size % 8 == 0;
  auto load_block = [&](u32x4 (&x)[NV], const __bf16* pool, int blk) __attribute__((always_inline)) {
    const int j0 = j_begin + blk * BLK;
    unsigned have = 0;                                // bit i: row i of the block has a place in the pool
    if (by_eight && j0 + BLK <= min(n, j_end)) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int j = j0 + 8 * t, at = (int)p.pg.by_page.div((unsigned)j), page = __builtin_amdgcn_readfirstlane(pages[at - page0]);
        const u32x4* rows = (const u32x4*)(pool + row_offset<D>(p.pg, max(page, 0), c, j - at * p.pg.page_size));
        have |= page >= 0 ? 0xffu << (8 * t) : 0u;
#pragma unroll
        for (int i = 0; i < NV / 4; ++i) x[t * (NV / 4) + i] = STREAMED ? __builtin_nontemporal_load(rows + lane + kWave * i) : rows[lane + kWave * i];
      }
      return have;
    }
    int own = lane;                                   // (opaque: what follows from it is not worth registers over the loop)
    asm volatile("" : "+v"(own));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int unit = own + kWave * i, j = min(j0 + unit / UPR, max(min(n, j_end) - 1, j_begin));
      const int at = (int)p.pg.by_page.div((unsigned)j), page = pages[at - page0];
      x[i] = *(const u32x4*)(pool + row_offset<D>(p.pg, max(page, 0), c, j - at * p.pg.page_size) + unit % UPR * 8);
      const unsigned long long who = __ballot(page >= 0 && j0 + unit / UPR < min(n, j_end));
#pragma unroll
      for (int r = 0; r < RPI; ++r) have |= (unsigned)(who >> (r * UPR) & 1) << (i * RPI + r);
      asm volatile("" ::: "memory");                  // one row's address at a time: together they do not fit the registers
    }
    return have;
  };
  const u32x4 newest = *(const u32x4*)(new_v + r16 % UPR * 8);
  u32x4 kr[NV], vr[NV];
  unsigned there = 0;
  f32x4 o[DB];
  float mrow, lrow;
  __bf16* smv = tile[wave].v;
  // Byte addresses in the tile.  Unit lane + 64 i is chunk lane % UPR of row lane / UPR + RPI i, and lies at that chunk ^ swizzle(row):
  // the lane's own part of it, ^ what the row's RPI i adds.
  int key_write = lane / UPR * (2 * D) + ((lane % UPR ^ key_swz<D>(lane / UPR)) << 4), key_read = r16 * (2 * D) + ((quad ^ key_swz<D>(r16)) << 4);
  int value_write = lane / UPR * (2 * D) + ((lane % UPR ^ short_v_swz<D>(lane / UPR)) << 4);
  // of the transposing reads of 16 elements by 8 keys: keys 4 quad + (0..3), and 16 rows on
  int value_read = (4 * quad + (r16 >> 2)) * (2 * D) + (((r16 & 3) >> 1 ^ short_v_swz<D>(4 * quad + (r16 >> 2))) << 4) + 8 * (r16 & 1);
  auto key_step = [](int i) { return key_swz<D>(RPI * i) << 4; };
  auto value_step = [](int i) { return short_v_swz<D>(RPI * i) << 4; };
  const int q_row = min(r16, na - 1);                 // columns beyond the group repeat its last query
  float* scores = p.scores ? p.scores + ((long long)u * p.hq + c * gq + a0 + q_row) * p.score_stride : nullptr;
  auto walk = [&](auto careful_c) {
    constexpr bool CAREFUL = decltype(careful_c)::value;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    mrow = -INFINITY;
    lrow = 0.f;
    if (wave < n_blocks) {
      there = load_block(kr, (const __bf16*)p.pg.k, wave);
      load_block(vr, (const __bf16*)p.pg.v, wave);
    }
    for (int blk = wave; blk < n_blocks; blk += WAVES) {
      const int j0 = j_begin + blk * BLK;
      const unsigned stored = there;
      const bool more = blk + WAVES < n_blocks;
      const int j_new = blk == n_blocks - 1 && j_end == n + 1 ? n - j0 : BLK;   // the new token's row of the block
      const unsigned mask = j_new < BLK ? stored | 1u << j_new : stored;
      // (opaque: eight addresses a register each, kept over the loop, would not fit)
      asm volatile("" : "+v"(key_write), "+v"(key_read), "+v"(value_write), "+v"(value_read));
      // the wave's LDS operations complete in order: only the compiler has to keep theirs
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        *(u32x4*)((char*)smv + (key_write ^ key_step(i)) + 1024 * i) = kr[i];
      }
      if (j_new < BLK && lane < UPR) *(u32x4*)(smv + j_new * D + ((lane ^ key_swz<D>(j_new)) << 3)) = *(const u32x4*)&rot[0][QR][lane * 8];
      if (more) there = load_block(kr, (const __bf16*)p.pg.k, blk + WAVES);
      asm volatile("" ::: "memory");
      // products with the queries' first terms and with what is left of them, apart: an infinite key element gives its
      // infinity with the first term, and NaN where the terms differ in sign
      f32x4 sc[2], rest[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) sc[t] = rest[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[2], q[3];
#pragma unroll
        for (int t = 0; t < 2; ++t) kf[t] = *(const bf16x8*)((const char*)smv + (key_read ^ (64 * ks)) + 32 * D * t);
#pragma unroll
        for (int i = 0; i < 3; ++i) q[i] = *(const bf16x8*)&rot[i][q_row][32 * ks + 8 * quad];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          rest[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t], q[2], rest[t], 0, 0, 0);
          sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t], q[0], sc[t], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) rest[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t], q[1], rest[t], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) short_settle(sc[t], rest[t]);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < NV; ++i) *(u32x4*)((char*)smv + (value_write ^ value_step(i)) + 1024 * i) = vr[i];
      if (stored != 0xffffffffu) {                     // rows that are not there weigh 0: their values have to be finite
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (!(stored >> (RPI * i + lane / UPR) & 1)) *(u32x4*)((char*)smv + (value_write ^ value_step(i)) + 1024 * i) = u32x4{0u, 0u, 0u, 0u};
        asm volatile("" ::: "memory");
        if (j_new < BLK && lane < UPR) *(u32x4*)(smv + j_new * D + ((lane ^ short_v_swz<D>(j_new)) << 3)) = newest;
      }
      if (more) load_block(vr, (const __bf16*)p.pg.v, blk + WAVES);
      if (scores && r16 < na) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          u32x4 x = __builtin_bit_cast(u32x4, sc[t]);
          if (mask != 0xffffffffu) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = mask >> (16 * t + 4 * quad + i) & 1 ? x[i] : kNoRow;
          }
          *(u32x4*)(scores + j0 + 16 * t + 4 * quad) = x;
        }
      }
      if (mask != 0xffffffffu) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(mask >> (16 * t + 4 * quad + i) & 1)) sc[t][i] = -INFINITY;
      }
      u32x4 pw[3];
      const float alpha = short_softmax(sc, mrow, lrow, pw);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const char* at = (const char*)smv + (value_read ^ (32 * db));
        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)at);
        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + 32 * D));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int i = 0; i < 4; ++i) o[db][i] *= alpha;
        f32x4 small = CAREFUL ? f32x4{0.f, 0.f, 0.f, 0.f} : o[db];
        small = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pw[2]), small, 0, 0, 0);
        small = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pw[1]), small, 0, 0, 0);
        if (CAREFUL) {
          o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pw[0]), o[db], 0, 0, 0);
          short_settle(o[db], small);
        } else o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pw[0]), small, 0, 0, 0);
      }
      asm volatile("" ::: "memory");
    }
  };
  walk(std::false_type{});
  float probe = lrow;                                 // NaN where anything is, or where infinities of both signs meet
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) probe += o[db][i];
  if (__any(probe != probe)) walk(std::true_type{});
  lrow += __shfl_xor(lrow, 16, kWave);
  lrow += __shfl_xor(lrow, 32, kWave);
  if (r16 < na) {
#pragma unroll
    for (int db = 0; db < DB; ++db) *(f32x4*)&tile[wave].o[r16][16 * db + 4 * quad] = o[db];
    if (quad == 0) ml[wave][r16] = f32x2{mrow, lrow};
  }
  __syncthreads();
  for (int i = tid; i < na * UPR; i += THREADS) {
    const int a = i / UPR, e = (i % UPR) * 8;
    float m = -INFINITY, l = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, ml[w][a][0]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w >= n_blocks) continue;                    // a wave without rows: its tile holds nothing
      const float f = ml[w][a][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w][a][0] - m);
      l += f * ml[w][a][1];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(f, tile[w].o[a][e + j], x[j]);
    }
    finish_group<__bf16, D>(p, (long long)u * p.hq, c * gq + a0 + a, z, e, m, l, x);
    if (e == 0) states[a] = f32x2{m, 1.f / l};
  }
  if (p.scores && !p.part_o) add_weights<THREADS>(p, u, c, n, 0, min(n + 1, p.w_cap), states, [] { __syncthreads(); });
}

// Joins the splits' states.  Bound by its trips to memory, one behind the other: 128 splits of 12 heads with the weights of 65521 rows
// 7 us (83 with a thread walking all splits).  Blocks x < Hq / Hkv of a (kv head, stream) give one query head's output each: 256 / (D / 8) lanes
// share the splits, then meet in LDS.  The blocks behind them give
// join_rows rows' weights each.
constexpr int kJoinThreads = kPagedThreads, kMaxGroup = 128;
template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedParams p) {
  constexpr int LPK = D / 8, LANES = kJoinThreads / LPK;
  const int c = blockIdx.y, u = blockIdx.z, gq = p.hq / p.hkv, tid = threadIdx.x;
  const int n = length_of(p.cache_len, u, p.max_len, p.pg);
  if (n < 0) return;
  const int used = (n + p.chunk) / p.chunk;    // splits that have rows: n + 1 rows
  const long long head0 = (long long)u * p.hq + c * gq;
  if ((int)blockIdx.x < gq) {
    const int a = blockIdx.x, sb = tid % LPK, part = tid / LPK;
    __shared__ float sm[LANES][LPK][10];
    float m = -INFINITY, l = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int z0 = part; z0 < used; z0 += 4 * LANES) {   // four splits' states on their way together
      f32x4 x2[4][2];
      f32x2 state[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long slot = (head0 + a) * p.n_splits + min(z0 + i * LANES, used - 1);
        state[i] = *(const f32x2*)(p.part_ml + slot * 2);
        x2[i][0] = *(const f32x4*)(p.part_o + slot * D + sb * 8);
        x2[i][1] = *(const f32x4*)(p.part_o + slot * D + sb * 8 + 4);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (z0 + i * LANES >= used) continue;
        const float y[8] = {x2[i][0][0], x2[i][0][1], x2[i][0][2], x2[i][0][3], x2[i][1][0], x2[i][1][1], x2[i][1][2], x2[i][1][3]};
        merge_state<8>(m, l, x, state[i][0], state[i][1], y);
      }
    }
    sm[part][sb][0] = m;
    sm[part][sb][1] = l;
#pragma unroll
    for (int e = 0; e < 8; ++e) sm[part][sb][2 + e] = x[e];
    __syncthreads();
    if (part > 0) return;
#pragma unroll 4
    for (int i = 1; i < min(LANES, used); ++i) merge_state<8>(m, l, x, sm[i][sb][0], sm[i][sb][1], &sm[i][sb][2]);
    const float inv = 1.f / l;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    Row8<T>::store((T*)p.out + ((long long)u * p.hq + head_of_slot(p.heads, c * gq + a)) * D + sb * 8, x);
    return;
  }
  const int j0 = (int)(blockIdx.x - gq) * p.join_rows, j1 = min(min(n + 1, j0 + p.join_rows), p.w_cap);
  if (j0 >= j1) return;
  __shared__ f32x2 state[kMaxGroup];
  add_weights<kJoinThreads>(p, u, c, n, j0, j1, state, [&]() {
    for (int a = tid / kWave; a < gq; a += kJoinThreads / kWave) {   // a wave per head
      const f32x2* split = (const f32x2*)p.part_ml + (head0 + a) * p.n_splits;
      float m = -INFINITY, l = 0.f;
      for (int z = tid % kWave; z < used; z += kWave) merge_state<0>(m, l, nullptr, split[z][0], split[z][1], nullptr);
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const float m2 = __shfl_xor(m, o, kWave), l2 = __shfl_xor(l, o, kWave);
        merge_state<0>(m, l, nullptr, m2, l2, nullptr);
      }
      if (tid % kWave == 0) state[a] = f32x2{m, 1.f / l};
    }
    __syncthreads();
  });
}

// ------------------------------------------------------------------------------------------------------------------
// evict
// ------------------------------------------------------------------------------------------------------------------
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave;

struct EvictParams {
  Pages pg;
  const int32_t* cache_len; const float* w_in; float* w_out; const int32_t* new_table;
  int32_t* kept; int32_t* len_out;
  int max_len, w_cap, w_out_cap, budget, first, last, new_pages;
};

// a weight as an integer of the same order: NaN below everything, zeros of either sign equal; 0 is no weight's
__device__ __forceinline__ unsigned weight_key(float w) {
  if (w != w) return 1u;
  const unsigned b = __float_as_uint(w == 0.f ? 0.f : w);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// One workgroup per (kv head, stream): the key of the last row that is kept by weight, 11, 11 and 10 bits of it at a time from
// histograms of the rows that agree so far, then the kept rows in their order.  A wave has a run of rows of its own, ROWS / 16 of
// them, whose keys stay in registers (ROWS = 0: any number, read again in every pass).  Weights crowd: most of the first histogram's
// additions go to a few neighbouring bins, so that eight copies of it, a lane's by its number, take them in turn.  The rows
// that agree in the first 11 bits are listed, a few hundred as a rule, and the other digits come from the list.  One workgroup
// does all of it, so what bounds it is the vector instructions that every row takes in its few passes: the first histogram, the list,
// two counts, the result.  8 x 8 heads of 32768 rows 26 us (one bit a pass, rows read again, 252), 64 x 2 of 1024-2048 rows 10 (25).
constexpr int kDigitBins = 2048, kDigitCopies = 8, kDigitList = 4096;
struct SelectSmem {
  int bins[kDigitBins * kDigitCopies];
  unsigned list[kDigitList];
  int wave_sum[kSelectWaves], wave_above[kSelectWaves], wave_equal[kSelectWaves];
  int digit, above, in_bin, listed;
};
// The bin, from the top, in which the need-th entry lies (need >= 1, at most all entries); `above`: entries in higher bins, `in_bin`:
// in this one.
template <int COPIES>
__device__ __forceinline__ int select_digit(SelectSmem& sm, int need, int& above, int& in_bin) {
  constexpr int PER = kDigitBins / kSelectThreads;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  int count[PER], all = 0;                       // this thread's bins, from the top
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int bin = kDigitBins - 1 - (tid * PER + i);
    count[i] = 0;
#pragma unroll
    for (int k = 0; k < COPIES; ++k) count[i] += sm.bins[bin * COPIES + (k + tid) % COPIES];
    all += count[i];
  }
  int sum = all;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(sum, o, kWave);
    if (lane >= o) sum += y;
  }
  if (lane == kWave - 1) sm.wave_sum[wave] = sum;
  __syncthreads();
  int before = sum - all;
  for (int i = 0; i < wave; ++i) before += sm.wave_sum[i];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < need && before + count[i] >= need) { sm.digit = kDigitBins - 1 - (tid * PER + i); sm.above = before; sm.in_bin = count[i]; }
    before += count[i];
  }
  __syncthreads();
  above = sm.above;
  in_bin = sm.in_bin;
  return sm.digit;
}

template <int ROWS>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictParams p) {
  constexpr int PER = ROWS / kSelectThreads;     // rows of a thread
  __shared__ SelectSmem sm;
  const int c = blockIdx.x, u = blockIdx.y, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int n = length_of(p.cache_len, u, min(p.max_len, p.w_cap), p.pg);
  const long long pair = (long long)u * p.pg.hkv + c;
  const float* w = p.w_in + pair * p.w_cap;
  int32_t* kept = p.kept + pair * p.budget;
  const int m = min(n, p.budget);
  for (int i = max(m, 0) + tid; i < p.budget; i += kSelectThreads) kept[i] = -1;
  if (n < 0) return;
  if (n <= p.budget) {
    for (int i = tid; i < n; i += kSelectThreads) kept[i] = i;
    return;
  }
  const int lo = p.first, hi = n - p.last, need = p.budget - p.first - p.last;   // rows [lo, hi) compete for `need` places
  // lane's rows: begin + 64 i + lane
  const int per = ((hi - lo + kSelectWaves - 1) / kSelectWaves + kWave - 1) / kWave * kWave;
  const int begin = lo + wave * per, end = min(hi, begin + per);
  unsigned held[PER > 0 ? PER : 1];
  if constexpr (PER > 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) held[i] = __float_as_uint(begin + i * kWave + lane < end ? w[begin + i * kWave + lane] : 0.f);
  }
  for (int i = tid; i < p.first; i += kSelectThreads) kept[i] = i;
  for (int i = tid; i < p.last; i += kSelectThreads) kept[p.budget - p.last + i] = hi + i;
  if (need <= 0) return;
  for (int i = tid; i < kDigitBins * kDigitCopies / 4; i += kSelectThreads) *(u32x4*)&sm.bins[4 * i] = u32x4{0u, 0u, 0u, 0u};
  if (tid == 0) sm.listed = 0;
  if constexpr (PER > 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) held[i] = begin + i * kWave + lane < end ? weight_key(__uint_as_float(held[i])) : 0u;
  }
  auto each = [&](auto f) {                      // f(row, key), all lanes of a wave together; key 0 where there is no row
    if constexpr (PER > 0) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (begin + i * kWave < end) f(begin + i * kWave + lane, held[i]);
    } else {
      for (int j0 = begin; j0 < end; j0 += kWave) f(j0 + lane, j0 + lane < end ? weight_key(w[j0 + lane]) : 0u);
    }
  };
  __syncthreads();
  each([&](int, unsigned k) { atomicAdd(&sm.bins[(k >> 21) * kDigitCopies + lane % kDigitCopies], 1); });
  __syncthreads();
  int above, in_bin;                             // rows whose key exceeds what is known of t, that agree with it
  unsigned t = (unsigned)select_digit<kDigitCopies>(sm, need, above, in_bin) << 21;
  const bool listed = in_bin <= kDigitList;
  if (listed) {                                  // a place in the list for each wave's, then the keys
    int mine = 0;
    each([&](int, unsigned k) { mine += __popcll(__ballot(k >> 21 == t >> 21)); });
    int to = 0;
    if (lane == 0 && mine) to = atomicAdd(&sm.listed, mine);
    to = __builtin_amdgcn_readfirstlane(to);
    each([&](int, unsigned k) {
      const bool here = k >> 21 == t >> 21;
      const unsigned long long mask = __ballot(here);
      if (here) sm.list[to + __popcll(mask & ((1ull << lane) - 1))] = k;
      to += __popcll(mask);
    });
  }
  const int n_list = in_bin;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    const int shift = pass == 0 ? 10 : 0, known = pass == 0 ? 21 : 10, digit = pass == 0 ? 2047 : 1023;
    for (int i = tid; i < kDigitBins / 4; i += kSelectThreads) *(u32x4*)&sm.bins[4 * i] = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
    auto count = [&](unsigned k) {
      if ((k ^ t) >> known == 0) atomicAdd(&sm.bins[k >> shift & digit], 1);
    };
    if (listed) {
      for (int i = tid; i < n_list; i += kSelectThreads) count(sm.list[i]);
    } else {
      each([&](int, unsigned k) { count(k); });
    }
    __syncthreads();
    int over;
    t |= (unsigned)select_digit<1>(sm, need - above, over, in_bin) << shift;
    above += over;
  }
  const int equal_kept = need - above;           // of the rows whose key is t, the first ones
  int mine_above = 0, mine_equal = 0;
  each([&](int, unsigned k) {
    mine_above += __popcll(__ballot(k > t));
    mine_equal += __popcll(__ballot(k == t));
  });
  if (lane == 0) { sm.wave_above[wave] = mine_above; sm.wave_equal[wave] = mine_equal; }
  __syncthreads();
  int at = p.first, eq = 0;
  for (int i = 0; i < wave; ++i) { at += sm.wave_above[i]; eq += sm.wave_equal[i]; }
  at += min(eq, equal_kept);
  int left = __builtin_amdgcn_readfirstlane(max(equal_kept - eq, 0));   // equal rows that this wave still keeps
  at = __builtin_amdgcn_readfirstlane(at);
  each([&](int j, unsigned k) {
    unsigned long long mask = __ballot(k > t), same = __ballot(k == t);
    for (int drop = __popcll(same) - left; drop > 0; --drop) same &= ~(1ull << (63 - __builtin_clzll(same)));
    left -= __popcll(same);
    mask |= same;
    if (mask >> lane & 1) kept[at + __popcll(mask & ((1ull << lane) - 1))] = j;
    at += __popcll(mask);
  });
}

// 16 bytes of a K and a V row per thread, and the kept rows' sums.  A gathering copy: 8 x 8 heads x 4096 rows of 128 (268 MB read and written) 55 us, 4.9 TB/s, what
// a large copy reaches; 64 x 2 x 1000 rows (131 MB) 25.5.
template <typename T, int D>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictParams p) {
  constexpr int UPR = D * (int)sizeof(T) / 16;
  const int i = (int)(blockIdx.x * (256 / UPR) + threadIdx.x / UPR), unit = threadIdx.x % UPR, c = blockIdx.y, u = blockIdx.z;
  if (blockIdx.x == 0 && c == 0 && threadIdx.x == 0) {
    const int n = length_of(p.cache_len, u, min(p.max_len, p.w_cap), p.pg);
    p.len_out[u] = min(n, p.budget);
  }
  if (i >= p.budget) return;
  const long long pair = (long long)u * p.pg.hkv + c;
  const int r = p.kept[pair * p.budget + i];
  if (r < 0) return;
  if (unit == 0 && p.w_out) p.w_out[pair * p.w_out_cap + i] = p.w_in[pair * p.w_cap + r];
  int in_old;
  const int old = page_of_row(p.pg, u, r, in_old);
  const int at = (int)p.pg.by_page.div((unsigned)i), page = p.new_table[(long long)u * p.new_pages + at];
  if ((unsigned)page >= (unsigned)p.pg.n_pages) return;
  const long long to = row_offset<D>(p.pg, page, c, i - at * p.pg.page_size) * (long long)sizeof(T) / 16 + unit;
  u32x4 k = {0u, 0u, 0u, 0u}, v = k;             // a row without a page, which no caller hands over: zeros, not what the new page held
  if (old >= 0) {
    const long long from = row_offset<D>(p.pg, old, c, in_old) * (long long)sizeof(T) / 16 + unit;
    k = __builtin_nontemporal_load((const u32x4*)p.pg.k + from);
    v = __builtin_nontemporal_load((const u32x4*)p.pg.v + from);
  }
  ((u32x4*)p.pg.k)[to] = k;
  ((u32x4*)p.pg.v)[to] = v;
}

// ------------------------------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------------------------------
static Pages make_pages(void* k, void* v, const int32_t* table, int max_pages, int n_pages, int page_size, int hkv) {
  return Pages{k, v, table, max_pages, n_pages, page_size, hkv, FastDiv::of((unsigned)page_size)};
}
static int launched() {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return EARN_OK;
  set_error("launch failed: %s", hipGetErrorString(e));
  return EARN_ERR_HIP;
}
// f(T{}, std::integral_constant<int, D>{}) for the description's type and head size
template <typename F>
static void for_type(const earn_attn_desc* desc, F f) {
  const bool f32 = desc->dtype == EARN_F32;
  if (desc->head_dim == 64) { if (f32) f(float{}, std::integral_constant<int, 64>{}); else f(__bf16{}, std::integral_constant<int, 64>{}); }
  else { if (f32) f(float{}, std::integral_constant<int, 128>{}); else f(__bf16{}, std::integral_constant<int, 128>{}); }
}

int launch_cache_store(const earn_attn_desc* desc, const void* k, const void* v, const int32_t* cu, const int32_t* start, int batch,
                       int total, void* k_pages, void* v_pages, const int32_t* table, int max_pages, int n_pages, int page_size,
                       hipStream_t stream) {
  const Pages pg = make_pages(k_pages, v_pages, table, max_pages, n_pages, page_size, desc->n_kv_heads);
  for_type(desc, [&](auto t, auto d) {
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value, rows = 256 / (D * (int)sizeof(T) / 16) * kStoreUnits;   // of a workgroup
    const long long blocks = ((long long)total * desc->n_kv_heads + rows - 1) / rows;
    hipLaunchKernelGGL((paged_store_kernel<T, D>), dim3((unsigned)blocks), dim3(256), 0, stream, (const u32x4*)k, (const u32x4*)v, pg, cu,
                       start, batch, total, FastDiv::of((unsigned)desc->n_kv_heads));
  });
  return launched();
}

struct PagedPlan { int n_splits, chunk, score_stride; size_t part_o, part_ml, scores; };
constexpr int kWholeRows = 640, kMinChunk = 256, kMostChunk = 1088;
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }
// query heads that a workgroup serves, and the workgroups of a group of heads
static int paged_heads(const earn_attn_desc* desc) {
  const int gq = desc->n_q_heads / desc->n_kv_heads;
  if (desc->dtype == EARN_BF16) return gq > 8 ? 16 : 8;
  return gq > 4 ? 8 : gq > 2 ? 4 : gq;
}
static int paged_parts(const earn_attn_desc* desc) {
  const int gq = desc->n_q_heads / desc->n_kv_heads, heads = paged_heads(desc);
  return (gq + heads - 1) / heads;
}
static int wanted_workgroups(const earn_attn_desc* desc) { return desc->dtype == EARN_F32 ? 512 : 256; }
// `forced`: the setting of "paged_chunk", 0 for none; a call reads it once, for the size that it asks for and for what it launches
static PagedPlan plan_paged(const earn_attn_desc* desc, int n_streams, int max_len, bool weights, int forced) {
  PagedPlan pl{};
  const long long pairs = (long long)n_streams * desc->n_kv_heads, rows = (long long)max_len + 1;
  // Rows of a split: what leaves a workgroup per CU (fp32, whose workgroups are lighter: two), from kMinChunk, below
  // which a workgroup's start costs more than its rows, to kMostChunk, above which the long streams' last splits run on their own (1088: a
  // cache of 1024 rows and its new row are one split).  Up to kWholeRows rows nothing is split: the joining launch costs as much as it
  // saves.  us, 256 / 512 / 1024 / 1088 / 2048 rows: 8 streams of 2000 rows, 32 / 32 heads 61 / 58 / 56 / 58 / 53; 4 of 8192, 32 / 8 heads
  // 40 / 38 / 33 / 34 / 42; one of 4096 14 / 17 / 24 / 26 / 40; 16 of 8192-32768 256 / 212 / 201 / 202 / 199; 64 of 1024, 8 / 8 heads 68 / 65
  // / 63 / 56 / 57; one of 65521, 12 / 2 heads, weights 26 / 24 / 30 / 31 / 46; one of 32768, fp32 72 / 63 / 71 / 73 / 119; 32 of 256-528, 14 / 2
  // heads of 64 11.6 / 14.4 / 10.1 whole; 256 of 100-500, 12 / 2 heads 29 / 21 whole.
  long long chunk = rows * pairs / wanted_workgroups(desc);
  if (chunk < kMinChunk) chunk = kMinChunk;
  if (chunk > kMostChunk) chunk = kMostChunk;
  if (rows <= kWholeRows) chunk = rows;
  if (forced > 0) chunk = forced < kPagedMaxChunk ? forced : kPagedMaxChunk;
  if (chunk > rows) chunk = rows;
  if (chunk < rows / 65535 + 1) chunk = rows / 65535 + 1;   // a grid dimension
  pl.chunk = (int)((chunk + 63) / 64 * 64);
  pl.n_splits = (int)((rows + pl.chunk - 1) / pl.chunk);
  pl.score_stride = (int)((rows + 31) / 32 * 32);   // whole blocks of rows
  const size_t heads = (size_t)n_streams * desc->n_q_heads;
  // without splits, and with all heads of a group in one workgroup, that workgroup finishes weights and outputs by itself
  if (pl.n_splits > 1 || (weights && paged_parts(desc) > 1)) {
    pl.part_o = up256(heads * pl.n_splits * desc->head_dim * 4);
    pl.part_ml = up256(heads * pl.n_splits * 8);
  }
  if (weights) pl.scores = up256(heads * pl.score_stride * 4);
  return pl;
}
// What any call of at most n_streams streams and max_len rows takes by plan_paged: splits get longer, and fewer, as either grows, but
// a workspace sized for the largest call has to serve the smaller ones.  With n streams of hkv heads, r rows, c rows a split and W
// workgroups wanted:  c >= kMinChunk, so n splits <= n ceil(r / kMinChunk);  and either c = kMostChunk, so n splits <= n ceil(r /
// kMostChunk), or r n hkv / W < c + 1 (its division leaves a rest), so n splits < n (r / c + 1) < W (kMinChunk + 1) / (kMinChunk hkv) + n.
size_t decode_paged_workspace_bytes(const earn_attn_desc* desc, int n_streams, int max_len, bool weights, int forced) {
  const long long rows = (long long)max_len + 1, n = n_streams;
  auto of = [](long long r, long long c) { return (r + c - 1) / c; };
  long long splits = n;                          // of all streams
  if (forced > 0) splits = n * min(of(rows, (min(forced, kPagedMaxChunk) + 63) / 64 * 64), 65535ll);
  else if (rows > kWholeRows)
    splits = min(n * of(rows, kMinChunk),
                 max(n * of(rows, kMostChunk), (long long)wanted_workgroups(desc) * (kMinChunk + 1) / (kMinChunk * desc->n_kv_heads) + n));
  const size_t heads = (size_t)n * desc->n_q_heads;
  size_t bytes = weights ? up256(heads * ((rows + 31) / 32 * 32) * 4) : 0;
  if (splits > n || (weights && paged_parts(desc) > 1))
    bytes += up256((size_t)splits * desc->n_q_heads * desc->head_dim * 4) + up256((size_t)splits * desc->n_q_heads * 8);
  return bytes;
}

int launch_decode_paged(const earn_attn_desc* desc, const void* q, const void* k_new, const void* v_new, const int32_t* q_pos,
                        void* k_pages, void* v_pages, const int32_t* table, const int32_t* cache_len, int n_streams, int max_pages,
                        int n_pages, int page_size, int max_len, const float* w_in, float* w_out, int w_cap, void* out,
                        void* workspace, int forced, hipStream_t stream) {
  const PagedPlan pl = plan_paged(desc, n_streams, max_len, w_out != nullptr, forced);
  PagedParams p;
  p.pg = make_pages(k_pages, v_pages, table, max_pages, n_pages, page_size, desc->n_kv_heads);
  p.q = q; p.k_new = k_new; p.v_new = v_new; p.q_pos = q_pos; p.cache_len = cache_len;
  p.w_in = w_in; p.w_out = w_out; p.out = out; p.w_cap = w_cap;
  p.part_o = pl.part_o ? (float*)workspace : nullptr;
  p.part_ml = (float*)((char*)workspace + pl.part_o);
  p.scores = pl.scores ? (float*)((char*)workspace + pl.part_o + pl.part_ml) : nullptr;
  p.hq = desc->n_q_heads; p.hkv = desc->n_kv_heads; p.max_len = max_len;
  p.n_splits = pl.n_splits; p.chunk = pl.chunk; p.score_stride = pl.score_stride;
  const float scale = desc->softmax_scale > 0.f ? desc->softmax_scale : 1.f / sqrtf((float)desc->head_dim);
  p.scale_log2 = scale * 1.4426950408889634f;
  p.rope = make_rope_table(desc->rope_base, desc->head_dim);
  const int rc = make_head_map(desc, &p.heads, "earn_decode_attn_paged");
  if (rc != EARN_OK) return rc;
  const bool mfma = desc->dtype == EARN_BF16;
  // bf16 rows that the caches in front of the memory (256 MB) cannot hold until the next step are loaded without a place there, whole
  // lines at a time: 16 streams of 8192-32768 rows, 32 / 8 heads of 128, 240 -> 223 us; 32 of 4000-16000, 4 heads of 64, 72 -> 66; but 256
  // streams of 100-500 rows, 63 MB, 22 -> 24.  An fp32 row leaves memory in halves of 16 bytes a lane, half lines, which such loads fetch
  // twice (16 of 3000-12000, 4 heads of 128, 106 -> 131; 8 of 16384, 32 / 8 heads, which gain, 217 -> 209): always through the caches.
  const bool streamed = mfma && 2ll * n_streams * p.hkv * max_len * desc->head_dim * 2 > (256ll << 20);
  const int gq = p.hq / p.hkv, g = paged_heads(desc), parts = paged_parts(desc);
  // Eight waves share the rows of a stream that is not split, where no other workgroup would fill the CU: us, 32 streams of 256-528
  // rows, 14 / 2 heads of 64, 13.3 -> 11.7; 8 of 500, 32 / 8 heads, 16.0 -> 13.3; 16 of 100-300, 12 / 2 heads, 13.7 -> 12.5; but 256 of 100-500, 12 / 2
  // heads (512 workgroups), 22 -> 27, and split caches gain nothing (one of 65521 rows 24.3 -> 25.7).
  const bool wide = pl.n_splits == 1 && (long long)p.hkv * parts * n_streams <= 256 && pl.chunk > 128;
  // splits last: consecutive workgroups go to the XCDs in turn, and with two splits side by side every other XCD had short ones only
  // (64 streams of 256-2080 rows, 32 heads, two splits: 277 us, this way 209)
  const dim3 grid(p.hkv * parts, n_streams, pl.n_splits);
  for_type(desc, [&](auto t, auto d) {
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value;
    auto mfma_launch = [&](auto qr, auto nt, auto waves) {
      hipLaunchKernelGGL((paged_decode_mfma_kernel<D, decltype(qr)::value, decltype(nt)::value, decltype(waves)::value>), grid, dim3(kWave * decltype(waves)::value), 0, stream, p);
    };
    constexpr std::integral_constant<int, 4> four;
    constexpr std::integral_constant<int, 8> eight;
    constexpr std::integral_constant<int, 16> sixteen;
    if (mfma && g == 8 && streamed) mfma_launch(eight, std::true_type{}, four);
    else if (mfma && streamed) mfma_launch(sixteen, std::true_type{}, four);
    else if (mfma && g == 8 && wide) mfma_launch(eight, std::false_type{}, eight);
    else if (mfma && wide) mfma_launch(sixteen, std::false_type{}, eight);
    else if (mfma && g == 8) mfma_launch(eight, std::false_type{}, four);
    else if (mfma) mfma_launch(sixteen, std::false_type{}, four);
    else if constexpr (sizeof(T) == 4) {
      auto vector_launch = [&](auto heads) {
        constexpr int G = decltype(heads)::value;
        hipLaunchKernelGGL((paged_decode_kernel<T, D, G>), grid, dim3(kPagedThreads), 0, stream, p);
      };
      if (g == 1) vector_launch(std::integral_constant<int, 1>{});
      else if (g == 2) vector_launch(std::integral_constant<int, 2>{});
      else if (g == 4) vector_launch(std::integral_constant<int, 4>{});
      else vector_launch(eight);
    }
  });
  if (p.part_o) for_type(desc, [&](auto t, auto d) {
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value;
    {
      // rows of a block: 1024, more where the blocks are many (64 streams of up to 2080 rows, 32 heads: 16 -> 12 us)
      const long long blocks = ((long long)max_len + kWeightRows) / kWeightRows, more = blocks * p.hkv * n_streams / 2048;
      p.join_rows = kWeightRows * (int)(more < 1 ? 1 : more > 8 ? 8 : more);
      const int row_blocks = w_out ? (int)(((long long)max_len + p.join_rows) / p.join_rows) : 0;
      hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3(gq + row_blocks, p.hkv, n_streams), dim3(kJoinThreads), 0, stream, p);
    }
  });
  return launched();
}

int launch_cache_evict(const earn_attn_desc* desc, void* k_pages, void* v_pages, const int32_t* table, const int32_t* cache_len,
                       int n_streams, int max_pages, int n_pages, int page_size, int max_len, const float* w_in, int w_cap, int budget,
                       int first, int last, const int32_t* new_table, int new_pages, int32_t* kept, int32_t* len_out, float* w_out,
                       int w_out_cap, hipStream_t stream) {
  EvictParams p;
  p.pg = make_pages(k_pages, v_pages, table, max_pages, n_pages, page_size, desc->n_kv_heads);
  p.cache_len = cache_len; p.w_in = w_in; p.w_out = w_out; p.new_table = new_table; p.kept = kept; p.len_out = len_out;
  p.max_len = max_len; p.w_cap = w_cap; p.w_out_cap = w_out_cap;
  p.budget = budget; p.first = first; p.last = last; p.new_pages = new_pages;
  const dim3 pairs(desc->n_kv_heads, n_streams);
  if (max_len <= 4096) hipLaunchKernelGGL(evict_select_kernel<4096>, pairs, dim3(kSelectThreads), 0, stream, p);
  else if (max_len <= 32768) hipLaunchKernelGGL(evict_select_kernel<32768>, pairs, dim3(kSelectThreads), 0, stream, p);
  else hipLaunchKernelGGL(evict_select_kernel<0>, pairs, dim3(kSelectThreads), 0, stream, p);
  for_type(desc, [&](auto t, auto d) {
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value, rows = 256 / (D * (int)sizeof(T) / 16);
    hipLaunchKernelGGL((evict_move_kernel<T, D>), dim3((budget + rows - 1) / rows, desc->n_kv_heads, n_streams), dim3(256), 0, stream, p);
  });
  return launched();
}

}  // namespace earn
