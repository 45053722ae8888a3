// Pieces that the decode kernels share, over contiguous caches and over pages: rows in 16-byte pieces, softmax states, and
// blocks of 32 keys on the 16x16x32 matrix products.
#pragma once
#include "mfma_tiles.h"

namespace earn {

template <typename T>
struct Row8;  // 8 consecutive elements of a row as floats
template <>
struct Row8<float> {
  static __device__ __forceinline__ void load(const float* p, float* x) {
    f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
    x[0] = a[0]; x[1] = a[1]; x[2] = a[2]; x[3] = a[3]; x[4] = b[0]; x[5] = b[1]; x[6] = b[2]; x[7] = b[3];
  }
  static __device__ __forceinline__ void store(float* p, const float* x) {
    f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
    *(f32x4*)p = a;
    *(f32x4*)(p + 4) = b;
  }
  // value as it will be read back from storage
  static __device__ __forceinline__ float round(float x) { return x; }
  // the 8 elements as loaded, converted on use: lets several rows be in flight without holding their floats
  struct Raw { f32x4 a, b; };
  static __device__ __forceinline__ Raw load_raw(const float* p) { return Raw{*(const f32x4*)p, *(const f32x4*)(p + 4)}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float* x) {
    x[0] = r.a[0]; x[1] = r.a[1]; x[2] = r.a[2]; x[3] = r.a[3]; x[4] = r.b[0]; x[5] = r.b[1]; x[6] = r.b[2]; x[7] = r.b[3];
  }
  static constexpr int kRowsInFlight = 2;
};
template <>
struct Row8<__bf16> {
  static __device__ __forceinline__ void load(const __bf16* p, float* x) {
    u32x4 w = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  }
  static __device__ __forceinline__ void store(__bf16* p, const float* x) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    *(u32x4*)p = w;
  }
  static __device__ __forceinline__ float round(float x) { return bf16_lo(pack_bf16(x, 0.f) & 0xffffu); }
  typedef u32x4 Raw;
  static __device__ __forceinline__ Raw load_raw(const __bf16* p) { return *(const u32x4*)p; }
  static __device__ __forceinline__ void unpack(const Raw& w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  }
  static constexpr int kRowsInFlight = 4;
};

// Sum over the LPK (8 or 16) adjacent lanes that hold one key row, left in every lane of the group.  Data-parallel
// primitives instead of shuffles through LDS: pairs, quads, the mirrored half (lane i <-> 7-i: the other quad), the
// mirrored row (lane i <-> 15-i: the other half).
template <int CTRL>
__device__ __forceinline__ float dpp_move(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LPK>
__device__ __forceinline__ float group_sum(float x) {
  static_assert(LPK == 8 || LPK == 16);
  x += dpp_move<0xB1>(x);   // quad_perm [1,0,3,2]
  x += dpp_move<0x4E>(x);   // quad_perm [2,3,0,1]
  x += dpp_move<0x141>(x);  // row_half_mirror
  if (LPK == 16) x += dpp_move<0x140>(x);  // row_mirror
  return x;
}

// merge (m2,l2,o2) into (m,l,o); all in base-2 exponent units
template <int N>
__device__ __forceinline__ void merge_state(float& m, float& l, float* o, float m2, float l2, const float* o2) {
  float mn = fmaxf(m, m2);
  float a = (m == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m - mn);
  float b = (m2 == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m2 - mn);
  l = l * a + l2 * b;
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = o[i] * a + o2[i] * b;
  m = mn;
}

// Two fp32 numbers as three words of bf16 pairs whose sum they are: w[0] = the numbers rounded, w[1] = the remainders
// rounded, w[2] = what is left.  (With two words, 16 to 17 bits, large scores and values that cancel lost what fp32 keeps:
// 64 rows, 8 heads of 128, relative error of the outputs 1.6585039e-3 against 1.6585009e-3 of their rounding alone; with
// three, as in fp32 arithmetic, the last digit at most differs from the rounding's.)
__device__ __forceinline__ void split_pair(float a, float b, unsigned (&w)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    w[i] = pack_bf16(a, b);
    a -= bf16_lo(w[i]);
    b -= bf16_hi(w[i]);
  }
}

// 16 consecutive rows share a chunk of a transposing read: two rows per chunk position at most
template <int D>
__device__ __forceinline__ int short_v_swz(int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }
// An operand in three terms times an infinite key or value element is inf - inf where the terms differ in sign, or 0 * inf
// where one is zero, instead of the infinity that the whole operand gives.  So a result that came out as NaN is worked out
// again (CAREFUL) with the first term's products on their own: where they are infinite, they are the result.
__device__ __forceinline__ void short_settle(f32x4& first, const f32x4& rest) {
#pragma unroll
  for (int i = 0; i < 4; ++i) first[i] = __builtin_isinf(first[i]) ? first[i] : first[i] + rest[i];
}
template <int D, int ROWS, bool CAREFUL>
__device__ __forceinline__ void short_scores(const bf16x8 (&kf)[2][D / 32], const __bf16 (*rot)[ROWS][D + 8], int q_row, int quad, f32x4 (&sc)[2]) {
  f32x4 sc_rest[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 2; i >= 0; --i) {
    if (CAREFUL && i == 0) {
#pragma unroll
      for (int t = 0; t < 2; ++t) { sc_rest[t] = sc[t]; sc[t] = f32x4{0.f, 0.f, 0.f, 0.f}; }
    }
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      const bf16x8 q = *(const bf16x8*)&rot[i][q_row][32 * ks + 8 * quad];
#pragma unroll
      for (int t = 0; t < 2; ++t) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][ks], q, sc[t], 0, 0, 0);
    }
  }
  if (CAREFUL) {
#pragma unroll
    for (int t = 0; t < 2; ++t) short_settle(sc[t], sc_rest[t]);
  }
}
// Masked scores -> weights (three terms), the running maximum and sum; returns what earlier sums are scaled by.
__device__ __forceinline__ float short_softmax(const f32x4 (&sc)[2], float& mrow, float& lrow, u32x4 (&pw)[3]) {
  float m = -INFINITY;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, sc[t][i]);
  m = fmaxf(m, __shfl_xor(m, 16, kWave));
  m = fmaxf(m, __shfl_xor(m, 32, kWave));
  const float mnew = fmaxf(mrow, m), ref = mnew == -INFINITY ? 0.f : mnew;
  const float alpha = __builtin_amdgcn_exp2f(mrow - ref);
  mrow = mnew;
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const float a = __builtin_amdgcn_exp2f(sc[t][i] - ref), b = __builtin_amdgcn_exp2f(sc[t][i + 1] - ref);
      sum += a + b;
      unsigned w[3];
      split_pair(a, b, w);
#pragma unroll
      for (int j = 0; j < 3; ++j) pw[j][2 * t + i / 2] = w[j];
    }
  lrow = lrow * alpha + sum;
  return alpha;
}
// o = o alpha + V^T P^T over the 32 value rows at smv; only in lanes where `mine`
template <int D, bool CAREFUL>
__device__ __forceinline__ void short_weigh(const __bf16* smv, const u32x4 (&pw)[3], float alpha, int lane, f32x4 (&o)[D / 16], bool mine = true) {
  const int r16 = lane & 15, quad = lane >> 4;
#pragma unroll
  for (int db = 0; db < D / 16; ++db) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const int row = 4 * quad + (r16 >> 2), chunk = 2 * db + ((r16 & 3) >> 1);
    const __bf16* a0 = smv + row * D + ((chunk ^ short_v_swz<D>(row)) << 3) + 4 * (r16 & 1);
    const __bf16* a1 = smv + (row + 16) * D + ((chunk ^ short_v_swz<D>(row + 16)) << 3) + 4 * (r16 & 1);
    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)a0);
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)a1);
    const bf16x8 vf = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    f32x4 was = o[db];
#pragma unroll
    for (int i = 0; i < 4; ++i) was[i] *= alpha;
    f32x4 acc = CAREFUL ? f32x4{0.f, 0.f, 0.f, 0.f} : was, acc_rest;
#pragma unroll
    for (int j = 2; j >= 0; --j) {
      if (CAREFUL && j == 0) { acc_rest = acc; acc = was; }
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pw[j]), acc, 0, 0, 0);
    }
    if (CAREFUL) short_settle(acc, acc_rest);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[db][i] = mine ? acc[i] : o[db][i];
  }
}

}  // namespace earn
