// One row of one head against the paged key-value cache, key by key: the definition itself.  The fast kernels fall
// back on it for rows that a value which is not finite has reached although the row does not see it.
#pragma once
#include "gorgo_attn.cuh"

namespace gorgo {

// A lane's elements of pool row `row` times its power of two.
template <typename T, int D>
__device__ __forceinline__ void load_row(const void* pool, const int8_t* exps, int64_t row, uint32_t lane, float* f) {
  constexpr int kPer = D / 32;
  if (exps) {
    const uint8_t* p = static_cast<const uint8_t*>(pool) + row * D + lane * kPer;
    const float m = pow2i(exps[row]);
#pragma unroll
    for (int i = 0; i < kPer; i += 2) {
      const float2 v = unpack_e4m3(*reinterpret_cast<const uint16_t*>(p + i));
      f[i] = v.x * m;
      f[i + 1] = v.y * m;
    }
  } else {
    const T* p = static_cast<const T*>(pool) + row * D + lane * kPer;
#pragma unroll
    for (int i = 0; i < kPer; i += 2) {
      const float2 v = unpack2(*reinterpret_cast<const uint32_t*>(p + i), T());
      f[i] = v.x;
      f[i + 1] = v.y;
    }
  }
}

// By a warp: writes the row's result over the keys 0..seen-1 of sequence s, with the running maximum and sum of
// the softmax in 32 bits.
template <typename T, int D>
__device__ __noinline__ void attend_row(const AttnArgs& a, uint32_t s, int seen, uint32_t row, uint32_t h, uint32_t lane) {
  constexpr int kPer = D / 32;
  const uint32_t g = h / a.group;
  float q[kPer], o[kPer], k[kPer];
  const T* qp = static_cast<const T*>(a.q) + (size_t)row * a.q_stride + (size_t)h * D + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) {
    const float2 v = unpack2(*reinterpret_cast<const uint32_t*>(qp + i), T());
    q[i] = v.x;
    q[i + 1] = v.y;
    o[i] = o[i + 1] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int j = 0; j < seen; ++j) {
    const int64_t at = pool_row(a.kv, a.b, s, g, j);
    if (at < 0) return;                   // (reported, and NaN already)
    load_row<T, D>(a.kv.k, a.kv.k_exp, at, lane, k);
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) z = __fmaf_rn(q[i], k[i], z);
#pragma unroll
    for (int d = 16; d; d /= 2) z += __shfl_xor_sync(0xffffffffu, z, d);
    z *= a.scale_log2;
    load_row<T, D>(a.kv.v, a.kv.v_exp, at, lane, k);
    const float top = fmaxf(m, z);
    const float keep = m == top ? 1.f : exp2f(m - top), p = z == -INFINITY ? 0.f : exp2f(z - top);   // (a NaN in z stays)
    l = __fmaf_rn(l, keep, p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = __fmaf_rn(o[i], keep, p * k[i]);
    m = top;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* op = static_cast<T*>(a.out) + (size_t)row * a.out_stride + (size_t)h * D + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) *reinterpret_cast<uint32_t*>(op + i) = pack2(o[i] * inv, o[i + 1] * inv, T());
}

// By a warp, for a row at position `pos` whose result is not finite: is one of the values behind it that its tile
// of rows took, keys pos + 1 to min(end, kv) - 1, the cause?  Then it is computed again.
template <typename T, int D>
__device__ __forceinline__ void mend_row(const AttnArgs& a, uint32_t s, int pos, int end, int kv, uint32_t row, uint32_t h, uint32_t lane) {
  constexpr int kPer = D / 32;
  bool cause = false;
  for (int j = max(pos + 1, 0); j < min(end, kv); ++j) {
    const int64_t at = pool_row(a.kv, a.b, s, h / a.group, j);
    if (at < 0) { cause = true; break; }  // (its stand-in may be anything)
    float v[kPer];
    load_row<T, D>(a.kv.v, a.kv.v_exp, at, lane, v);
#pragma unroll
    for (int i = 0; i < kPer; ++i) cause |= !(fabsf(v[i]) < INFINITY);
  }
  if (__any_sync(0xffffffffu, cause)) attend_row<T, D>(a, s, pos + 1, row, h, lane);
}

}  // namespace gorgo
