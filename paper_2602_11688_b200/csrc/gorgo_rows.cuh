// One row of one head against the paged key-value cache, key by key: the definition itself.  Prefill falls back on it for
// rows that a value which is not finite has reached although the row does not see it.
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
// the softmax in 32 bits.  32 keys at a time, a lane looks up each one's page; eight rows are in flight.
template <typename T, int D>
__device__ __noinline__ void attend_row(const AttnArgs& a, uint32_t s, int seen, uint32_t row, uint32_t h, uint32_t lane) {
  constexpr int kPer = D / 32, kFly = 4;
  const uint32_t g = h / a.group;
  float q[kPer], o[kPer];
  const T* qp = static_cast<const T*>(a.q) + (size_t)row * a.q_stride + (size_t)h * D + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) {
    const float2 v = unpack2(*reinterpret_cast<const uint32_t*>(qp + i), T());
    q[i] = v.x;
    q[i + 1] = v.y;
    o[i] = o[i + 1] = 0.f;
  }
  float m = -INFINITY, l = 0.f;           // l: this lane's keys
  for (int j0 = 0; j0 < seen; j0 += 32) {
    const int n = min(32, seen - j0);
    const int64_t at = (int)lane < n ? pool_row(a.kv, a.b, s, g, j0 + lane) : 0;
    if (__any_sync(0xffffffffu, at < 0)) return;               // (reported, and NaN already)
    float z = -INFINITY;                  // of key j0 + lane
    for (int k0 = 0; k0 < n; k0 += kFly) {
      float k[kFly][kPer], dot[kFly];
#pragma unroll
      for (int x = 0; x < kFly; ++x) {    // (keys behind the last one: the last one once more)
        const int64_t r = __shfl_sync(0xffffffffu, at, min(k0 + x, n - 1));
        load_row<T, D>(a.kv.k, a.kv.k_exp, r, lane, k[x]);
      }
#pragma unroll
      for (int x = 0; x < kFly; ++x) {
        dot[x] = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) dot[x] = __fmaf_rn(q[i], k[x][i], dot[x]);
      }
#pragma unroll
      for (int d = 16; d; d /= 2)
#pragma unroll
        for (int x = 0; x < kFly; ++x) dot[x] += __shfl_xor_sync(0xffffffffu, dot[x], d);
#pragma unroll
      for (int x = 0; x < kFly; ++x)
        if ((int)lane == k0 + x && k0 + x < n) z = dot[x] * a.scale_log2;
    }
    float top = z;                        // (NaN is taken care of below)
#pragma unroll
    for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    top = fmaxf(top, m);
    if (__any_sync(0xffffffffu, !(z < INFINITY))) {            // a score that is NaN or infinite: so is the row
      l = NAN;
      break;
    }
    const float keep = m == top ? 1.f : exp2f(m - top), p = z == -INFINITY ? 0.f : exp2f(z - top);
    l = __fmaf_rn(l, keep, p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] *= keep;
    for (int k0 = 0; k0 < n; k0 += kFly) {
      float v[kFly][kPer];
#pragma unroll
      for (int x = 0; x < kFly; ++x) load_row<T, D>(a.kv.v, a.kv.v_exp, __shfl_sync(0xffffffffu, at, min(k0 + x, n - 1)), lane, v[x]);
#pragma unroll
      for (int x = 0; x < kFly; ++x) {
        const float w = __shfl_sync(0xffffffffu, p, min(k0 + x, n - 1));
        if (k0 + x < n)
#pragma unroll
          for (int i = 0; i < kPer; ++i) o[i] = __fmaf_rn(w, v[x][i], o[i]);
      }
    }
    m = top;
  }
#pragma unroll
  for (int d = 16; d; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* op = static_cast<T*>(a.out) + (size_t)row * a.out_stride + (size_t)h * D + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) *reinterpret_cast<uint32_t*>(op + i) = pack2(o[i] * inv, o[i + 1] * inv, T());
}

// By a warp, for a row at position `pos` whose tile of rows took the keys up to `end`: computes it again if an element is not
// finite and a value behind pos is the cause.  Where a value that the row sees among the keys from..pos is not finite either,
// the element would be that anyway.
template <typename T, int D>
__device__ __noinline__ void mend_row(const AttnArgs& a, uint32_t s, int from, int pos, int end, uint32_t row, uint32_t h, uint32_t lane) {
  constexpr int kPer = D / 32;
  const T* op = static_cast<const T*>(a.out) + (size_t)row * a.out_stride + (size_t)h * D + lane * kPer;
  bool seen[kPer], behind[kPer];          // whether a value there is not finite; elements that are finite count as seen
#pragma unroll
  for (int i = 0; i < kPer; i += 2) {
    const float2 v = unpack2(*reinterpret_cast<const uint32_t*>(op + i), T());
    seen[i] = fabsf(v.x) < INFINITY;
    seen[i + 1] = fabsf(v.y) < INFINITY;
    behind[i] = behind[i + 1] = false;
  }
  for (int j = from; j < end; ++j) {
    const int64_t at = pool_row(a.kv, a.b, s, h / a.group, j);
    float v[kPer];
    if (at >= 0) load_row<T, D>(a.kv.v, a.kv.v_exp, at, lane, v);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const bool none = at < 0 || !(fabsf(v[i]) < INFINITY);   // (a wrong page's stand-in may be anything)
      seen[i] |= none && j <= pos;
      behind[i] |= none && j > pos;
    }
  }
  bool cause = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) cause |= behind[i] && !seen[i];
  if (__any_sync(0xffffffffu, cause)) attend_row<T, D>(a, s, pos + 1, row, h, lane);
}

}  // namespace gorgo
