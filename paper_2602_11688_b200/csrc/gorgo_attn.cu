// Attention against a paged key-value cache (sm_100a): one warp per query row and head.
#include "gorgo_attn.cuh"

namespace gorgo {

namespace {

// Element i of pool row `row` times its power of two.
template <typename T, bool kQuant, int D>
__device__ __forceinline__ void load_row(const void* pool, const int8_t* exps, int64_t row, uint32_t lane, float* f) {
  constexpr int kPer = D / 32;            // elements of a lane
  if (kQuant) {
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

// One row of one head by a warp, key by key, with the running maximum and sum of the softmax in 32 bits: the
// definition itself, for the keys 0..seen-1 of sequence s.
template <typename T, bool kQuant, int D>
__device__ void attend_row(const AttnArgs& a, uint32_t s, int seen, uint32_t row, uint32_t h, bool bad, uint32_t lane) {
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
  for (int j = 0; j < seen && !bad; ++j) {
    const int64_t at = pool_row(a.kv, a.b, s, g, j);
    if (at < 0) { bad = true; if (lane == 0) report(a.b.status, GORGO_KV_BAD_PAGE); break; }
    load_row<T, kQuant, D>(a.kv.k, a.kv.k_exp, at, lane, k);
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) z = __fmaf_rn(q[i], k[i], z);
#pragma unroll
    for (int d = 16; d; d /= 2) z += __shfl_xor_sync(0xffffffffu, z, d);
    z *= a.scale_log2;
    load_row<T, kQuant, D>(a.kv.v, a.kv.v_exp, at, lane, k);
    const float top = fmaxf(m, z);
    const float keep = top == -INFINITY ? 1.f : exp2f(m - top), p = top == -INFINITY ? 0.f : exp2f(z - top);
    l = __fmaf_rn(l, keep, p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = __fmaf_rn(o[i], keep, p * k[i]);
    m = top;
  }
  const float inv = bad ? NAN : l == 0.f ? 0.f : 1.f / l;
  T* op = static_cast<T*>(a.out) + (size_t)row * a.out_stride + (size_t)h * D + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) *reinterpret_cast<uint32_t*>(op + i) = pack2(o[i] * inv, o[i + 1] * inv, T());
  if (a.lse && lane == 0)
    a.lse[(size_t)row * a.n_heads + h] = bad ? NAN : (m + log2f(l)) * 0.693147180559945309f;
}

template <typename T, bool kQuant, int D>
__global__ void attn_rows_kernel(const AttnArgs a, bool decode) {
  const uint32_t lane = threadIdx.x % 32;
  const uint64_t w = (uint64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
  const uint32_t h = (uint32_t)(w % a.n_heads), row = (uint32_t)(w / a.n_heads);
  if (row >= (decode ? a.b.n_seqs : a.b.total_new)) return;
  uint32_t s = row;
  int seen;
  bool bad = false;
  if (decode) {
    seen = a.b.kv_len[s];
    if (!kv_len_ok(a.b, seen)) { bad = true; report(a.b.status, GORGO_KV_BAD_LENGTH); }
  } else {
    s = warp_find_seq(a.b, row, lane);
    if (s >= a.b.n_seqs) return;
    const SeqLen q = seq_len(a.b, s);
    if (q.ok && (int)row < q.first) return;
    bad = !q.ok;
    seen = q.kv - q.n + ((int)row - q.first) + 1;
  }
  attend_row<T, kQuant, D>(a, s, seen, row, h, bad, lane);
}

template <typename T, bool kQuant, int D>
cudaError_t launch_rows(const AttnArgs& a, bool decode, cudaStream_t st) {
  const uint64_t warps = (uint64_t)(decode ? a.b.n_seqs : a.b.total_new) * a.n_heads;
  if (warps == 0) return cudaSuccess;
  attn_rows_kernel<T, kQuant, D><<<(uint32_t)((warps + 3) / 4), 128, 0, st>>>(a, decode);
  return cudaGetLastError();
}

cudaError_t dispatch_rows(const AttnArgs& a, bool decode, cudaStream_t st) {
  const bool q = a.store == GORGO_E4M3, b = a.type == GORGO_BF16, d = a.head_dim == 128;
  if (b) {
    if (q) return d ? launch_rows<__nv_bfloat16, true, 128>(a, decode, st) : launch_rows<__nv_bfloat16, true, 64>(a, decode, st);
    return d ? launch_rows<__nv_bfloat16, false, 128>(a, decode, st) : launch_rows<__nv_bfloat16, false, 64>(a, decode, st);
  }
  if (q) return d ? launch_rows<__half, true, 128>(a, decode, st) : launch_rows<__half, true, 64>(a, decode, st);
  return d ? launch_rows<__half, false, 128>(a, decode, st) : launch_rows<__half, false, 64>(a, decode, st);
}

}  // namespace

uint64_t attn_workspace(const AttnArgs& a, bool decode, int sms) { return decode ? decode_workspace(a, sms) : 0; }
cudaError_t launch_attn_prefill(const AttnArgs& a, cudaStream_t st) { return dispatch_rows(a, false, st); }

}  // namespace gorgo
