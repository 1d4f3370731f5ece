// Kernels of the paged key-value cache (sm_100a): new tokens into their pages and tokens out of them.
//
// Both move each byte once and compute next to nothing, so the bound is HBM: 2 * T * n_kv_heads * head_dim *
// (2 + stored bytes) bytes for T tokens, and for a handful of tokens the launch and the chain
// cu_new -> table -> row.  A block takes a few tokens with all their heads: one warp per token finds the sequence, the
// page and the slot while the rows are already being loaded; 16 bytes a lane.
#include "gorgo_attn.cuh"

namespace gorgo {

namespace {

constexpr int kMoveThreads = 256;
constexpr int kMaxTok = 8;                // tokens of a block: one warp finds each one's place

struct Place {
  int64_t row;                            // pool row of kv head 0, -1: none
};

// Warp w of the block finds where token first + w lies.
__device__ __forceinline__ void find_places(const KvView& kv, const BatchView& b, uint32_t first, uint32_t n_tok,
                                            int64_t* place) {
  const uint32_t w = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (w >= n_tok) return;
  const uint32_t t = first + w;
  const uint32_t s = warp_find_seq(b, t, lane);
  if (lane) return;
  int64_t row = -1;
  if (s < b.n_seqs) {                     // (rows behind the last sequence belong to nobody)
    const SeqLen q = seq_len(b, s);
    const int j = q.kv - q.n + ((int)t - q.first);
    if (q.ok && (j < 0 || (int)t < q.first)) { report(b.status, GORGO_KV_BAD_LENGTH); }
    else if (q.ok) {
      row = pool_row(kv, b, s, 0, (uint32_t)j);
      if (row < 0) report(b.status, GORGO_KV_BAD_PAGE);
    }
    if (row < 0) row = -2;                // a token of a sequence, with no place
  }
  place[w] = row;
}

// One row of a token and kv head belongs to D / 8 lanes, 8 elements each.
template <typename T, bool kQuant, int D>
__global__ void __launch_bounds__(kMoveThreads) kv_write_kernel(const KvMoveArgs a, const uint32_t n_tok) {
  constexpr uint32_t kLanes = D / 8;
  __shared__ int64_t place[kMaxTok];
  const uint32_t first = blockIdx.x * n_tok;
  const uint32_t here = min(n_tok, a.b.total_new - first), hk = a.kv.n_kv_heads;
  const uint32_t l = threadIdx.x % kLanes;
  const uint32_t rows = here * hk;
  bool known = false;
  // the lanes of a row have the same rows, and a warp runs as long as any of its lanes has one
  for (uint32_t r0 = threadIdx.x / kLanes; r0 - (threadIdx.x % 32) / kLanes < rows || !known; r0 += kMoveThreads / kLanes) {
    const bool mine = r0 < rows;
    const uint32_t tok = mine ? r0 / hk : 0, h = mine ? r0 - tok * hk : 0;
    uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (mine) {
      const size_t col = (size_t)h * D + l * 8;
      x[0] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(a.k_in) + (size_t)(first + tok) * a.k_stride + col));
      x[1] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(a.v_in) + (size_t)(first + tok) * a.v_stride + col));
    }
    if (!known) {
      find_places(a.kv, a.b, first, here, place);
      __syncthreads();
      known = true;
    }
    const int64_t base = mine ? place[tok] : -1;
    const int64_t row = base + ((int64_t)h << a.kv.page_shift);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      void* pool = w ? a.kv.v : a.kv.k;
      if (!kQuant) {
        if (base >= 0) *reinterpret_cast<uint4*>(static_cast<T*>(pool) + row * D + l * 8) = x[w];
        continue;
      }
      float f[8];
      const uint32_t* u = reinterpret_cast<const uint32_t*>(&x[w]);
      uint32_t top = 0;                   // |x| as bits: their order is that of the values, infinity and NaN on top
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 p = unpack2(u[i], T());
        f[2 * i] = p.x;
        f[2 * i + 1] = p.y;
        top = max(top, max(__float_as_uint(p.x) & 0x7fffffffu, __float_as_uint(p.y) & 0x7fffffffu));
      }
#pragma unroll
      for (uint32_t m = kLanes / 2; m; m /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
      if (base < 0) continue;
      // max|x| = f * 2^x, 1 <= f < 2, and 448 = 1.75 * 2^8: e = x - 8, one more if f > 1.75
      const int e = max(kExpMin, (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u));
      const float inv = pow2i(-e);        // exact, and so is x * inv: the code is rounded once
      uint32_t c[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i] * inv, f[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i + 2] * inv, f[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
        c[i] = lo | hi << 16;
      }
      if (top >= 0x7f800000u) c[0] = c[1] = 0x7f7f7f7fu;   // an infinity or NaN: the row is NaN
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + row * D + l * 8) = make_uint2(c[0], c[1]);
      if (l == 0) (w ? a.kv.v_exp : a.kv.k_exp)[row] = (int8_t)(top >= 0x7f800000u ? 0 : e);
    }
  }
}

template <typename T, bool kQuant, int D>
__global__ void __launch_bounds__(kMoveThreads) kv_read_kernel(const KvMoveArgs a, const uint32_t n_tok) {
  constexpr uint32_t kLanes = D / 8;
  __shared__ int64_t place[kMaxTok];
  const uint32_t first = blockIdx.x * n_tok;
  const uint32_t here = min(n_tok, a.b.total_new - first), hk = a.kv.n_kv_heads;
  find_places(a.kv, a.b, first, here, place);
  __syncthreads();
  const uint32_t l = threadIdx.x % kLanes;
  for (uint32_t r0 = threadIdx.x / kLanes; r0 < here * hk; r0 += kMoveThreads / kLanes) {
    const uint32_t tok = r0 / hk, h = r0 - tok * hk;
    const int64_t base = place[tok];
    if (base == -1) continue;
    const int64_t row = base + ((int64_t)h << a.kv.page_shift);
    const size_t col = (size_t)h * D + l * 8;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const void* pool = w ? a.kv.v : a.kv.k;
      uint4 x;
      if (base < 0) {
        x = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);   // NaN in either type
      } else if (!kQuant) {
        x = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(pool) + row * D + l * 8));
      } else {
        const uint2 c = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pool) + row * D + l * 8));
        const float m = pow2i((w ? a.kv.v_exp : a.kv.k_exp)[row]);
        uint32_t* u = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 p = unpack_e4m3((i < 2 ? c.x : c.y) >> 16 * (i & 1) & 0xffffu);
          u[i] = pack2(p.x * m, p.y * m, T());             // (the product is exact up to the type's range)
        }
      }
      T* out = static_cast<T*>(w ? a.v_out : a.k_out);
      __stcs(reinterpret_cast<uint4*>(out + (size_t)(first + tok) * (w ? a.v_stride : a.k_stride) + col), x);
    }
  }
}

template <bool kWrite, typename T, bool kQuant, int D>
cudaError_t launch_move(const KvMoveArgs& a, cudaStream_t st) {
  // Few tokens: one a block, so that their chains run side by side; else as many as keep 148 SMs in work.
  const uint32_t n_tok = a.b.total_new < 8u * 148u ? 1 : kMaxTok;
  const uint32_t grid = (a.b.total_new + n_tok - 1) / n_tok;
  if (kWrite) kv_write_kernel<T, kQuant, D><<<grid, kMoveThreads, 0, st>>>(a, n_tok);
  else kv_read_kernel<T, kQuant, D><<<grid, kMoveThreads, 0, st>>>(a, n_tok);
  return cudaGetLastError();
}

template <bool kWrite>
cudaError_t dispatch_move(const KvMoveArgs& a, cudaStream_t st) {
  const bool q = a.store == GORGO_E4M3, b = a.type == GORGO_BF16, d = a.head_dim == 128;
  if (b) {
    if (q) return d ? launch_move<kWrite, __nv_bfloat16, true, 128>(a, st) : launch_move<kWrite, __nv_bfloat16, true, 64>(a, st);
    return d ? launch_move<kWrite, __nv_bfloat16, false, 128>(a, st) : launch_move<kWrite, __nv_bfloat16, false, 64>(a, st);
  }
  if (q) return d ? launch_move<kWrite, __half, true, 128>(a, st) : launch_move<kWrite, __half, true, 64>(a, st);
  return d ? launch_move<kWrite, __half, false, 128>(a, st) : launch_move<kWrite, __half, false, 64>(a, st);
}

}  // namespace

cudaError_t launch_kv_write(const KvMoveArgs& a, cudaStream_t st) { return dispatch_move<true>(a, st); }
cudaError_t launch_kv_read(const KvMoveArgs& a, cudaStream_t st) { return dispatch_move<false>(a, st); }

}  // namespace gorgo
