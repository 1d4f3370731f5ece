// Kernels of the paged key-value cache (sm_100a): new tokens into their pages and tokens out of them.
//
// Both move each byte once and compute next to nothing, so the bound is HBM: 2 * T * n_kv_heads * head_dim *
// (2 + stored bytes) bytes for T tokens, and for a handful of tokens the launch and the chain
// cu_new -> table -> row.  A block takes a few tokens with all their heads: one warp finds the sequences, pages and slots
// while the rows are already being loaded; 16 bytes a lane.
// Measured, of 6,538 GB/s that a copy reaches: new turns in bf16 (273 MB) 47.7 us, 5.7 TB/s; 128,000 tokens written in e4m3
// (789 MB) 161 us back to back, 4.9 TB/s (with pauses 154), bound by its instructions; e4m3 prefixes read in bf16 (2.2 GB)
// 356 us, 6.2 TB/s.
#include "gorgo_attn.cuh"

namespace gorgo {

namespace {

constexpr int kMoveThreads = 256;
constexpr int kMaxTok = 32;               // tokens of a block at most: a lane finds each one's place

// By the first warp: where the tokens first, first + 1, ... lie: the pool row of their kv head 0; -1: the token belongs to no
// sequence, or to one whose place in the packed array makes no sense; -2: to one, but has no place.
__device__ __forceinline__ void find_places(const KvView& kv, const BatchView& b, uint32_t first, uint32_t n_tok,
                                            int64_t* place) {
  if (threadIdx.x >= 32) return;
  const uint32_t lane = threadIdx.x, t = first + lane;
  uint32_t s = warp_find_seq(b, first, lane);
  if (lane >= n_tok) return;
  for (; s < b.n_seqs; ++s) {             // neighbours: their sequences are near (and a decreasing cu_new is reported below)
    const int e = b.cu_new[s + 1];
    if (e > (int)t || e < b.cu_new[s]) break;
  }
  int64_t row = -1;
  if (s < b.n_seqs) {                     // (rows behind the last sequence belong to nobody)
    const SeqLen q = seq_len(b, s);
    const int j = q.kv - q.n + ((int)t - q.first);
    if (q.ok && (j < 0 || (int)t < q.first)) { report(b.status, GORGO_KV_BAD_LENGTH); }
    else if (q.ok) {
      row = pool_row(kv, b, s, 0, (uint32_t)j);
      if (row < 0) report(b.status, GORGO_KV_BAD_PAGE);
    }
    if (row < 0 && q.placed) row = -2;
  }
  place[lane] = row;
}

// The larger of two values in each half; NaN if one is.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, __nv_bfloat16) {
  uint32_t y;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, __half) {
  uint32_t y;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}

// One row of a token and kv head belongs to D / 8 lanes, 8 elements each; a thread has kAhead rows of K and of V in
// flight.  The powers of two of neighbouring tokens lie side by side: they are gathered and go out together.
constexpr int kAhead = 2;

template <typename T, bool kQuant, int D>
__global__ void __launch_bounds__(kMoveThreads) kv_write_kernel(const KvMoveArgs a, const uint32_t n_tok) {
  constexpr uint32_t kLanes = D / 8, kRows = kMoveThreads / kLanes;
  extern __shared__ __align__(16) int8_t gathered[];           // [2][heads][n_tok], quantised only; read eight at a time
  __shared__ int64_t place[kMaxTok];
  const uint32_t first = blockIdx.x * n_tok;
  const uint32_t here = min(n_tok, a.b.total_new - first), hk = a.kv.n_kv_heads;
  const uint32_t l = threadIdx.x % kLanes, rows = here * hk;
  bool known = false;
  // a warp runs as long as any of its lanes has a row: lanes of a row take part in its maximum together
  for (uint32_t r0 = threadIdx.x / kLanes; r0 - (threadIdx.x % 32) / kLanes < rows || !known; r0 += kAhead * kRows) {
    uint4 x[kAhead][2];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const uint32_t r = r0 + n * kRows, tok = (uint32_t)(r * a.per_head >> 32), h = r - tok * hk;
      x[n][0] = x[n][1] = make_uint4(0, 0, 0, 0);
      if (r >= rows) continue;
      const size_t col = (size_t)h * D + l * 8;
      x[n][0] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(a.k_in) + (size_t)(first + tok) * a.k_stride + col));
      x[n][1] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(a.v_in) + (size_t)(first + tok) * a.v_stride + col));
    }
    if (!known) {
      find_places(a.kv, a.b, first, here, place);
      __syncthreads();
      known = true;
    }
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const uint32_t r = r0 + n * kRows, tok = (uint32_t)(r * a.per_head >> 32), h = r - tok * hk;
      const int64_t base = r < rows ? place[tok] : -1;
      const int64_t row = base + ((int64_t)h << a.kv.page_shift);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        void* pool = w ? a.kv.v : a.kv.k;
        if (!kQuant) {
          if (base >= 0) *reinterpret_cast<uint4*>(static_cast<T*>(pool) + row * D + l * 8) = x[n][w];
          continue;
        }
        float f[8];
        const uint32_t* u = reinterpret_cast<const uint32_t*>(&x[n][w]);
        // max|x|, two at a time
        uint32_t most = max2(max2(u[0] & 0x7fff7fffu, u[1] & 0x7fff7fffu, T()), max2(u[2] & 0x7fff7fffu, u[3] & 0x7fff7fffu, T()), T());
#pragma unroll
        for (uint32_t m = kLanes / 2; m; m /= 2) most = max2(most, __shfl_xor_sync(0xffffffffu, most, m), T());
        most = max(most & 0xffffu, most >> 16);
        const uint32_t top = __float_as_uint(unpack2(most, T()).x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 p = unpack2(u[i], T());
          f[2 * i] = p.x;
          f[2 * i + 1] = p.y;
        }
        if (base < 0) continue;
        // max|x| = f * 2^x, 1 <= f < 2, and 448 = 1.75 * 2^8: e = x - 8, one more if f > 1.75
        const int e = max(kExpMin, (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u));
        const float inv = pow2i(-e);      // exact, and so is x * inv: the code is rounded once
        uint32_t c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          c[i] = codes_of(f[4 * i] * inv, f[4 * i + 1] * inv, f[4 * i + 2] * inv, f[4 * i + 3] * inv);
        }
        if (top >= 0x7f800000u) c[0] = c[1] = 0x7f7f7f7fu;     // an infinity or NaN: the row is NaN
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + row * D + l * 8) = make_uint2(c[0], c[1]);
        if (l == 0) gathered[(w * hk + h) * n_tok + tok] = (int8_t)(top >= 0x7f800000u ? 0 : e);
      }
    }
  }
  if (!kQuant) return;
  __syncthreads();
  for (uint32_t t0 = 0; t0 < here; t0 += 8) {                  // eight neighbours of a page are one store
    bool side = t0 + 8 <= here && place[t0] >= 0 && place[t0] % 8 == 0;
    for (uint32_t t = 1; side && t < 8; ++t) side = place[t0 + t] == place[t0] + t;
    for (uint32_t y = threadIdx.x; y < 2 * hk; y += kMoveThreads) {
      int8_t* out = (y >= hk ? a.kv.v_exp : a.kv.k_exp) + ((int64_t)(y >= hk ? y - hk : y) << a.kv.page_shift);
      const int8_t* in = gathered + y * n_tok + t0;
      if (side) {
        *reinterpret_cast<uint2*>(out + place[t0]) = *reinterpret_cast<const uint2*>(in);
      } else {
        for (uint32_t t = 0; t < min(8u, here - t0); ++t)
          if (place[t0 + t] >= 0) out[place[t0 + t]] = in[t];
      }
    }
  }
}

template <typename T, bool kQuant, int D>
__global__ void __launch_bounds__(kMoveThreads) kv_read_kernel(const KvMoveArgs a, const uint32_t n_tok) {
  constexpr uint32_t kLanes = D / 8, kRows = kMoveThreads / kLanes;
  __shared__ int64_t place[kMaxTok];
  const uint32_t first = blockIdx.x * n_tok;
  const uint32_t here = min(n_tok, a.b.total_new - first), hk = a.kv.n_kv_heads;
  find_places(a.kv, a.b, first, here, place);
  __syncthreads();
  const uint32_t l = threadIdx.x % kLanes, rows = here * hk;
  for (uint32_t r0 = threadIdx.x / kLanes; r0 < rows; r0 += kAhead * kRows) {
    uint4 x[kAhead][2];
    int e[kAhead][2];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const uint32_t r = r0 + n * kRows, tok = (uint32_t)(r * a.per_head >> 32), h = r - tok * hk;
      const int64_t base = r < rows ? place[tok] : -1;
      const int64_t row = base + ((int64_t)h << a.kv.page_shift);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const void* pool = w ? a.kv.v : a.kv.k;
        e[n][w] = 0;
        if (base < 0) {
          x[n][w] = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);   // NaN in all of the types
        } else if (!kQuant) {
          x[n][w] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(pool) + row * D + l * 8));
        } else {
          const uint2 c = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pool) + row * D + l * 8));
          x[n][w] = make_uint4(c.x, c.y, 0, 0);
          e[n][w] = (w ? a.kv.v_exp : a.kv.k_exp)[row];
        }
      }
    }
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const uint32_t r = r0 + n * kRows, tok = (uint32_t)(r * a.per_head >> 32), h = r - tok * hk;
      const int64_t base = r < rows ? place[tok] : -1;
      if (base == -1) continue;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        uint4 y = x[n][w];
        if (kQuant && base >= 0) {
          const float m = pow2i(e[n][w]);
          uint32_t* u = reinterpret_cast<uint32_t*>(&y);
          const uint32_t c[2] = {x[n][w].x, x[n][w].y};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 p = unpack_e4m3(c[i >> 1] >> 16 * (i & 1) & 0xffffu);
            u[i] = pack2(p.x * m, p.y * m, T());               // (the product is exact up to the type's range)
          }
        }
        T* out = static_cast<T*>(w ? a.v_out : a.k_out);
        __stcs(reinterpret_cast<uint4*>(out + (size_t)(first + tok) * (w ? a.v_stride : a.k_stride) + (size_t)h * D + l * 8), y);
      }
    }
  }
}

template <bool kWrite, typename T, bool kQuant, int D>
cudaError_t launch_move(const KvMoveArgs& a, cudaStream_t st) {
  // Few tokens: one a block, so that their chains run side by side (1,000 tokens read with eight a block are 2.6 us, with one
  // 4.9; 400 written in e4m3 the other way round 4.6 and 3.7, 1,000 again 4.7 and 5.8).  Many: eight, or 32 where codes are written (128,000 tokens:
  // 154 against 165 us; read, 32 are 360 against 349 us), if the gathered powers of two leave room for them.
  const bool codes = kWrite && kQuant;
  const uint32_t n_tok = a.b.total_new < (codes ? 4u : 2u) * a.sms ? 1
                         : a.b.total_new < 8u * a.sms * 32u || !codes || a.kv.n_kv_heads > 64 ? 8 : kMaxTok;
  const uint32_t grid = (a.b.total_new + n_tok - 1) / n_tok;
  if (kWrite) kv_write_kernel<T, kQuant, D><<<grid, kMoveThreads, kQuant ? 2 * a.kv.n_kv_heads * n_tok : 0, st>>>(a, n_tok);
  else kv_read_kernel<T, kQuant, D><<<grid, kMoveThreads, 0, st>>>(a, n_tok);
  return cudaGetLastError();
}

template <bool kWrite>
cudaError_t dispatch_move(KvMoveArgs a, cudaStream_t st) {
  // r / n_kv_heads = r * per_head / 2^32 for r < 2^22: per_head is too large by less than 1
  a.per_head = ((1ull << 32) + a.kv.n_kv_heads - 1) / a.kv.n_kv_heads;
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
