// What the kernels of the paged key-value cache share: views of the cache and of a batch, where a token
// lies, and the two 16-bit types.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/gorgo.h"

namespace gorgo {

constexpr int kExpMin = -24;              // least exponent of a quantised row

struct KvView {
  void* k;
  void* v;
  int8_t* k_exp;                          // null unless quantised
  int8_t* v_exp;
  uint32_t n_pages, page_shift, n_kv_heads;
};

struct BatchView {
  const int32_t* cu_new;
  const int32_t* kv_len;
  const int32_t* table;
  uint32_t* status;
  uint32_t n_seqs, total_new, max_new, max_kv, table_stride;
};

// Launchers; every size has been checked by the caller.
struct KvMoveArgs {
  KvView kv;
  BatchView b;
  const void* k_in;                       // write: rows of new tokens
  const void* v_in;
  void* k_out;                            // read
  void* v_out;
  uint64_t k_stride, v_stride;            // elements from token to token
  uint32_t head_dim, type, store;
  uint32_t sms;                           // of the device
  uint64_t per_head;                      // set by the launcher: a division as a product
};
cudaError_t launch_kv_write(const KvMoveArgs& a, cudaStream_t st);
cudaError_t launch_kv_read(const KvMoveArgs& a, cudaStream_t st);

struct AttnArgs {
  KvView kv;
  BatchView b;
  const void* q;
  void* out;
  float* lse;                             // or null
  uint64_t q_stride, out_stride;          // elements from row to row
  uint32_t n_heads, group;                // group: query heads of a kv head
  uint32_t head_dim, type, store;
  float scale_log2;                       // scale * log2(e)
  uint64_t total_kv;
  void* workspace;
  long long wait_ticks;                   // clock ticks after which a wait gives up
};
void set_kv_wait_ticks(uint32_t ticks);   // 2^32 - 1: the default
uint64_t decode_workspace(const AttnArgs& a, int sms);
bool prefill_fits(const AttnArgs& a);           // whether the 16-bit copy of e4m3 pages has fewer than 2^31 rows
uint64_t prefill_workspace(const AttnArgs& a, int sms);
cudaError_t launch_attn_prefill(const AttnArgs& a, int sms, cudaStream_t st);
cudaError_t launch_attn_decode(const AttnArgs& a, int sms, cudaStream_t st);

#ifdef __CUDACC__

__device__ __forceinline__ void report(uint32_t* status, uint32_t bits) {
  if (status) atomicOr(status, bits);
}

// 2^e for -126 <= e <= 127, exactly.
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }

__device__ __forceinline__ float2 unpack2(uint32_t x, __nv_bfloat16) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t x, __half) {
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Two e4m3 codes (low byte first) as fp16 and as floats, exactly.
__device__ __forceinline__ uint32_t codes_to_half2(uint16_t two) {
  uint32_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"(two));
  return y;
}
__device__ __forceinline__ float2 unpack_e4m3(uint32_t two) { return unpack2(codes_to_half2((uint16_t)two), __half()); }

// Four floats as e4m3 codes (the first in the low byte), each rounded to nearest even.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  uint32_t y;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}"
      : "=r"(y) : "f"(a), "f"(b), "f"(c), "f"(d));
  return y;
}

// New tokens and all tokens of sequence s; a wrong length is reported and counts as no tokens.
// (a, e: cu_new of a sequence and of the one behind it)
__device__ __forceinline__ bool placed_ok(const BatchView& b, int a, int e) {
  return a >= 0 && e >= a && (uint32_t)e <= b.total_new && (uint32_t)(e - a) <= b.max_new;
}
struct SeqLen {
  int first, n, kv;                       // first row, new tokens, tokens in all
  bool placed, ok;                        // its place in the packed array makes sense; so does its length
};
__device__ __forceinline__ bool kv_len_ok(const BatchView& b, int kv) { return kv >= 0 && (uint32_t)kv <= b.max_kv; }
__device__ __forceinline__ SeqLen seq_len(const BatchView& b, uint32_t s) {
  const int a = b.cu_new[s], e = b.cu_new[s + 1], kv = b.kv_len[s];
  SeqLen r = {a, e - a, kv, placed_ok(b, a, e), false};
  r.ok = r.placed && kv_len_ok(b, kv);
  if (!r.ok) report(b.status, GORGO_KV_BAD_LENGTH);
  return r;
}

// Row of the pool (in units of head_dim elements) of token `j` of sequence s in kv head h; -1 if its page is
// none.  Needs j < table_stride << page_shift.
__device__ __forceinline__ int64_t pool_row(const KvView& kv, const BatchView& b, uint32_t s, uint32_t h, uint32_t j) {
  const uint32_t page = (uint32_t)b.table[(size_t)s * b.table_stride + (j >> kv.page_shift)];
  if (page >= kv.n_pages) return -1;
  return (((int64_t)page * kv.n_kv_heads + h) << kv.page_shift) + (j & ((1u << kv.page_shift) - 1));
}

// Sequence whose rows hold row t, by a warp: the number of cu_new[1..n] that are <= t.  n_seqs if none holds it.
__device__ __forceinline__ uint32_t warp_find_seq(const BatchView& b, uint32_t t, uint32_t lane) {
  // 32 places at a time narrow the range (cu_new does not decrease; where it does, what is found is checked)
  uint32_t lo = 0, hi = b.n_seqs;                          // the count lies in [lo, hi]
  while (lo < hi) {
    const uint32_t step = (hi - lo + 31) / 32;
    const uint32_t at = lo + (lane + 1) * step;            // cu_new[at] <= t: at least `at` sequences end before t
    const bool le = at <= hi && b.cu_new[at] <= (int)t;
    const uint32_t c = __popc(__ballot_sync(0xffffffffu, le));
    const uint32_t nlo = lo + c * step;
    hi = min(hi, nlo + step - 1);
    lo = min(nlo, hi);
  }
  return lo;
}

#endif  // __CUDACC__

}  // namespace gorgo
