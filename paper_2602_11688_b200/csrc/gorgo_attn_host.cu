// C ABI of the paged key-value cache and its attention: argument checks and launches.  Nothing here allocates,
// waits or keeps anything between calls.
#include <cmath>

#include "gorgo_tma.cuh"

using namespace gorgo;

namespace gorgo {

namespace {

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool encode3(CUtensorMap* map, uint32_t type, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
             const cuuint32_t* box) {
  static const Encode encode = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      fn = nullptr;
    return reinterpret_cast<Encode>(fn);
  }();
  const cuuint32_t step[3] = {1, 1, 1};
  const CUtensorMapDataType t = type == GORGO_E4M3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                : type == GORGO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return encode && encode(map, t, 3, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          box[0] * (type == GORGO_E4M3 ? 1 : 2) == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

bool make_pool_map(CUtensorMap* map, const void* pool, uint64_t rows, uint32_t head_dim, uint32_t type, uint32_t box_rows,
                   uint32_t box_planes) {
  const uint32_t size = type == GORGO_E4M3 ? 1 : 2;
  const uint32_t cols = head_dim * size < 128 ? head_dim : 128 / size;     // elements of a plane's row
  const cuuint64_t dims[3] = {cols, rows, head_dim / cols};
  const cuuint64_t strides[2] = {(cuuint64_t)head_dim * size, (cuuint64_t)cols * size};
  const cuuint32_t box[3] = {cols, box_rows, box_planes};
  return encode3(map, type, pool, dims, strides, box);
}

bool make_rows_map(CUtensorMap* map, const void* q, uint32_t rows, uint32_t n_heads, uint32_t head_dim, uint64_t stride,
                   uint32_t type, uint32_t box_rows, uint32_t box_heads) {
  const cuuint64_t dims[3] = {head_dim, n_heads, rows};
  const cuuint64_t strides[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {64, box_heads, box_rows};
  return encode3(map, type, q, dims, strides, box);
}

// (a test switch of the process: nothing that a call depends on otherwise)
static std::atomic<uint32_t> kv_wait_ticks{UINT32_MAX};
void set_kv_wait_ticks(uint32_t ticks) { kv_wait_ticks.store(ticks, std::memory_order_relaxed); }

}  // namespace gorgo

namespace {

// The device of the call for its duration.
struct DeviceScope {
  int prev = -1;
  bool ok = true;
  explicit DeviceScope(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; prev = -1; return; }
    if (prev == dev) prev = -1;
    else if (cudaSetDevice(dev) != cudaSuccess) ok = false;
  }
  ~DeviceScope() { if (prev >= 0) cudaSetDevice(prev); }
};

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool pow2(uint64_t x) { return x && (x & (x - 1)) == 0; }

bool cache_ok(const gorgo_kv_cache_t* c) {
  if (!c || !c->k || !c->v || !aligned(c->k, 128) || !aligned(c->v, 128)) return false;
  if (c->type > GORGO_E4M3 || (c->head_dim != 64 && c->head_dim != 128) || c->device < 0) return false;
  if (!pow2(c->page_tokens) || c->page_tokens < 16 || c->page_tokens > 1024) return false;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_pages < 1) return false;
  if ((uint64_t)c->n_pages * c->n_kv_heads * c->page_tokens >= (1ull << 31)) return false;   // rows: coordinates of a bulk copy
  const bool exps = c->k_exp && c->v_exp && aligned(c->k_exp, 16) && aligned(c->v_exp, 16);
  return c->type == GORGO_E4M3 ? exps : !c->k_exp && !c->v_exp;
}

bool batch_ok(const gorgo_kv_cache_t* c, const gorgo_kv_batch_t* b, bool decode) {
  if (!b || b->reserved || b->n_seqs > 65535) return false;
  if (b->n_seqs == 0) return true;
  if (b->total_kv >= 1ull << 40) return false;
  if (!b->kv_len || (!b->table && b->max_kv) || (!decode && !b->cu_new)) return false;
  if (!aligned(b->kv_len, 4) || !aligned(b->table, 4) || !aligned(b->status, 4) || (!decode && !aligned(b->cu_new, 4))) return false;
  if (!decode && (b->total_new >= (1u << 24) || b->max_new > b->total_new)) return false;
  return b->max_kv < (1u << 24) && (uint64_t)b->table_stride * c->page_tokens >= b->max_kv;
}

bool type_ok(const gorgo_kv_cache_t* c, uint32_t type) {
  return type <= GORGO_FP16 && (c->type == GORGO_E4M3 || c->type == type);
}

bool rows_ok(const void* p, uint64_t stride, uint64_t width) {
  return p && aligned(p, 16) && stride % 8 == 0 && stride >= width && stride < (1ull << 32);
}

KvView view(const gorgo_kv_cache_t* c) {
  return {c->k, c->v, c->k_exp, c->v_exp, c->n_pages, (uint32_t)__builtin_ctz(c->page_tokens), c->n_kv_heads};
}
BatchView view(const gorgo_kv_batch_t* b) {
  return {b->cu_new, b->kv_len, b->table, b->status, b->n_seqs, b->total_new, b->max_new, b->max_kv, b->table_stride};
}

int sm_count(int device) {
  static std::atomic<int> known[64];
  int n = device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
  if (n) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 0;
  if (device < 64) known[device].store(n, std::memory_order_relaxed);
  return n;
}

int move(bool write, const gorgo_kv_cache_t* c, const gorgo_kv_batch_t* b, const void* k, const void* v, uint32_t type,
         uint64_t ks, uint64_t vs, void* stream) {
  if (!cache_ok(c) || !batch_ok(c, b, false) || !type_ok(c, type)) return GORGO_ERR_INVALID_ARG;
  if (b->n_seqs == 0 || b->total_new == 0) return GORGO_OK;
  const uint64_t width = (uint64_t)c->n_kv_heads * c->head_dim;
  if (!rows_ok(k, ks, width) || !rows_ok(v, vs, width)) return GORGO_ERR_INVALID_ARG;
  DeviceScope dev(c->device);
  const int sms = dev.ok ? sm_count(c->device) : 0;
  if (!sms) return GORGO_ERR_CUDA;
  KvMoveArgs a = {view(c), view(b), k, v, const_cast<void*>(k), const_cast<void*>(v), ks, vs, c->head_dim, type, c->type, (uint32_t)sms};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (write ? launch_kv_write(a, st) : launch_kv_read(a, st)) == cudaSuccess ? GORGO_OK : GORGO_ERR_CUDA;
}

bool heads_ok(const gorgo_kv_cache_t* c, uint32_t n_heads) {
  return n_heads && n_heads % c->n_kv_heads == 0 && n_heads / c->n_kv_heads <= 128;
}

AttnArgs attn_args(const gorgo_kv_cache_t* c, const gorgo_kv_batch_t* b, uint32_t n_heads, uint32_t type) {
  AttnArgs a = {};
  a.kv = view(c);
  a.b = view(b);
  a.n_heads = n_heads;
  a.group = n_heads / c->n_kv_heads;
  a.head_dim = c->head_dim;
  a.type = type;
  a.store = c->type;
  a.total_kv = b->total_kv;
  return a;
}

int attend(bool decode, const gorgo_kv_cache_t* c, const gorgo_kv_batch_t* b, const void* q, uint32_t n_heads, uint32_t type,
           uint64_t qs, double scale, void* out, uint64_t os, float* lse, void* ws, uint64_t ws_bytes, void* stream) {
  if (!cache_ok(c) || !batch_ok(c, b, decode) || !type_ok(c, type) || !heads_ok(c, n_heads)) return GORGO_ERR_INVALID_ARG;
  const float scale_log2 = (float)(scale * 1.4426950408889634074);
  if (!std::isfinite(scale_log2)) return GORGO_ERR_NONFINITE_PARAM;
  const uint64_t rows = b->n_seqs == 0 ? 0 : decode ? b->n_seqs : b->total_new;
  if (rows == 0) return GORGO_OK;
  const uint64_t width = (uint64_t)n_heads * c->head_dim;
  if (rows * n_heads >= (1ull << 31) || !rows_ok(q, qs, width) || !rows_ok(out, os, width) || !aligned(lse, 4)) return GORGO_ERR_INVALID_ARG;
  AttnArgs a = attn_args(c, b, n_heads, type);
  if (!decode && !prefill_fits(a)) return GORGO_ERR_INVALID_ARG;
  DeviceScope dev(c->device);
  const int sms = dev.ok ? sm_count(c->device) : 0;
  if (!sms) return GORGO_ERR_CUDA;
  const uint64_t need = (decode ? decode_workspace(a, sms) : prefill_workspace(a, sms));
  if (need && (!ws || !aligned(ws, 256))) return GORGO_ERR_INVALID_ARG;
  if (ws_bytes < need) return GORGO_ERR_WORKSPACE_TOO_SMALL;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.q_stride = qs;
  a.out_stride = os;
  a.scale_log2 = scale_log2;
  a.workspace = ws;
  const uint32_t ticks = kv_wait_ticks.load(std::memory_order_relaxed);
  a.wait_ticks = ticks == UINT32_MAX ? kWaitTicks : (long long)ticks;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (decode ? launch_attn_decode(a, sms, st) : launch_attn_prefill(a, sms, st)) == cudaSuccess ? GORGO_OK : GORGO_ERR_CUDA;
}

}  // namespace

extern "C" {

int gorgo_kv_write(const gorgo_kv_cache_t* cache, const gorgo_kv_batch_t* batch, const void* k_new, const void* v_new,
                   uint32_t type, uint64_t k_stride, uint64_t v_stride, void* cuda_stream) {
  return move(true, cache, batch, k_new, v_new, type, k_stride, v_stride, cuda_stream);
}

int gorgo_kv_read(const gorgo_kv_cache_t* cache, const gorgo_kv_batch_t* batch, void* k_out, void* v_out, uint32_t type,
                  uint64_t k_stride, uint64_t v_stride, void* cuda_stream) {
  return move(false, cache, batch, k_out, v_out, type, k_stride, v_stride, cuda_stream);
}

int gorgo_attn_workspace_bytes(const gorgo_kv_cache_t* cache, const gorgo_kv_batch_t* batch, uint32_t n_heads, uint32_t type,
                               int decode, uint64_t* bytes_out) {
  if (!bytes_out || !cache_ok(cache) || !batch_ok(cache, batch, decode != 0) || !type_ok(cache, type) ||
      !heads_ok(cache, n_heads))
    return GORGO_ERR_INVALID_ARG;
  *bytes_out = 0;
  if (batch->n_seqs == 0) return GORGO_OK;
  const AttnArgs a = attn_args(cache, batch, n_heads, type);
  if (!decode && !prefill_fits(a)) return GORGO_ERR_INVALID_ARG;
  const int sms = sm_count(cache->device);
  if (!sms) return GORGO_ERR_CUDA;
  *bytes_out = decode ? decode_workspace(a, sms) : prefill_workspace(a, sms);
  return GORGO_OK;
}

int gorgo_attn_prefill(const gorgo_kv_cache_t* cache, const gorgo_kv_batch_t* batch, const void* q, uint32_t n_heads,
                       uint32_t type, uint64_t q_stride, double scale, void* out, uint64_t out_stride, float* lse,
                       void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
  return attend(false, cache, batch, q, n_heads, type, q_stride, scale, out, out_stride, lse, workspace, workspace_bytes,
                cuda_stream);
}

int gorgo_attn_decode(const gorgo_kv_cache_t* cache, const gorgo_kv_batch_t* batch, const void* q, uint32_t n_heads,
                      uint32_t type, uint64_t q_stride, double scale, void* out, uint64_t out_stride, float* lse,
                      void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
  return attend(true, cache, batch, q, n_heads, type, q_stride, scale, out, out_stride, lse, workspace, workspace_bytes,
                cuda_stream);
}

}  // extern "C"
