// Attention of the uncached tokens of packed prompts over the paged key-value cache (sm_100a).
//
// Mathematics.  Rows are (token, head) pairs of one kv head; with S = Q K^T, running maximum m and sum l of a row in
// 32 bits, P = 2^(c S - c m): O <- O 2^(c (m_old - m)) + P V, out = O / l.  The maximum that P is taken against
// moves only when a row's true maximum has grown by more than 2^8 beyond it: that leaves the result the same (O and l
// carry the same factor) and makes rescaling O rare; P stays below 2^8.
//
// What bounds it: 4 * 128 * 128 * D operations of the tensor pipe for each 128 x 128 piece of S and as many
// exponentials as elements, which at D = 128 take the same 1,024 cycles of an SM.  So one tile's softmax has to run
// under the other tile's products.
//
// A block takes one kv head and two tiles of 128 rows, floor(128 / group) tokens each with all their query heads, so
// that keys and values serve a whole group and both tiles.  Warps: 0-3 and 4-7 softmax of the tiles, a row a thread
// (TMEM lane), no shuffles; 8 copies; 9 issues tcgen05.mma (10 and 11 only hand in registers), S of one tile while the other is in softmax.  TMEM: S of
// both tiles (P of 16 bits takes the place of the S it came from, and is the first operand of P V there), O of both.
// Keys and values come page by page in tiled bulk copies, 128 keys a slot, each as planes of 128-byte rows with
// the 128-byte swizzle; V is the second operand as it lies (its dims contiguous).
//
// Values behind the last key of a sequence may be anything: they are overwritten with zeros in shared memory.  A value
// that is not finite and that a row of its tile does not see would reach the row as 0 * x: rows whose result is not
// finite look at the values behind their own last key, and are computed again key by key if one of those is the cause.
//
// Few rows against long prefixes: the keys are split among blocks and joined by a second kernel.
//
// e4m3 pages are first written out in 16 bits (exactly) into the workspace, once for all rows that read them.
#include "gorgo_rows.cuh"
#include "gorgo_tma.cuh"

namespace gorgo {

namespace {

constexpr int kThreads = 384;            // three warpgroups: registers can be moved between these only
constexpr int kKeys = 128;                // keys of a tile
constexpr uint32_t kPlane = kKeys * 128;  // bytes of 128 rows of 128 bytes

template <int D>
struct Sizes {
  static constexpr int kPlanes = D / 64;
  static constexpr int kTile = kPlanes * kPlane;               // bytes of 128 rows of Q, K or V
  static constexpr int kSlots = D == 128 ? 5 : 10;
  static constexpr int kBars = 2 * kSlots + 11;
  static constexpr int kBytes = 2 * kTile + kSlots * kTile + 8 * kBars + 128;
  static constexpr int kO = 256;                               // first TMEM column of O; S of tile i begins at 128 i
};

struct Plan {
  uint32_t tq;                            // tokens of a tile: floor(128 / group)
  uint32_t splits;
  uint32_t box;                           // keys of one bulk copy
  uint64_t linear;                        // rows of a head in the 16-bit copy of e4m3 pages; 0: the pages themselves
  uint32_t negate;                        // the scale is negative: S takes -Q
  float scale;                            // |scale| * log2(e)
  float* part_o;                          // [splits][rows][heads][D]
  float* part_ml;                         // [splits][rows][heads][2]
};

struct Work {                             // what a block does
  uint32_t s, h;                          // sequence, kv head
  int first, n, kv;                       // its first row, new tokens, tokens in all
  int q0;                                 // first token of the block
  int tiles[2];                           // tiles of keys of either tile of rows, from 0
  int lo, hi;                             // the block's share of them
  uint32_t bad;
  uint64_t base;                          // first row of the sequence in the 16-bit copy
};

// ------------------------------------------------------------------ tcgen05
// One thread of a converged warp; the compiler knows that what follows runs alone and keeps operands in uniform registers.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Operands in shared memory, rows of 128 bytes in the 128-byte swizzle, groups of 8 rows 1,024 bytes apart: the low word
// has the address and `lead`, the bytes from one 64-element plane to the next where the rows run along the summed
// dimension (V; else unused), in units of 16; the high word is the same for all.
constexpr uint32_t kOperandHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t operand(uint32_t addr, uint32_t lead) { return addr >> 4 | (lead >> 4) << 16; }

__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 x, {%1, %3};\n\tmov.b64 y, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "n"(kOperandHigh), "r"(shape), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 y, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "n"(kOperandHigh), "r"(shape), "r"(acc) : "memory");
}
#define GORGO_R32(r, o)                                                                                              \
  "=r"((r)[(o) + 0]), "=r"((r)[(o) + 1]), "=r"((r)[(o) + 2]), "=r"((r)[(o) + 3]), "=r"((r)[(o) + 4]),                \
      "=r"((r)[(o) + 5]), "=r"((r)[(o) + 6]), "=r"((r)[(o) + 7]), "=r"((r)[(o) + 8]), "=r"((r)[(o) + 9]),            \
      "=r"((r)[(o) + 10]), "=r"((r)[(o) + 11]), "=r"((r)[(o) + 12]), "=r"((r)[(o) + 13]), "=r"((r)[(o) + 14]),       \
      "=r"((r)[(o) + 15]), "=r"((r)[(o) + 16]), "=r"((r)[(o) + 17]), "=r"((r)[(o) + 18]), "=r"((r)[(o) + 19]),       \
      "=r"((r)[(o) + 20]), "=r"((r)[(o) + 21]), "=r"((r)[(o) + 22]), "=r"((r)[(o) + 23]), "=r"((r)[(o) + 24]),       \
      "=r"((r)[(o) + 25]), "=r"((r)[(o) + 26]), "=r"((r)[(o) + 27]), "=r"((r)[(o) + 28]), "=r"((r)[(o) + 29]),       \
      "=r"((r)[(o) + 30]), "=r"((r)[(o) + 31])
#define GORGO_I32(r)                                                                                                 \
  "r"((r)[0]), "r"((r)[1]), "r"((r)[2]), "r"((r)[3]), "r"((r)[4]), "r"((r)[5]), "r"((r)[6]), "r"((r)[7]),            \
      "r"((r)[8]), "r"((r)[9]), "r"((r)[10]), "r"((r)[11]), "r"((r)[12]), "r"((r)[13]), "r"((r)[14]), "r"((r)[15]),  \
      "r"((r)[16]), "r"((r)[17]), "r"((r)[18]), "r"((r)[19]), "r"((r)[20]), "r"((r)[21]), "r"((r)[22]),              \
      "r"((r)[23]), "r"((r)[24]), "r"((r)[25]), "r"((r)[26]), "r"((r)[27]), "r"((r)[28]), "r"((r)[29]),              \
      "r"((r)[30]), "r"((r)[31])
__device__ __forceinline__ void tmem_ld32(uint32_t* r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : GORGO_R32(r, 0) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
      ::GORGO_I32(r), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 128 x n product of 16-bit operands, summed in 32 bits.
__device__ __forceinline__ uint32_t mma_shape(uint32_t n, bool bf16, bool negate_a, bool b_by_rows) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (negate_a ? 1u << 13 : 0u) | (b_by_rows ? 1u << 16 : 0u) |
         (n >> 3) << 17 | (128u >> 4) << 24;
}

// ------------------------------------------------------------------ who does what
// New rows of sequence s if its place in the packed array makes sense, else none.
__device__ __forceinline__ int rows_of(const BatchView& b, uint32_t s) {
  const int a = b.cu_new[s], e = b.cu_new[s + 1];
  return a < 0 || e < a || (uint32_t)e > b.total_new ? 0 : e - a;
}

// By one warp: the block's sequence and tokens, the last blocks of a sequence first (they see the most keys).
__device__ bool find_work(const AttnArgs& a, const Plan& p, Work& w, uint32_t lane) {
  const int step = 2 * p.tq;
  uint32_t total = 0;
  uint64_t base = 0;
  for (uint32_t s = lane; s < a.b.n_seqs; s += 32) total += (rows_of(a.b, s) + step - 1) / step;
  total = __reduce_add_sync(0xffffffffu, total);
  if (blockIdx.x >= total) return false;
  const uint32_t want = total - 1 - blockIdx.x;
  uint32_t before = 0;
  for (uint32_t s0 = 0;; s0 += 32) {
    const uint32_t s = s0 + lane;
    const int n = s < a.b.n_seqs ? rows_of(a.b, s) : 0;
    uint32_t mine = (n + step - 1) / step, upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= (uint32_t)d) upto += o;
    }
    const uint32_t over = __ballot_sync(0xffffffffu, before + upto > want);
    const uint32_t here = over ? __ffs(over) - 1 : 32;
    if (p.linear) {                       // the sequences before it in the 16-bit copy, each from a multiple of 128
      const int kv = s < a.b.n_seqs && lane < here ? a.b.kv_len[s] : 0;
      base += __reduce_add_sync(0xffffffffu, kv_len_ok(a.b, kv) ? (uint32_t)(kv + kKeys - 1) / kKeys : 0);
    }
    if (over) {
      w.s = s0 + here;
      w.n = __shfl_sync(0xffffffffu, n, here);
      w.q0 = (int)(want - before - __shfl_sync(0xffffffffu, upto - mine, here)) * step;
      break;
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
  }
  w.h = blockIdx.y;
  w.first = a.b.cu_new[w.s];
  w.kv = a.b.kv_len[w.s];
  w.base = base * kKeys;
  w.bad = !kv_len_ok(a.b, w.kv) || (p.linear && w.base + w.kv > p.linear);
  if (w.bad) {
    if (lane == 0) report(a.b.status, GORGO_KV_BAD_LENGTH);
    w.kv = 0;
  }
  int most = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = w.q0 + i * (int)p.tq;   // first token of the tile
    const int last = w.kv - w.n + min(t + (int)p.tq, w.n) - 1;   // position of its last
    w.tiles[i] = t >= w.n || last < 0 ? 0 : last / kKeys + 1;
    most = max(most, w.tiles[i]);
  }
  const int share = (most + (int)p.splits - 1) / (int)p.splits;
  w.lo = min(most, (int)blockIdx.z * share);
  w.hi = min(most, w.lo + share);
  return true;
}

// Waits; on the limit tells the block (and the host) to give up.
__device__ __forceinline__ bool wait_or_give_up(uint32_t bar, uint32_t parity, volatile uint32_t* quit, uint32_t* status) {
  if (mbar_try(bar, parity)) return true;
  const long long from = clock64();
  while (!mbar_try(bar, parity)) {
    if (*quit) return false;
    if (clock64() - from > kWaitTicks) {
      *quit = 1;
      report(status, GORGO_KV_WAIT_LIMIT);
      return false;
    }
  }
  return true;
}

template <typename T> constexpr float kShift = 0.f;      // P = 2^(c (S - m) + kShift)
template <> constexpr float kShift<__half> = 6.f;        // fp16: normal down to 2^-20 of the largest, below 2^15

// The larger of three; NaN if one is.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// Two floats in one register pair, and arithmetic on both at once.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 both(float x, float y) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 apart(f32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
prefill_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Plan p, const __grid_constant__ CUtensorMap q_map,
               const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using Z = Sizes<D>;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ Work work;
  __shared__ uint32_t tmem_base, quit, found;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t q_a = smem_u32(smem), ring_a = q_a + 2 * Z::kTile;
  const uint32_t bars = ring_a + Z::kSlots * Z::kTile;
  const uint32_t full = bars, empty = full + 8 * Z::kSlots, q_full = empty + 8 * Z::kSlots, s_full = q_full + 8,
                 p_full = s_full + 16, o_full = p_full + 32, drained = o_full + 16, tail = drained + 8;

  if (warp == 8) {
    Work w;
    const bool some = find_work(a, p, w, lane);
    if (lane == 0) {
      if (some) work = w;
      found = some;
      quit = 0;
      for (int i = 0; i < Z::kSlots; ++i) {
        mbar_init(full + 8 * i, 1);
        mbar_init(empty + 8 * i, 1);
      }
      mbar_init(q_full, 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(s_full + 8 * i, 1);
        mbar_init(p_full + 16 * i, 128);
        mbar_init(p_full + 16 * i + 8, 128);
        mbar_init(o_full + 8 * i, 1);
      }
      mbar_init(drained, 1);
      mbar_init(tail, 1);
      mbar_init_fence();
    }
  }
  if (warp == 9 && lane == 0) {
    prefetch_map(&q_map);
    prefetch_map(&k_map);
    prefetch_map(&v_map);
  }
  __syncthreads();
  if (!found) return;
  if (warp == 9) tmem_alloc(smem_u32(&tmem_base), 512);
  fence_before();
  __syncthreads();
  fence_after();
  const Work w = work;
  const uint32_t tmem = tmem_base;
  const int steps[2] = {max(0, min(w.hi, w.tiles[0]) - w.lo), max(0, min(w.hi, w.tiles[1]) - w.lo)};
  const int most = max(steps[0], steps[1]);
  const bool ragged = most > 0 && (w.lo + most) * kKeys > w.kv;  // the last tile of keys is not full

  // Registers: 384 threads of 168 at the launch; the softmax takes what the last warpgroup does not need
  // (2 * 200 + 104 = 3 * 168).
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // ---------------------------------------------------------------- softmax, a row a thread
    const int i = warp / 4;
    const uint32_t r = warp % 4 * 32 + lane, at = tmem + (warp % 4 * 32 << 16);
    const uint32_t s_at = at + 128 * i, o_at = at + Z::kO + D * i;
    const uint32_t tok = r / a.group;
    const int t = w.q0 + i * (int)p.tq + (int)tok;             // token of the row
    const bool mine = tok < p.tq && t < w.n;
    const int pos = w.kv - w.n + t;
    const float c = p.scale, slack = 8.f / c;
    float m = -INFINITY, l = 0.f;
    bool go = true;
    for (int j = 0; j < steps[i]; ++j) {
      go = __all_sync(0xffffffffu, wait_or_give_up(s_full + 8 * i, j & 1, &quit, a.b.status));
      if (!go) break;
      fence_after();
      const int seen = pos - (w.lo + j) * kKeys + 1;           // columns that the row sees
      const bool masked = __any_sync(0xffffffffu, seen < kKeys);
      // Half of a row at a time: the second half is read twice, which costs less than the registers for all of it.
      uint32_t x[64];
      auto read = [&](int k) {
        tmem_ld32(x, s_at + 64 * k);
        tmem_ld32(x + 32, s_at + 64 * k + 32);
        tmem_wait_ld();
        if (masked) {
          const int left = seen - 64 * k;
#pragma unroll
          for (int y = 0; y < 64; ++y)
            if (y >= left) x[y] = 0xff800000u;
        }
      };
      float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int k = 1; k >= 0; --k) {
        read(k);
#pragma unroll
        for (int y = 0; y < 64; y += 2) top[y / 2 % 4] = max3(top[y / 2 % 4], __uint_as_float(x[y]), __uint_as_float(x[y + 1]));
      }
      float now = max3(max3(top[0], top[1], top[2]), top[3], -INFINITY);
      const bool grow = !(now <= m + slack);                   // (also for NaN)
      if (__any_sync(0xffffffffu, grow)) {
        if (now == INFINITY) now = NAN;                        // infinity - infinity: the row is NaN
        const float f = grow ? fast_exp2((m - now) * c) : 1.f;
        if (grow) m = now;
        l *= f;
        if (j > 0) {
#pragma unroll
          for (int k = 0; k < D / 32; ++k) {
            uint32_t o[32];
            tmem_ld32(o, o_at + 32 * k);
            tmem_wait_ld();
#pragma unroll
            for (int y = 0; y < 32; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * f);
            tmem_st32(o_at + 32 * k, o);
          }
        }
      }
      const float off = m == -INFINITY ? 0.f : kShift<T> - m * c;
      // P in halves of 64 keys: their products with V begin while the other half is computed
      f32x2 sum[4] = {0, 0, 0, 0};
      const f32x2 c2 = both(c, c), off2 = both(off, off);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (k) read(1);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t pk[16];
#pragma unroll
          for (int y = 0; y < 16; ++y) {
            float2 e = apart(fma2(both(__uint_as_float(x[32 * q + 2 * y]), __uint_as_float(x[32 * q + 2 * y + 1])), c2, off2));
            e.x = fast_exp2(e.x);
            e.y = fast_exp2(e.y);
            sum[y % 4] = add2(sum[y % 4], both(e.x, e.y));
            pk[y] = pack2(e.x, e.y, T());
          }
          tmem_st16(s_at + 32 * k + 16 * q, pk);
        }
        tmem_wait_st();
        fence_before();
        mbar_arrive(p_full + 8 * (2 * i + k));
      }
      const float2 l2 = apart(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
      l += l2.x + l2.y;
    }
    if (steps[i] && go) {
      go = __all_sync(0xffffffffu, wait_or_give_up(o_full + 8 * i, 0, &quit, a.b.status));
      fence_after();
    }
    const uint32_t head = w.h * a.group + r % a.group;
    const size_t row = (size_t)(w.first + t);
    const bool bad = work.bad != 0 || !go;
    if (p.splits > 1) {
      const size_t part = ((size_t)blockIdx.z * a.b.total_new + row) * a.n_heads + head;
      if (mine) *reinterpret_cast<float2*>(p.part_ml + 2 * part) = make_float2(m * c, bad ? NAN : l);
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        if (!steps[i] || !go) break;
        uint32_t o[32];
        tmem_ld32(o, o_at + 32 * k);
        tmem_wait_ld();
        if (mine)
#pragma unroll
          for (int y = 0; y < 8; ++y)
            *reinterpret_cast<uint4*>(p.part_o + part * D + 32 * k + 4 * y) = make_uint4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]);
      }
    } else {
      // a row without keys: zeros
      const float inv = bad ? NAN : l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
      bool odd = false;
      T* out = static_cast<T*>(a.out) + row * a.out_stride + (size_t)head * D;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        uint32_t o[32];
        if (steps[i] && go) {
          tmem_ld32(o, o_at + 32 * k);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int y = 0; y < 32; ++y) o[y] = 0;
        }
        uint4 v[4];
        uint32_t* u = reinterpret_cast<uint32_t*>(v);
#pragma unroll
        for (int y = 0; y < 16; ++y) {
          const float f = __uint_as_float(o[2 * y]) * inv, g = __uint_as_float(o[2 * y + 1]) * inv;
          odd |= !(fabsf(f) < INFINITY) || !(fabsf(g) < INFINITY);
          u[y] = pack2(f, g, T());
        }
        if (mine)
#pragma unroll
          for (int y = 0; y < 4; ++y) *reinterpret_cast<uint4*>(out + 32 * k + 8 * y) = v[y];
      }
      if (mine && a.lse) a.lse[row * a.n_heads + head] = bad ? NAN : l == 0.f ? -INFINITY : (m * c - kShift<T> + log2f(l)) * 0.693147180559945309f;
      uint32_t again = __ballot_sync(0xffffffffu, mine && odd && !bad);
      for (; again; again &= again - 1) {
        const uint32_t b = __ffs(again) - 1;
        mend_row<T, D>(a, w.s, __shfl_sync(0xffffffffu, pos, b), w.tiles[i] * kKeys, w.kv, (uint32_t)__shfl_sync(0xffffffffu, (int)row, b),
                       __shfl_sync(0xffffffffu, head, b), lane);
      }
    }
    fence_before();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == 8) {
      // ---------------------------------------------------------------- copies
      if (most > 0) {
        if (lane == 0) {
          const uint32_t rows = p.tq * a.group;
          uint32_t bytes = 0;
          for (int i = 0; i < 2; ++i) bytes += steps[i] ? Z::kPlanes * rows * 128 : 0;
          mbar_expect(q_full, bytes);
          for (int i = 0; i < 2; ++i)
            for (int c = 0; steps[i] && c < Z::kPlanes; ++c)
              asm volatile(
                  "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                  ::"r"(q_a + i * Z::kTile + c * kPlane), "l"(reinterpret_cast<uint64_t>(&q_map)), "r"(c * 64),
                  "r"((int)(w.h * a.group)), "r"(w.first + w.q0 + i * (int)p.tq), "r"(q_full) : "memory");
        }
        // a lane a piece: the piece's page is looked up a tile ahead
        const uint32_t most_pieces = kKeys / p.box;
        auto row_of = [&](int j) -> int64_t {
          const int key = (w.lo + j) * kKeys + (int)(lane * p.box);
          if (lane >= most_pieces || key >= w.kv) return -2;
          if (p.linear) return (int64_t)(w.h * p.linear + w.base + key);
          return pool_row(a.kv, a.b, w.s, w.h, (uint32_t)key);
        };
        int64_t row = row_of(0);
        uint32_t slot = 0, phase = 1, copied = 0;
        bool go = true;
        for (int j = 0; go && j < most; ++j) {
          if (row == -1) {                  // a wrong page: copies something that is there, and says so
            report(a.b.status, GORGO_KV_BAD_PAGE);
            work.bad = 1;
            row = 0;
          }
          const uint32_t pieces = __popc(__ballot_sync(0xffffffffu, row >= 0));
          const int64_t next = j + 1 < most ? row_of(j + 1) : -2;
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            go = __all_sync(0xffffffffu, wait_or_give_up(empty + 8 * slot, phase, &quit, a.b.status));
            if (!go) break;
            if (lane == 0) mbar_expect(full + 8 * slot, pieces * p.box * D * 2);
            __syncwarp();
            if (row >= 0)
              for (int c = 0; c < Z::kPlanes; ++c)
                tma_plane(ring_a + slot * Z::kTile + c * kPlane + lane * p.box * 128, v ? &v_map : &k_map, (int)row, c, full + 8 * slot);
            ++copied;
            if (++slot == (uint32_t)Z::kSlots) { slot = 0; phase ^= 1; }
          }
          row = next;
        }
        if (ragged && go) {                 // what lies behind the last key becomes zeros
          const uint32_t last = copied - 1, at = last % Z::kSlots;
          if (__all_sync(0xffffffffu, wait_or_give_up(full + 8 * at, last / Z::kSlots & 1, &quit, a.b.status))) {
            const uint32_t here = w.kv - (w.lo + most - 1) * kKeys, rest = (kKeys - here) * 8;
            for (uint32_t x = lane; x < rest * Z::kPlanes; x += 32)
              *reinterpret_cast<uint4*>(smem + 2 * Z::kTile + at * Z::kTile + x / rest * kPlane + here * 128 + x % rest * 16) =
                  make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(tail);
          }
        }
        if (quit) {                         // what flies has to land before the block ends
          mbar_wait(q_full, 0);
          for (uint32_t i = 0; i < min(copied, (uint32_t)Z::kSlots); ++i)
            mbar_wait(full + 8 * i, i < slot ? phase ^ 1 : phase);         // the last copy into the slot
        }
      }
    } else if (warp == 9) {
      // -------------------------------------------------------------- products: one thread, nothing between two waits
      // but the issue itself (the tensor pipe takes few instructions ahead, so what this thread does besides shows)
      if (most > 0 && elect_one()) {
        constexpr bool kBf = std::is_same<T, __nv_bfloat16>::value;
        const uint32_t s_shape = mma_shape(kKeys, kBf, p.negate != 0, false), o_shape = mma_shape(D, kBf, false, true);
        const uint32_t q_op = operand(q_a, 16), k_op = operand(ring_a, 16), v_op = operand(ring_a, kPlane);
        auto scores = [&](int i, uint32_t slot) {              // S_i = Q_i K^T
          const uint32_t x = q_op + i * (Z::kTile >> 4), y = k_op + slot * (Z::kTile >> 4);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = ((k / 4) * kPlane + (k % 4) * 32) >> 4;
            mma_ss(tmem + 128 * i, x + off, y + off, s_shape, k > 0);
          }
          mma_commit(s_full + 8 * i);
        };
        auto values = [&](int i, uint32_t slot, int half, bool acc) {   // O_i (+)= P_i V, 64 keys
          const uint32_t y = v_op + slot * (Z::kTile >> 4);
#pragma unroll
          for (int k = 4 * half; k < 4 * half + 4; ++k)
            mma_ts(tmem + Z::kO + D * i, tmem + 128 * i + 8 * k, y + (k * 2048 >> 4), o_shape, acc || k > 0);
        };
        uint32_t slot = 0, phase = 0;
        auto take = [&](uint32_t bar) {                        // the next slot, when it is there
          if (!wait_or_give_up(bar, bar == tail ? 0 : phase, &quit, a.b.status)) return false;
          if (++slot == (uint32_t)Z::kSlots) { slot = 0; phase ^= 1; }
          return true;
        };
        bool go = wait_or_give_up(q_full, 0, &quit, a.b.status) && take(full);
        if (go) {
          fence_after();
          for (int i = 0; i < 2; ++i)
            if (steps[i]) scores(i, 0);
          mma_commit(empty);
        }
        for (int j = 0; go && j < most; ++j) {
          const uint32_t v_slot = slot;
          if (!take(ragged && j + 1 == most ? tail : full + 8 * slot)) break;
          uint32_t k_slot = slot;
          bool have_k = false;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (!go || j >= steps[i]) continue;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              go = go && wait_or_give_up(p_full + 8 * (2 * i + k), j & 1, &quit, a.b.status);
              fence_after();
              if (go) values(i, v_slot, k, j > 0);
            }
            if (j + 1 < steps[i]) {
              if (!have_k) go = go && take(full + 8 * slot);
              have_k = true;
              if (go) scores(i, k_slot);
            } else if (go) {
              mma_commit(o_full + 8 * i);
            }
          }
          if (!go) break;
          mma_commit(empty + 8 * v_slot);
          if (have_k) mma_commit(empty + 8 * k_slot);
        }
        if (quit) {                       // products in flight end before the block does
          mma_commit(drained);
          mbar_wait(drained, 0);
        }
      }
      __syncwarp();
    }
  }
  __syncthreads();
  fence_after();
  if (warp == 9) tmem_free(tmem, 512);
}

// Joins the parts of one row and head, a warp each.
template <typename T, int D>
__global__ void __launch_bounds__(128) prefill_join_kernel(const __grid_constant__ AttnArgs a, const Plan p) {
  constexpr int kPer = D / 32;
  const uint32_t lane = threadIdx.x % 32;
  const uint64_t id = (uint64_t)blockIdx.x * 4 + threadIdx.x / 32;
  const uint32_t head = (uint32_t)(id % a.n_heads), row = (uint32_t)(id / a.n_heads);
  if (row >= a.b.total_new) return;
  const uint32_t s = warp_find_seq(a.b, row, lane);
  if (s >= a.b.n_seqs) return;
  const SeqLen q = seq_len(a.b, s);
  if ((int)row < q.first || rows_of(a.b, s) == 0) return;
  float top = -INFINITY, sum = 0.f, acc[kPer];
  const size_t step = (size_t)a.b.total_new * a.n_heads, at = (size_t)row * a.n_heads + head;
  for (uint32_t i = 0; i < p.splits; ++i) top = fmaxf(top, p.part_ml[2 * (i * step + at)]);
#pragma unroll
  for (int y = 0; y < kPer; ++y) acc[y] = 0.f;
  for (uint32_t i = 0; i < p.splits; ++i) {
    const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * (i * step + at));
    if (ml.y == 0.f) continue;            // (it has no O)
    const float f = ml.x == top ? 1.f : fast_exp2(ml.x - top);
    sum = __fmaf_rn(ml.y, f, sum);
    const float* o = p.part_o + (i * step + at) * D + lane * kPer;
#pragma unroll
    for (int y = 0; y < kPer; ++y) acc[y] = __fmaf_rn(o[y], f, acc[y]);
  }
  const float inv = !q.ok ? NAN : sum == 0.f ? 0.f : 1.f / sum;
  bool odd = false;
  T* out = static_cast<T*>(a.out) + (size_t)row * a.out_stride + (size_t)head * D + lane * kPer;
#pragma unroll
  for (int y = 0; y < kPer; y += 2) {
    const float f = acc[y] * inv, g = acc[y + 1] * inv;
    odd |= !(fabsf(f) < INFINITY) || !(fabsf(g) < INFINITY);
    *reinterpret_cast<uint32_t*>(out + y) = pack2(f, g, T());
  }
  if (a.lse && lane == 0) a.lse[at] = !q.ok ? NAN : sum == 0.f ? -INFINITY : (top - kShift<T> + log2f(sum)) * 0.693147180559945309f;
  if (__any_sync(0xffffffffu, odd) && q.ok && sum == sum) {
    // keys that the row's tile took: the tile's last token sees the most
    const int t = (int)row - q.first, pos = q.kv - q.n + t;
    const int last = q.kv - q.n + min((t / (int)p.tq + 1) * (int)p.tq, q.n) - 1;
    mend_row<T, D>(a, s, pos, (last / kKeys + 1) * kKeys, q.kv, row, head, lane);
  }
}

// e4m3 pages as 16-bit rows [kv head][linear][D], a sequence after the other from multiples of 128 rows.
template <typename T, int D>
__global__ void __launch_bounds__(256) widen_kernel(const AttnArgs a, const uint64_t linear, T* k_out, T* v_out) {
  constexpr uint32_t kLanes = D / 8;
  __shared__ uint32_t seq, tile;
  const uint32_t lane = threadIdx.x % 32;
  if (threadIdx.x < 32) {
    uint32_t before = 0, s0 = 0;
    uint32_t s = a.b.n_seqs, t = 0;
    for (; s0 < a.b.n_seqs; s0 += 32) {
      const int kv = s0 + lane < a.b.n_seqs ? a.b.kv_len[s0 + lane] : 0;
      const uint32_t mine = kv_len_ok(a.b, kv) ? (uint32_t)(kv + kKeys - 1) / kKeys : 0;
      uint32_t upto = mine;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= (uint32_t)d) upto += o;
      }
      const uint32_t over = __ballot_sync(0xffffffffu, before + upto > blockIdx.x);
      if (over) {
        const uint32_t here = __ffs(over) - 1;
        s = s0 + here;
        t = blockIdx.x - before - __shfl_sync(0xffffffffu, upto - mine, here);
        break;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) { seq = s; tile = t; }
  }
  __syncthreads();
  if (seq >= a.b.n_seqs) return;
  const int kv = a.b.kv_len[seq];
  const uint32_t h = blockIdx.y, l = threadIdx.x % kLanes;
#pragma unroll 4
  for (uint32_t r = threadIdx.x / kLanes; r < kKeys; r += 256 / kLanes) {
    const uint32_t j = tile * kKeys + r;
    if ((int)j >= kv) break;
    const int64_t from = pool_row(a.kv, a.b, seq, h, j);
    if (from < 0) continue;               // (reported by the attention kernel of that sequence)
    const size_t to = (size_t)h * linear + (size_t)blockIdx.x * kKeys + r;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const uint2 x = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(v ? a.kv.v : a.kv.k) + from * D + l * 8));
      const float f = pow2i((v ? a.kv.v_exp : a.kv.k_exp)[from]);
      uint32_t u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 y = unpack_e4m3((i < 2 ? x.x : x.y) >> 16 * (i & 1) & 0xffffu);
        u[i] = pack2(y.x * f, y.y * f, T());
      }
      *reinterpret_cast<uint4*>((v ? v_out : k_out) + to * D + l * 8) = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
}

uint64_t round_up(uint64_t x, uint64_t n) { return (x + n - 1) / n * n; }

struct Layout {
  Plan p;
  uint32_t blocks;                        // (sequence, tokens) pieces at most
  uint64_t wide, parts, bytes;            // of the 16-bit copy of K (and V), of the parts' O, of all
};

Layout layout(const AttnArgs& a, int sms) {
  Layout y = {};
  y.p.tq = 128 / a.group;
  const uint32_t n = a.b.n_seqs < a.b.total_new ? a.b.n_seqs : a.b.total_new;
  y.blocks = (a.b.total_new - n) / (2 * y.p.tq) + n;           // sum of ceil(n_s / step) is the most when all but one have one token
  // Keys are split where the blocks would leave half of the SMs idle, in shares of four tiles or more.
  const uint64_t units = (uint64_t)y.blocks * a.kv.n_kv_heads;
  uint32_t splits = units * 2 <= (uint64_t)sms ? (uint32_t)(sms / units) : 1;
  const uint32_t most = (a.b.max_kv + 4 * kKeys - 1) / (4 * kKeys);
  if (splits > most) splits = most;
  y.p.splits = splits < 1 ? 1 : splits;
  if (a.store == GORGO_E4M3) {
    y.p.linear = round_up(a.total_kv, kKeys) + (uint64_t)kKeys * a.b.n_seqs;
    y.wide = round_up(y.p.linear * a.kv.n_kv_heads * a.head_dim * 2, 256);
  }
  y.p.box = a.store == GORGO_E4M3 ? kKeys : (1u << a.kv.page_shift) < (uint32_t)kKeys ? 1u << a.kv.page_shift : kKeys;
  if (y.p.splits > 1) y.parts = round_up((uint64_t)y.p.splits * a.b.total_new * a.n_heads * a.head_dim * 4, 256);
  y.bytes = 2 * y.wide + y.parts + (y.p.splits > 1 ? (uint64_t)y.p.splits * a.b.total_new * a.n_heads * 8 : 0);
  return y;
}

template <typename T, int D>
cudaError_t launch(const AttnArgs& a, int sms, cudaStream_t st) {
  using Z = Sizes<D>;
  Layout y = layout(a, sms);
  Plan& p = y.p;
  unsigned char* ws = static_cast<unsigned char*>(a.workspace);
  p.part_o = reinterpret_cast<float*>(ws + 2 * y.wide);
  p.part_ml = reinterpret_cast<float*>(ws + 2 * y.wide + y.parts);
  p.negate = a.scale_log2 < 0.f;
  // (a scale of zero: all scores next to nothing, and what is not seen still at minus infinity)
  p.scale = fmaxf(fabsf(a.scale_log2), 1e-30f);
  CUtensorMap qm, km, vm;
  const void *k = a.kv.k, *v = a.kv.v;
  uint64_t rows = (uint64_t)a.kv.n_pages * a.kv.n_kv_heads << a.kv.page_shift;
  if (p.linear) {
    k = ws;
    v = ws + y.wide;
    rows = p.linear * a.kv.n_kv_heads;
    const uint64_t tiles = p.linear / kKeys;
    widen_kernel<T, D><<<dim3((uint32_t)tiles, a.kv.n_kv_heads), 256, 0, st>>>(a, p.linear, reinterpret_cast<T*>(ws), reinterpret_cast<T*>(ws + y.wide));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!make_rows_map(&qm, a.q, a.b.total_new, a.n_heads, D, a.q_stride, a.type, p.tq, a.group) ||
      !make_pool_map(&km, k, rows, D, a.type, p.box, 1) || !make_pool_map(&vm, v, rows, D, a.type, p.box, 1))
    return cudaErrorUnknown;
  cudaError_t e = allow_smem<prefill_kernel<T, D>>(Z::kBytes);
  if (e != cudaSuccess) return e;
  prefill_kernel<T, D><<<dim3(y.blocks, a.kv.n_kv_heads, p.splits), kThreads, Z::kBytes, st>>>(a, p, qm, km, vm);
  if ((e = cudaGetLastError()) != cudaSuccess || p.splits == 1) return e;
  const uint64_t warps = (uint64_t)a.b.total_new * a.n_heads;
  prefill_join_kernel<T, D><<<(uint32_t)((warps + 3) / 4), 128, 0, st>>>(a, p);
  return cudaGetLastError();
}

}  // namespace

bool prefill_fits(const AttnArgs& a) {
  return a.store != GORGO_E4M3 || (round_up(a.total_kv, kKeys) + (uint64_t)kKeys * a.b.n_seqs) * a.kv.n_kv_heads < 1ull << 31;
}

uint64_t prefill_workspace(const AttnArgs& a, int sms) { return a.b.total_new ? layout(a, sms).bytes : 0; }

cudaError_t launch_attn_prefill(const AttnArgs& a, int sms, cudaStream_t st) {
  if (a.type == GORGO_BF16) return a.head_dim == 128 ? launch<__nv_bfloat16, 128>(a, sms, st) : launch<__nv_bfloat16, 64>(a, sms, st);
  return a.head_dim == 128 ? launch<__half, 128>(a, sms, st) : launch<__half, 64>(a, sms, st);
}

}  // namespace gorgo
