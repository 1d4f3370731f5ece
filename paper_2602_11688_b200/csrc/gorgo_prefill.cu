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
// (TMEM lane), no shuffles; 8 copies; 9 issues tcgen05.mma, S of one tile while the other is in softmax; 10 finds the
// work; 11 clears what lies behind a sequence's last key.  TMEM: S of both tiles (P of 16 bits takes the place of the S it came from, and is the first operand of P V there), O of both.
// Keys and values come page by page in tiled bulk copies, 128 keys a slot, each as planes of 128-byte rows with
// the 128-byte swizzle; V is the second operand as it lies (its dims contiguous).
//
// Values behind the last key of a sequence may be anything: they are overwritten with zeros in shared memory.  A value
// that is not finite and that a row of its tile does not see would reach the row as 0 * x: rows whose result is not
// finite are listed (a byte a row and head), and the second kernel, in which nothing waits for another warp, looks at the
// values behind their own last key and computes them again key by key if one of those is the cause (one row of
// 100,000 keys: 34 ms; 18,900 rows of 30,000: 108 ms).
//
// All (sequence, kv head, tokens) units with their tiles of keys, and two places more for what a unit costs besides, are
// laid out as one line that is cut into as many equal pieces as SMs: no batch, no lengths and no long prefix under a few
// rows leave an SM idle, and a block has at most two units in part, which a second, small kernel joins.  Warp 10 walks
// the line ahead of the others, so the next unit's copies and first products run under the last one's end.
//
// e4m3 pages are first written out in bf16 (exactly) into the workspace, once for all rows that read them.  fp16 queries on
// them: what a code stands for need not fit fp16, and q need not fit bf16; so q is taken as the sum of two bf16 numbers
// (exactly) and P, too, is held as two: twice the products, 16 bits of P.
//
// P is rounded to 16 bits once, and l sums it before that: the result is off by 2.1e-3 in bf16 (2-norm) where its own
// rounding makes 1.6e-3; to hold P as two numbers always would cost half again as many products.
//
// Measured (32 query heads, 8 kv heads, head dim 128, bf16), passes with pauses and, in brackets, back to back under the power
// cap: 20,000 tokens 2.57 (2.97) ms, 1,277 (1,105) TFLOP/s of 1,679 (1,389) that the library's products reach; sixteen prompts
// of about 1,000 tokens 416 (472) us, 882 (778); two turns of 1,000 on 20,000 1.45 ms, 1,066, in e4m3 1.54 (1.79) ms, with fp16
// queries 2.30 ms.  Head dim 64, 20,000 tokens: 2.3 to 2.6 ms, 630 to 710 TFLOP/s.
#include "gorgo_rows.cuh"
#include "gorgo_tma.cuh"

namespace gorgo {

namespace {

constexpr int kThreads = 384;            // three warpgroups: registers can be moved between these only
constexpr int kKeys = 128;                // keys of a tile
constexpr uint32_t kPlane = kKeys * 128;  // bytes of 128 rows of 128 bytes

constexpr int kEntries = 4;               // units that the roles of a block may be apart
constexpr int kUnit = 2;                  // what a unit costs besides its tiles, in tiles (with 1: 747 instead of 894 TFLOP/s on
                                          // sixteen prompts of about 1,000 tokens; with 3 and 4: 890 and 878)

template <int D, bool kTwo>
struct Sizes {
  static constexpr int kPlanes = D / 64;
  static constexpr int kTile = kPlanes * kPlane;               // bytes of 128 rows of Q, K or V
  static constexpr int kQ = kTwo ? 2 : 1;                      // tiles of Q for a tile of rows
  static constexpr int kSlots = D == 64 ? 10 : kTwo ? 3 : 5;
  static constexpr int kBars = 2 * kSlots + 2 * kEntries + 13;
  static constexpr int kBytes = 2 * kQ * kTile + kSlots * kTile + 8 * kBars;
  static constexpr int kO = 256;                               // first TMEM column of O; S of tile i begins at 128 i
};

struct Plan {
  uint32_t tq;                            // tokens of a tile: floor(128 / group)
  uint32_t box;                           // keys of one bulk copy
  uint64_t linear;                        // rows of a head in the 16-bit copy of e4m3 pages; 0: the pages themselves
  uint32_t negate;                        // the scale is negative: S takes -Q
  float scale;                            // |scale| * log2(e)
  float* part_o;                          // [2 * grid][256][D]
  float* part_ml;                         // [2 * grid][256][2]
  struct Split* split;                    // [grid]
  uint8_t* again;                         // [total_new][n_heads]: 1: the row is looked at again; only rows whose result is not
                                          // finite, and rows of split units (0), are written: a byte left over costs a look
  uint32_t* odd;                          // [grid]: 1: a block has such rows; 2: it gave up
};

struct Work {                             // a unit, or a block's part of it
  uint32_t s, h;                          // sequence, kv head
  int first, n, kv;                       // the sequence's first row, new tokens, tokens in all
  int q0;                                 // first token of the unit
  int tiles[2];                           // tiles of keys of either tile of rows, from 0
  int lo, hi;                             // the block's share of them
  uint32_t slot;                          // where a part goes; kWhole: the result is written
  int none_from;                          // first key that has no page: rows at this position or behind it are NaN
  uint32_t last;                          // nothing comes after the one before
  uint64_t base;                          // first row of the sequence in the 16-bit copy
};
constexpr uint32_t kWhole = 0xffffffffu;
constexpr int kAllKeys = 0x7fffffff, kNoRow = -kAllKeys - 1;   // none_from: every key has a page; a wrong length, all rows are NaN

struct Split {                            // a unit whose first part a block has: what the second kernel needs
  Work w;
  uint32_t parts;                         // 0: none; else blocks that hold parts, this one and those after it
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
  if (placed_ok(b, a, e)) return e - a;
  report(b.status, GORGO_KV_BAD_LENGTH);
  return 0;
}

// sum of floor((a i + b) / m) over 0 <= i < n, for a n + b < 2^32: by the steps of Euclid's algorithm on (a, m).
__device__ uint64_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
  uint64_t sum = 0;
  while (n) {
    sum += (uint64_t)n * (n - 1) / 2 * (a / m) + (uint64_t)n * (b / m);
    a %= m;
    b %= m;
    const uint32_t y = a * n + b;
    if (y < m) break;
    n = y / m;
    b = y % m;
    const uint32_t t = m;
    m = a;
    a = t;
  }
  return sum;
}

// Tiles of keys of unit q of a sequence with n new tokens of kv: its last token sees the most.
__device__ __forceinline__ int unit_tiles(int q, int step, int n, int kv) {
  const int last = kv - n + min((q + 1) * step, n) - 1;
  return last < 0 ? 0 : last / kKeys + 1;
}
// Places on the line before unit q (<= ceil(n / step)) of one kv head: each unit's tiles and kUnit more.
__device__ uint64_t places_before(int q, int step, int n, int kv) {
  uint64_t sum = (uint64_t)q * kUnit;
  const int units = (n + step - 1) / step;
  if (q == units && q) {                  // the last unit may be short
    sum += unit_tiles(q - 1, step, n, kv);
    --q;
  }
  // units i < q: ceil((kv - n + (i + 1) step) / 128), none below zero
  const int none = kv < n ? (n - kv) / step : 0;               // units whose last token sees nothing
  if (q > none) sum += floor_sum(q - none, kKeys, step, (uint32_t)(kv - n + (none + 1) * step + kKeys - 1));
  return sum;
}

struct SeqPlace {
  int first, n, kv;
  bool bad;
};
__device__ __forceinline__ SeqPlace seq_place(const AttnArgs& a, uint32_t s) {
  SeqPlace r = {0, 0, 0, false};
  if (s >= a.b.n_seqs) return r;
  r.first = a.b.cu_new[s];
  r.n = rows_of(a.b, s);
  r.kv = a.b.kv_len[s];
  if (!kv_len_ok(a.b, r.kv)) { r.kv = 0; r.bad = true; }       // (its units see no keys, and say NaN)
  return r;
}

// Walks a block's piece of the line; all lanes of one warp together.
struct Walk {
  uint64_t left;                          // places of the piece from here on
  uint64_t at;                            // place on the whole line
  uint64_t total;
  uint32_t pieces;
  uint32_t s, h;
  int q, units;
  uint64_t off;                           // place inside the unit
  SeqPlace seq;
  uint64_t base;                          // tiles of 128 keys of the sequences before

  // False if the block has no piece.
  __device__ bool begin(const AttnArgs& a, int step, uint32_t lane) {
    const uint32_t hk = a.kv.n_kv_heads;
    total = 0;
    for (uint32_t x = lane; x < a.b.n_seqs; x += 32) {
      const SeqPlace y = seq_place(a, x);
      total += places_before((y.n + step - 1) / step, step, y.n, y.kv);
    }
#pragma unroll
    for (int d = 16; d; d /= 2) total += __shfl_xor_sync(0xffffffffu, total, d);
    total *= hk;
    pieces = total / 4 >= gridDim.x ? gridDim.x : total < 8 ? 1 : (uint32_t)(total / 4);
    if (blockIdx.x >= pieces || total == 0) return false;
    at = total * blockIdx.x / pieces;
    left = total * (blockIdx.x + 1) / pieces - at;
    uint64_t before = 0;
    base = 0;
    for (uint32_t s0 = 0;; s0 += 32) {
      const SeqPlace y = seq_place(a, s0 + lane);
      const uint64_t mine = places_before((y.n + step - 1) / step, step, y.n, y.kv) * hk;
      uint64_t upto = mine;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const uint64_t o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= (uint32_t)d) upto += o;
      }
      const uint32_t over = __ballot_sync(0xffffffffu, before + upto > at);
      const uint32_t here = over ? __ffs(over) - 1 : 32;
      base += __reduce_add_sync(0xffffffffu, lane < here ? (uint32_t)(y.kv + kKeys - 1) / kKeys : 0);
      if (over) {
        s = s0 + here;
        before += __shfl_sync(0xffffffffu, upto - mine, here);
        break;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    seq = seq_place(a, s);
    units = (seq.n + step - 1) / step;
    const uint64_t each = places_before(units, step, seq.n, seq.kv);
    off = at - before;
    h = (uint32_t)(off / each);
    off %= each;
    // the unit that holds place `off` of the head: 32 candidates at a time
    int lo = 0, hi = units;                                    // places_before(lo) <= off < places_before(hi)
    while (hi - lo > 1) {
      const int gap = (hi - lo + 31) / 32, x = lo + (int)(lane + 1) * gap;
      const uint32_t c = __popc(__ballot_sync(0xffffffffu, x < hi && places_before(x, step, seq.n, seq.kv) <= off));
      lo += (int)c * gap;
      hi = min(hi, lo + gap);
    }
    q = lo;
    off -= places_before(q, step, seq.n, seq.kv);
    return true;
  }

  // The next unit or part of one; false at the end of the piece.
  __device__ bool next(const AttnArgs& a, const Plan& p, int step, Work& w) {
    while (left) {
      const int tiles = unit_tiles(q, step, seq.n, seq.kv);
      const uint64_t take = min(left, (uint64_t)tiles + kUnit - off);
      // the first places of a unit are what it costs besides; place kUnit + i is tile i
      w.lo = max(0, (int)off - kUnit);
      w.hi = max(0, (int)(off + take) - kUnit);
      const bool some = w.hi > w.lo || (tiles == 0 && off == 0);
      w.s = s;
      w.h = h;
      w.first = seq.first;
      w.n = seq.n;
      w.kv = seq.kv;
      w.q0 = q * step;
      w.base = base * kKeys;
      w.none_from = seq.bad || (p.linear && w.base + seq.kv > p.linear) ? kNoRow : kAllKeys;
      w.last = 0;
      for (int i = 0; i < 2; ++i) {
        const int t = w.q0 + i * (int)p.tq;                    // first token of the tile
        const int last = seq.kv - seq.n + min(t + (int)p.tq, seq.n) - 1;
        w.tiles[i] = t >= seq.n || last < 0 ? 0 : last / kKeys + 1;
      }
      w.slot = w.lo == 0 && w.hi == tiles ? kWhole : 2 * blockIdx.x + (w.lo == 0 ? 1 : 0);
      const uint64_t end = at + (uint64_t)tiles + kUnit - off;     // of the unit, on the line
      at += take;
      left -= take;
      off += take;
      if (off == (uint64_t)tiles + kUnit) {
        off = 0;
        if (++q == units) {
          q = 0;
          if (++h == a.kv.n_kv_heads) {
            h = 0;
            do {
              base += (uint64_t)(seq.kv + kKeys - 1) / kKeys;
              seq = seq_place(a, ++s);
            } while (seq.n == 0 && s < a.b.n_seqs);
            units = (seq.n + step - 1) / step;
          }
        }
      }
      if (!some) continue;
      unit_end = end;
      return true;
    }
    return false;
  }
  uint64_t unit_end;                      // of the unit that next() gave

  // Blocks after this one that hold parts of it.
  __device__ uint32_t blocks_after() const { return (uint32_t)((unit_end * pieces - 1) / total) - blockIdx.x; }
};

// Waits; on the limit tells the block (and the host) to give up.  Every role then leaves at its next wait, with what it has
// started complete: copies landed, products done, entries of the ring of units as they were.
__device__ __forceinline__ bool wait_or_give_up(uint32_t bar, uint32_t parity, long long limit, volatile uint32_t* quit, uint32_t* status) {
  if (mbar_try(bar, parity)) return true;
  const long long from = clock64();
  while (!mbar_try(bar, parity)) {
    if (*quit) return false;
    if (clock64() - from > limit) {
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

// kTwo: rows are fp16, keys and values bf16; Q comes as two bf16 numbers whose sum it is, and P is held as two.
template <typename T, int D, bool kTwo>
__global__ void __launch_bounds__(kThreads, 1)
prefill_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Plan p, const __grid_constant__ CUtensorMap q_map,
               const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using Z = Sizes<D, kTwo>;
  using M = typename std::conditional<kTwo, __nv_bfloat16, T>::type;     // type of the matrix instructions' operands
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ Work ring[kEntries];
  __shared__ uint32_t tmem_base, quit, clear_slot, clear_from, any_odd;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t q_a = smem_u32(smem), ring_a = q_a + 2 * Z::kQ * Z::kTile;
  const uint32_t full = ring_a + Z::kSlots * Z::kTile, empty = full + 8 * Z::kSlots, work_full = empty + 8 * Z::kSlots,
                 work_empty = work_full + 8 * kEntries, q_full = work_empty + 8 * kEntries, q_empty = q_full + 8,
                 s_full = q_empty + 8, p_full = s_full + 16, o_full = p_full + 32, drained = o_full + 16,
                 clear = drained + 8, cleared = clear + 8;

  if (threadIdx.x == 0) {
    quit = any_odd = 0;
    for (int i = 0; i < Z::kSlots; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < kEntries; ++i) {
      mbar_init(work_full + 8 * i, 1);
      mbar_init(work_empty + 8 * i, 10);                       // copies, products, eight warps of softmax
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(p_full + 16 * i, 128);
      mbar_init(p_full + 16 * i + 8, 128);
      mbar_init(o_full + 8 * i, 1);
    }
    mbar_init(drained, 1);
    mbar_init(clear, 1);
    mbar_init(cleared, 1);
    mbar_init_fence();
    prefetch_map(&q_map);
    prefetch_map(&k_map);
    prefetch_map(&v_map);
  }
  if (warp == 9) tmem_alloc(smem_u32(&tmem_base), 512);
  launch_dependents();
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_base;
  auto wait = [&](uint32_t bar, uint32_t parity) { return wait_or_give_up(bar, parity, a.wait_ticks, &quit, a.b.status); };
  auto steps_of = [](const Work& w, int i) { return max(0, min(w.hi, w.tiles[i]) - w.lo); };

  // Registers: 384 threads of 168 at the launch; the softmax takes what the last warpgroup does not need
  // (2 * 200 + 104 = 3 * 168).
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // ---------------------------------------------------------------- softmax, a row a thread
    const int i = warp / 4;
    const uint32_t r = warp % 4 * 32 + lane, at = tmem + (warp % 4 * 32 << 16);
    const uint32_t s_at = at + 128 * i, o_at = at + Z::kO + D * i;
    const uint32_t tok = r / a.group, in_group = r % a.group;
    const float c = p.scale, slack = 8.f / c;
    uint32_t s_phase = 0, o_phase = 0;
    bool go = true;
    for (uint32_t e = 0, e_phase = 0; go; e = (e + 1) % kEntries, e_phase ^= e == 0) {
      go = __all_sync(0xffffffffu, wait(work_full + 8 * e, e_phase));
      if (!go || ring[e].last) break;
      const Work& w = ring[e];
      const int steps = steps_of(w, i), lo = w.lo;
      const int t = w.q0 + i * (int)p.tq + (int)tok;           // token of the row
      const bool mine = tok < p.tq && t < w.n;
      const int pos = w.kv - w.n + t;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < steps; ++j) {
        go = __all_sync(0xffffffffu, wait(s_full + 8 * i, s_phase));
        if (!go) break;
        s_phase ^= 1;
        fence_after();
        const int seen = pos - (lo + j) * kKeys + 1;           // columns that the row sees
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
        const bool grow = !(now <= m + slack);                 // (also for NaN)
        if (__any_sync(0xffffffffu, grow)) {
          // m * c stays finite: a score beyond 32 bits makes the row NaN, below them it is minus infinity
          const float z = now * c;
          if (z == INFINITY) now = NAN;
          if (z == -INFINITY) now = -INFINITY;
          const bool up = grow && now != m;
          const float f = up ? fast_exp2(m * c - now * c) : 1.f;
          if (up) m = now;
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
        const float off = m == -INFINITY ? 0.f : kShift<M> - m * c;
        // P in halves of 64 keys: their products with V begin while the other half is computed
        f32x2 sum[4] = {0, 0, 0, 0};
        const f32x2 c2 = both(c, c), off2 = both(off, off);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (k) read(1);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t pk[16], low[kTwo ? 16 : 1];
#pragma unroll
            for (int y = 0; y < 16; ++y) {
              float2 u = apart(fma2(both(__uint_as_float(x[32 * q + 2 * y]), __uint_as_float(x[32 * q + 2 * y + 1])), c2, off2));
              u.x = fast_exp2(u.x);
              u.y = fast_exp2(u.y);
              sum[y % 4] = add2(sum[y % 4], both(u.x, u.y));
              pk[y] = pack2(u.x, u.y, M());
              if (kTwo) {
                const float2 h = unpack2(pk[y], M());
                low[y % (kTwo ? 16 : 1)] = pack2(u.x - h.x, u.y - h.y, M());
              }
            }
            tmem_st16(s_at + (kTwo ? 64 : 32) * k + 16 * q, pk);
            if (kTwo) tmem_st16(s_at + 64 * k + 32 + 16 * q, low);
          }
          tmem_wait_st();
          fence_before();
          mbar_arrive(p_full + 8 * (2 * i + k));
        }
        const float2 l2 = apart(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
        l += l2.x + l2.y;
      }
      if (steps && go) {
        go = __all_sync(0xffffffffu, wait(o_full + 8 * i, o_phase));
        o_phase ^= 1;
        fence_after();
      }
      const bool bad = pos >= w.none_from || !go;
      if (w.slot != kWhole) {
        // (the second kernel sees these rows' results first)
        if (mine && lo == 0) p.again[(size_t)(w.first + t) * a.n_heads + w.h * a.group + in_group] = 0;
        const size_t part = (size_t)w.slot * 256 + i * 128 + r;
        *reinterpret_cast<float2*>(p.part_ml + 2 * part) = make_float2(m * c, bad ? NAN : l);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          if (!steps || !go) break;
          uint32_t o[32];
          tmem_ld32(o, o_at + 32 * k);
          tmem_wait_ld();
          if (mine)
#pragma unroll
            for (int y = 0; y < 8; ++y)
              *reinterpret_cast<uint4*>(p.part_o + part * D + 32 * k + 4 * y) = make_uint4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]);
        }
      } else {
        const uint32_t head = w.h * a.group + in_group;
        const size_t row = (size_t)(w.first + t);
        // a row without keys: zeros
        const float inv = bad ? NAN : l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
        f32x2 none = 0;                    // 0 x the elements: NaN if one is not finite
        T* out = static_cast<T*>(a.out) + row * a.out_stride + (size_t)head * D;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          uint32_t o[32];
          if (steps && go) {
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
            none = fma2(both(__uint_as_float(o[2 * y]), __uint_as_float(o[2 * y + 1])), 0, none);
            u[y] = pack2(f, g, T());
          }
          if (mine)
#pragma unroll
            for (int y = 0; y < 4; ++y) *reinterpret_cast<uint4*>(out + 32 * k + 8 * y) = v[y];
        }
        if (mine && a.lse) a.lse[row * a.n_heads + head] = bad ? NAN : l == 0.f ? -INFINITY : (m * c - kShift<M> + log2f(l)) * 0.693147180559945309f;
        // (a sum that is not finite: the scores are the cause; a byte for every row would cost 12 us in 410 with units of 1,000
        // tokens, and so would a comparison for every element)
        const float2 n2 = apart(none);
        if (mine && !(n2.x == 0.f && n2.y == 0.f) && !bad && l < INFINITY) p.again[row * a.n_heads + head] = any_odd = 1;
      }
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(work_empty + 8 * e);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == 8) {
      // -------------------------------------------------------------- copies
      const uint32_t most_pieces = kKeys / p.box;
      uint32_t slot = 0, phase = 1, copied = 0, q_phase = 1;
      bool go = true;
      for (uint32_t e = 0, e_phase = 0; go; e = (e + 1) % kEntries, e_phase ^= e == 0) {
        go = __all_sync(0xffffffffu, wait(work_full + 8 * e, e_phase));
        if (!go || ring[e].last) break;
        const Work w = ring[e];
        const int steps[2] = {steps_of(w, 0), steps_of(w, 1)}, most = max(steps[0], steps[1]);
        // a lane a piece: the piece's page is looked up a tile ahead
        auto row_of = [&](int j) -> int64_t {
          const int key = (w.lo + j) * kKeys + (int)(lane * p.box);
          if (j >= most || lane >= most_pieces || key >= w.kv) return -2;
          if (p.linear) return w.none_from == kNoRow ? 0 : (int64_t)(w.h * p.linear + w.base + key);
          return pool_row(a.kv, a.b, w.s, w.h, (uint32_t)key);
        };
        int64_t row = row_of(0);
        for (int j = 0; go && j < most; ++j) {
          const uint32_t wrong = __ballot_sync(0xffffffffu, row == -1);
          if (row == -1) {                // a wrong page: copies something that is there, and says so
            report(a.b.status, GORGO_KV_BAD_PAGE);
            const int key = (w.lo + j) * kKeys + (int)(lane * p.box);
            if (lane == (uint32_t)__ffs(wrong) - 1 && key < ring[e].none_from) ring[e].none_from = key;
            row = 0;
          }
          const uint32_t pieces = __popc(__ballot_sync(0xffffffffu, row >= 0));
          const int64_t next = row_of(j + 1);
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            go = __all_sync(0xffffffffu, wait(empty + 8 * slot, phase));
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
          if (j == 0 && go) {             // Q behind the first keys: its place is free only after the last unit's scores
            go = __all_sync(0xffffffffu, wait(q_empty, q_phase));
            if (!go) break;
            q_phase ^= 1;
            if (lane == 0) {
              const uint32_t bytes = p.tq * a.group * 128 * Z::kPlanes * Z::kQ;
              mbar_expect(q_full, (steps[0] ? bytes : 0) + (steps[1] ? bytes : 0));
              for (int i = 0; i < 2; ++i)
                for (int c = 0; steps[i] && c < Z::kPlanes * Z::kQ; ++c)         // (the second numbers: total_new rows behind)
                  asm volatile(
                      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                      ::"r"(q_a + i * Z::kQ * Z::kTile + c * kPlane), "l"(reinterpret_cast<uint64_t>(&q_map)), "r"(c % Z::kPlanes * 64),
                      "r"((int)(w.h * a.group)), "r"(w.first + w.q0 + i * (int)p.tq + (c / Z::kPlanes ? (int)a.b.total_new : 0)), "r"(q_full) : "memory");
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(work_empty + 8 * e);
      }
      // what flies has to land before the block ends, whichever role gives up, and when
      mbar_wait(q_full, q_phase);
      for (uint32_t i = 0; i < min(copied, (uint32_t)Z::kSlots); ++i)
        mbar_wait(full + 8 * i, i < slot ? phase ^ 1 : phase);           // the last copy into the slot
    } else if (warp == 9) {
      // -------------------------------------------------------------- products: one thread, nothing between two waits
      // but the issue itself (the tensor pipe takes few instructions ahead, so what this thread does besides shows)
      // At D = 64 the exponentials are the bound and a thread that issues a little later serves them better: the tiles
      // fall into turns (20,000 tokens: 733 against 694 TFLOP/s; at D = 128 it is 1,240 against 1,306).
      if (D == 64 ? lane == 0 : elect_one()) {
        constexpr bool kBf = std::is_same<M, __nv_bfloat16>::value;
        const uint32_t s_shape = mma_shape(kKeys, kBf, p.negate != 0, false), o_shape = mma_shape(D, kBf, false, true);
        const uint32_t q_op = operand(q_a, 16), k_op = operand(ring_a, 16), v_op = operand(ring_a, kPlane);
        auto scores = [&](int i, uint32_t slot) {              // S_i = Q_i K^T
          const uint32_t x = q_op + i * (Z::kQ * Z::kTile >> 4), y = k_op + slot * (Z::kTile >> 4);
#pragma unroll
          for (int k = 0; k < Z::kQ * (D / 16); ++k) {
            const uint32_t off = ((k / 4) * kPlane + (k % 4) * 32) >> 4, k_off = off % (Z::kTile >> 4);
            mma_ss(tmem + 128 * i, x + off, y + k_off, s_shape, k > 0);
          }
          mma_commit(s_full + 8 * i);
        };
        auto values = [&](int i, uint32_t slot, int half, bool acc) {   // O_i (+)= P_i V, 64 keys
          const uint32_t y = v_op + slot * (Z::kTile >> 4);
#pragma unroll
          for (int k = 4 * half; k < 4 * half + 4; ++k)
#pragma unroll
            for (int n = 0; n < Z::kQ; ++n)
              mma_ts(tmem + Z::kO + D * i, tmem + 128 * i + 8 * k + (kTwo ? 32 * (half + n) : 0), y + (k * 2048 >> 4), o_shape,
                     acc || k > 0 || n > 0);
        };
        uint32_t slot = 0, phase = 0, q_phase = 0, c_phase = 0, p_phase[2] = {0, 0};
        auto take = [&] {                                      // the next slot, when it is there
          if (!wait(full + 8 * slot, phase)) return false;
          if (++slot == (uint32_t)Z::kSlots) { slot = 0; phase ^= 1; }
          return true;
        };
        bool go = true;
        for (uint32_t e = 0, e_phase = 0; go; e = (e + 1) % kEntries, e_phase ^= e == 0) {
          go = wait(work_full + 8 * e, e_phase);
          if (!go || ring[e].last) break;
          const int steps[2] = {steps_of(ring[e], 0), steps_of(ring[e], 1)}, most = max(steps[0], steps[1]);
          const int behind = ring[e].kv - (ring[e].lo + most - 1) * kKeys;   // keys of the last tile
          mbar_arrive(work_empty + 8 * e);
          if (most == 0) continue;
          const uint32_t first_slot = slot;
          go = take() && wait(q_full, q_phase);
          q_phase ^= 1;
          if (!go) break;
          fence_after();
          for (int i = 0; i < 2; ++i)
            if (steps[i]) scores(i, first_slot);
          mma_commit(empty + 8 * first_slot);
          if (most == 1) mma_commit(q_empty);
          for (int j = 0; go && j < most; ++j) {
            const uint32_t v_slot = slot;
            if (!(go = take())) break;
            if (behind < kKeys && j + 1 == most) {             // what lies behind the last key becomes zeros
              clear_slot = v_slot;
              clear_from = behind;
              mbar_arrive(clear);
              if (!(go = mbar_wait(cleared, c_phase))) break;  // (always answered, so never left: the next request would
                                                               // take `clear` past the phase that warp 11 waits for)
              c_phase ^= 1;
            }
            const uint32_t k_slot = slot;
            bool have_k = false;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              if (!go || j >= steps[i]) continue;
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                go = go && wait(p_full + 8 * (2 * i + k), p_phase[i]);
                fence_after();
                if (go) values(i, v_slot, k, j > 0);
              }
              p_phase[i] ^= 1;
              if (j + 1 < steps[i]) {
                if (!have_k) go = go && take();
                have_k = true;
                if (go) scores(i, k_slot);
              } else if (go) {
                mma_commit(o_full + 8 * i);
              }
            }
            if (!go) break;
            mma_commit(empty + 8 * v_slot);
            if (have_k) mma_commit(empty + 8 * k_slot);
            if (j + 2 == most) mma_commit(q_empty);
          }
        }
        mma_commit(drained);              // products in flight end before the block does
        mbar_wait(drained, 0);
        clear_slot = kWhole;              // (ends warp 11)
        mbar_arrive(clear);
      }
      __syncwarp();
    } else if (warp == 10) {
      // -------------------------------------------------------------- the work, ahead of the others
      const int step = 2 * (int)p.tq;
      Walk walk;
      Work w;
      uint32_t parts = 0;
      bool more = walk.begin(a, step, lane), go = true;
      for (uint32_t e = 0, e_phase = 1; go; e = (e + 1) % kEntries, e_phase ^= e == 0) {
        more = more && walk.next(a, p, step, w);
        go = __all_sync(0xffffffffu, wait(work_empty + 8 * e, e_phase));
        if (!go) break;                   // (the entry is still read)
        if (lane == 0) {
          if (more) {
            ring[e] = w;
            if (w.none_from == kNoRow) report(a.b.status, GORGO_KV_BAD_LENGTH);
            if (w.slot != kWhole && w.lo == 0) {               // the second kernel finds its parts here and in the blocks behind
              parts = 1 + walk.blocks_after();
              p.split[blockIdx.x].w = w;
            }
          } else {
            ring[e].last = 1;
          }
          mbar_arrive(work_full + 8 * e);
        }
        __syncwarp();
        if (!more) break;
      }
      if (lane == 0) p.split[blockIdx.x].parts = parts;
    } else {
      // -------------------------------------------------------------- clears values behind a sequence's last key
      for (uint32_t c_phase = 0;; c_phase ^= 1) {
        // (the products' thread always comes to an end and says so; this wait may last as long as all of the work)
        const long long began = clock64();
        bool asked;
        while (!(asked = mbar_try(clear, c_phase)) && clock64() - began < 64 * kWaitTicks) {}   // (not the limit a test sets)
        if (!__all_sync(0xffffffffu, asked)) break;
        const uint32_t slot = __shfl_sync(0xffffffffu, clear_slot, 0), from = __shfl_sync(0xffffffffu, clear_from, 0);
        if (slot == kWhole) break;
        const uint32_t rest = (kKeys - from) * 8;              // 16-byte pieces of a plane
        for (uint32_t x = lane; x < rest * Z::kPlanes; x += 32)
          *reinterpret_cast<uint4*>(smem + 2 * Z::kQ * Z::kTile + slot * Z::kTile + x / rest * kPlane + from * 128 + x % rest * 16) = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(cleared);
      }
    }
  }
  __syncthreads();
  fence_after();
  if (warp == 9) tmem_free(tmem, 512);
  if (threadIdx.x == 0) p.odd[blockIdx.x] = any_odd | (quit ? 2 : 0);
}

// Keys that the tile of rows of a sequence's new token t took.
__device__ __forceinline__ int keys_taken(int t, int tq, int n, int kv) {
  const int last = kv - n + min((t / tq + 1) * tq, n) - 1;
  return last < 0 ? 0 : min((last / kKeys + 1) * kKeys, kv);
}

// By all warps of the blocks y < kListBlocks of the second kernel: rows on the list.  Neighbours go to different warps: they
// are long.
constexpr uint32_t kListBlocks = 4;
template <typename T, int D>
__device__ __noinline__ void mend_list(const AttnArgs& a, const Plan& p, uint32_t lane) {
  const uint64_t rows = (uint64_t)a.b.total_new * a.n_heads, warps = (uint64_t)gridDim.x * kListBlocks * 8;
  const uint64_t me = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * 8 + threadIdx.x / 32;
  for (uint64_t x0 = 0; x0 * warps + me < rows; x0 += 32) {
    const uint64_t mine = (x0 + lane) * warps + me;
    uint32_t left = __ballot_sync(0xffffffffu, mine < rows && p.again[mine < rows ? mine : 0] == 1);
    for (; left; left &= left - 1) {
      const uint64_t x = (x0 + __ffs(left) - 1) * warps + me;
      const uint32_t row = (uint32_t)(x / a.n_heads);
      if ((int)row >= a.b.cu_new[a.b.n_seqs]) continue;        // (nobody's rows are not on the list: what is there is left over)
      const uint32_t s = warp_find_seq(a.b, row, lane);
      const SeqPlace q = seq_place(a, s);
      const int t = (int)row - q.first, pos = q.kv - q.n + t;
      if (q.bad || t < 0 || t >= q.n || pos < 0) continue;
      mend_row<T, D>(a, s, pos / kKeys * kKeys, pos, keys_taken(t, p.tq, q.n, q.kv), row, (uint32_t)(x % a.n_heads), lane);
    }
  }
}

// Joins the parts of the units that several blocks hold: a block of this kernel takes eight rows, a warp each, of the unit
// whose first part block x of the first kernel has.  Before that some blocks see to the rows on the list, if there are any.
template <typename T, int D, bool kTwo>
__global__ void __launch_bounds__(256, 6)
prefill_join_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Plan p) {
  constexpr int kPer = D / 32;
  constexpr float kUp = kTwo ? 0.f : kShift<T>;
  const uint32_t lane = threadIdx.x % 32, c0 = blockIdx.x;
  wait_primary();
  if (blockIdx.y < kListBlocks) {
    uint32_t odd_rows = 0;
    for (uint32_t x = lane; x < gridDim.x; x += 32) odd_rows |= p.odd[x];
    if (__any_sync(0xffffffffu, odd_rows & 1)) mend_list<T, D>(a, p, lane);
  }
  const Work w = p.split[c0].w;           // (read beside `parts`, whatever that says)
  const uint32_t parts = p.split[c0].parts;
  if (parts == 0) return;
  const uint32_t r = blockIdx.y * 8 + threadIdx.x / 32;
  const uint32_t i = r / 128, tok = r % 128 / a.group, head = w.h * a.group + r % 128 % a.group;
  const int t = w.q0 + (int)(i * p.tq + tok);
  if (tok >= p.tq || t >= w.n) return;
  // the first block holds its last unit's part, the others their first one's
  auto at = [&](uint32_t k) { return (size_t)(2 * (c0 + k) + (k == 0 ? 1 : 0)) * 256 + r; };
  float top = -INFINITY, sum = 0.f, acc[kPer];
#pragma unroll
  for (int y = 0; y < kPer; ++y) acc[y] = 0.f;
#pragma unroll 4
  for (uint32_t k = 0; k < parts; ++k) {
    const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * at(k));
    float o[kPer];
#pragma unroll
    for (int y = 0; y < kPer; ++y) o[y] = p.part_o[at(k) * D + lane * kPer + y];
    if (p.odd[c0 + k] & 2) sum = NAN;     // (its part may not be there)
    if (ml.y == 0.f) continue;            // (it has no O: what was read is nothing)
    const float now = fmaxf(top, ml.x);
    const float f = top == now ? 1.f : fast_exp2(top - now), g = ml.x == now ? 1.f : fast_exp2(ml.x - now);
    top = now;
    sum = __fmaf_rn(ml.y, g, sum * f);
#pragma unroll
    for (int y = 0; y < kPer; ++y) acc[y] = __fmaf_rn(o[y], g, acc[y] * f);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  bool odd = false;
  const size_t row = (size_t)(w.first + t);
  T* out = static_cast<T*>(a.out) + row * a.out_stride + (size_t)head * D + lane * kPer;
#pragma unroll
  for (int y = 0; y < kPer; y += 2) {
    const float f = acc[y] * inv, g = acc[y + 1] * inv;
    odd |= !(fabsf(f) < INFINITY) || !(fabsf(g) < INFINITY);
    *reinterpret_cast<uint32_t*>(out + y) = pack2(f, g, T());
  }
  if (a.lse && lane == 0) a.lse[row * a.n_heads + head] = sum == 0.f ? -INFINITY : (top - kUp + log2f(sum)) * 0.693147180559945309f;
  // (a sum that is NaN: a wrong page, or a score that is none)
  const int pos = w.kv - w.n + t;
  if (__any_sync(0xffffffffu, odd) && sum < INFINITY && pos >= 0)
    mend_row<T, D>(a, w.s, pos / kKeys * kKeys, pos, keys_taken(t, p.tq, w.n, w.kv), (uint32_t)row, head, lane);
}

// e4m3 pages as bf16 rows [kv head][linear][D], a sequence after the other from multiples of 128 rows.  Exact: a code has
// four bits, and code * 2^e is between 2^-33 and bf16's largest value, but for 2^128, which the largest rows of bf16 may round to.
template <int D>
__global__ void __launch_bounds__(256) widen_kernel(const AttnArgs a, const uint64_t linear, __nv_bfloat16* k_out, __nv_bfloat16* v_out) {
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
  if (seq >= a.b.n_seqs || rows_of(a.b, seq) == 0) return;     // (nobody reads it)
  const int kv = a.b.kv_len[seq];
  const uint32_t h = blockIdx.y, l = threadIdx.x % kLanes;
#pragma unroll 4
  for (uint32_t r = threadIdx.x / kLanes; r < kKeys; r += 256 / kLanes) {
    const uint32_t j = tile * kKeys + r;
    if ((int)j >= kv) break;
    const int64_t from = pool_row(a.kv, a.b, seq, h, j);
    const size_t to = (size_t)h * linear + (size_t)blockIdx.x * kKeys + r;
    if (from < 0) report(a.b.status, GORGO_KV_BAD_PAGE);       // the attention kernel does not look at the table: rows that
                                                               // see this key are NaN because the key is
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      uint4* out = reinterpret_cast<uint4*>((v ? v_out : k_out) + to * D + l * 8);
      if (from < 0) {
        *out = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
        continue;
      }
      const uint2 x = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(v ? a.kv.v : a.kv.k) + from * D + l * 8));
      const float f = pow2i((v ? a.kv.v_exp : a.kv.k_exp)[from]);
      uint32_t u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 y = unpack_e4m3((i < 2 ? x.x : x.y) >> 16 * (i & 1) & 0xffffu);
        u[i] = pack2(y.x * f, y.y * f, __nv_bfloat16());
      }
      *out = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
}

// fp16 rows of queries as two bf16 numbers whose sum they are: [2][rows][n_heads][D].
__global__ void __launch_bounds__(256) split_kernel(const AttnArgs a, uint4* out) {
  const uint32_t width = a.n_heads * a.head_dim / 8;           // 16-byte pieces of a row
  const uint64_t n = (uint64_t)a.b.total_new * width, x = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (x >= n) return;
  const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const __half*>(a.q) + x / width * a.q_stride + x % width * 8);
  const uint32_t in[4] = {v.x, v.y, v.z, v.w};
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack2(in[i], __half());
    hi[i] = pack2(f.x, f.y, __nv_bfloat16());
    const float2 h = unpack2(hi[i], __nv_bfloat16());          // (infinities and NaN are in the first alone)
    lo[i] = pack2(fabsf(f.x) < INFINITY ? f.x - h.x : 0.f, fabsf(f.y) < INFINITY ? f.y - h.y : 0.f, __nv_bfloat16());
  }
  out[x] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  out[n + x] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

uint64_t round_up(uint64_t x, uint64_t n) { return (x + n - 1) / n * n; }

struct Layout {
  Plan p;
  uint64_t wide, two, parts, bytes;       // of the 16-bit copy of K (and V), of Q as two numbers, of the parts' O, of all
};

Layout layout(const AttnArgs& a, int sms) {
  Layout y = {};
  y.p.tq = 128 / a.group;
  if (a.store == GORGO_E4M3) {
    y.p.linear = round_up(a.total_kv, kKeys) + (uint64_t)kKeys * a.b.n_seqs;
    y.wide = round_up(y.p.linear * a.kv.n_kv_heads * a.head_dim * 2, 256);
    if (a.type == GORGO_FP16) y.two = round_up((uint64_t)2 * a.b.total_new * a.n_heads * a.head_dim * 2, 256);
  }
  y.p.box = a.store == GORGO_E4M3 ? kKeys : (1u << a.kv.page_shift) < (uint32_t)kKeys ? 1u << a.kv.page_shift : kKeys;
  y.parts = (uint64_t)2 * sms * 256 * a.head_dim * 4;
  y.bytes = 2 * y.wide + y.two + y.parts + (uint64_t)2 * sms * 256 * 8 + round_up((uint64_t)sms * sizeof(Split), 256) +
            round_up((uint64_t)sms * 4, 256) + round_up((uint64_t)a.b.total_new * a.n_heads, 256);
  return y;
}

template <typename T, int D, bool kTwo>
cudaError_t launch(const AttnArgs& a, int sms, cudaStream_t st) {
  using Z = Sizes<D, kTwo>;
  Layout y = layout(a, sms);
  Plan& p = y.p;
  unsigned char* ws = static_cast<unsigned char*>(a.workspace);
  p.part_o = reinterpret_cast<float*>(ws + 2 * y.wide + y.two);
  p.part_ml = reinterpret_cast<float*>(ws + 2 * y.wide + y.two + y.parts);
  p.split = reinterpret_cast<Split*>(p.part_ml + (size_t)2 * sms * 256 * 2);
  p.odd = reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(p.split) + round_up((uint64_t)sms * sizeof(Split), 256));
  p.again = reinterpret_cast<uint8_t*>(p.odd) + round_up((uint64_t)sms * 4, 256);
  p.negate = a.scale_log2 < 0.f;
  // A scale of zero is the smallest number there is, 2^-149: its scores are below 2^-21 however large the products, and
  // what is not seen stays at minus infinity.
  p.scale = fmaxf(fabsf(a.scale_log2), 1.401298464e-45f);
  CUtensorMap qm, km, vm;
  const void *q = a.q, *k = a.kv.k, *v = a.kv.v;
  uint64_t q_rows = a.b.total_new, q_stride = a.q_stride;
  const uint32_t type = kTwo ? (uint32_t)GORGO_BF16 : a.type;
  uint64_t rows = (uint64_t)a.kv.n_pages * a.kv.n_kv_heads << a.kv.page_shift;
  if (p.linear) {
    k = ws;
    v = ws + y.wide;
    rows = p.linear * a.kv.n_kv_heads;
    const uint64_t tiles = p.linear / kKeys;
    widen_kernel<D><<<dim3((uint32_t)tiles, a.kv.n_kv_heads), 256, 0, st>>>(a, p.linear, reinterpret_cast<__nv_bfloat16*>(ws),
                                                                            reinterpret_cast<__nv_bfloat16*>(ws + y.wide));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (kTwo) {
    q = ws + 2 * y.wide;
    q_rows *= 2;
    q_stride = (uint64_t)a.n_heads * D;
    const uint64_t pieces = a.b.total_new * q_stride / 8;
    split_kernel<<<(uint32_t)((pieces + 255) / 256), 256, 0, st>>>(a, reinterpret_cast<uint4*>(ws + 2 * y.wide));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!make_rows_map(&qm, q, (uint32_t)q_rows, a.n_heads, D, q_stride, type, p.tq, a.group) ||
      !make_pool_map(&km, k, rows, D, type, p.box, 1) || !make_pool_map(&vm, v, rows, D, type, p.box, 1))
    return cudaErrorUnknown;
  cudaError_t e = allow_smem<prefill_kernel<T, D, kTwo>>(Z::kBytes);
  if (e != cudaSuccess) return e;
  prefill_kernel<T, D, kTwo><<<sms, kThreads, Z::kBytes, st>>>(a, p, qm, km, vm);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sms, 32);
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute early = {};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, prefill_join_kernel<T, D, kTwo>, a, p);
}

template <int D>
cudaError_t launch(const AttnArgs& a, int sms, cudaStream_t st) {
  if (a.type == GORGO_BF16) return launch<__nv_bfloat16, D, false>(a, sms, st);
  return a.store == GORGO_E4M3 ? launch<__half, D, true>(a, sms, st) : launch<__half, D, false>(a, sms, st);
}

}  // namespace

bool prefill_fits(const AttnArgs& a) {
  return a.store != GORGO_E4M3 || (round_up(a.total_kv, kKeys) + (uint64_t)kKeys * a.b.n_seqs) * a.kv.n_kv_heads < 1ull << 31;
}

uint64_t prefill_workspace(const AttnArgs& a, int sms) { return a.b.total_new ? layout(a, sms).bytes : 0; }

cudaError_t launch_attn_prefill(const AttnArgs& a, int sms, cudaStream_t st) {
  return a.head_dim == 128 ? launch<128>(a, sms, st) : launch<64>(a, sms, st);
}

}  // namespace gorgo
