// One new token per sequence against the paged key-value cache (sm_100a).
//
// Mathematics.  For the query heads of one kv head and a run of keys: z = K q, p = exp2(z' - m), o = V^T p,
// l = sum p with the running maximum m, all sums in 32 bits; runs are joined by
//   m = max m_i,  l = sum l_i 2^(m_i - m),  o = sum o_i 2^(m_i - m) / l.
//
// What bounds it: every key and value is read once and used for `group` heads only, so HBM.  The work, all
// (sequence, kv head) pairs with their keys in tiles of four slices, is laid out as one line and cut into as many equal pieces as
// blocks fit the GPU at once: no length and no batch leaves an SM idle, and at most two pieces of a block are
// partial; a second, small kernel joins those (it starts early and waits for the first one's end).
//
// Each of a block's four warps takes a slice of every tile, 4 KB of keys (16 to 64), and is on
// its own: its own ring of bulk copies, its own running maximum and sum; warps meet only at the end of a
// (sequence, head).  Keys are the rows of the
// matrix instructions (S^T = K q^T, O^T = V^T P^T, 16 x 8 x 16), so that up to eight query heads cost what one
// does; P is transposed between the two products by matrix moves.  P enters as the sum of two 16-bit numbers, so
// that it is not what limits the result; the tensor pipe is nearly idle here.
//
// e4m3 pages: codes become fp16, exactly; q as fp16 after a power of two per head that makes its largest value about
// 2^10 (exact but for what is 2^-34 of it); the keys' powers of two multiply the scores, the values' are added to the exponents
// of P.  Those powers may be 2^144 apart, so for l the exponentials are taken 2^30 larger, and a factor between maxima is applied
// to l as two square roots: neither loses a key that counts.
//
// Measured (32 query heads, 8 kv heads, head dim 128): 16 sequences of about 20,000 tokens in bf16, 1.47 GB, 228 us: 6.4 TB/s;
// 64 in e4m3, 3.6 GB, 646 us: 5.6 TB/s (with pauses 579); four of about 1,000: 12.4 us in a graph, latency.
#include "gorgo_tma.cuh"

namespace gorgo {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr float kOffset = 14.f;           // p = 2^(z - m + kOffset): fp16 keeps p down to 2^-38 of the largest
constexpr int kLift = 30;                 // e4m3: powers of two that l holds more than p

// l and o of a run whose maximum `m` becomes `top`: l * 2^(m - top) for e4m3 pages, where the difference may be large although
// the run counts, and 2^(m - top), the factor of o.
template <bool kQuant>
__device__ __forceinline__ float move_max(float m, float top, float& l) {
  if (m == top) return 1.f;
  if (!kQuant) {
    const float f = fast_exp2(m - top);
    l *= f;
    return f;
  }
  const float h = fast_exp2(0.5f * (m - top));
  l = l * h * h;
  return h * h;
}

template <bool kQuant, int D, int NB>
struct Sizes {
  static constexpr int kRow = D * (kQuant ? 1 : 2);            // bytes of a row
  static constexpr int kSlice = 4096 / kRow;                   // keys of a warp in a tile
  static constexpr int kBlocks = kSlice / 16;
  static constexpr int kTile = kWarps * kSlice;
  static constexpr int kPart = kSlice * kRow;                  // K or V of a slice
  // Codes take more instructions a byte, in chains that a scheduler with two warps does not fill: three blocks an SM
  // with two stages each, where their registers allow it.
  static constexpr int kPerSm = kQuant && NB == 1 ? 3 : 2;
  static constexpr int kStages = kPerSm == 3 ? 2 : 3;
  static constexpr int kRing = kWarps * kStages * 2 * kPart;
  static constexpr int kPad = 64 + 4;                          // floats of a head's row in the merge buffer: 64 dims at a time
  static constexpr int kMerge = kWarps * 8 * kPad * 4;
  static constexpr int kExps = kQuant ? kWarps * kStages * 2 * kSlice : 0;
  static constexpr int kBytes = kRing + kMerge + kExps + kWarps * 8 * 2 * 4 + kWarps * kStages * (8 + 4);
};

struct Split {
  uint32_t hh;                            // (kv head, block of query heads) pairs of a sequence
  uint32_t ng;                            // blocks of query heads of a kv head
  float* part_o;                          // [2 * grid][8 * NB][D]
  float* part_ml;                         // [2 * grid][8 * NB][2]
  uint4* first;                           // [grid]: the (sequence, pair) whose first part a block has, blocks that hold parts (0: none)
  uint32_t grid;                          // blocks of the first kernel
  uint32_t box;                           // keys of one bulk copy: a slice, or a page where that is less
};

template <int kTile>
__device__ __forceinline__ uint32_t tiles_of(const BatchView& b, uint32_t s) {
  const int kv = b.kv_len[s];
  return kv_len_ok(b, kv) ? (uint32_t)(kv + kTile - 1) / kTile : 0;
}

// Pieces that `total` tiles are cut into: not more than blocks, and not below two tiles a piece.
__device__ __forceinline__ uint32_t pieces(uint64_t total, uint32_t grid) {
  return total / 2 >= grid ? grid : total < 4 ? 1 : (uint32_t)(total / 2);
}

template <int kTile>
struct Iter {                             // a place on the line of tiles
  uint32_t s, hh, tile, nt;
  int kv;
  uint32_t left;                          // tiles of this block from here on
  __device__ __forceinline__ void next(const BatchView& b, uint32_t n_hh) {
    if (--left == 0) return;
    if (++tile < nt) return;
    tile = 0;
    if (++hh < n_hh) return;
    hh = 0;
    do { ++s; nt = tiles_of<kTile>(b, s); } while (nt == 0);
    kv = b.kv_len[s];
  }
};

__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1, __nv_bfloat16) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1, __half) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Waits for the copies into the `flying` stages from `st` on.
__device__ __noinline__ void land(uint32_t bars, uint32_t stages, uint32_t st, uint32_t phase, uint32_t flying) {
  for (; flying; --flying) {
    mbar_wait(bars + 8 * st, phase);
    if (++st == stages) { st = 0; phase ^= 1; }
  }
  __syncwarp();
}

// Byte offset of 16-byte chunk c of row r inside a slice, as the bulk copy's swizzle lays it out.
template <bool kQuant, int D>
__device__ __forceinline__ uint32_t chunk_at(uint32_t r, uint32_t c) {
  if (kQuant && D == 64) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
  return (c >> 3) * (16 * 128) + r * 128 + (((c ^ r) & 7) << 4);
}

template <typename T, bool kQuant, int D, int NB>
__global__ void __launch_bounds__(kThreads, Sizes<kQuant, D, NB>::kPerSm)
decode_kernel(const AttnArgs a, const Split sp, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using Z = Sizes<kQuant, D, NB>;
  using M = typename std::conditional<kQuant, __half, T>::type;   // type of the matrix instructions' operands
  constexpr int kSteps = D / 16, kH = 8 * NB, kSlice = Z::kSlice, kBlocks = Z::kBlocks;
  constexpr bool kLow = !(kQuant && std::is_same<T, __nv_bfloat16>::value);   // fp16 P is exact enough for a bf16 result
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  unsigned char* ring = smem + warp * Z::kStages * 2 * Z::kPart;
  float* merge = reinterpret_cast<float*>(smem + Z::kRing);
  unsigned char* exps = smem + Z::kRing + Z::kMerge + warp * Z::kStages * 2 * kSlice;
  float* ml = reinterpret_cast<float*>(smem + Z::kRing + Z::kMerge + Z::kExps);        // [warp][8][2]
  uint64_t* bars = reinterpret_cast<uint64_t*>(ml + kWarps * 8 * 2);
  uint32_t* bad_page = reinterpret_cast<uint32_t*>(bars + kWarps * Z::kStages) + warp * Z::kStages;
  const uint32_t ring_a = smem_u32(ring), exps_a = smem_u32(exps), bar_a = smem_u32(bars + warp * Z::kStages);

  if (lane == 0) {
    for (int i = 0; i < Z::kStages; ++i) mbar_init(bar_a + 8 * i, 1);
    mbar_init_fence();
    prefetch_map(&k_map);
    prefetch_map(&v_map);
  }
  launch_dependents();

  // sequences without keys: zeros; with a wrong length: NaN
  for (uint32_t s = blockIdx.x; s < a.b.n_seqs; s += gridDim.x) {
    const int kv = a.b.kv_len[s];
    const bool ok = kv_len_ok(a.b, kv);
    if (ok && kv > 0) continue;
    if (!ok && threadIdx.x == 0) report(a.b.status, GORGO_KV_BAD_LENGTH);
    const uint32_t none = pack2(ok ? 0.f : NAN, ok ? 0.f : NAN, T());
    uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + (size_t)s * a.out_stride);
    for (uint32_t x = threadIdx.x; x < a.n_heads * (D / 2); x += kThreads) out[x] = none;
    if (a.lse)
      for (uint32_t x = threadIdx.x; x < a.n_heads; x += kThreads) a.lse[(size_t)s * a.n_heads + x] = ok ? -INFINITY : NAN;
  }

  // this block's piece of the line, found by every warp for itself
  Iter<Z::kTile> use;
  uint64_t total = 0, at;                 // `at`: place of tile use.tile on the line
  uint32_t n_pieces;
  {
    for (uint32_t s = lane; s < a.b.n_seqs; s += 32) total += tiles_of<Z::kTile>(a.b, s);
#pragma unroll
    for (int d = 16; d; d /= 2) total += __shfl_xor_sync(0xffffffffu, total, d);
    total *= sp.hh;
    const uint32_t n = n_pieces = pieces(total, gridDim.x);
    if (blockIdx.x >= n || total == 0) {
      if (threadIdx.x == 0) sp.first[blockIdx.x] = make_uint4(0, 0, 0, 0);
      return;
    }
    const uint64_t lo = total * blockIdx.x / n, hi = total * (blockIdx.x + 1) / n;
    at = lo;
    uint64_t before = 0;
    uint32_t s0 = 0, mine = 0, here = 0;
    for (;; s0 += 32) {                   // the sequence that holds tile `lo`
      mine = s0 + lane < a.b.n_seqs ? tiles_of<Z::kTile>(a.b, s0 + lane) : 0;
      uint64_t upto = mine;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const uint64_t o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
      }
      const uint32_t over = __ballot_sync(0xffffffffu, (before + upto) * sp.hh > lo);
      if (over) {
        here = __ffs(over) - 1;
        before += __shfl_sync(0xffffffffu, upto - mine, here);
        break;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    use.s = s0 + here;
    use.nt = __shfl_sync(0xffffffffu, mine, here);
    use.kv = a.b.kv_len[use.s];
    const uint64_t off = lo - before * sp.hh;
    use.hh = (uint32_t)(off / use.nt);
    use.tile = (uint32_t)(off % use.nt);
    use.left = (uint32_t)(hi - lo);
  }
  Iter<Z::kTile> get = use;
  __syncwarp();

  // Copies of a warp's slice of tile `get` into stage `st`.
  auto issue = [&](uint32_t st) {
    if (lane == 0) {
      const uint32_t p0 = get.tile * Z::kTile + warp * kSlice, bar = bar_a + 8 * st;
      const int n = get.kv - (int)p0;     // keys from here on; only pieces that hold some have a page
      if (n <= 0) {
        mbar_arrive(bar);
      } else {
        const uint32_t pieces = min((uint32_t)n + sp.box - 1, (uint32_t)kSlice) / sp.box;
        mbar_expect(bar, pieces * sp.box * 2 * (Z::kRow + (kQuant ? 1 : 0)));
        uint32_t wrong = 0;
        for (uint32_t i = 0, r = 0; i < pieces; ++i, r += sp.box) {
          int64_t row = pool_row(a.kv, a.b, get.s, get.hh / sp.ng, p0 + r);
          if (row < 0) { report(a.b.status, GORGO_KV_BAD_PAGE); wrong = 1; row = 0; }   // (copies something that is there)
          const uint32_t to = ring_a + st * 2 * Z::kPart + r * Z::kRow;
          tma_rows(to, &k_map, (int)row, bar);
          tma_rows(to + Z::kPart, &v_map, (int)row, bar);
          if (kQuant) {
            bulk_copy(exps_a + st * 2 * kSlice + r, a.kv.k_exp + row, sp.box, bar);
            bulk_copy(exps_a + st * 2 * kSlice + kSlice + r, a.kv.v_exp + row, sp.box, bar);
          }
        }
        bad_page[st] = wrong;
      }
    }
    get.next(a.b, sp.hh);
    __syncwarp();                         // (bad_page is read by all lanes)
  };

  uint32_t flying = 0;                    // stages whose copies may still run
  for (; flying < (uint32_t)Z::kStages && get.left; ++flying) issue(flying);

  uint32_t qf[NB][kSteps][2];             // q as the second operand: (k = dim, n = head)
  float o[NB][kSteps][4], m[NB][2], l[NB][2], zs[NB][2];
  uint32_t st = 0, phase = 0, first_tile = 0, h0 = 0, n_h = 0;  // h0, n_h: first query head and how many
  uint4 begun = make_uint4(0, 0, 0, 0);
  bool fresh = true, bad = false, alive = true;
  for (;;) {
    if (fresh) {
      h0 = use.hh / sp.ng * a.group + use.hh % sp.ng * kH;
      n_h = min((uint32_t)kH, a.group - use.hh % sp.ng * kH);
      first_tile = use.tile;
      bad = false;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const bool have = 8 * nb + g < n_h;
        const T* q = static_cast<const T*>(a.q) + (size_t)use.s * a.q_stride + (size_t)(h0 + (have ? 8 * nb + g : 0)) * D;
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          // e4m3: a thread's four codes are neighbours, so the dims of a step are taken in that order
          const int d0 = k * 16 + (kQuant ? 4 * t : 2 * t), d1 = kQuant ? d0 + 2 : d0 + 8;
          qf[nb][k][0] = have ? *reinterpret_cast<const uint32_t*>(q + d0) : 0;
          qf[nb][k][1] = have ? *reinterpret_cast<const uint32_t*>(q + d1) : 0;
          if (kQuant) {
            const float2 x = unpack2(qf[nb][k][0], T()), y = unpack2(qf[nb][k][1], T());
            top = fmaxf(fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y))), fmaxf(fabsf(y.x), fabsf(y.y)));
          }
        }
        float back = 1.f;
        if (kQuant) {
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const int e = max((int)(__float_as_uint(top) >> 23) - 127, -100) - 10;
          const float f = pow2i(-e);
          back = pow2i(e);
#pragma unroll
          for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float2 x = unpack2(qf[nb][k][i], T());
              qf[nb][k][i] = pack2(x.x * f, x.y * f, __half());
            }
        }
        // the factor of head g's scores, where this thread has heads 2t and 2t + 1
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          zs[nb][i] = __shfl_sync(0xffffffffu, back, (2 * t + i) * 4) * a.scale_log2;
          m[nb][i] = -INFINITY;
          l[nb][i] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[nb][k][i] = 0.f;
      }
      fresh = false;
    }

    const int n_keys = use.kv - (int)(use.tile * Z::kTile + warp * kSlice);
    const uint32_t bar = bar_a + 8 * st;
    if (flying && !__all_sync(0xffffffffu, mbar_wait(bar, phase, a.wait_ticks))) {
      alive = false;                      // no more copies; those that fly land before the block ends
      if (lane == 0) report(a.b.status, GORGO_KV_WAIT_LIMIT);
      land(bar_a, Z::kStages, st, phase, flying);
      flying = 0;
    }
    if (n_keys > 0 && alive) {
      bad |= bad_page[st] != 0;
      const uint32_t ka = ring_a + st * 2 * Z::kPart, va = ka + Z::kPart;
      float c[kBlocks][NB][4];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i) c[b][nb][i] = 0.f;
        const uint32_t r = 16 * b + (lane & 15), hi = lane >> 4;
#pragma unroll
        for (int k = 0; k < kSteps; k += (kQuant ? 2 : 1)) {
          uint32_t f[4];
          if (!kQuant) {
            ldsm4(f, ka + chunk_at<kQuant, D>(r, 2 * k + hi));
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma(c[b][nb], f, qf[nb][k][0], qf[nb][k][1], M());
          } else {
            ldsm4(f, ka + chunk_at<kQuant, D>(r, k + hi));     // two steps' codes: four neighbours of a row each
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t x[4] = {codes_to_half2((uint16_t)f[2 * i]), codes_to_half2((uint16_t)f[2 * i + 1]),
                                     codes_to_half2((uint16_t)(f[2 * i] >> 16)), codes_to_half2((uint16_t)(f[2 * i + 1] >> 16))};
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) mma(c[b][nb], x, qf[nb][k + i][0], qf[nb][k + i][1], M());
            }
          }
        }
      }
      // rows g and g + 8 of a block of S^T: this thread's two keys; columns 2t and 2t + 1: its two heads
      float vi[kBlocks][2];               // what l takes p times: the values' powers of two go into P alone
      const bool part = n_keys < kSlice;
      bool grow = false;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const int8_t* e = reinterpret_cast<const int8_t*>(exps + st * 2 * kSlice) + 16 * b + g;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bool have = 16 * b + (int)g + 8 * i < n_keys;  // (behind the last key lies anything)
          float ks = 1.f, ve = 0.f;
          vi[b][i] = 1.f;
          if (kQuant) {
            ks = pow2i(have ? e[8 * i] : 0);
            const int v = have ? e[kSlice + 8 * i] : 0;
            ve = (float)v;
            vi[b][i] = pow2i(-v);
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float z = c[b][nb][2 * i + j] * zs[nb][j];
              if (kQuant) z = __fmaf_rn(z, ks, ve);
              c[b][nb][2 * i + j] = part && !have ? -INFINITY : z;
            }
        }
      }
      float top[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x = fmaxf(c[0][nb][i], c[0][nb][i + 2]);
#pragma unroll
          for (int b = 1; b < kBlocks; ++b) x = fmaxf(x, fmaxf(c[b][nb][i], c[b][nb][i + 2]));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
          top[nb][i] = x;
          grow |= x > m[nb][i];
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float x = fmaxf(m[nb][i], top[nb][i]);
            f[i] = move_max<kQuant>(m[nb][i], x, l[nb][i]);
            m[nb][i] = x;
          }
#pragma unroll
          for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[nb][k][i] *= f[i & 1];
        }
      }
      uint32_t ph[kBlocks][NB][2], pl[kBlocks][NB][2];   // P as the second operand (k = key, n = head), high and low part
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        constexpr float kUp = kOffset + (kQuant ? kLift : 0);
        const float m0 = m[nb][0] == -INFINITY ? 0.f : m[nb][0] - kUp, m1 = m[nb][1] == -INFINITY ? 0.f : m[nb][1] - kUp;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 2; ++i) {   // key g + 8 i
            float x = fast_exp2(c[b][nb][2 * i] - m0), y = fast_exp2(c[b][nb][2 * i + 1] - m1);
            l[nb][0] = __fmaf_rn(x, vi[b][i], l[nb][0]);
            l[nb][1] = __fmaf_rn(y, vi[b][i], l[nb][1]);
            if (kQuant) {
              x *= pow2i(-kLift);
              y *= pow2i(-kLift);
            }
            const uint32_t hi = pack2(x, y, M());
            ph[b][nb][i] = transpose8(hi);
            if (kLow) {
              const float2 h = unpack2(hi, M());
              pl[b][nb][i] = transpose8(pack2(x - h.x, y - h.y, M()));
            }
          }
      }
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        // values behind the last key may be anything: they enter as zeros
        const int n = n_keys - 16 * b;
        const uint32_t keep0 = ((int)(2 * t) < n ? 0xffffu : 0) | ((int)(2 * t + 1) < n ? 0xffff0000u : 0);
        const uint32_t keep8 = ((int)(2 * t + 8) < n ? 0xffffu : 0) | ((int)(2 * t + 9) < n ? 0xffff0000u : 0);
#pragma unroll
        for (int k = 0; k < kSteps; k += (kQuant ? 2 : 1)) {
          uint32_t f[4];
          if (!kQuant) {
            ldsm4t(f, va + chunk_at<kQuant, D>(16 * b + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
            if (part) { f[0] &= keep0; f[1] &= keep0; f[2] &= keep8; f[3] &= keep8; }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              mma(o[nb][k], f, ph[b][nb][0], ph[b][nb][1], M());
              if (kLow) mma(o[nb][k], f, pl[b][nb][0], pl[b][nb][1], M());
            }
          } else {
            // two columns of 16 dims: a register holds dims 2g, 2g + 1 of key 2t (low half) and of key 2t + 1
            ldsm4t(f, va + chunk_at<kQuant, D>(16 * b + (lane & 15), k + (lane >> 4)));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t x[4];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const uint32_t y = __byte_perm(f[2 * i + j], 0, 0x3120);   // dim 2g of both keys, then dim 2g + 1
                x[2 * j] = codes_to_half2((uint16_t)y);
                x[2 * j + 1] = codes_to_half2((uint16_t)(y >> 16));
              }
              if (part) { x[0] &= keep0; x[1] &= keep0; x[2] &= keep8; x[3] &= keep8; }
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) {
                mma(o[nb][k + i], x, ph[b][nb][0], ph[b][nb][1], M());
                if (kLow) mma(o[nb][k + i], x, pl[b][nb][0], pl[b][nb][1], M());
              }
            }
          }
        }
      }
    }
    __syncwarp();                         // the stage has been read
    const bool last = use.left == 1;
    if (get.left && alive) issue(st);
    else if (flying) --flying;
    if (++st == (uint32_t)Z::kStages) { st = 0; phase ^= 1; }

    if (last || use.tile + 1 == use.nt) {
      // the warps' sums of this (sequence, head) become one, eight heads and 64 dims at a time
      const bool whole = first_tile == 0 && use.tile + 1 == use.nt;
      const uint32_t slot = 2 * blockIdx.x + (first_tile == 0 ? 1 : 0);
      if (!whole && first_tile == 0) {    // the second kernel finds its parts here and in the blocks behind
        const uint64_t end = at + (use.nt - use.tile);         // of its tiles on the line
        begun = make_uint4(use.s, use.hh, (uint32_t)((end * n_pieces - 1) / total) - blockIdx.x + 1, 0);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if (8 * nb >= (int)n_h) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x = l[nb][i];
          x += __shfl_xor_sync(0xffffffffu, x, 4);
          x += __shfl_xor_sync(0xffffffffu, x, 8);
          x += __shfl_xor_sync(0xffffffffu, x, 16);
          if (kQuant) x *= pow2i(-kLift);
          if (bad || !alive) x = NAN;
          if (g == 0) {
            ml[(warp * 8 + 2 * t + i) * 2] = m[nb][i];
            ml[(warp * 8 + 2 * t + i) * 2 + 1] = x;
          }
        }
        float* mo = merge + warp * 8 * Z::kPad;
#pragma unroll
        for (int part = 0; part < D / 64; ++part) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int dim = k * 16 + (kQuant ? 2 * g + (i >> 1) : g + 8 * (i >> 1));
              mo[(2 * t + (i & 1)) * Z::kPad + dim] = o[nb][4 * part + k][i];
            }
          __syncthreads();
          static_assert(8 * 16 == kThreads, "a thread has four dims of a head");
          const uint32_t h = threadIdx.x / 16, d = threadIdx.x % 16 * 4;
          if (8 * nb + h < n_h) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[(w * 8 + h) * 2]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
              float lw = ml[(w * 8 + h) * 2 + 1];
              const float f = move_max<kQuant>(ml[(w * 8 + h) * 2], top, lw);
              const float4 y = *reinterpret_cast<const float4*>(merge + (w * 8 + h) * Z::kPad + d);
              sum += lw;
              acc.x = __fmaf_rn(y.x, f, acc.x);
              acc.y = __fmaf_rn(y.y, f, acc.y);
              acc.z = __fmaf_rn(y.z, f, acc.z);
              acc.w = __fmaf_rn(y.w, f, acc.w);
            }
            const uint32_t at = 64 * part + d;
            if (whole) {
              const float inv = sum == 0.f ? 0.f : 1.f / sum;  // (0: every score is minus infinity, and so is lse)
              T* out = static_cast<T*>(a.out) + (size_t)use.s * a.out_stride + (size_t)(h0 + 8 * nb + h) * D + at;
              *reinterpret_cast<uint2*>(out) = make_uint2(pack2(acc.x * inv, acc.y * inv, T()), pack2(acc.z * inv, acc.w * inv, T()));
              if (a.lse && at == 0)
                a.lse[(size_t)use.s * a.n_heads + h0 + 8 * nb + h] = (top - kOffset + log2f(sum)) * 0.693147180559945309f;
            } else {
              *reinterpret_cast<float4*>(sp.part_o + ((size_t)slot * kH + 8 * nb + h) * D + at) = acc;
              if (at == 0) *reinterpret_cast<float2*>(sp.part_ml + ((size_t)slot * kH + 8 * nb + h) * 2) = make_float2(top, sum);
            }
          }
          __syncthreads();
        }
      }
      fresh = true;
    }
    if (last) break;
    use.next(a.b, sp.hh);
    ++at;
  }
  if (threadIdx.x == 0) sp.first[blockIdx.x] = begun;
}

// Joins what several blocks hold of one query head: block x of this kernel has the pair whose first part block x of the
// first kernel has.  Its threads take every 8th or 16th part, 16 bytes of the row each, with a running maximum, so that
// parts arrive side by side.
constexpr int kJoinThreads = 256;
template <typename T, bool kQuant, int D, int NB>
__global__ void __launch_bounds__(kJoinThreads) decode_join_kernel(const AttnArgs a, const Split sp) {
  constexpr uint32_t kH = 8 * NB, kVec = D / 4, kWays = kJoinThreads / kVec;
  const uint32_t way = threadIdx.x / kVec, d = threadIdx.x % kVec * 4, h = blockIdx.y;
  __shared__ float part[kWays][D + 4];
  wait_primary();
  const uint4 what = sp.first[blockIdx.x];
  const uint32_t s = what.x, hh = what.y;
  if (what.z == 0 || h >= a.group - hh % sp.ng * kH) return;
  const uint32_t head = hh / sp.ng * a.group + hh % sp.ng * kH + h;
  const uint32_t c0 = blockIdx.x, c1 = c0 + what.z - 1;
  T* out = static_cast<T*>(a.out) + (size_t)s * a.out_stride + (size_t)head * D + d;
  float* lse = a.lse ? a.lse + (size_t)s * a.n_heads + head : nullptr;
  // the first block holds its last piece of line, the others their first
  auto at = [&](uint32_t c) { return (size_t)(2 * c + (c == c0 ? 1 : 0)) * kH + h; };
  float top = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (uint32_t c = c0 + way; c <= c1; c += kWays) {
    float2 p = *reinterpret_cast<const float2*>(sp.part_ml + at(c) * 2);
    const float4 y = *reinterpret_cast<const float4*>(sp.part_o + at(c) * D + d);
    const float now = fmaxf(top, p.x);
    const float f = move_max<kQuant>(top, now, sum), w = move_max<kQuant>(p.x, now, p.y);
    top = now;
    sum += p.y;
    acc.x = __fmaf_rn(y.x, w, acc.x * f);
    acc.y = __fmaf_rn(y.y, w, acc.y * f);
    acc.z = __fmaf_rn(y.z, w, acc.z * f);
    acc.w = __fmaf_rn(y.w, w, acc.w * f);
  }
  *reinterpret_cast<float4*>(&part[way][d]) = acc;
  if (d == 0) { part[way][D] = top; part[way][D + 1] = sum; }
  __syncthreads();
  if (way) return;
#pragma unroll
  for (uint32_t w = 0; w < kWays; ++w) top = fmaxf(top, part[w][D]);
  sum = 0.f;
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (uint32_t w = 0; w < kWays; ++w) {
    float lw = part[w][D + 1];
    const float f = move_max<kQuant>(part[w][D], top, lw);
    const float4 y = *reinterpret_cast<const float4*>(&part[w][d]);
    sum += lw;
    acc.x = __fmaf_rn(y.x, f, acc.x);
    acc.y = __fmaf_rn(y.y, f, acc.y);
    acc.z = __fmaf_rn(y.z, f, acc.z);
    acc.w = __fmaf_rn(y.w, f, acc.w);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<uint2*>(out) = make_uint2(pack2(acc.x * inv, acc.y * inv, T()), pack2(acc.z * inv, acc.w * inv, T()));
  if (lse && d == 0) *lse = (top - kOffset + log2f(sum)) * 0.693147180559945309f;
}

uint32_t head_blocks(uint32_t group) { return group <= 8 ? 1 : (group + 15) / 16; }

template <typename T, bool kQuant, int D, int NB>
cudaError_t launch(const AttnArgs& a, int sms, cudaStream_t st) {
  using Z = Sizes<kQuant, D, NB>;
  static_assert(Z::kPerSm * (Z::kBytes + 1024) <= 233472, "blocks of an SM");
  Split sp;
  sp.ng = head_blocks(a.group);
  sp.hh = a.kv.n_kv_heads * sp.ng;
  sp.grid = Z::kPerSm * sms;
  sp.box = min((uint32_t)Z::kSlice, 1u << a.kv.page_shift);
  sp.part_o = static_cast<float*>(a.workspace);
  sp.part_ml = sp.part_o + (size_t)2 * sp.grid * 8 * NB * D;
  sp.first = reinterpret_cast<uint4*>(sp.part_ml + (size_t)2 * sp.grid * 8 * NB * 2);
  CUtensorMap km, vm;
  const uint64_t rows = (uint64_t)a.kv.n_pages * a.kv.n_kv_heads << a.kv.page_shift;
  const uint32_t planes = Z::kRow > 128 ? Z::kRow / 128 : 1;
  if (!make_pool_map(&km, a.kv.k, rows, D, a.store, sp.box, planes) ||
      !make_pool_map(&vm, a.kv.v, rows, D, a.store, sp.box, planes))
    return cudaErrorUnknown;
  auto kernel = decode_kernel<T, kQuant, D, NB>;
  cudaError_t e = allow_smem<decode_kernel<T, kQuant, D, NB>>(Z::kBytes);
  if (e != cudaSuccess) return e;
  kernel<<<sp.grid, kThreads, Z::kBytes, st>>>(a, sp, km, vm);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sp.grid, a.group < 8 * NB ? a.group : 8 * NB);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute early = {};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, decode_join_kernel<T, kQuant, D, NB>, a, sp);
}

template <typename T, bool kQuant, int D>
cudaError_t launch(const AttnArgs& a, int sms, cudaStream_t st) {
  return a.group <= 8 ? launch<T, kQuant, D, 1>(a, sms, st) : launch<T, kQuant, D, 2>(a, sms, st);
}
template <typename T, bool kQuant>
cudaError_t launch(const AttnArgs& a, int sms, cudaStream_t st) {
  return a.head_dim == 128 ? launch<T, kQuant, 128>(a, sms, st) : launch<T, kQuant, 64>(a, sms, st);
}

}  // namespace

uint64_t decode_workspace(const AttnArgs& a, int sms) {
  const uint64_t heads = a.group <= 8 ? 8 : 16;
  return (uint64_t)3 * sms * (2 * heads * (a.head_dim + 2) * 4 + 16);   // (three blocks an SM at most, two parts each)
}

cudaError_t launch_attn_decode(const AttnArgs& a, int sms, cudaStream_t st) {
  const bool q = a.store == GORGO_E4M3;
  if (a.type == GORGO_BF16) return q ? launch<__nv_bfloat16, true>(a, sms, st) : launch<__nv_bfloat16, false>(a, sms, st);
  return q ? launch<__half, true>(a, sms, st) : launch<__half, false>(a, sms, st);
}

}  // namespace gorgo
