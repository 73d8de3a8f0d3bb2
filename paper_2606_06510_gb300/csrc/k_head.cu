// Losses over a vocabulary from the last layer's input x and the head's weights w,
// without keeping the logits z = scale·x·wᵀ:
//
//   forward    per token the sum of exponentials and its targets' logits
//   gradient   dz = a·((1 + e)·exp(z - lse) - weights of its targets), z formed again;
//              dx = dz·w and dw = dzᵀ·x are k_linear.cu's products
//
// A hard target has the weight 1, a teacher's listed rows the softmax of its logits.
#include <algorithm>

#include "lin_mma.cuh"
#include "lm_common.cuh"

namespace oz2 {
namespace {

constexpr int kEpiWarps = 16;
constexpr int kThreads = 64 + 32 * kEpiWarps;  // TMA warp, MMA warp, epilogue warps
constexpr int kStages = 5;
constexpr int kTile = 256;                     // tokens and vocabulary rows of a CTA pair's tile
constexpr int kStage = 2 * kTileBytes;
constexpr int kChunk = 32;                     // columns that an epilogue warp takes at a time
constexpr int kBuffer = 32 * 2 * kChunk;       // its 32 rows of them in 16 bits
constexpr int kSmem = 1024 + kStages * kStage + kEpiWarps * kBuffer + 256;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.402823466e38f;    // no maximum is below it: z - max is a number then, but for infinities

struct HeadMaps {
  CUtensorMap x, w, w_half;                    // w in boxes of 128 and of 64 rows
};
struct HeadUnits {
  int ntm, ntn, units, half_units;             // whole tiles, and after those halves of tiles
  int steps;                                   // of 64 elements of depth
};

// The unit's tile: bands of 8 tile rows, so that the tiles in flight share rows in L2.
struct HeadTile {
  int tm, col, width;
};
__device__ __forceinline__ bool head_tile(const HeadUnits& u, int i, HeadTile& t) {
  if (i >= u.units + u.half_units) return false;
  const int half = i - u.units, at = half >= 0 ? u.units + half / 2 : i;
  const int per = 8 * u.ntn, band = at / per, in = at - band * per;
  const int h = min(8, u.ntm - band * 8), tn = in / h;
  t.tm = band * 8 + (in - tn * h);
  t.col = tn * kTile;
  t.width = kTile;
  if (half >= 0) {
    t.width = kTile / 2;
    t.col += (half & 1) * t.width;
  }
  return true;
}

// A token's terms: of its target, or as they were prepared for listed rows.
__device__ __forceinline__ HeadRow head_row(const HeadTerms& t, Ids ids, int64_t n, int64_t row) {
  if (t.rows) {
    const float4 f = __ldg(reinterpret_cast<const float4*>(t.rows) + row);
    return HeadRow{f.x, f.y, f.z, __float_as_int(f.w)};
  }
  const int64_t id = ids[row];
  if (id < 0) return HeadRow{0.f, 0.f, 0.f, 0};
  const float l = __ldg(t.lse + row), g = __ldg(t.dloss + (t.dloss_each ? row : 0)) * t.scale;
  return HeadRow{id < n ? g : __int_as_float(0x7FC00000), l, t.z_loss != 0.f ? 2.f * t.z_loss * l : 0.f, 1};
}
// The largest |dz| that a token's terms can give: a·(1 + e)·p, or a target's a·((1 + e)·p - 1), for
// p up to 1.  (What is no number does not count.)
__device__ __forceinline__ float head_size(const HeadRow& r) {
  const float size = fabsf(r.a) * fmaxf(fmaxf(1.f, fabsf(r.e)), fabsf(1.f + r.e));
  return size < INFINITY ? size : 0.f;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// v[j] for a j that the compiler does not know.
__device__ __forceinline__ float pick32(const uint32_t (&v)[32], int j) {
  uint32_t t[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) t[i] = j & 1 ? v[2 * i + 1] : v[2 * i];
#pragma unroll
  for (int n = 8, b = 2; n; n >>= 1, b <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) t[i] = j & b ? t[2 * i + 1] : t[2 * i];
  return __uint_as_float(t[0]);
}
__device__ __forceinline__ void set32(float (&v)[32], int j, float d) {
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (i == j) v[i] = d;
}

// The larger one; NaN where either is NaN: a maximum of infinity then says that there is none, and
// lse is infinity (the sum beside it is no number in both cases).
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A lane's maximum of v·to2 over its 64 sums (the first `cols` where not WHOLE), and the sum
// of exp2 of the differences: the largest sum first, in its own units (NEGATIVE to2: the
// smallest), then one multiply-add for two differences.
template <bool NEGATIVE>
__device__ __forceinline__ float extreme(float a, float b, float c) {
  float r;
  if (NEGATIVE) {
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  } else {
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  }
  return r;
}
template <bool WHOLE, bool NEGATIVE>
__device__ __forceinline__ void head_sums(const uint32_t (&v0)[32], const uint32_t (&v1)[32], int cols, float to2, float& most,
                                          float& sum) {
  auto t = [&](int j) {  // past the vocabulary's end: the first one again
    const float v = __uint_as_float(j < 32 ? v0[j & 31] : v1[j & 31]);
    return WHOLE || j < cols ? v : __uint_as_float(v0[0]);
  };
  float top[4] = {t(0), t(1), t(2), t(3)};
#pragma unroll
  for (int j = 4; j < 60; j += 8)
#pragma unroll
    for (int e = 0; e < 4; ++e) top[e] = extreme<NEGATIVE>(top[e], t(j + e), t(j + 4 + e));
  top[0] = extreme<NEGATIVE>(top[0], top[1], t(60));
  top[1] = extreme<NEGATIVE>(top[2], t(61), t(62));
  top[2] = extreme<NEGATIVE>(top[3], t(63), t(63));
  most = max_nan(extreme<NEGATIVE>(top[0], top[1], top[2]) * to2, kLowest);
  const Two to = two(to2, to2), less = two(-most, -most);
  Two s[2] = {two(0.f, 0.f), two(0.f, 0.f)};
#pragma unroll
  for (int j = 0; j < 64; j += 2) {
    const float2 x = both(fma(two(t(j), t(j + 1)), to, less));
    float a = exp2_fast(x.x), b = exp2_fast(x.y);
    if (!WHOLE) a = j < cols ? a : 0.f, b = j + 1 < cols ? b : 0.f;
    s[j >> 1 & 1] = s[j >> 1 & 1] + two(a, b);
  }
  const float2 r = both(s[0] + s[1]);
  sum = r.x + r.y;
}

// ---------------------------------------------------------------------------
// Tiles of 256 tokens × 256 rows of w on CTA pairs as in linear_pair_kernel: 128 rows
// of each operand a CTA, two accumulators in tensor memory, so that a tile's epilogue
// runs beside the next one's products.  An epilogue warp has 32 tokens, one a lane, and
// 64 columns.
//
// Forward, a lane takes the maximum of its logits in powers of two and sums exp2 of the
// differences; its group's two numbers are joined to the others' by head_join_kernel.  Gradient,
// it turns them into dz, which goes to memory by way of its warp's two KB.
//
// Fewer bits: exp2 is the approximate one (2^-22 of the value, a few steps of FP32), and dz is
// rounded to the operands' 16 bits, the type in which the tensor cores take both sides of a
// product.  dX and dW then carry that rounding beside their own: 1.4 times the error of one, up to
// 1.65 where few terms make a sum.  Two 16-bit terms for each dz would take it away and run dX's and
// dW's products, over half of the gradient's time, twice.
//
// What bounds it: the tensor pipes (4096×50257×1024 bf16: 96% of their cycles, 209 µs alone, 238
// back to back under the power cap; the gradient's 84%, 239 µs, its epilogue being nearly as
// long as 16 steps of products).  A depth of 128 is all epilogue: 2 µs a tile forward, 4 with dz,
// whose bytes are then the memory's rate.  What a lane reads of its token for the next tile is on
// its way while it works on this one.
// ---------------------------------------------------------------------------
template <int TYPE, bool GRAD, bool SOFT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    head_kernel(const __grid_constant__ HeadMaps maps, const __grid_constant__ HeadArgs A, const HeadUnits U,
                Oz2Device* dev) {
  constexpr bool BF16 = TYPE == OZ2_TYPE_BF16;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* epi = smem + kStages * kStage;
  uint64_t* bars = reinterpret_cast<uint64_t*>(epi + kEpiWarps * kBuffer);
  // bars: full[S], empty[S], acc_full[2], acc_empty[2], drain
  __shared__ uint32_t tmem_base_s;

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + kStages);
  const uint32_t acc_full = smem_u32(bars + 2 * kStages), acc_empty = smem_u32(bars + 2 * kStages + 2);
  const uint32_t drain_bar = smem_u32(bars + 2 * kStages + 4);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full + 8 * a, 1);
      mbar_init(acc_empty + 8 * a, 2 * kEpiWarps);
    }
    mbar_init(drain_bar, 1);
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&tmem_base_s), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_s, 0);
  bool ok = true;
  pdl_wait();

  HeadTile tile;
  const int steps = U.steps;
  if (warp == 0) {
    // ---------------- TMA producer (both CTAs) ----------------
    if (elect_one()) {
      const uint32_t full_leader0 = mapa_shared(full0, 0), ring0 = smem_u32(smem);
      uint32_t it = 0, s = 0, ph = 1;
      for (int i = pair; ok && steps && head_tile(U, i, tile); i += npairs) {
        const bool half = tile.width != kTile;
        const int xrow = tile.tm * kTile + rank * kRows, wrow = tile.col + rank * (tile.width / 2);
        const CUtensorMap* mw = half ? &maps.w_half : &maps.w;
        const uint32_t bytes = 2u * (kTileBytes + (half ? kTileBytes / 2 : kTileBytes));
        for (int t = 0, d = 0; t < steps; ++t, d += 64) {
          if (!mbar_wait_bounded(empty0 + 8 * s, ph, kWaitLimit)) {
            ok = false;
            break;
          }
          const uint32_t sa = ring0 + s * kStage, bar = full_leader0 + 8 * s;
          if (leader) mbar_arrive_expect_tx(full0 + 8 * s, bytes);
          tma_load_2d_pair(sa, &maps.x, bar, d, xrow);
          tma_load_2d_pair(sa + kTileBytes, mw, bar, d, wrow);
          ++it;
          if (++s == kStages) {
            s = 0;
            ph ^= 1;
          }
        }
      }
      if (!ok) {
        dev->status = kStatusTimeout;
        dev->timeout_site = 31;
      }
      pdl_trigger();
      if (leader)  // the leader's stage barriers also count the peer's bytes
        for (uint32_t j = (it > kStages ? it - kStages : 0); j < it; ++j)
          mbar_wait_bounded(full0 + 8 * (j % kStages), (j / kStages) & 1, kWaitLimit);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------- MMA issuer (leader CTA) ----------------
    if (leader) {  // the whole warp; lane 0 issues
      const uint32_t me = lane == 0;
      const uint32_t base = smem_u32(smem);
      const uint64_t xd = operand_desc<false>(base), wd = operand_desc<false>(base + kTileBytes);
      uint32_t s = 0, ph = 0, acc = 0, accph = 1;
      auto multiply = [&](auto shape, uint32_t d) {
        for (int t = 0; t < steps && ok; ++t) {
          if (!(ok = mbar_wait_warp(full0 + 8 * s, ph, kWaitLimit))) break;
          tc_fence_after();
          const uint64_t a = xd + s * (kStage >> 4), b = wd + s * (kStage >> 4);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_pair<false>(me, d, a + kk * shape.a_next, b + kk * shape.b_next, shape.idesc, (t | kk) ? 1u : 0u);
          mma_commit_pair_mc(me, empty0 + 8 * s, 0x3);
          if (++s == kStages) {
            s = 0;
            ph ^= 1;
          }
        }
      };
      for (int i = pair; ok && steps && head_tile(U, i, tile); i += npairs) {
        ok = mbar_wait_warp(acc_empty + 8 * acc, accph, kWaitLimit);
        tc_fence_after();
        if (tile.width == kTile) {
          multiply(MmaShape<TYPE, false, false, kTile, kTile>{}, tmem + acc * kTile);
        } else {
          multiply(MmaShape<TYPE, false, false, kTile, kTile / 2>{}, tmem + acc * kTile);
        }
        if (!ok) break;
        mma_commit_pair_mc(me, acc_full + 8 * acc, 0x3);
        acc ^= 1;
        if (acc == 0) accph ^= 1;
      }
      if (!ok && me) {
        dev->status = kStatusTimeout;
        dev->timeout_site = 32;
      }
      mma_commit_pair(me, drain_bar);
      mbar_wait_bounded(drain_bar, 0, kWaitLimit);
    }
    __syncwarp();
  } else {
    // ---------------- epilogue (warps 2..17, both CTAs) ----------------
    const int ew = warp - 2;
    const int q = warp & 3, h = ew >> 2;  // TMEM lane quarter, column quarter
    uint8_t* buf = epi + ew * kBuffer;
    const uint32_t acc_empty_leader = mapa_shared(acc_empty, 0);
    const float to2 = A.scale * kLog2E;   // logits in powers of two
    float up = 1.f;                       // dz's scale
    if (GRAD && A.largest) {
      float most = 0.f;
#pragma unroll 16
      for (int i = lane; i < A.maxima; i += 32) most = fmaxf(most, __ldg(A.largest + i));
      const int bits = __float_as_int(warp_max(most)), e = (bits >> 23) - 127;
      const int s = bits > 0 ? max(-100, min(100, 14 - e)) : 0;
      up = __int_as_float((127 + s) << 23);
      if (blockIdx.x == 0 && threadIdx.x == 64) *A.unscale = __int_as_float((127 - s) << 23);
    }
    uint32_t acc = 0, accph = 0;
    // What a lane has to know of its token for a tile, and where in the tile its warp is: read
    // while the tile before is worked on.
    struct Part {
      int row;
      int col0, cols;        // in the piece; of the warp (a half tile is two warps' columns)
      int next;              // the token's target here: its row of w (in the piece)
      int at, end;           // or its entries here
      HeadRow terms;
    };
    auto entry_at = [&](const Part& p, int at) {
      return at < p.end ? __ldg(A.entries + static_cast<int64_t>(p.row) * A.top + at) : make_int2(kNoTarget, 0);
    };
    auto find = [&](int i, Part& p) {
      if (!head_tile(U, i, tile)) return false;
      p.row = tile.tm * kTile + rank * kRows + 32 * q + lane;
      p.col0 = tile.col + kHeadGroup * h;
      p.cols = kHeadGroup * h < tile.width && p.col0 < A.cols ? min(static_cast<int64_t>(kHeadGroup), A.cols - p.col0) : 0;
      p.next = kNoTarget;
      if (SOFT) p.at = p.end = 0;
      p.terms = HeadRow{0.f, 0.f, 0.f, 0};
      if (p.row < A.m && p.cols > 0) {
        const int first = static_cast<int>(A.c0) + p.col0;
        if (GRAD) {
          p.terms = head_row(A.terms, A.ids, A.n, p.row);
          p.terms.a *= up;
        }
        if (!SOFT) {
          const int64_t id = A.ids[p.row];
          if (id >= first && id < A.n) p.next = static_cast<int>(id - A.c0);
        }
      }
      if (SOFT && p.cols > 0 && p.row < A.m) {
        const uint16_t* offset = A.offsets + (A.c0 + p.col0) / kHeadGroup * A.ld_offsets + p.row;
        p.at = __ldg(offset), p.end = __ldg(offset + A.ld_offsets);
      }
      return true;
    };
    Part now, then;
    bool more = find(pair, now);
    for (int i = pair; more; now = then) {
      i += npairs;
      int2 entry, after;  // the lane's next two entries, whose loads are on their way while it waits
      if (SOFT) entry = entry_at(now, now.at), after = entry_at(now, now.at + 1);
      if (steps) {
        if (!mbar_wait_bounded(acc_full + 8 * acc, accph, kWaitLimit)) ok = false;
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        tc_fence_after();
      }
      const int row = now.row;
      const int col0 = now.col0, cols = now.cols;
      const uint32_t from = tmem + (static_cast<uint32_t>(32 * q) << 16) + acc * kTile + kHeadGroup * h;
      auto load = [&](int c, uint32_t (&v)[32]) {
        if (steps) {
          tmem_ld32(from + c, v);
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0u;
        }
      };
      auto release = [&] {  // the sums are in registers: the next but one tile's products may begin
        if (steps) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote_relaxed(acc_empty_leader + 8 * acc);
          acc ^= 1;
          if (acc == 0) accph ^= 1;
        }
      };
      if (cols == 0) {
        release();
        more = find(i, then);
        continue;
      }
      // The column in the piece of the lane's next entry.
      int column = kNoTarget;
      auto look = [&] { column = entry.x != kNoTarget ? entry.x - static_cast<int>(A.c0) : kNoTarget; };
      auto advance = [&] {
        entry = after;
        ++now.at;
        after = entry_at(now, now.at + 1);
        look();
      };
      if (SOFT) look();
      if (!GRAD) {
        auto pick = [&](const uint32_t (&v)[32], int from) {
          if (SOFT) {
#pragma unroll
            for (int g = 0; g < 32; g += 8) {
              while (__any_sync(0xffffffffu, column < from + g + 8)) {
                if (column < from + g + 8) {
                  const int at = column - (from + g);
                  uint32_t e = v[g];
#pragma unroll
                  for (int j = 1; j < 8; ++j) e = j == at ? v[g + j] : e;
                  A.picked[static_cast<int64_t>(row) * A.top + entry.y] = __uint_as_float(e) * A.scale;
                  advance();
                }
              }
            }
            __syncwarp();
          } else if (__any_sync(0xffffffffu, now.next < from + 32)) {
            if (now.next < from + 32) {
              A.picked[row] = pick32(v, now.next - from) * A.scale;
              now.next = kNoTarget;
            }
            __syncwarp();
          }
        };
        uint32_t v0[32], v1[32];
        load(0, v0);
        load(32, v1);
        tmem_ld_wait();
        release();
        more = find(i, then);
        pick(v0, col0);
        pick(v1, col0 + 32);
        float most, sum;
        if (to2 >= 0.f) {
          cols == kHeadGroup ? head_sums<true, false>(v0, v1, cols, to2, most, sum)
                             : head_sums<false, false>(v0, v1, cols, to2, most, sum);
        } else {
          head_sums<false, true>(v0, v1, cols, to2, most, sum);
        }
        if (row < A.m) A.stats[static_cast<int64_t>(col0 / kHeadGroup) * A.ld_stats + row] = make_float2(most, sum);
      } else {
        const int row0 = row - lane;
        auto gradients = [&](const uint32_t (&v)[32], int c) {
          const HeadRow& t = now.terms;
          const int from = col0 + c, end = from + 32;
          float hard = 0.f;
          if (!SOFT && now.next < end) hard = pick32(v, now.next - from);
          const float main = t.a * (1.f + t.e);
          const float lse2 = t.lse * kLog2E;
          const Two to = two(to2, to2), less = two(-lse2, -lse2), by = two(main, main);
          float z[32];
#pragma unroll
          for (int g = 0; g < 32; g += 8) {
#pragma unroll
            for (int j = g; j < g + 8; j += 2) {
              const float2 x = both(fma(two(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), to, less));
              const float2 d = both(two(exp2_fast(x.x), exp2_fast(x.y)) * by);
              z[j] = d.x, z[j + 1] = d.y;
            }
            if (SOFT) {
              while (__any_sync(0xffffffffu, column < from + g + 8)) {
                if (column < from + g + 8) {
                  const int at = column - (from + g);
                  const float weight = -t.a * __int_as_float(entry.y);
#pragma unroll
                  for (int j = 0; j < 8; ++j)
                    if (j == at) z[g + j] += weight;
                  advance();
                }
              }
            }
          }
          if (!SOFT && __any_sync(0xffffffffu, now.next < end)) {
            if (now.next < end) {  // (1 + e)·p - 1 with p near 1: by p - 1, of z - lse rounded once
              set32(z, now.next - from, t.a * fmaf(1.f + t.e, expm1f(fmaf(hard, A.scale, -t.lse)), t.e));
              now.next = kNoTarget;
            }
          }
          __syncwarp();
          if (!t.live) {
#pragma unroll
            for (int j = 0; j < 32; ++j) z[j] = 0.f;
          }
#pragma unroll
          for (int j = 0; j < 32; j += 8)
            sts128(buf + piece_at(lane, j >> 3),
                   make_uint4(pack16(z[j], z[j + 1], BF16), pack16(z[j + 2], z[j + 3], BF16),
                              pack16(z[j + 4], z[j + 5], BF16), pack16(z[j + 6], z[j + 7], BF16)));
          __syncwarp();
          // (dz's rows are on 16-byte boundaries, and there are multiples of 64 of its columns.)
          if (row0 + 32 <= A.m) {
            store_fast(A.dz + static_cast<int64_t>(row0 + (lane >> 2)) * A.ld_dz + from + 8 * (lane & 3), A.ld_dz, lane, buf);
          } else {
            store_slow(A.dz, A.ld_dz, A.m, A.cols, row0, from, lane, buf);
          }
          __syncwarp();
        };
        uint32_t v[32];
        load(0, v);
        tmem_ld_wait();
        more = find(i, then);
        gradients(v, 0);
        if (cols > 32) load(32, v);
        tmem_ld_wait();
        release();
        if (cols > 32) gradients(v, 32);
      }
    }
    if (!ok) {
      dev->status = kStatusTimeout;
      dev->timeout_site = 33;
    }
  }
  tc_fence_before();
  cluster_sync_all();  // neither CTA leaves while the pair's MMAs or loads may touch it
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

// ---------------------------------------------------------------------------
// A token's listed rows, sorted by row of w and place, and where those of each group of 64
// rows of w begin: an epilogue's lane then reads its own two places, beside its neighbours'.
// (Found by search in every tile, 32 lanes reading 32 lists, the entries took more than the
// products: 350 µs for 4096 tokens × 50257×1024 with 64 entries, 250 without any.  Sorted for
// 32 tokens together and handed out by shuffles, short lists were as fast, long ones not.)
// With `rows` the entries' weights and the token's terms of the gradient.  One warp to a token.
// ---------------------------------------------------------------------------
constexpr int kListWarps = 16;  // (whose offsets of a group are a sector)

__device__ __forceinline__ float teacher_at(const HeadTargets& t, int64_t row, int i) {
  const int64_t at = row * t.ld_teacher + i;
  return t.teacher_type == OZ2_TYPE_F32 ? __ldg(static_cast<const float*>(t.teacher) + at)
                                        : load16(static_cast<const uint16_t*>(t.teacher) + at,
                                                 t.teacher_type == OZ2_TYPE_BF16);
}
// A logit's distance from the largest one, which is then divided: the type's lowest value over a
// temperature below 1 would be minus infinity, and a list of nothing else no softmax.
__device__ __forceinline__ float below(float v, float most, const HeadTargets& t) { return (v - most) / t.temperature; }
// The listed logits' maximum, and the sum of the exponentials of their distances from it.
__device__ __forceinline__ void teacher_sums(const HeadTargets& t, int64_t row, int lane, float* top, float* sum) {
  float m = kLowest, s = 0.f;
  for (int i = lane; i < t.top; i += 32)
    if (t.ids[row * t.ld + i] >= 0) m = fmaxf(m, teacher_at(t, row, i));
  m = warp_max(m);
  for (int i = lane; i < t.top; i += 32)
    if (t.ids[row * t.ld + i] >= 0) s += expf(below(teacher_at(t, row, i), m, t));
  *top = m;
  *sum = warp_add(s);
}

// Steps of 32 and less of a bitonic merge of `size`, 64 keys to a warp in registers (a lane
// has two of them next to each other); with `first`, of all sizes up to 64.
template <typename Key>
__device__ __forceinline__ void sort_64(Key* keys, int at, int size, bool first, int lane) {
  Key a = keys[at + 2 * lane], b = keys[at + 2 * lane + 1];
  for (int n = first ? 2 : size; n <= size; n <<= 1) {
    const bool up = ((at + 2 * lane) & n) == 0;
    for (int step = min(n >> 1, 32); step > 1; step >>= 1) {
      const int other = step >> 1;  // lanes away
      const bool low = (lane & other) == 0;
      const Key c = __shfl_xor_sync(0xffffffffu, a, other), d = __shfl_xor_sync(0xffffffffu, b, other);
      a = (a > c) == (low == up) ? c : a;
      b = (b > d) == (low == up) ? d : b;
    }
    if ((a > b) == up) {
      const Key c = a;
      a = b, b = c;
    }
  }
  keys[at + 2 * lane] = a, keys[at + 2 * lane + 1] = b;
}

// A key is the row of w and, in its low `bits` bits, the place: 32 bits of them where that is
// enough (its shuffles and comparisons are half).
template <typename Key>
__global__ void __launch_bounds__(32 * kListWarps)
    head_targets_kernel(int64_t m, int64_t n, HeadTargets t, int padded, int bits, int table, int64_t groups1,
                        int64_t ld_offsets, int2* entries, uint16_t* offsets, HeadRow* rows, HeadTerms terms) {
  // The warps' keys, then the teacher's logits, and `table` bytes on (0: it does not fit) the offsets.
  extern __shared__ __align__(16) unsigned long long list_smem[];
  constexpr Key kNone = ~Key(0), kBad = kNone - 1;   // not there; no row of w
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, top = t.top;
  __shared__ uint16_t offsets_s[2][32][kListWarps];
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kListWarps, row = row0 + warp;
  const bool there = row < m;
  Key* keys = reinterpret_cast<Key*>(list_smem) + warp * padded;
  float* logits = reinterpret_cast<float*>(reinterpret_cast<Key*>(list_smem) + kListWarps * padded) + warp * top;
  float g = 0.f, l = 0.f;
  if (rows && there) g = terms.dloss[terms.dloss_each ? row : 0], l = terms.lse[row];
  bool live = false, bad = false;
  float most = kLowest, sum = 0.f;
  for (int i = lane; i < padded; i += 32) {
    int64_t id = -1;
    if (i < top && there) {
      id = t.ids[row * t.ld + i];
      if (rows) {
        const float u = teacher_at(t, row, i);
        logits[i] = u;
        if (id >= 0) most = fmaxf(most, u);
      }
    }
    live = live || id >= 0;
    bad = bad || id >= n;
    keys[i] = id < 0 ? kNone : id >= n ? kBad : static_cast<Key>(id) << bits | static_cast<Key>(i);
  }
  if (rows) {
    live = __any_sync(0xffffffffu, live);
    bad = __any_sync(0xffffffffu, bad);
    most = warp_max(most);
    for (int i = lane; i < top; i += 32)
      if (keys[i] != kNone) sum += expf(logits[i] = below(logits[i], most, t));
    sum = warp_add(sum);
    if (lane == 0 && there) rows[row] = HeadRow{bad ? __int_as_float(0x7FC00000) : live ? g * terms.scale : 0.f, live ? l : 0.f, 0.f, live};
  }
  __syncwarp();
  for (int at = 0; at < padded; at += 64) sort_64(keys, at, 64, true, lane);
  __syncwarp();
  for (int size = 128; size <= padded; size <<= 1) {
    for (int step = size >> 1; step >= 64; step >>= 1) {
      for (int p = lane; p < padded / 2; p += 32) {
        const int i = 2 * p - (p & (step - 1)), j = i + step;
        const Key a = keys[i], b = keys[j];
        if ((a > b) == ((i & size) == 0)) keys[i] = b, keys[j] = a;
      }
      __syncwarp();
    }
    for (int at = 0; at < padded; at += 64) sort_64(keys, at, size, false, lane);
    __syncwarp();
  }
  for (int i = lane; i < top && there; i += 32) {
    const Key key = keys[i];
    int2 e = make_int2(kNoTarget, 0);
    if (key < kBad) {
      const int place = static_cast<int>(key & ((Key(1) << bits) - 1));
      e.x = static_cast<int>(key >> bits);
      e.y = rows ? __float_as_int(expf(logits[place]) / sum) : place;
    }
    entries[row * top + i] = e;
  }
  // The offsets, all of them in shared memory where they fit: between two entries' groups they are
  // the number of entries before.
  if (table) {
    uint16_t* mine = reinterpret_cast<uint16_t*>(reinterpret_cast<uint8_t*>(list_smem) + table) + warp;
    for (int i = lane; i <= top; i += 32) {
      if (i > 0 && keys[i - 1] >= kBad) continue;
      const int before = i > 0 ? static_cast<int>(static_cast<int64_t>(keys[i - 1] >> bits) / kHeadGroup) : -1;
      const int last = i < top && keys[i] < kBad ? static_cast<int>(static_cast<int64_t>(keys[i] >> bits) / kHeadGroup)
                                                 : static_cast<int>(groups1) - 1;
      for (int q = before + 1; q <= last; ++q) mine[q * kListWarps] = static_cast<uint16_t>(i);
    }
    __syncthreads();
    const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(list_smem) + table);
    for (int i = threadIdx.x; i < 2 * groups1; i += 32 * kListWarps)  // (a group's 16 tokens: 32 bytes)
      *reinterpret_cast<uint4*>(offsets + (i >> 1) * ld_offsets + row0 + 8 * (i & 1)) = from[i];
    return;
  }
  // The offsets, 32 groups at a time: the warp walks over its entries there once.  By way of
  // shared memory: a group's are beside each other.
  int turn = 0, next = 0;
  for (int64_t q0 = 0; q0 < groups1; q0 += 32, turn ^= 1) {
    int at = next;
    while (next < top) {
      const Key key = keys[next];
      if (key >= kBad) break;  // (as the offset of what is past the last group: of the ones that are rows of w)
      const int64_t group = static_cast<int64_t>(key >> bits) / kHeadGroup - q0;
      if (group >= 32) break;
      at += group < lane;
      ++next;
    }
    offsets_s[turn][lane][warp] = static_cast<uint16_t>(at);
    __syncthreads();  // (the other set is written again behind the next one)
    const int64_t to = q0 + threadIdx.x / kListWarps;
    if (to < groups1) offsets[to * ld_offsets + row0 + threadIdx.x % kListWarps] = offsets_s[turn][threadIdx.x / kListWarps][threadIdx.x % kListWarps];
  }
}

// ---------------------------------------------------------------------------
// lse and losses.  A block has 32 tokens, one a lane; its warps take the groups of
// columns in turn, eight loads at once, and their maxima and sums are joined in shared
// memory.  4096 tokens of 50257 rows, 26 MB, take 8 µs.
// ---------------------------------------------------------------------------
constexpr int kJoinWarps = 32, kJoinAhead = 8;

__global__ void __launch_bounds__(32 * kJoinWarps)
    head_join_kernel(int64_t m, int64_t n, HeadTargets t, const float2* __restrict__ stats, int64_t ld_stats, int groups,
                     int join_warps, float z_loss, float* __restrict__ loss, float* __restrict__ lse, float* picked) {
  __shared__ float2 parts[kJoinWarps][32];
  __shared__ float lse_s[32];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * 32, row = row0 + lane;
  float most = kLowest, sum = 0.f;
  auto join = [&](float2 p) {
    const float top = max_nan(most, p.x);
    sum = sum * exp2_fast(most - top) + p.y * exp2_fast(p.x - top);
    most = top;
  };
  if (row < m && warp < join_warps) {
    for (int g = warp; g < groups; g += kJoinAhead * join_warps) {
      float2 p[kJoinAhead];
#pragma unroll
      for (int i = 0; i < kJoinAhead; ++i)
        p[i] = g + i * join_warps < groups ? stats[(g + i * join_warps) * ld_stats + row] : make_float2(kLowest, 0.f);
      float2 all = p[0];
#pragma unroll
      for (int i = 1; i < kJoinAhead; ++i) all.x = max_nan(all.x, p[i].x);
      all.y = 0.f;
#pragma unroll
      for (int i = 0; i < kJoinAhead; ++i) all.y = fmaf(p[i].y, exp2_fast(p[i].x - all.x), all.y);
      join(all);
    }
  }
  parts[warp][lane] = make_float2(most, sum);
  __syncthreads();
  if (warp == 0) {
    for (int w = 1; w < join_warps; ++w) join(parts[w][lane]);
    const float l = most == INFINITY ? INFINITY : kLn2 * most + logf(sum);
    lse_s[lane] = l;
    if (row < m) {
      lse[row] = l;
      if (!t.soft) {
        const int64_t id = t.ids[row * t.ld];
        float p = id >= n ? __int_as_float(0x7FC00000) : 0.f;
        if (id >= 0 && id < n) {
          p = picked[row];
        } else {
          picked[row] = p;
        }
        loss[row] = id < 0 ? 0.f : l - p + (z_loss != 0.f ? z_loss * l * l : 0.f);
      }
    }
  }
  if (!t.soft) return;
  __syncthreads();
  for (int64_t mine = row0 + warp; mine < min(m, row0 + 32); mine += warps) {
    float top, all;
    teacher_sums(t, mine, lane, &top, &all);
    const float log_all = logf(all);
    float s = 0.f;
    bool live = false;
    for (int i = lane; i < t.top; i += 32) {
      const int64_t id = t.ids[mine * t.ld + i];
      float* p = picked + mine * t.top + i;
      float z = 0.f;
      if (id >= 0 && id < n) {
        z = *p;
      } else {
        *p = z = id >= n ? __int_as_float(0x7FC00000) : 0.f;
      }
      if (id >= 0) {
        live = true;
        const float log_q = below(teacher_at(t, mine, i), top, t) - log_all, weight = expf(log_q);
        if (weight != 0.f || id >= n) s = fmaf(weight, log_q - z, s);  // (a row that the teacher rules out weighs nothing)
      }
    }
    s = warp_add(s);
    live = __any_sync(0xffffffffu, live);
    if (lane == 0) loss[mine] = live ? s + lse_s[mine - row0] : 0.f;
  }
}

// ---------------------------------------------------------------------------
// Rows of x, zeros for the tokens that do not count: their gradient is zero times what
// they hold, which need not be a number.  Memory bounds it (4096×1024 4 µs).
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(256) live_rows_kernel(int64_t m, int64_t n, int64_t k, const uint16_t* __restrict__ x,
                                                        int64_t ldx, Ids ids, HeadTerms terms, float* __restrict__ largest,
                                                        uint16_t* __restrict__ dst, int64_t ld_dst) {
  __shared__ float most_s[8];
  pdl_trigger();
  pdl_wait();
  // 16-byte pieces, one grid's stride apart.
  const uint32_t per = static_cast<uint32_t>((k + 7) / 8);
  const uint32_t first = blockIdx.x * blockDim.x + threadIdx.x, stride = gridDim.x * blockDim.x;
  const uint32_t stride_rows = stride / per, stride_pieces = stride - stride_rows * per;
  const uint16_t* end = x + (m - 1) * ldx + k;
  float most = 0.f;
  int64_t r = first / per;
  uint32_t c = first - static_cast<uint32_t>(r) * per;
  while (r < m) {
    const bool live = terms.rows ? __ldg(&terms.rows[r].live) != 0 : ids[r] >= 0;
    if (largest && c == 0) most = fmaxf(most, head_size(head_row(terms, ids, n, r)));
    const uint16_t* p = x + r * ldx + 8 * c;
    *reinterpret_cast<uint4*>(dst + r * ld_dst + 8 * c) =
        live ? load16_any(p, x, end, static_cast<int>(min(int64_t(8), k - 8 * c))) : make_uint4(0, 0, 0, 0);
    r += stride_rows;
    c += stride_pieces;
    if (c >= per) c -= per, ++r;
  }
  if (!largest) return;
  most = warp_max(most);
  if ((threadIdx.x & 31) == 0) most_s[threadIdx.x >> 5] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 8; ++w) most = fmaxf(most, most_s[w]);
    largest[blockIdx.x] = most;
  }
}

// FP32 sums to the rows' type.
template <bool BF16>
__global__ void __launch_bounds__(256) round_rows_kernel(int64_t m, int64_t k, const float* __restrict__ src, int64_t ld_src,
                                                         const float* __restrict__ unscale, uint16_t* __restrict__ dst,
                                                         int64_t ld_dst, bool vec) {
  pdl_trigger();
  pdl_wait();
  const float f = unscale ? *unscale : 1.f;
  const int per = static_cast<int>((k + 7) / 8);
  for (int64_t r = blockIdx.x; r < m; r += gridDim.x)
    for (int c = threadIdx.x; c < per; c += 256) {
      const float4 *p = reinterpret_cast<const float4*>(src + r * ld_src + 8 * c), a = p[0], b = p[1];  // (rows of multiples of 8)
      const int n = static_cast<int>(min(int64_t(8), k - 8 * c));
      store16_any(dst + r * ld_dst + 8 * c,
                  make_uint4(pack16(a.x * f, a.y * f, BF16), pack16(a.z * f, a.w * f, BF16), pack16(b.x * f, b.y * f, BF16),
                             pack16(b.z * f, b.w * f, BF16)),
                  n, vec && n == 8);
    }
}

bool make_rows_map(CUtensorMap* map, const void* base, int64_t rows, int64_t depth, int64_t ld, int box_rows) {
  EncodeTiledFn enc = get_encode_fn();
  if (!enc) return false;
  cuuint64_t dims[2] = {static_cast<cuuint64_t>(depth), static_cast<cuuint64_t>(rows)};
  cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * 2};
  cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)}, estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int TYPE, bool GRAD, bool SOFT>
cudaError_t launch(const HeadArgs& a, Oz2Device* dev, cudaStream_t st) {
  auto kern = head_kernel<TYPE, GRAD, SOFT>;
  cudaError_t err = allow_smem(reinterpret_cast<const void*>(kern), kSmem);
  if (err != cudaSuccess) return err;
  const int64_t ntm = (a.m + kTile - 1) / kTile, ntn = (a.cols + kTile - 1) / kTile;
  if (ntm * ntn > 0x1FFFFFFF) return cudaErrorInvalidValue;
  const int64_t resident = resident_pairs(reinterpret_cast<const void*>(kern), kThreads, kSmem);
  HeadUnits u{static_cast<int>(ntm), static_cast<int>(ntn), static_cast<int>(ntm * ntn), 0,
              static_cast<int>((a.k + 63) / 64)};
  // A last round of few tiles: they are taken as halves, by twice as many pairs.
  const int last = static_cast<int>(u.units % resident);
  if (2 * last <= resident) {
    u.units -= last;
    u.half_units = 2 * last;
  }
  HeadMaps maps{};
  if (u.steps && (!make_rows_map(&maps.x, a.x, a.m, a.k, a.ldx, kRows) || !make_rows_map(&maps.w, a.w, a.cols, a.k, a.ldw, kRows) ||
                  !make_rows_map(&maps.w_half, a.w, a.cols, a.k, a.ldw, kRows / 2)))
    return cudaErrorInvalidValue;
  const int64_t pairs = std::min<int64_t>(u.units + u.half_units, resident);
  count_launch();
  return launch_dependent(kern, dim3(static_cast<unsigned>(2 * pairs)), dim3(kThreads), kSmem, st, maps, a, u, dev);
}

int padded_top(int top) {
  int p = 1;
  while (p < top) p *= 2;
  return p;
}

}  // namespace

HeadLists head_lists(int64_t m, int64_t n, int top) {
  return HeadLists{m * top, (n + kHeadGroup - 1) / kHeadGroup + 1, (m + 31) / 32 * 32};
}

cudaError_t launch_head_targets(int64_t m, int64_t n, const HeadTargets& t, int2* entries, uint16_t* offsets, HeadRow* rows,
                                const HeadTerms& terms, cudaStream_t st) {
  const HeadLists l = head_lists(m, n, t.top);
  const int padded = std::max(64, padded_top(t.top));
  int bits = 0;
  while ((t.top - 1) >> bits) ++bits;
  const bool narrow = n < (int64_t(1) << (32 - bits)) - 1;
  const size_t lists = (kListWarps * ((narrow ? 4 : 8) * padded + (rows ? sizeof(float) * t.top : 0)) + 15) / 16 * 16;
  const size_t table = sizeof(uint16_t) * kListWarps * l.groups1;
  const bool fits = lists + table <= 200 * 1024;
  const size_t smem = lists + (fits ? table : 0);
  auto kern = narrow ? head_targets_kernel<uint32_t> : head_targets_kernel<unsigned long long>;
  const cudaError_t err = allow_smem(reinterpret_cast<const void*>(kern), smem);
  if (err != cudaSuccess) return err;
  count_launch();
  return launch_dependent(kern, dim3(static_cast<unsigned>((m + kListWarps - 1) / kListWarps)), dim3(32 * kListWarps), smem, st, m, n, t,
                          padded, bits, fits ? static_cast<int>(lists) : 0, l.groups1, l.ld_offsets, entries, offsets, rows, terms);
}

int live_rows_maxima(int64_t m, int64_t k) {
  return static_cast<int>(std::min<int64_t>((m * ((k + 7) / 8) + 255) / 256, 8 * static_cast<int64_t>(num_sms())));
}

cudaError_t launch_live_rows(int64_t m, int64_t n, int64_t k, const void* x, int64_t ldx, Ids ids, const HeadTerms& terms,
                             float* largest, void* dst, int64_t ld_dst, cudaStream_t st) {
  count_launch();
  return launch_dependent(live_rows_kernel, dim3(static_cast<unsigned>(live_rows_maxima(m, k))), dim3(256), 0, st, m, n, k,
                          static_cast<const uint16_t*>(x), ldx, ids, terms, largest, static_cast<uint16_t*>(dst), ld_dst);
}

cudaError_t launch_head_forward(const HeadArgs& a, int type, Oz2Device* dev, cudaStream_t st) {
  const bool soft = a.soft != 0;
  if (type == OZ2_TYPE_BF16) return soft ? launch<OZ2_TYPE_BF16, false, true>(a, dev, st) : launch<OZ2_TYPE_BF16, false, false>(a, dev, st);
  return soft ? launch<OZ2_TYPE_F16, false, true>(a, dev, st) : launch<OZ2_TYPE_F16, false, false>(a, dev, st);
}

cudaError_t launch_head_grad(const HeadArgs& a, int type, Oz2Device* dev, cudaStream_t st) {
  const bool soft = a.soft != 0;
  if (type == OZ2_TYPE_BF16) return soft ? launch<OZ2_TYPE_BF16, true, true>(a, dev, st) : launch<OZ2_TYPE_BF16, true, false>(a, dev, st);
  return soft ? launch<OZ2_TYPE_F16, true, true>(a, dev, st) : launch<OZ2_TYPE_F16, true, false>(a, dev, st);
}

cudaError_t launch_head_join(int64_t m, int64_t n, const HeadTargets& t, const float2* stats, int64_t ld_stats,
                             float z_loss, float* loss, float* lse, float* picked, cudaStream_t st) {
  // As many warps as have eight groups each; listed rows, which are a warp's each, want all.
  const int groups = static_cast<int>((n + kHeadGroup - 1) / kHeadGroup);
  const int join_warps = std::min(kJoinWarps, (groups + kJoinAhead - 1) / kJoinAhead);
  const int warps = t.soft ? kJoinWarps : join_warps;
  count_launch();
  return launch_dependent(head_join_kernel, dim3(static_cast<unsigned>((m + 31) / 32)), dim3(32 * warps), 0, st, m, n, t,
                          stats, ld_stats, groups, join_warps, z_loss, loss, lse, picked);
}

cudaError_t launch_round_rows(int64_t m, int64_t k, int type, const float* src, int64_t ld_src, const float* unscale,
                              void* dst, int64_t ld_dst, cudaStream_t st) {
  count_launch();
  return launch_dependent(type == OZ2_TYPE_BF16 ? round_rows_kernel<true> : round_rows_kernel<false>,
                          dim3(static_cast<unsigned>(std::min<int64_t>(m, 8 * num_sms()))), dim3(256), 0, st, m, k, src, ld_src,
                          unscale, static_cast<uint16_t*>(dst), ld_dst, rows_on16(dst, ld_dst, 2));
}

}  // namespace oz2
