// The products of a linear layer and of its gradient: D = epilogue(P·Qᵀ) on
// tcgen05 (16-bit types by kind::f16, E4M3 by kind::f8f6f4), FP32 sums.
//
//   forward   Y = act(X·Wᵀ·scales + b) + R   P = X, Q = W, both K-major
//   gradient  dX = dZ·W                      P = dZ K-major, Q = W MN-major
//             dW = dZᵀ·X                     both MN-major
//
// An operand tile is 128 rows × 128 bytes of depth in K-major storage (rows of
// 128 bytes), or 64 depth rows × two 64-element row blocks in MN-major storage;
// both land in shared memory with the 128-byte swizzle, and the descriptor and
// the instruction's transpose bits tell them apart.
#include <algorithm>
#include <type_traits>

#include "lin_common.cuh"

namespace oz2 {
namespace {

constexpr int kLinEpiWarps = 16;
constexpr int kLinThreads = 64 + 32 * kLinEpiWarps;  // TMA warp, MMA warp, epilogue warps
constexpr int kLinStages = 5;
constexpr int kLinTile = 256;         // rows and columns of a CTA pair's tile
constexpr int kLinStage = 2 * kTileBytes;
constexpr int kLinCols = kLinTile / (kLinEpiWarps / 4);  // columns of an epilogue warp
constexpr int kChunk = 32;            // of which it takes this many at a time
constexpr int kStageBytes = 32 * 2 * kChunk;             // an epilogue warp's 32 rows × 32 columns of 16 bits
constexpr int kLinSmem = 1024 + kLinStages * kLinStage + kLinEpiWarps * (kStageBytes + 2 * 4 * kLinCols) + 256;
constexpr int kMaxPairSplit = 16;     // parts of a tile's depth on pairs
constexpr int kPartFloats = kLinTile * kLinTile;         // a part of a tile's sums in the workspace

struct LinUnits {                     // one product of a launch
  int64_t rows, cols;
  int ntm, ntn, units;
  int steps;                          // of 128 bytes of depth
  int split;                          // on pairs: parts that the depth of each tile is cut into
  int halves;                         // on pairs: last tiles that are taken as two halves
  uint32_t p_mn, q_mn;
  LinEpilogue ep;
};
struct LinLaunch {
  int count;
  int units;                          // whole tiles (of the products with split = 1)
  int half_units;                     // on pairs: halves of tiles, after those, all of the last product
  // On pairs: the parts of the tiles of products with split > 1, one to a pair from
  // the first on; the pairs without one take whole tiles in `ahead` rounds of their
  // own meanwhile.
  int parts, ahead;
  float* sums;                        // the parts' sums: kPartFloats each
  int* arrived;                       // parts done, for each of their tiles, CTA and epilogue warp
  LinUnits u[kMaxProducts];
};
struct LinMaps {
  CUtensorMap p[kMaxProducts], q[kMaxProducts];
  CUtensorMap q_half;                 // the last product's Q in boxes of half the rows (K-major)
};

// Instruction descriptor of kind::f16 with FP32 sums: D = F32 (bits 4-5 = 1), A
// and B BF16 (1) or F16 (0) in bits 7-9 and 10-12, MN-major A and B in bits 15
// and 16, N >> 3 in 17-22, M >> 4 in 24-28.
constexpr uint32_t idesc_16(int M, int N, bool bf16, bool a_mn, bool b_mn) {
  return (1u << 4) | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
         (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// The instruction descriptor and the operands' descriptors of the MMAs of one
// operand type and storage, constants but for the tile's address.
template <int TYPE, bool A_MN, bool B_MN, int M, int N>
struct MmaShape {
  static constexpr uint32_t idesc =
      TYPE == OZ2_TYPE_E4M3 ? idesc_f8_f32(M, N) : idesc_16(M, N, TYPE == OZ2_TYPE_BF16, A_MN, B_MN);
  // 32 bytes of depth an instruction: 32 bytes along a K-major row, 16 depth rows
  // of 128 bytes in MN-major storage (in the descriptors' units of 16 bytes).
  static constexpr uint32_t a_next = A_MN ? 128 : 2, b_next = B_MN ? 128 : 2;
};

// The descriptor of a tile in MN-major storage: 64-element (128-byte) row
// blocks kTileBytes/2 apart (leading byte offset), groups of 8 depth rows 1024
// bytes apart (stride byte offset), 128-byte swizzle.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t saddr) {
  return (smem_desc_sw128(saddr) & ~(0x3FFFull << 16)) | (static_cast<uint64_t>(kTileBytes / 2 >> 4) << 16);
}

// One lane of a whole warp, known to the compiler as one: its TMA and tensor-core
// instructions take their operands from uniform registers as they are.  Under
// `lane == 0` each is issued in a loop over the lanes that might be there (a
// producer's step of two loads took 660 cycles in place of 300).
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred P;\n elect.sync _|P, 0xffffffff;\n selp.u32 %0, 1, 0, P;\n}\n" : "=r"(p));
  return p != 0;
}

template <bool MN>
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr) {
  return MN ? smem_desc_mn(saddr) : smem_desc_sw128(saddr);
}

template <bool F8>
__device__ __forceinline__ void mma_pair(uint32_t me, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                         uint32_t accumulate) {
  if (F8) {
    mma_f8_pair(me, d_tmem, a_desc, b_desc, idesc, accumulate);
  } else {
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
        " @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(me)
        : "memory");
  }
}

// Tile (tm, tn) of unit u: bands of 8 tile rows, so that the tiles in flight
// share operand rows in L2.
__device__ __forceinline__ void unit_tile(const LinUnits& x, int u, int* tm, int* tn) {
  const int per = 8 * x.ntn, band = u / per, in = u - band * per;
  const int h = min(8, x.ntm - band * 8);
  *tn = in / h;
  *tm = band * 8 + (in - *tn * h);
}

// --- an epilogue warp's 32 rows × 64 bytes in shared memory ---------------------
// 16-byte piece c of row r at r·64 + (c ^ (r/2 & 3))·16: eight threads' own rows and
// two rows' eight pieces are both free of bank conflicts.
__device__ __forceinline__ uint32_t piece_at(int row, int c) { return row * 64 + ((c ^ (row >> 1 & 3)) << 4); }

__device__ __forceinline__ uint4 lds128(const uint8_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void sts128(uint8_t* p, uint4 v) { *reinterpret_cast<uint4*>(p) = v; }

__device__ __forceinline__ bool vec_ok(const void* p, int64_t ld, int bytes) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * bytes)) & 15) == 0;
}

// A warp's 32 rows × 32 columns of 16 bits between global and shared memory: by 16
// bytes a lane, eight rows at a time, where the whole of them lies inside the matrix
// and on 16-byte boundaries (`from`, `to`: this lane's place in the first eight rows),
// else by single values, and what lies past the matrix is not touched.  The fetch is
// in two halves, so that all its loads are on their way before the first is waited for
// (value by value in turn, 4096×4095 with a residual at a depth of 1024 took 95 µs; so 39).
struct Fetched {
  uint32_t v[16];
};
__device__ __forceinline__ void fetch_begin(const uint16_t* from, int64_t ld, Fetched& f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 v = *reinterpret_cast<const uint4*>(from + 8 * i * ld);
    f.v[4 * i] = v.x, f.v[4 * i + 1] = v.y, f.v[4 * i + 2] = v.z, f.v[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ void fetch_end(const Fetched& f, int lane, uint8_t* buf) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    sts128(buf + piece_at(8 * i + (lane >> 2), lane & 3),
           make_uint4(f.v[4 * i], f.v[4 * i + 1], f.v[4 * i + 2], f.v[4 * i + 3]));
}
__device__ __forceinline__ void store_fast(uint16_t* to, int64_t ld, int lane, const uint8_t* buf) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<uint4*>(to + 8 * i * ld) = lds128(buf + piece_at(8 * i + (lane >> 2), lane & 3));
}
__device__ __forceinline__ uint8_t* value_at(uint8_t* buf, int row, int col) {
  return buf + piece_at(row, col >> 3) + 2 * (col & 7);
}
// Two columns a lane, two rows at a time.
__device__ __forceinline__ void fetch_begin_slow(const void* src, int64_t ld, int64_t rows, int64_t cols, int64_t row0,
                                                 int64_t col0, int lane, Fetched& f) {
  const int64_t row = row0 + (lane >> 4), col = col0 + 2 * (lane & 15);
  const uint16_t* s = static_cast<const uint16_t*>(src) + row * ld + col;
  const int n = static_cast<int>(min(int64_t(32), rows - row));  // of these rows, 2·i < n are there
  const bool one = col < cols, two = col + 1 < cols;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const bool there = 2 * i < n;
    const uint32_t a = there && one ? s[2 * i * ld] : 0, b = there && two ? s[2 * i * ld + 1] : 0;
    f.v[i] = a | b << 16;
  }
}
__device__ __forceinline__ void fetch_end_slow(const Fetched& f, int lane, uint8_t* buf) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    *reinterpret_cast<uint32_t*>(value_at(buf, 2 * i + (lane >> 4), 2 * (lane & 15))) = f.v[i];
}
__device__ __noinline__ void store_slow(void* dst, int64_t ld, int64_t rows, int64_t cols, int64_t row0, int64_t col0,
                                        int lane, uint8_t* buf) {
  uint16_t* d = static_cast<uint16_t*>(dst) + row0 * ld + col0 + lane;
  if (col0 + lane >= cols) return;
#pragma unroll 8
  for (int r = 0; r < 32; ++r)
    if (row0 + r < rows) d[r * ld] = *reinterpret_cast<const uint16_t*>(value_at(buf, r, lane));
}
// 16 columns of FP32, stored or added to.
__device__ __noinline__ void store32(const LinUnits& x, void* dst, int64_t ld, int64_t row0, int64_t col0, int lane,
                                        const uint8_t* buf, bool add) {
  float* d = static_cast<float*>(dst);
  const int c = lane & 15;
  if (col0 + c >= x.cols) return;
  for (int r = lane >> 4; r < 32 && row0 + r < x.rows; r += 2) {
    float* at = d + (row0 + r) * ld + col0 + c;
    const float v = *reinterpret_cast<const float*>(buf + piece_at(r, c >> 2) + 4 * (c & 3));
    *at = add ? *at + v : v;
  }
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr));
}

// 32 sums of one row (columns c.. of the warp's) with their scales and biases.
__device__ __forceinline__ void scale32(const float* scale_s, float row_scale, int c, float (&z)[32]) {
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    const float4 s = *reinterpret_cast<const float4*>(scale_s + c + j);
    z[j] *= row_scale * s.x;
    z[j + 1] *= row_scale * s.y;
    z[j + 2] *= row_scale * s.z;
    z[j + 3] *= row_scale * s.w;
  }
}
__device__ __forceinline__ void bias32(const float* bias_s, int c, float (&z)[32]) {
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    const float4 b = *reinterpret_cast<const float4*>(bias_s + c + j);
    z[j] += b.x;
    z[j + 1] += b.y;
    z[j + 2] += b.z;
    z[j + 3] += b.w;
  }
}

// act(z) + r for 32 columns, into the warp's buffer (which holds r there).
template <int ACT>
__device__ __forceinline__ void finish32(const float (&z)[32], bool add, bool bf16, uint8_t* buf, int lane) {
#pragma unroll
  for (int j = 0; j < 32; j += 8) {
    uint8_t* at = buf + piece_at(lane, j >> 3);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = activate<ACT>(z[j + e]);
    if (add) {
      const uint4 r = lds128(at);
      const uint32_t rw[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = unpack16(rw[e], bf16);
        y[2 * e] += f.x;
        y[2 * e + 1] += f.y;
      }
    }
    sts128(at, make_uint4(pack16(y[0], y[1], bf16), pack16(y[2], y[3], bf16), pack16(y[4], y[5], bf16),
                          pack16(y[6], y[7], bf16)));
  }
}

__device__ __forceinline__ int count_part(int* at) {
  int before;
  asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(at) : "memory");
  return before;
}

// --- the work of a CTA pair --------------------------------------------------------
// First a part of a tile whose depth is split, then whole tiles.  The parts come
// first so that the last of a tile's parts, which joins them, is not at the launch's
// end, and all at once so that tiles that share rows of an operand read the same
// depth at the same time.
struct Piece {
  int i;               // product
  int tm, tn;          // tile
  int col, width;      // its first column of the result and how many (256, or 128 of a half)
  int t0, t1;          // steps of its depth
  int parts;           // of the tile (1: whole)
  int slot, first_slot, stride;  // of its sums: this part's, the first part's, from part to part
  int tile;            // number among the tiles whose depth is split
};
struct PairWork {
  const LinLaunch& L;
  int pair, npairs, round;
  __device__ PairWork(const LinLaunch& launch, int p, int np) : L(launch), pair(p), npairs(np), round(p < launch.parts ? -1 : 0) {}
  __device__ bool next(Piece& p) {
    p.width = kLinTile;
    if (round < 0) {
      round = L.ahead;
      const int first = L.u[0].split > 1 ? L.u[0].units * L.u[0].split : 0;
      p.i = pair >= first ? 1 : 0;
      const LinUnits& x = L.u[p.i];
      const int v = p.i ? pair - first : pair, part = v / x.units, tile = v - part * x.units;
      const int per = (x.steps + x.split - 1) / x.split;
      unit_tile(x, tile, &p.tm, &p.tn);
      p.col = p.tn * kLinTile;
      p.t0 = min(x.steps, part * per);
      p.t1 = min(x.steps, p.t0 + per);
      p.parts = x.split;
      p.slot = pair;
      p.first_slot = pair - part * x.units;
      p.stride = x.units;
      p.tile = tile + (p.i && first ? L.u[0].units : 0);
      return true;
    }
    const int others = npairs - L.parts;
    int u = round < L.ahead ? round * others + pair - L.parts : L.ahead * others + (round - L.ahead) * npairs + pair;
    ++round;
    if (u >= L.units + L.half_units) return false;
    const int first = L.u[0].split > 1 ? 0 : L.u[0].units - L.u[0].halves, half = u - L.units;
    p.i = half >= 0 ? L.count - 1 : u >= first ? 1 : 0;
    const LinUnits& x = L.u[p.i];
    unit_tile(x, half >= 0 ? x.units - x.halves + half / 2 : p.i ? u - first : u, &p.tm, &p.tn);
    p.col = p.tn * kLinTile;
    if (half >= 0) {
      p.width = kLinTile / 2;
      p.col += (half & 1) * p.width;
    }
    p.t0 = 0;
    p.t1 = x.steps;
    p.parts = 1;
    return true;
  }
};

// ---------------------------------------------------------------------------
// Tiles of 256 × 256 on CTA pairs (cta_group::2: each CTA stages 128 rows of P
// and 128 of Q), persistent, two accumulators in tensor memory so that a
// tile's epilogue runs beside the next tile's products.
//
// A product of few tiles and a long depth (a weight's gradient over many tokens)
// has its tiles' depth split over pairs.  A part's sums go to the workspace in FP32;
// each epilogue warp counts its own 32 × 64 corner in, and the warp that comes last
// adds up the tile's parts, in their order whoever is last, and finishes them.
//
// What bounds it: the tensor pipes and, as closely, what an SM takes in.  A step of
// 64 elements of depth is 512 cycles of MMAs and 32 KB a CTA at 64 bytes a cycle, 247
// ns at 2.07 GHz; one pair alone takes 262, all 76 together 282 (and the power cap the
// rest).  So a narrower tile would only load more for its MMAs, and five stages are
// wanted (four: 339 ns).  4864×4096×4096 bf16, four even rounds of tiles, takes 86 µs
// (1.89 PFLOP/s); 4096³ 78; 16384²×4096 1.12 ms; E4M3 of normal values
// 8192³ 298 µs (3.7 PFLOP/s).  A last round that is at most half full takes its tiles
// as halves on twice as many pairs (a half's step, its loads, 390 cycles of 535: 4096³
// 80 to 76 µs, the gradient of 2504×3008×2048 44 to 39).  Sharing out that round's steps
// of depth evenly instead (parts of every tile's) won 1% at 4096³ and lost elsewhere: a
// part's sums are 256 KB to write and to read.  Split depths: 65536 tokens' dX and dW at
// 1024×1024 take 160 µs, 344 with dW's 16 tiles whole.
//
// The epilogue is 16 warps, 32 rows × 64 columns each, in 32-column chunks through
// two KB of shared memory that turn a thread's row into 64-byte pieces of eight rows.
// At a depth of 64, where it is all there is, a round takes 3.5 µs, 10 MB at a fill's
// rate (relu adds 0.4, silu 1.1, gelu_tanh 1.3, gelu 2.1, a residual 2.1, which is
// memory's): it hides behind the next tile's products from a depth of about 1024 on.
// ---------------------------------------------------------------------------
template <int TYPE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLinThreads, 1)
    linear_pair_kernel(const __grid_constant__ LinMaps maps, const __grid_constant__ LinLaunch L, Oz2Device* dev) {
  constexpr bool F8 = TYPE == OZ2_TYPE_E4M3;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* epi = smem + kLinStages * kLinStage;
  uint64_t* bars = reinterpret_cast<uint64_t*>(epi + kLinEpiWarps * (kStageBytes + 2 * 4 * kLinCols));
  // bars: full[S], empty[S], acc_full[2], acc_empty[2], drain
  __shared__ uint32_t tmem_base_s;

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + kLinStages);
  const uint32_t acc_full = smem_u32(bars + 2 * kLinStages), acc_empty = smem_u32(bars + 2 * kLinStages + 2);
  const uint32_t drain_bar = smem_u32(bars + 2 * kLinStages + 4);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kLinStages; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full + 8 * a, 1);
      mbar_init(acc_empty + 8 * a, 2 * kLinEpiWarps);
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
  pdl_wait();  // the operands are written; the set-up above overlaps that kernel's tail

  PairWork work(L, pair, npairs);
  Piece pc;

  if (warp == 0) {
    // ---------------- TMA producer (both CTAs) ----------------
    if (elect_one()) {
      const uint32_t full_leader0 = mapa_shared(full0, 0), ring0 = smem_u32(smem);
      uint32_t it = 0, s = 0, ph = 1;
      while (ok && work.next(pc)) {
        const LinUnits& x = L.u[pc.i];
        // In registers: what is read from the launch's parameters is read again at
        // every step (and each TMA instruction's operands wait for it).
        const int prow = pc.tm * kLinTile + rank * kRows;
        const int qrow = pc.col + rank * (pc.width / 2);
        const int t1 = pc.t1;
        const bool p_mn = x.p_mn != 0, q_mn = x.q_mn != 0, half = pc.width != kLinTile;
        const CUtensorMap *mp = &maps.p[pc.i], *mq = half ? &maps.q_half : &maps.q[pc.i];
        const uint32_t bytes = 2u * (kTileBytes + (half ? kTileBytes / 2 : kTileBytes));
        for (int t = pc.t0, d = t * (F8 ? 128 : 64); t < t1; ++t, d += F8 ? 128 : 64) {
          if (!mbar_wait_bounded(empty0 + 8 * s, ph, kWaitLimit)) {
            ok = false;
            break;
          }
          const uint32_t sa = ring0 + s * kLinStage, sb = sa + kTileBytes, bar = full_leader0 + 8 * s;
          if (leader) mbar_arrive_expect_tx(full0 + 8 * s, bytes);
          if (!p_mn) {
            tma_load_2d_pair(sa, mp, bar, d, prow);
          } else {
            tma_load_2d_pair(sa, mp, bar, prow, d);
            tma_load_2d_pair(sa + kTileBytes / 2, mp, bar, prow + 64, d);
          }
          if (!q_mn) {
            tma_load_2d_pair(sb, mq, bar, d, qrow);
          } else {
            tma_load_2d_pair(sb, mq, bar, qrow, d);
            if (!half) tma_load_2d_pair(sb + kTileBytes / 2, mq, bar, qrow + 64, d);
          }
          ++it;
          if (++s == kLinStages) {
            s = 0;
            ph ^= 1;
          }
        }
      }
      if (!ok) {
        dev->status = kStatusTimeout;
        dev->timeout_site = 21;
      }
      pdl_trigger();  // the next kernel's start overlaps the last tiles
      if (leader)  // the leader's stage barriers also count the peer's bytes
        for (uint32_t j = (it > kLinStages ? it - kLinStages : 0); j < it; ++j)
          mbar_wait_bounded(full0 + 8 * (j % kLinStages), (j / kLinStages) & 1, kWaitLimit);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------- MMA issuer (leader CTA) ----------------
    if (leader) {  // the whole warp; lane 0 issues
      const uint32_t me = lane == 0;
      const uint32_t base = smem_u32(smem);
      uint32_t s = 0, ph = 0, acc = 0, accph = 1;
      auto multiply = [&](auto shape, uint64_t pd, uint64_t qd, int steps, uint32_t d) {
        for (int t = 0; t < steps && ok; ++t) {
          if (!(ok = mbar_wait_warp(full0 + 8 * s, ph, kWaitLimit))) break;
          tc_fence_after();
          const uint64_t a = pd + s * (kLinStage >> 4), b = qd + s * (kLinStage >> 4);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_pair<F8>(me, d, a + kk * shape.a_next, b + kk * shape.b_next, shape.idesc, (t | kk) ? 1u : 0u);
          mma_commit_pair_mc(me, empty0 + 8 * s, 0x3);
          if (++s == kLinStages) {
            s = 0;
            ph ^= 1;
          }
        }
      };
      while (ok && work.next(pc)) {
        const LinUnits& x = L.u[pc.i];
        if (pc.t0 == pc.t1) continue;
        ok = mbar_wait_warp(acc_empty + 8 * acc, accph, kWaitLimit);
        tc_fence_after();
        const int steps = pc.t1 - pc.t0;
        auto by_width = [&](auto p_mn, auto q_mn) {
          constexpr bool PM = decltype(p_mn)::value, QM = decltype(q_mn)::value;
          const uint64_t pd = operand_desc<PM>(base), qd = operand_desc<QM>(base + kTileBytes);
          if (pc.width == kLinTile) {
            multiply(MmaShape<TYPE, PM, QM, kLinTile, kLinTile>{}, pd, qd, steps, tmem + acc * kLinTile);
          } else {
            multiply(MmaShape<TYPE, PM, QM, kLinTile, kLinTile / 2>{}, pd, qd, steps, tmem + acc * kLinTile);
          }
        };
        if (F8 || !x.q_mn) {
          by_width(std::false_type{}, std::false_type{});
        } else if (!x.p_mn) {
          by_width(std::false_type{}, std::true_type{});
        } else {
          by_width(std::true_type{}, std::true_type{});
        }
        if (!ok) break;
        mma_commit_pair_mc(me, acc_full + 8 * acc, 0x3);
        acc ^= 1;
        if (acc == 0) accph ^= 1;
      }
      if (!ok && me) {
        dev->status = kStatusTimeout;
        dev->timeout_site = 22;
      }
      mma_commit_pair(me, drain_bar);
      mbar_wait_bounded(drain_bar, 0, kWaitLimit);
    }
    __syncwarp();
  } else {
    // ---------------- epilogue (warps 2..17, both CTAs) ----------------
    const int ew = warp - 2;
    const int q = warp & 3, h = ew >> 2;  // TMEM lane quarter, column quarter
    uint8_t* buf = epi + ew * kStageBytes;
    float* bias_s = reinterpret_cast<float*>(epi + kLinEpiWarps * kStageBytes) + ew * 2 * kLinCols;
    float* scale_s = bias_s + kLinCols;
    const uint32_t acc_empty_leader = mapa_shared(acc_empty, 0);
    uint32_t acc = 0, accph = 0;
    while (work.next(pc)) {
      const LinUnits& x = L.u[pc.i];
      const LinEpilogue& ep = x.ep;
      const int cols = pc.width / 4;  // of this warp
      const int64_t row0 = pc.tm * kLinTile + rank * kRows + 32 * q, col0 = pc.col + cols * h;
      const bool bf16 = TYPE == OZ2_TYPE_BF16 || (F8 && ep.out_type == OZ2_TYPE_BF16);
      const bool scales = F8 && ep.row_scale != nullptr, add = ep.add != nullptr;
      const bool sums = pc.t1 > pc.t0;
      // Where this warp's corner is inside the matrix and on 16-byte boundaries.
      const bool inside = row0 + 32 <= x.rows && col0 + cols <= x.cols;
      const bool fast_add = inside && vec_ok(ep.add, ep.ld_add, 2), fast_pre = inside && vec_ok(ep.pre, ep.ld_pre, 2),
                 fast_out = inside && vec_ok(ep.out, ep.ld_out, 2);
      const int64_t lane_row = row0 + (lane >> 2), lane_col = col0 + 8 * (lane & 3);
      __syncwarp();
      if (ep.bias) {
        for (int c = lane; c < cols; c += 32) {
          const int64_t j = col0 + c;
          float b = 0.f;
          if (j < x.cols)
            b = ep.bias_type == OZ2_TYPE_F32 ? __ldg(static_cast<const float*>(ep.bias) + j)
                                             : load16(static_cast<const uint16_t*>(ep.bias) + j, bf16);
          bias_s[c] = b;
        }
      }
      float row_scale = 0.f;
      if (scales) {
        for (int c = lane; c < cols; c += 32) scale_s[c] = col0 + c < x.cols ? __ldg(ep.col_scale + col0 + c) : 0.f;
        if (row0 + lane < x.rows) row_scale = __ldg(ep.row_scale + row0 + lane);
      }
      Fetched r;
      const uint16_t* from = static_cast<const uint16_t*>(ep.add) + lane_row * ep.ld_add + lane_col;
      if (fast_add && add) fetch_begin(from, ep.ld_add, r);
      if (add && !fast_add) fetch_begin_slow(ep.add, ep.ld_add, x.rows, x.cols, row0, col0, lane, r);
      __syncwarp();
      if (sums) {
        if (!mbar_wait_bounded(acc_full + 8 * acc, accph, kWaitLimit)) ok = false;
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        tc_fence_after();
      }
      const uint32_t at = tmem + (static_cast<uint32_t>(32 * q) << 16) + acc * kLinTile + cols * h;
      auto release = [&] {
        if (sums) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote_relaxed(acc_empty_leader + 8 * acc);
          acc ^= 1;
          if (acc == 0) accph ^= 1;
        }
      };
      // This warp's corner of a slot: chunks of 32 columns, four at a time, 32 rows.
      const int corner = ((rank * kLinEpiWarps + ew) * (kLinCols / 4)) * 128 + 4 * lane;
      if (pc.parts > 1) {
        float* to = L.sums + static_cast<int64_t>(pc.slot) * kPartFloats + corner;
#pragma unroll 1
        for (int c = 0; c < kLinCols; c += kChunk) {
          uint32_t v[32];
          if (sums) {
            tmem_ld32(at + c, v);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0u;
          }
#pragma unroll
          for (int j = 0; j < 32; j += 4)
            __stcg(reinterpret_cast<uint4*>(to + (c + j) * 32), make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]));
        }
        release();
        // The warp's stores come before its lane's count (which releases them, and
        // takes over those that it counts after), the last warp's loads after it.
        __syncwarp();
        int before = 0;
        if (lane == 0) before = count_part(L.arrived + (pc.tile * 2 + rank) * kLinEpiWarps + ew);
        if (__shfl_sync(0xffffffffu, before, 0) != pc.parts - 1) continue;
        __syncwarp();
      }
#pragma unroll 1
      for (int c = 0; c < cols; c += kChunk) {
        float z[32];
        if (pc.parts > 1) {
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const float4 a = __ldcg(reinterpret_cast<const float4*>(L.sums + static_cast<int64_t>(pc.first_slot) * kPartFloats +
                                                                    corner + (c + j) * 32));
            z[j] = a.x, z[j + 1] = a.y, z[j + 2] = a.z, z[j + 3] = a.w;
          }
#pragma unroll 2
          for (int p = 1; p < pc.parts; ++p) {
            const float* part = L.sums + static_cast<int64_t>(pc.first_slot + p * pc.stride) * kPartFloats + corner;
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const float4 a = __ldcg(reinterpret_cast<const float4*>(part + (c + j) * 32));
              z[j] += a.x, z[j + 1] += a.y, z[j + 2] += a.z, z[j + 3] += a.w;
            }
          }
        } else if (sums) {
          uint32_t v[32];
          tmem_ld32(at + c, v);
          tmem_ld_wait();
          if (c == cols - kChunk) release();
#pragma unroll
          for (int j = 0; j < 32; ++j) z[j] = __uint_as_float(v[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) z[j] = 0.f;
        }
        if (ep.out_type == OZ2_TYPE_F32) {
#pragma unroll
          for (int g = 0; g < 32; g += 16) {
#pragma unroll
            for (int j = 0; j < 16; j += 4)
              sts128(buf + piece_at(lane, j >> 2), make_uint4(__float_as_uint(z[g + j]), __float_as_uint(z[g + j + 1]),
                                                              __float_as_uint(z[g + j + 2]), __float_as_uint(z[g + j + 3])));
            __syncwarp();
            store32(x, ep.out, ep.ld_out, row0, col0 + c + g, lane, buf, ep.accumulate != 0);
            __syncwarp();
          }
          continue;
        }
        if (scales) scale32(scale_s, row_scale, c, z);
        if (ep.bias) bias32(bias_s, c, z);
        if (ep.pre) {
          finish32<OZ2_ACT_NONE>(z, false, bf16, buf, lane);
          __syncwarp();
          if (fast_pre) {
            store_fast(static_cast<uint16_t*>(ep.pre) + lane_row * ep.ld_pre + lane_col + c, ep.ld_pre, lane, buf);
          } else {
            store_slow(ep.pre, ep.ld_pre, x.rows, x.cols, row0, col0 + c, lane, buf);
          }
          __syncwarp();
        }
        if (add) {
          if (fast_add) {
            fetch_end(r, lane, buf);
            if (c + kChunk < cols) fetch_begin(from + c + kChunk, ep.ld_add, r);
          } else {
            fetch_end_slow(r, lane, buf);
          }
          __syncwarp();
        }
        switch (ep.act) {
          case OZ2_ACT_RELU: finish32<OZ2_ACT_RELU>(z, add, bf16, buf, lane); break;
          case OZ2_ACT_GELU: finish32<OZ2_ACT_GELU>(z, add, bf16, buf, lane); break;
          case OZ2_ACT_GELU_TANH: finish32<OZ2_ACT_GELU_TANH>(z, add, bf16, buf, lane); break;
          case OZ2_ACT_SILU: finish32<OZ2_ACT_SILU>(z, add, bf16, buf, lane); break;
          default: finish32<OZ2_ACT_NONE>(z, add, bf16, buf, lane);
        }
        if (add && !fast_add && c + kChunk < cols)  // z's registers are free now for its loads
          fetch_begin_slow(ep.add, ep.ld_add, x.rows, x.cols, row0, col0 + c + kChunk, lane, r);
        __syncwarp();
        if (fast_out) {
          store_fast(static_cast<uint16_t*>(ep.out) + lane_row * ep.ld_out + lane_col + c, ep.ld_out, lane, buf);
        } else {
          store_slow(ep.out, ep.ld_out, x.rows, x.cols, row0, col0 + c, lane, buf);
        }
        __syncwarp();
      }
    }
    if (!ok) {
      dev->status = kStatusTimeout;
      dev->timeout_site = 23;
    }
  }
  tc_fence_before();
  cluster_sync_all();  // neither CTA leaves while the pair's MMAs or loads may touch it
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

// ---------------------------------------------------------------------------
// Tiles of NT rows × 128 columns of D on single CTAs, the depth split over the
// CTAs of a cluster: for a D of few tiles.  The tile is formed transposed: Q's
// 128 rows are the MMA's M (D's columns on tensor-memory lanes), P's NT rows its
// N, so that a few tokens fill a small N, and a warp's lanes are consecutive
// columns of D.  Each CTA leaves its sums in its shared memory (where the operands
// were), and after a cluster barrier takes an equal share of the tile's rows, adds
// up the parts in the order of the CTAs and finishes them: no workspace, and the
// same bits every time.
//
// What bounds it: memory, where the weights stream through (16 tokens × 16384² E4M3
// 45 µs, 6.0 TB/s; bf16 85 µs, 6.3), else the chain of a launch, its first loads, the
// MMAs, the parts' exchange and the stores: 1 × 512 × 512 takes 3.7 µs, one token × 4096²
// bf16 9.1 (34 MB in 128 CTAs), 256³ 3.7, 1024×2048×2048 12.6.  A thread's columns of the
// tile are the same for every row it finishes, so biases and scales are in registers
// before the sums come, and a residual's row is loaded one ahead.
// ---------------------------------------------------------------------------
constexpr int kSplitThreads = 256;    // TMA warp, MMA warp, 4 that drain, all 8 finish
constexpr int kMaxSplit = 8;
constexpr int kSplitMaxStages = 12;
constexpr int split_stage_bytes(int nt) { return (kRows + nt) * 128; }
constexpr int split_smem(int nt, int stages) {
  const int ring = stages * split_stage_bytes(nt), sums = nt * kRows * 4;
  return 1024 + (ring > sums ? ring : sums) + 8 * (2 * kSplitMaxStages + 2);
}

template <bool F8>
__device__ __forceinline__ void mma_one(uint32_t me, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                        uint32_t accumulate) {
  if (F8) {
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
        " @q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(me)
        : "memory");
  } else {
    mma_f16_by(me, d_tmem, a_desc, b_desc, idesc, accumulate);
  }
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

template <int ACT>
__device__ __forceinline__ void activate8(float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = activate<ACT>(z[e]);
}

// Eight 16-bit values of a row of R, from its column col on (n of them there).
__device__ __forceinline__ uint4 load8(const LinUnits& x, const void* src, int64_t ld, int64_t row, int64_t col, int n) {
  const uint16_t* s = static_cast<const uint16_t*>(src);
  return load16_any<false>(s + row * ld + col, s, s + (x.rows - 1) * ld + x.cols, n);
}
__device__ __forceinline__ void store8(void* dst, int64_t ld, int64_t row, int64_t col, int n, const float (&z)[8],
                                       bool bf16) {
  uint16_t* d = static_cast<uint16_t*>(dst) + row * ld + col;
  const uint32_t w[4] = {pack16(z[0], z[1], bf16), pack16(z[2], z[3], bf16), pack16(z[4], z[5], bf16),
                         pack16(z[6], z[7], bf16)};
  if (n == 8 && vec_ok(dst, ld, 2)) {
    *reinterpret_cast<uint4*>(d) = make_uint4(w[0], w[1], w[2], w[3]);
  } else if (n == 8 && (reinterpret_cast<uintptr_t>(d) & 2) == 0) {
#pragma unroll
    for (int e = 0; e < 4; ++e) reinterpret_cast<uint32_t*>(d)[e] = w[e];
  } else if (n == 8) {
    d[0] = static_cast<uint16_t>(w[0]);
#pragma unroll
    for (int e = 0; e < 3; ++e) reinterpret_cast<uint32_t*>(d + 1)[e] = __funnelshift_r(w[e], w[e + 1], 16);
    d[7] = static_cast<uint16_t>(w[3] >> 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) d[e] = static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
  }
}

// What a thread needs of its eight columns of D, whichever the row.
struct ColumnTerms {
  float bias[8], scale[8];
};
__device__ __forceinline__ void load_terms(const LinEpilogue& ep, int64_t cols, int64_t col, int n, ColumnTerms& t) {
#pragma unroll
  for (int e = 0; e < 8; ++e) t.bias[e] = 0.f, t.scale[e] = 1.f;
  if (ep.bias && ep.bias_type == OZ2_TYPE_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) t.bias[e] = __ldg(static_cast<const float*>(ep.bias) + col + e);
  } else if (ep.bias) {
    const uint16_t* b = static_cast<const uint16_t*>(ep.bias);
    const uint4 v = load16_any(b + col, b, b + cols, n);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = unpack16(w[e], ep.bias_type == OZ2_TYPE_BF16);
      t.bias[2 * e] = f.x;
      t.bias[2 * e + 1] = f.y;
    }
  }
  if (ep.col_scale) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) t.scale[e] = __ldg(ep.col_scale + col + e);
  }
}

// Eight columns of one row of D from their sums; r holds R's, where there is one.
__device__ __forceinline__ void finish8(const LinEpilogue& ep, int64_t row, int64_t col, int n, const ColumnTerms& t,
                                        uint4 r, float (&z)[8]) {
  if (ep.out_type == OZ2_TYPE_F32) {
    float* d = static_cast<float*>(ep.out) + row * ep.ld_out + col;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) d[e] = ep.accumulate ? d[e] + z[e] : z[e];
    return;
  }
  const bool bf16 = ep.out_type == OZ2_TYPE_BF16;
  const float rs = ep.row_scale ? __ldg(ep.row_scale + row) : 1.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = fmaf(z[e], rs * t.scale[e], t.bias[e]);
  if (ep.pre) store8(ep.pre, ep.ld_pre, row, col, n, z, bf16);
  switch (ep.act) {
    case OZ2_ACT_RELU: activate8<OZ2_ACT_RELU>(z); break;
    case OZ2_ACT_GELU: activate8<OZ2_ACT_GELU>(z); break;
    case OZ2_ACT_GELU_TANH: activate8<OZ2_ACT_GELU_TANH>(z); break;
    case OZ2_ACT_SILU: activate8<OZ2_ACT_SILU>(z); break;
    default: break;
  }
  if (ep.add) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = unpack16(w[e], bf16);
      z[2 * e] += f.x;
      z[2 * e + 1] += f.y;
    }
  }
  store8(ep.out, ep.ld_out, row, col, n, z, bf16);
}

// The rows of the tile that a CTA finishes: from row r on, every 16th, of SPLIT
// CTAs' sums (`at`: this thread's columns of row 0 in this CTA's).  All of a row's
// loads are under way before the first is added.
template <int SPLIT>
__device__ __forceinline__ void finish_rows(const LinUnits& x, int64_t row0, int64_t col, int n, int r, int end,
                                            uint32_t at, const ColumnTerms& t, uint4 add) {
#pragma unroll 1
  for (; r < end && row0 + r < x.rows; r += 16) {
    float4 a[SPLIT], b[SPLIT];
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {
      const uint32_t from = (SPLIT > 1 ? mapa_shared(at, p) : at) + r * kRows * 4;
      a[p] = ld_cluster_f4(from);
      b[p] = ld_cluster_f4(from + 16);
    }
    const uint4 now = add;  // R's values of the next row are on their way while this one is finished
    if (x.ep.add && r + 16 < end && row0 + r + 16 < x.rows) add = load8(x, x.ep.add, x.ep.ld_add, row0 + r + 16, col, n);
    float z[8] = {a[0].x, a[0].y, a[0].z, a[0].w, b[0].x, b[0].y, b[0].z, b[0].w};
#pragma unroll
    for (int p = 1; p < SPLIT; ++p) {
      z[0] += a[p].x, z[1] += a[p].y, z[2] += a[p].z, z[3] += a[p].w;
      z[4] += b[p].x, z[5] += b[p].y, z[6] += b[p].z, z[7] += b[p].w;
    }
    finish8(x.ep, row0 + r, col, n, t, now, z);
  }
}

template <int TYPE, int NT>
__global__ void __launch_bounds__(kSplitThreads)
    linear_split_kernel(const __grid_constant__ LinMaps maps, const __grid_constant__ LinLaunch L, int stages, int split,
                        Oz2Device* dev) {
  constexpr bool F8 = TYPE == OZ2_TYPE_E4M3;
  constexpr int kStage = split_stage_bytes(NT);
  constexpr int kCols = NT < 32 ? 32 : NT;   // tensor memory is allocated in powers of two from 32 columns
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t bars[2 * kSplitMaxStages + 1];
  __shared__ uint32_t tmem_base_s;
  __shared__ int failed_s;

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = split > 1 ? cluster_ctarank() : 0;
  const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + kSplitMaxStages);
  const uint32_t done = smem_u32(bars + 2 * kSplitMaxStages);
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    mbar_init(done, 1);
    fence_barrier_init();
    failed_s = 0;
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&tmem_base_s), kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_s, 0);
  pdl_trigger();
  pdl_wait();

  int u = blockIdx.x / split;
  const int i = L.count > 1 && u >= L.u[0].units ? 1 : 0;
  const LinUnits& x = L.u[i];
  if (i) u -= L.u[0].units;
  const int tn = u / x.ntm, tm = u - tn * x.ntm;   // tiles that share Q's rows run together
  const int per = (x.steps + split - 1) / split;
  const int t0 = min(x.steps, static_cast<int>(rank) * per), t1 = min(x.steps, t0 + per);

  if (warp == 0) {
    if (elect_one()) {
      const int prow = tm * NT, qrow = tn * kRows;
      uint32_t s = 0, ph = 1;
      bool ok = true;
      const bool p_mn = x.p_mn != 0, q_mn = x.q_mn != 0;
      const CUtensorMap *mp = &maps.p[i], *mq = &maps.q[i];
      const uint32_t ring0 = smem_u32(smem);
      const int steps = t1 - t0;
      int d = t0 * (F8 ? 128 : 64);
      for (int t = 0; t < steps; ++t, d += F8 ? 128 : 64) {
        if (!mbar_wait_bounded(empty0 + 8 * s, ph, kWaitLimit)) {
          ok = false;
          break;
        }
        const uint32_t sa = ring0 + s * kStage, sb = sa + kTileBytes, bar = full0 + 8 * s;
        mbar_arrive_expect_tx(bar, kStage);
        if (!q_mn) {
          tma_load_2d(sa, mq, bar, d, qrow);
        } else {
          tma_load_2d(sa, mq, bar, qrow, d);
          tma_load_2d(sa + kTileBytes / 2, mq, bar, qrow + 64, d);
        }
        if (!p_mn) {
          tma_load_2d(sb, mp, bar, d, prow);
        } else {
#pragma unroll
          for (int r = 0; r < NT; r += 64) tma_load_2d(sb + r * 128, mp, bar, prow + r, d);
        }
        if (++s == static_cast<uint32_t>(stages)) {
          s = 0;
          ph ^= 1;
        }
      }
      if (!ok) {
        failed_s = 1;
        dev->status = kStatusTimeout;
        dev->timeout_site = 24;
        // Copies in flight land before the block goes.
        for (int j = 0; j < stages; ++j)
          if (j < steps) mbar_wait_bounded(full0 + 8 * j, j < static_cast<int>(s) ? ph ^ 1 : ph, kWaitLimit);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t me = lane == 0, base = smem_u32(smem);
    const int steps = t1 - t0;
    uint32_t s = 0, ph = 0;
    auto multiply = [&](auto shape, uint64_t ad, uint64_t bd) {
      for (int t = 0; t < steps; ++t) {
        if (!mbar_wait_warp(full0 + 8 * s, ph, kWaitLimit)) {
          if (me) {
            failed_s = 1;
            dev->status = kStatusTimeout;
            dev->timeout_site = 25;
          }
          break;
        }
        tc_fence_after();
        const uint64_t a = ad + s * (kStage >> 4), b = bd + s * (kStage >> 4);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          mma_one<F8>(me, tmem, a + kk * shape.a_next, b + kk * shape.b_next, shape.idesc, (t | kk) ? 1u : 0u);
        mma_commit_by(me, empty0 + 8 * s);
        if (++s == static_cast<uint32_t>(stages)) {
          s = 0;
          ph ^= 1;
        }
      }
    };
    if (F8 || !x.q_mn) {
      multiply(MmaShape<TYPE, false, false, kRows, NT>{}, operand_desc<false>(base), operand_desc<false>(base + kTileBytes));
    } else if (!x.p_mn) {
      multiply(MmaShape<TYPE, true, false, kRows, NT>{}, operand_desc<true>(base), operand_desc<false>(base + kTileBytes));
    } else {
      multiply(MmaShape<TYPE, true, true, kRows, NT>{}, operand_desc<true>(base), operand_desc<true>(base + kTileBytes));
    }
    mma_commit_by(me, done);
    __syncwarp();
  }
  // This thread's part of the epilogue: eight columns of every 16th row of the CTA's
  // share of the tile.  What does not depend on the sums is loaded before them.
  const int share = NT / split, r_first = static_cast<int>(rank) * share + (threadIdx.x >> 4);
  const int64_t row0 = static_cast<int64_t>(tm) * NT, col = static_cast<int64_t>(tn) * kRows + (threadIdx.x & 15) * 8;
  const int n = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(8), x.cols - col)));
  const int r_end = n > 0 ? (static_cast<int>(rank) + 1) * share : 0;
  ColumnTerms terms;
  uint4 first = make_uint4(0, 0, 0, 0);
  if (r_first < r_end && row0 + r_first < x.rows) {
    load_terms(x.ep, x.cols, col, n, terms);
    if (x.ep.add) first = load8(x, x.ep.add, x.ep.ld_add, row0 + r_first, col, n);
  }
  // The sums, NT columns of 128 lanes, to shared memory: the operands there have
  // been multiplied.
  float* sums = reinterpret_cast<float*>(smem);
  if (warp >= 2 && warp < 6) {
    const int q = warp & 3;
    const bool ok = mbar_wait_warp(done, 0, kWaitLimit);
    if (!ok && lane == 0) {
      failed_s = 1;
      dev->status = kStatusTimeout;
      dev->timeout_site = 26;
    }
    tc_fence_after();
    if (ok && !*static_cast<volatile int*>(&failed_s)) {
#pragma unroll
      for (int c = 0; c < NT; c += 16) {
        uint32_t v[16];
        if (t1 > t0) {
          tmem_ld16(tmem + (static_cast<uint32_t>(32 * q) << 16) + c, v);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = 0u;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) sums[(c + j) * kRows + 32 * q + lane] = __uint_as_float(v[j]);
      }
    }
  }
  tc_fence_before();
  if (split > 1) {
    cluster_sync_all();
  } else {
    __syncthreads();
  }
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, kCols);
  const uint32_t at = smem_u32(sums) + (threadIdx.x & 15) * 32;
  switch (split) {
    case 1: finish_rows<1>(x, row0, col, n, r_first, r_end, at, terms, first); break;
    case 2: finish_rows<2>(x, row0, col, n, r_first, r_end, at, terms, first); break;
    case 4: finish_rows<4>(x, row0, col, n, r_first, r_end, at, terms, first); break;
    default: finish_rows<8>(x, row0, col, n, r_first, r_end, at, terms, first);
  }
  if (split > 1) cluster_sync_all();  // no CTA leaves while another reads its sums
}

// One operand as a 2-D tensor.  K-major: rows of `depth`, boxes of 128 bytes of
// depth × box_rows rows.  MN-major: depth rows of `rows`, boxes of 64 × 64.
bool make_operand_map(CUtensorMap* map, const void* base, int64_t rows, int64_t depth, int64_t ld, int type, bool mn,
                      int box_rows = kRows) {
  EncodeTiledFn enc = get_encode_fn();
  if (!enc) return false;
  const int es = type_bytes(type);
  cuuint64_t dims[2] = {static_cast<cuuint64_t>(mn ? rows : depth), static_cast<cuuint64_t>(mn ? depth : rows)};
  cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * es};
  cuuint32_t box[2] = {static_cast<cuuint32_t>(128 / es), mn ? 64u : static_cast<cuuint32_t>(box_rows)};
  cuuint32_t estr[2] = {1, 1};
  return enc(map, es == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(base),
             dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

namespace {

int64_t steps_of(const LinProduct& p, int type) {
  const int64_t step = 128 / type_bytes(type);
  return (p.depth + step - 1) / step;
}
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The estimates (cycles of an SM) behind a plan, fitted to measurements on one GB300.
//   Pairs: a step of a tile 535 (512 of MMAs), of half a tile 390 (its loads), a tile
//   at least 4600 (its epilogue) and 1000 more; the launch's start and its last epilogue 10000; the exchange of split
//   tiles' parts 26000.
//   Clusters: a CTA 5600 and for each step what its loads take of the SM's 61 bytes a
//   cycle or its MMAs of the tensor core; 26 for each row that it finishes; joining
//   the parts 1200 and 36 a row of the tile.  CTAs that share an SM share both rates.
//   From memory an SM gets 24 bytes a cycle, however few of them there are.
//   (Fitted on 70 shapes from 1 to 2500 rows, 64 to 16384 columns and depth.  On 96 others,
//   drawn from 1 to 4096 rows and 64 to 11000 columns and depth, the plan it picks takes
//   2% longer than the fastest in the mean, 41% at most.)
constexpr double kPairStep = 535, kPairTileLeast = 4600, kPairTile = 1000, kPairLaunch = 10000, kExchange = 26000;
constexpr double kCta = 5600, kLoadRate = 61, kFinishRow = 26, kJoin = 1200, kJoinRow = 36, kClusterLaunch = 800;
constexpr double kMemoryRate = 24;
constexpr double kTwoLaunches = 2500;  // what a launch of its own costs beside a product's time

constexpr double kHalfStep = 390;
double pair_tile_cycles(int64_t steps) { return std::max(steps * kPairStep, kPairTileLeast) + kPairTile; }
double half_tile_cycles(int64_t steps) { return std::max(steps * kHalfStep, kPairTileLeast / 2) + kPairTile; }

// CTAs in clusters of `split` that run at once, one or two to an SM (152 SMs in
// groups that clusters do not cross).
int64_t clustered_ctas(int64_t sms, int split, int per_sm) {
  const int64_t most = sms * per_sm;
  if (split <= 2) return most;
  if (per_sm == 1) return split == 4 ? most * 144 / 152 / 4 * 4 : most * 120 / 152 / 8 * 8;
  return split == 4 ? most * 296 / 304 / 4 * 4 : most * 288 / 304 / 8 * 8;
}

// On pairs: tiles whole, or split depths for the products of few tiles.
void plan_pairs(const int64_t (&tiles)[kMaxProducts], const int64_t (&steps)[kMaxProducts], int count, double bytes,
                int64_t pairs, LinPlan* best) {
  // Tiles go to the pairs in turn, the first product's first: the pair that takes the most
  // of those, and the first that takes one fewer.
  const double t0 = pair_tile_cycles(steps[0]), t1 = pair_tile_cycles(steps[count - 1]);
  const int64_t units = tiles[0] + (count > 1 ? tiles[1] : 0);
  const int64_t even = tiles[0] / pairs, odd = tiles[0] % pairs;
  const double most = (even + (odd > 0)) * t0 + (ceil_div(units, pairs) - even - (odd > 0)) * t1;
  const double fewer = even * t0 + (ceil_div(units - odd, pairs) - even) * t1;
  best->cost = kPairLaunch + std::max({most, fewer, bytes / (kMemoryRate * 2 * std::min(units, pairs))});
  // A last round of few tiles: they are taken as halves, by twice as many pairs.
  const int64_t last = units % pairs;
  if (units > pairs && last > 0 && 2 * last <= pairs && last <= tiles[count - 1]) {
    const double cost = best->cost - pair_tile_cycles(steps[count - 1]) + half_tile_cycles(steps[count - 1]);
    if (cost < best->cost) {
      best->cost = cost;
      best->halves = static_cast<int>(last);
    }
  }
  // The parts of the products of few tiles, while they fit, each next one to the
  // tile that takes longest.
  int split[kMaxProducts] = {1, 1};
  bool few[kMaxProducts] = {false, false};
  int64_t taken = 0;
  for (int i = 0; i < count; ++i) {
    few[i] = tiles[i] > 0 && 2 * tiles[i] <= pairs;
    if (few[i]) taken += tiles[i];
  }
  for (bool more = taken > 0; more;) {
    int at = -1;
    for (int i = 0; i < count; ++i)
      if (few[i] && split[i] < kMaxPairSplit && taken + tiles[i] <= pairs && steps[i] / (split[i] + 1) >= 8 &&
          (at < 0 || steps[i] / split[i] > steps[at] / split[at]))
        at = i;
    if ((more = at >= 0)) {
      ++split[at];
      taken += tiles[at];
    }
  }
  double part = 0, all = 0, tile = 0;
  int64_t parts = 0, whole = 0;
  for (int i = 0; i < count; ++i) {
    const double t = pair_tile_cycles(ceil_div(steps[i], split[i]));
    all += tiles[i] * split[i] * t;
    if (split[i] > 1) {
      parts += tiles[i] * split[i];
      part = std::max(part, t);
    } else if (tiles[i]) {
      whole += tiles[i];
      tile = std::max(tile, t);
    }
  }
  const double cost = kPairLaunch + kExchange + std::max(part, whole ? all / pairs + tile / 2 : part);
  if (parts == 0 || cost >= best->cost) return;
  best->cost = cost;
  best->halves = 0;
  for (int i = 0; i < count; ++i) best->pair_split[i] = split[i];
  best->parts = static_cast<int>(parts);
  // Rounds of whole tiles that the other pairs have time for beside a part.
  best->ahead = whole && parts < pairs ? static_cast<int>(std::min<int64_t>(part / tile, whole / (pairs - parts))) : 0;
  best->scratch = (sizeof(float) * kPartFloats + sizeof(int) * 2 * kLinEpiWarps) * best->parts;
}

}  // namespace

LinPlan plan_linear(const LinProduct* products, int count, int type) {
  LinPlan best;
  int64_t tiles[kMaxProducts] = {}, steps[kMaxProducts] = {}, units = 0;
  double bytes = 0;
  bool p_mn = false;
  for (int i = 0; i < count; ++i) {
    tiles[i] = ceil_div(products[i].rows, kLinTile) * ceil_div(products[i].cols, kLinTile);
    steps[i] = steps_of(products[i], type);
    units += tiles[i];
    bytes += static_cast<double>(products[i].rows + products[i].cols) * products[i].depth * type_bytes(type);
    p_mn = p_mn || products[i].p_mn;
  }
  if (units == 0) return best;
  const int64_t sms = num_sms();
  plan_pairs(tiles, steps, count, bytes, sms / 2, &best);
  for (int nt : {16, 32, 64, 128}) {
    if (p_mn && nt < 64) continue;
    for (int split = 1; split <= kMaxSplit; split *= 2) {
      int64_t ctas = 0, n[kMaxProducts];
      for (int i = 0; i < count; ++i) {
        n[i] = ceil_div(products[i].rows, nt) * ceil_div(products[i].cols, kRows) * split;
        ctas += n[i];
      }
      // One CTA to an SM while they fit, else two; split depths in one round only, and
      // beside another CTA only in pairs of small tiles (64 and 128 rows so: half as
      // fast again as the next smaller split).
      const int per_sm = ctas <= clustered_ctas(sms, split, 1) ? 1 : 2;
      const int64_t at_once = clustered_ctas(sms, split, per_sm);
      if (split > 1 && (ctas > at_once || (per_sm == 2 && (nt > 32 || split > 2)))) continue;
      // The CTA that takes longest, undisturbed, or all CTAs' work at the SMs' rates.
      const double step = std::max((kRows + nt) * 128 / kLoadRate, 2.0 * nt);
      double work = 0, longest = 0;
      for (int i = 0; i < count; ++i) {
        const int64_t each = ceil_div(steps[i], split);
        const double t = kCta + each * step + kFinishRow * nt / split + (split > 1 ? kJoin + kJoinRow * nt : 0.0);
        work += static_cast<double>(n[i]) * (each * step + kFinishRow * nt / split);
        if (n[i]) longest = std::max(longest, t);
      }
      // (In one round some SMs have one CTA more than others.)
      const double share = ctas <= at_once ? work / ctas * ceil_div(ctas, sms) : work / sms;
      const double cost = kClusterLaunch + std::max({longest, ceil_div(ctas, at_once) * kCta + share,
                                                     kCta + bytes / (kMemoryRate * std::min(ctas, sms))});
      if (cost < best.cost) {
        best = LinPlan{};
        best.cost = cost;
        best.nt = nt;
        best.split = split;
        best.stages = std::min(kSplitMaxStages, (per_sm == 2 ? 110 * 1024 : 220 * 1024) / split_stage_bytes(nt));
      }
    }
  }
  return best;
}

bool plan_apart(const LinPlan& together, const LinPlan& a, const LinPlan& b) {
  return a.cost + b.cost + kTwoLaunches < together.cost;
}

namespace {

using SplitKernel = void (*)(const LinMaps, const LinLaunch, int, int, Oz2Device*);
template <int TYPE>
SplitKernel split_kernel(int nt) {
  return nt == 16   ? linear_split_kernel<TYPE, 16>
         : nt == 32 ? linear_split_kernel<TYPE, 32>
         : nt == 64 ? linear_split_kernel<TYPE, 64>
                    : linear_split_kernel<TYPE, 128>;
}

// As launch_dependent, in clusters.
template <typename... KArgs, typename... Args>
cudaError_t launch_clusters(void (*kernel)(KArgs...), unsigned grid, unsigned block, size_t smem, unsigned cluster,
                            cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

}  // namespace

cudaError_t launch_linear(const LinProduct* products, int count, int type, const LinPlan& plan, void* scratch,
                          Oz2Device* dev, cudaStream_t st) {
  LinMaps maps{};
  LinLaunch L{};
  const int tile_rows = plan.nt ? plan.nt : kLinTile, tile_cols = plan.nt ? kRows : kLinTile;
  int split_tiles = 0;
  for (int i = 0; i < count; ++i) {
    const LinProduct& p = products[i];
    LinUnits& x = L.u[i];
    x.rows = p.rows;
    x.cols = p.cols;
    // (A result of more tiles than an int counts is larger than the memory.)
    const int64_t ntm = ceil_div(p.rows, tile_rows), ntn = ceil_div(p.cols, tile_cols);
    if (ntm * ntn * plan.split * 8 > 0x3FFFFFFFLL) return cudaErrorInvalidValue;
    x.ntm = static_cast<int>(ntm);
    x.ntn = static_cast<int>(ntn);
    x.units = x.ntm * x.ntn;
    x.split = plan.pair_split[i];
    x.halves = i + 1 == count ? plan.halves : 0;
    x.steps = static_cast<int>(steps_of(p, type));
    x.p_mn = p.p_mn;
    x.q_mn = p.q_mn;
    x.ep = p.ep;
    if (x.split > 1) {
      split_tiles += x.units;
    } else {
      L.units += x.units - x.halves;
      L.half_units += 2 * x.halves;
    }
    if (x.steps && (!make_operand_map(&maps.p[i], p.p, p.rows, p.depth, p.ldp, type, p.p_mn, plan.nt ? plan.nt : kRows) ||
                    !make_operand_map(&maps.q[i], p.q, p.cols, p.depth, p.ldq, type, p.q_mn) ||
                    (x.halves &&
                     !make_operand_map(&maps.q_half, p.q, p.cols, p.depth, p.ldq, type, p.q_mn, kRows / 2))))
      return cudaErrorInvalidValue;
  }
  L.count = count;
  if (L.units + split_tiles == 0) return cudaSuccess;
  if (plan.nt) {
    SplitKernel kern = type == OZ2_TYPE_BF16  ? split_kernel<OZ2_TYPE_BF16>(plan.nt)
                       : type == OZ2_TYPE_F16 ? split_kernel<OZ2_TYPE_F16>(plan.nt)
                                              : split_kernel<OZ2_TYPE_E4M3>(plan.nt);
    const size_t smem = split_smem(plan.nt, plan.stages);
    cudaError_t err = allow_smem(reinterpret_cast<const void*>(kern), smem);
    if (err != cudaSuccess) return err;
    count_launch();
    return launch_clusters(kern, static_cast<unsigned>(L.units * plan.split), kSplitThreads, smem, plan.split, st, maps, L,
                           plan.stages, plan.split, dev);
  }
  auto kern = type == OZ2_TYPE_BF16  ? linear_pair_kernel<OZ2_TYPE_BF16>
              : type == OZ2_TYPE_F16 ? linear_pair_kernel<OZ2_TYPE_F16>
                                     : linear_pair_kernel<OZ2_TYPE_E4M3>;
  cudaError_t err = allow_smem(reinterpret_cast<const void*>(kern), kLinSmem);
  if (err != cudaSuccess) return err;
  const int64_t resident = resident_pairs(reinterpret_cast<const void*>(kern), kLinThreads, kLinSmem);
  int64_t pairs = std::min<int64_t>(L.units, resident);
  if (plan.parts) {
    // Each part has a pair of its own, resident or not: no pair waits for another.
    pairs = num_sms() / 2;
    L.parts = plan.parts;
    L.ahead = plan.ahead;
    L.sums = static_cast<float*>(scratch);
    L.arrived = reinterpret_cast<int*>(L.sums + static_cast<int64_t>(plan.parts) * kPartFloats);
    err = cudaMemsetAsync(L.arrived, 0, sizeof(int) * split_tiles * 2 * kLinEpiWarps, st);
    if (err != cudaSuccess) return err;
  }
  count_launch();
  return launch_dependent(kern, dim3(static_cast<unsigned>(2 * pairs)), dim3(kLinThreads), kLinSmem, st, maps, L, dev);
}

}  // namespace oz2
