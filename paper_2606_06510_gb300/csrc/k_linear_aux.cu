// The memory-bound steps around the products of a linear layer: rows copied to
// 16-byte boundaries for operands that TMA cannot read where they are, and the
// gradient's dz = dy·act'(z) with its column sums db.
#include <algorithm>

#include "lin_common.cuh"

namespace oz2 {
namespace {

// ---------------------------------------------------------------------------
// Pack: a thread writes 16-byte pieces of the destination's rows, one grid's stride
// apart (consecutive threads' are consecutive).  Its row and place in it are found by one
// division and carried on from piece to piece.  Up to two operands in one launch: the
// blocks of the second grid row take the second.
//
// Memory bounds it, and at a few MB the launch: 3001×2047 and 2500×2047 of 16 bits, 45 MB
// there and back, 10 µs (13 with a 64-bit division for each piece).
// ---------------------------------------------------------------------------
constexpr int kPackAhead = 2;   // pieces of a thread on their way at once
constexpr int kPackBlocks = 8;  // blocks an SM

template <typename T>
__global__ void __launch_bounds__(256) pack_rows_kernel(PackJob a, PackJob b) {
  pdl_trigger();
  pdl_wait();
  constexpr int kVec = 16 / sizeof(T);
  const PackJob& x = blockIdx.y ? b : a;
  const T* src = static_cast<const T*>(x.src);
  T* dst = static_cast<T*>(x.dst);
  const uint32_t per = static_cast<uint32_t>((x.cols + kVec - 1) / kVec);
  const uint32_t first = blockIdx.x * blockDim.x + threadIdx.x, stride = gridDim.x * blockDim.x;
  const uint32_t stride_rows = stride / per, stride_pieces = stride - stride_rows * per;
  const T* end = src + (x.rows - 1) * x.ld_src + x.cols;
  int64_t r = first / per;
  uint32_t c = first - static_cast<uint32_t>(r) * per;
  while (r < x.rows) {
    const T* from[kPackAhead];
    T* to[kPackAhead];
    int n[kPackAhead];
    bool there[kPackAhead], inside = true;
#pragma unroll
    for (int j = 0; j < kPackAhead; ++j) {
      there[j] = r < x.rows;
      const int64_t row = there[j] ? r : 0, col = static_cast<int64_t>(c) * kVec;
      from[j] = src + row * x.ld_src + col;
      to[j] = dst + row * x.ld_dst + col;
      n[j] = static_cast<int>(min(static_cast<int64_t>(kVec), x.cols - col));
      inside = inside && words_inside(from[j], src, end);
      r += stride_rows;
      c += stride_pieces;
      if (c >= per) c -= per, ++r;
    }
    if (inside) {
      Words w[kPackAhead];
#pragma unroll
      for (int j = 0; j < kPackAhead; ++j) w[j] = load_words16(from[j]);
#pragma unroll
      for (int j = 0; j < kPackAhead; ++j)
        if (there[j]) *reinterpret_cast<uint4*>(to[j]) = shift_words16(from[j], w[j]);
    } else {
#pragma unroll
      for (int j = 0; j < kPackAhead; ++j)
        if (there[j]) *reinterpret_cast<uint4*>(to[j]) = load16_any(from[j], src, end, n[j]);
    }
  }
}

// ---------------------------------------------------------------------------
// dz and db.  A block takes 256 columns (a lane 8 of them) and a chunk of rows,
// which its 8 warps walk in turn; the warps' sums are joined in shared memory in
// a fixed order.  Up to 8 chunks (2048 rows) are a cluster, whose first block adds up
// the others' sums; more of them write theirs to `partial` (chunk, column) and a second
// kernel adds those.  Either way in order: the sums never depend on who came first.
//
// Memory bounds it without an activation (65536×1024 bf16: 134 MB in 23 µs, 5.9 TB/s),
// with one the load-work-store chain of three blocks an SM (4096² gelu_tanh: 101 MB in
// 19 µs; exp and erf by their slow functions it was 62).  Rows off the 16-byte grid
// are put together from two aligned loads each, all of a round's under way at once:
// 2500×3001 gelu 17 µs (27 when each row's bounds were asked before its loads).
// ---------------------------------------------------------------------------
constexpr int kGradCols = 256, kGradWarps = 8, kGradBlocks = 3;  // blocks an SM

// Eight columns of a row: g ← dy·act'(z), the sums, and dz.
template <int ACT>
__device__ __forceinline__ void grad8(const uint32_t (&aw)[4], const uint32_t (&bw)[4], bool bf16, float (&s)[8],
                                      uint16_t* dz) {
  float g[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = unpack16(aw[e], bf16);
    g[2 * e] = f.x;
    g[2 * e + 1] = f.y;
    if (ACT != OZ2_ACT_NONE) {
      const float2 t = unpack16(bw[e], bf16);
      // (Not fused into the sums: db does not depend on whether dz is wanted.)
      g[2 * e] = __fmul_rn(g[2 * e], act_slope<ACT>(t.x));
      g[2 * e + 1] = __fmul_rn(g[2 * e + 1], act_slope<ACT>(t.y));
    }
    s[2 * e] += g[2 * e];
    s[2 * e + 1] += g[2 * e + 1];
  }
  if (dz)  // rows of 16-byte pieces: what lies past n in the last one is padding
    *reinterpret_cast<uint4*>(dz) = make_uint4(pack16(g[0], g[1], bf16), pack16(g[2], g[3], bf16),
                                               pack16(g[4], g[5], bf16), pack16(g[6], g[7], bf16));
}

// Rows that a warp loads before it works on them (shifted loads take twice the
// registers).
template <bool ALIGNED>
constexpr int kGradAhead = ALIGNED ? 4 : 2;

// ALIGNED: rows start on 16-byte boundaries.
template <int ACT, bool BF16, bool ALIGNED>
__global__ void __launch_bounds__(32 * kGradWarps, kGradBlocks)
    act_grad_kernel(int64_t m, int64_t n, int64_t chunk_rows, const uint16_t* __restrict__ dy, int64_t ld_dy,
                    const uint16_t* __restrict__ z, int64_t ld_z, uint16_t* __restrict__ dz, int64_t ld_dz,
                    float* __restrict__ partial, float* __restrict__ db, bool accumulate) {
  __shared__ float sums[kGradWarps][kGradCols];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * kGradCols + 8 * lane;
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * chunk_rows, r1 = min(m, r0 + chunk_rows);
  const int left = static_cast<int>(min(static_cast<int64_t>(8), n - col));
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = 0.f;
  auto work = [&](uint4 a, uint4 b, int64_t r) {
    const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
    grad8<ACT>(aw, bw, BF16, s, dz ? dz + r * ld_dz + col : nullptr);
  };
  auto one = [&](const uint16_t* src, int64_t ld, int64_t r) {
    const uint16_t* p = src + r * ld + col;
    if (ALIGNED) return left == 8 ? __ldg(reinterpret_cast<const uint4*>(p)) : load16_singly(p, left);
    return load16_any(p, src, src + (m - 1) * ld + n, left);
  };
  if (left > 0) {
    constexpr int kAhead = kGradAhead<ALIGNED>;
    constexpr bool kZ = ACT != OZ2_ACT_NONE;
    int64_t r = r0 + warp;
    for (; r + (kAhead - 1) * kGradWarps < r1; r += kAhead * kGradWarps) {
      // The first and the last of these rows: what lies between them is inside too.
      const int64_t last = r + (kAhead - 1) * kGradWarps;
      const uint16_t *dy_end = dy + (m - 1) * ld_dy + n, *z_end = z + (m - 1) * ld_z + n;
      if (ALIGNED ? left == 8
                  : words_inside(dy + r * ld_dy + col, dy, dy_end) && words_inside(dy + last * ld_dy + col, dy, dy_end) &&
                        (!kZ || (words_inside(z + r * ld_z + col, z, z_end) && words_inside(z + last * ld_z + col, z, z_end)))) {
        if (ALIGNED) {
          uint4 a[kAhead], b[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            a[i] = __ldg(reinterpret_cast<const uint4*>(dy + (r + i * kGradWarps) * ld_dy + col));
            b[i] = kZ ? __ldg(reinterpret_cast<const uint4*>(z + (r + i * kGradWarps) * ld_z + col)) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < kAhead; ++i) work(a[i], b[i], r + i * kGradWarps);
        } else {
          Words a[kAhead], b[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            a[i] = load_words16(dy + (r + i * kGradWarps) * ld_dy + col);
            if (kZ) b[i] = load_words16(z + (r + i * kGradWarps) * ld_z + col);
          }
#pragma unroll
          for (int i = 0; i < kAhead; ++i)
            work(shift_words16(dy + (r + i * kGradWarps) * ld_dy + col, a[i]),
                 kZ ? shift_words16(z + (r + i * kGradWarps) * ld_z + col, b[i]) : make_uint4(0, 0, 0, 0), r + i * kGradWarps);
        }
      } else {
        for (int i = 0; i < kAhead; ++i) {
          const int64_t at = r + i * kGradWarps;
          work(one(dy, ld_dy, at), kZ ? one(z, ld_z, at) : make_uint4(0, 0, 0, 0), at);
        }
      }
    }
    for (; r < r1; r += kGradWarps) work(one(dy, ld_dy, r), kZ ? one(z, ld_z, r) : make_uint4(0, 0, 0, 0), r);
  }
  if (!db) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[warp][8 * lane + e] = s[e];
  __syncthreads();
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kGradCols + threadIdx.x;
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < kGradWarps; ++w) t += sums[w][threadIdx.x];
  if (partial) {
    if (j < n) partial[blockIdx.y * n + j] = t;
    return;
  }
  __syncthreads();
  sums[0][threadIdx.x] = t;
  cluster_sync_all();
  if (blockIdx.y == 0 && j < n) {
    const uint32_t at = smem_u32(&sums[0][threadIdx.x]);
    t = 0.f;
    for (uint32_t c = 0; c < gridDim.y; ++c) {
      float v;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(mapa_shared(at, c)));
      t += v;
    }
    db[j] = accumulate ? db[j] + t : t;
  }
  cluster_sync_all();  // no block leaves while the first reads its sums
}

// db from the chunks' sums: a warp's lanes are 32 columns, its 8 warps each add every
// eighth chunk, and their sums are joined in order.
__global__ void __launch_bounds__(256) sum_chunks_kernel(int64_t n, int64_t chunks, const float* __restrict__ partial,
                                                         float* __restrict__ db, bool accumulate) {
  __shared__ float sums[8][32];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t j = blockIdx.x * 32LL + lane;
  float t = 0.f;
  if (j < n) {
#pragma unroll 8
    for (int64_t c = warp; c < chunks; c += 8) t += partial[c * n + j];
  }
  sums[warp][lane] = t;
  __syncthreads();
  if (warp == 0 && j < n) {
    t = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += sums[w][lane];
    db[j] = accumulate ? db[j] + t : t;
  }
}

constexpr int kGradCluster = 8;      // blocks of a cluster, of up to 256 rows each

int64_t chunk_rows_for(int64_t m, int64_t n) {
  if (m <= kGradCluster * 256) return std::max<int64_t>(32, (m + kGradCluster - 1) / kGradCluster);
  // As many blocks as run at once, of whole rounds of the warps' rows.
  const int64_t across = (n + kGradCols - 1) / kGradCols;
  const int64_t chunks = std::max<int64_t>(1, kGradBlocks * static_cast<int64_t>(num_sms()) / across);
  const int64_t rows = std::max((m + chunks - 1) / chunks, (m + 65534) / 65535);  // (the grid's second axis)
  return (rows + 15) / 16 * 16;
}

template <bool BF16, bool ALIGNED>
auto grad_kernel(int act) {
  return act == OZ2_ACT_RELU        ? act_grad_kernel<OZ2_ACT_RELU, BF16, ALIGNED>
         : act == OZ2_ACT_GELU      ? act_grad_kernel<OZ2_ACT_GELU, BF16, ALIGNED>
         : act == OZ2_ACT_GELU_TANH ? act_grad_kernel<OZ2_ACT_GELU_TANH, BF16, ALIGNED>
         : act == OZ2_ACT_SILU      ? act_grad_kernel<OZ2_ACT_SILU, BF16, ALIGNED>
                                    : act_grad_kernel<OZ2_ACT_NONE, BF16, ALIGNED>;
}

}  // namespace

static int64_t chunks_of(int64_t m, int64_t n) {
  const int64_t r = chunk_rows_for(m, n);
  return std::max<int64_t>(1, (m + r - 1) / r);
}

int64_t lin_db_chunks(int64_t m, int64_t n) {
  const int64_t chunks = chunks_of(m, n);
  return chunks <= kGradCluster ? 0 : chunks;
}

cudaError_t launch_pack_rows(const PackJob* jobs, int count, int bytes, cudaStream_t st) {
  int64_t pieces = 0;
  for (int i = 0; i < count; ++i) pieces = std::max(pieces, jobs[i].rows * ((jobs[i].cols * bytes + 15) / 16));
  if (pieces == 0) return cudaSuccess;
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((pieces + 256 * kPackAhead - 1) / (256 * kPackAhead),
                                                                   kPackBlocks * static_cast<int64_t>(num_sms())));
  count_launch();
  return launch_dependent(bytes == 1 ? pack_rows_kernel<uint8_t> : pack_rows_kernel<uint16_t>,
                          dim3(blocks, static_cast<unsigned>(count)), dim3(256), 0, st, jobs[0], jobs[count - 1]);
}

cudaError_t launch_act_grad(int64_t m, int64_t n, int type, int act, const void* dy, int64_t ld_dy, const void* z,
                            int64_t ld_z, void* dz, int64_t ld_dz, float* db, float* partial, bool accumulate,
                            cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  const int64_t rows = chunk_rows_for(m, n), chunks = chunks_of(m, n);
  auto aligned = [](const void* p, int64_t ld) { return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(2 * ld)) & 15) == 0; };
  const bool vec = aligned(dy, ld_dy) && (act == OZ2_ACT_NONE || aligned(z, ld_z));
  auto kern = type == OZ2_TYPE_BF16 ? (vec ? grad_kernel<true, true>(act) : grad_kernel<true, false>(act))
                                    : (vec ? grad_kernel<false, true>(act) : grad_kernel<false, false>(act));
  const bool joined = chunks <= kGradCluster;
  count_launch();
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>((n + kGradCols - 1) / kGradCols), static_cast<unsigned>(chunks));
  cfg.blockDim = dim3(32 * kGradWarps);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = static_cast<unsigned>(joined ? chunks : 1);
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cudaError_t err = cudaLaunchKernelEx(&cfg, kern, m, n, rows, static_cast<const uint16_t*>(dy), ld_dy,
                                       static_cast<const uint16_t*>(z), ld_z, static_cast<uint16_t*>(dz), ld_dz,
                                       joined ? static_cast<float*>(nullptr) : partial, db, accumulate);
  if (err != cudaSuccess || !db || joined) return err;
  count_launch();
  return launch_dependent(sum_chunks_kernel, dim3(static_cast<unsigned>((n + 31) / 32)), dim3(256), 0, st, n, chunks,
                          static_cast<const float*>(partial), db, accumulate);
}

}  // namespace oz2
