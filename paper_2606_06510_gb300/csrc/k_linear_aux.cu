// The memory-bound steps around the products of a linear layer: rows copied to
// 16-byte boundaries for operands that TMA cannot read where they are, and the
// gradient's dz = dy·act'(z) with its column sums db.
#include <algorithm>

#include "lin_common.cuh"

namespace oz2 {
namespace {

// ---------------------------------------------------------------------------
// Pack: a thread writes 16 bytes of a destination row from its elements, one by one
// (consecutive threads' are consecutive).  Up to two operands in one launch: the
// blocks of the second grid row take the second.
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) pack_rows_kernel(PackJob a, PackJob b) {
  pdl_trigger();
  pdl_wait();
  constexpr int kVec = 16 / sizeof(T);
  const PackJob& x = blockIdx.y ? b : a;
  const T* src = static_cast<const T*>(x.src);
  T* dst = static_cast<T*>(x.dst);
  const int64_t per = (x.cols + kVec - 1) / kVec;
  for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < x.rows * per;
       i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t r = i / per, c = (i - r * per) * kVec;
    const T* s = src + r * x.ld_src + c;
    union {
      uint4 v;
      T e[kVec];
    } w;
    w.v = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      if (c + j < x.cols) w.e[j] = __ldg(s + j);
    *reinterpret_cast<uint4*>(dst + r * x.ld_dst + c) = w.v;
  }
}

// ---------------------------------------------------------------------------
// dz and db.  A block takes 256 columns (a lane 8 of them) and a chunk of rows,
// which its 8 warps walk in turn; the warps' sums are joined in shared memory in
// a fixed order and the block's written to `partial` (chunk, column).  A second
// kernel adds the chunks in order: the sums never depend on who came first.
// ---------------------------------------------------------------------------
constexpr int kGradCols = 256, kGradWarps = 8;

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
      g[2 * e] *= act_slope<ACT>(t.x);
      g[2 * e + 1] *= act_slope<ACT>(t.y);
    }
    s[2 * e] += g[2 * e];
    s[2 * e + 1] += g[2 * e + 1];
  }
  if (dz)  // rows of 16-byte pieces: what lies past n in the last one is padding
    *reinterpret_cast<uint4*>(dz) = make_uint4(pack16(g[0], g[1], bf16), pack16(g[2], g[3], bf16),
                                               pack16(g[4], g[5], bf16), pack16(g[6], g[7], bf16));
}

constexpr int kGradAhead = 4;        // rows that a warp loads before it works on them

template <int ACT, bool BF16>
__global__ void __launch_bounds__(32 * kGradWarps)
    act_grad_kernel(int64_t m, int64_t n, int64_t chunk_rows, bool vec, const uint16_t* __restrict__ dy,
                    int64_t ld_dy, const uint16_t* __restrict__ z, int64_t ld_z, uint16_t* __restrict__ dz,
                    int64_t ld_dz, float* __restrict__ partial) {
  __shared__ float sums[kGradWarps][kGradCols];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * kGradCols + 8 * lane;
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * chunk_rows, r1 = min(m, r0 + chunk_rows);
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = 0.f;
  if (vec && col + 8 <= n) {
    int64_t r = r0 + warp;
    for (; r + (kGradAhead - 1) * kGradWarps < r1; r += kGradAhead * kGradWarps) {
      uint4 a[kGradAhead], b[kGradAhead];
#pragma unroll
      for (int i = 0; i < kGradAhead; ++i) {
        a[i] = __ldg(reinterpret_cast<const uint4*>(dy + (r + i * kGradWarps) * ld_dy + col));
        b[i] = make_uint4(0, 0, 0, 0);
        if (ACT != OZ2_ACT_NONE) b[i] = __ldg(reinterpret_cast<const uint4*>(z + (r + i * kGradWarps) * ld_z + col));
      }
#pragma unroll
      for (int i = 0; i < kGradAhead; ++i) {
        const uint32_t aw[4] = {a[i].x, a[i].y, a[i].z, a[i].w}, bw[4] = {b[i].x, b[i].y, b[i].z, b[i].w};
        grad8<ACT>(aw, bw, BF16, s, dz ? dz + (r + i * kGradWarps) * ld_dz + col : nullptr);
      }
    }
    for (; r < r1; r += kGradWarps) {
      const uint4 a = __ldg(reinterpret_cast<const uint4*>(dy + r * ld_dy + col));
      uint4 b = make_uint4(0, 0, 0, 0);
      if (ACT != OZ2_ACT_NONE) b = __ldg(reinterpret_cast<const uint4*>(z + r * ld_z + col));
      const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
      grad8<ACT>(aw, bw, BF16, s, dz ? dz + r * ld_dz + col : nullptr);
    }
  } else if (col < n) {
#pragma unroll 2
    for (int64_t r = r0 + warp; r < r1; r += kGradWarps) {
      const uint16_t* a = dy + r * ld_dy + col;
      const uint16_t* b = ACT == OZ2_ACT_NONE ? nullptr : z + r * ld_z + col;
      uint32_t aw[4] = {0, 0, 0, 0}, bw[4] = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < n) {
          aw[e >> 1] |= static_cast<uint32_t>(__ldg(a + e)) << (16 * (e & 1));
          if (ACT != OZ2_ACT_NONE) bw[e >> 1] |= static_cast<uint32_t>(__ldg(b + e)) << (16 * (e & 1));
        }
      grad8<ACT>(aw, bw, BF16, s, dz ? dz + r * ld_dz + col : nullptr);
    }
  }
  if (partial) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[warp][8 * lane + e] = s[e];
    __syncthreads();
    const int64_t j = static_cast<int64_t>(blockIdx.x) * kGradCols + threadIdx.x;
    if (j < n) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < kGradWarps; ++w) t += sums[w][threadIdx.x];
      partial[blockIdx.y * n + j] = t;
    }
  }
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

int64_t chunk_rows_for(int64_t m, int64_t n) {
  // About four blocks an SM, of at least 32 rows.
  const int64_t across = (n + kGradCols - 1) / kGradCols;
  const int64_t chunks = std::max<int64_t>(1, 4 * static_cast<int64_t>(num_sms()) / across);
  int64_t rows = std::max<int64_t>(32, (m + chunks - 1) / chunks);
  return std::max(rows, (m + 65534) / 65535);  // the grid's second axis
}

template <bool BF16>
auto grad_kernel(int act) {
  return act == OZ2_ACT_RELU        ? act_grad_kernel<OZ2_ACT_RELU, BF16>
         : act == OZ2_ACT_GELU      ? act_grad_kernel<OZ2_ACT_GELU, BF16>
         : act == OZ2_ACT_GELU_TANH ? act_grad_kernel<OZ2_ACT_GELU_TANH, BF16>
         : act == OZ2_ACT_SILU      ? act_grad_kernel<OZ2_ACT_SILU, BF16>
                                    : act_grad_kernel<OZ2_ACT_NONE, BF16>;
}

}  // namespace

int64_t lin_db_chunks(int64_t m, int64_t n) {
  const int64_t r = chunk_rows_for(m, n);
  return std::max<int64_t>(1, (m + r - 1) / r);
}

cudaError_t launch_pack_rows(const PackJob* jobs, int count, int bytes, cudaStream_t st) {
  int64_t pieces = 0;
  for (int i = 0; i < count; ++i) pieces = std::max(pieces, jobs[i].rows * ((jobs[i].cols * bytes + 15) / 16));
  if (pieces == 0) return cudaSuccess;
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((pieces + 255) / 256, 16LL * num_sms()));
  count_launch();
  return launch_dependent(bytes == 1 ? pack_rows_kernel<uint8_t> : pack_rows_kernel<uint16_t>,
                          dim3(blocks, static_cast<unsigned>(count)), dim3(256), 0, st, jobs[0], jobs[count - 1]);
}

cudaError_t launch_act_grad(int64_t m, int64_t n, int type, int act, const void* dy, int64_t ld_dy, const void* z,
                            int64_t ld_z, void* dz, int64_t ld_dz, float* db, float* partial, bool accumulate,
                            cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  const int64_t rows = chunk_rows_for(m, n), chunks = lin_db_chunks(m, n);
  auto aligned = [](const void* p, int64_t ld) { return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(2 * ld)) & 15) == 0; };
  const bool vec = aligned(dy, ld_dy) && (act == OZ2_ACT_NONE || aligned(z, ld_z));
  auto kern = type == OZ2_TYPE_BF16 ? grad_kernel<true>(act) : grad_kernel<false>(act);
  count_launch();
  cudaError_t err = launch_dependent(
      kern, dim3(static_cast<unsigned>((n + kGradCols - 1) / kGradCols), static_cast<unsigned>(chunks)),
      dim3(32 * kGradWarps), 0, st, m, n, rows, vec, static_cast<const uint16_t*>(dy), ld_dy,
      static_cast<const uint16_t*>(z), ld_z, static_cast<uint16_t*>(dz), ld_dz, db ? partial : nullptr);
  if (err != cudaSuccess || !db) return err;
  count_launch();
  return launch_dependent(sum_chunks_kernel, dim3(static_cast<unsigned>((n + 31) / 32)), dim3(256), 0, st, n, chunks,
                          partial, db, accumulate);
}

}  // namespace oz2
