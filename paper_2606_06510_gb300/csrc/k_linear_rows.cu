// The linear layer of a few tokens whose operands lie off the 16-byte grid (an odd
// depth, a view): TMA cannot read such rows, and a copy of the weights would be
// written and read again for a product that is bound by reading them once.
#include <algorithm>

#include "lin_common.cuh"

namespace oz2 {
namespace {

// ---------------------------------------------------------------------------
// 16 of D's columns a block, for up to 8·MT tokens.  The warps of a cluster's blocks
// walk the depth in turn: a lane takes 16-byte pieces of two weight rows and MT
// tokens, each put together from the two aligned words that hold it, and they are
// operands of mma.sync as they are: its sum over the depth may run in any order that
// both operands share, so lane t of a quad's pieces stand for the k's that the
// instruction has it hold.  (Tensor memory would want the rows in shared memory
// first, and 128 of them.)  The warps' sums are joined in shared memory, the blocks' in
// the first one's, in order.
//
// What bounds it: memory, and beside it the aligned loads, two for a piece.  8 tokens ×
// 10240×7569 bf16 take 47 µs (3.3 TB/s), one × 16384×16383 124 (4.3), one × 4096×4097 13,
// one × 333×395 3.6; with the weights copied 78, 259, 17 and 6.  Two pieces ahead and one
// tile of weight rows a warp: one piece ahead 20% slower, three no faster; two tiles of
// rows, for fewer loads of the tokens, 10% slower.
// ---------------------------------------------------------------------------
constexpr int kRowsWarps = 8, kRowsCols = 16, kRowsSplit = 8;
constexpr int kRowsAhead = 2;  // a lane's pieces of a row on their way at once

struct RowsJob {
  const void *x, *w;
  int64_t ldx, ldw, n, k;
  int m;
  LinEpilogue ep;
};

template <int TYPE>
__device__ __forceinline__ void mma_16x8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
#define OZ2_MMA(shape, type)                                                                                  \
  asm("mma.sync.aligned." shape ".row.col.f32." type "." type ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, " \
      "{%0,%1,%2,%3};"                                                                                        \
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])                                                        \
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1))
  if (TYPE == OZ2_TYPE_E4M3) {
    OZ2_MMA("m16n8k32", "e4m3");
  } else if (TYPE == OZ2_TYPE_BF16) {
    OZ2_MMA("m16n8k16", "bf16");
  } else {
    OZ2_MMA("m16n8k16", "f16");
  }
#undef OZ2_MMA
}

// The first `bytes` bytes of a piece, the others 0.
__device__ __forceinline__ uint4 first_bytes(uint4 v, int bytes) {
  auto cut = [&](uint32_t w, int i) {
    const int b = bytes - 4 * i;
    return b >= 4 ? w : b <= 0 ? 0u : w & ((1u << (8 * b)) - 1);
  };
  return make_uint4(cut(v.x, 0), cut(v.y, 1), cut(v.z, 2), cut(v.w, 3));
}

// One value of D from its sum.
__device__ __forceinline__ void finish_one(const LinEpilogue& ep, int64_t token, int64_t col, float z) {
  const bool bf16 = ep.out_type == OZ2_TYPE_BF16;
  const float scale = ep.row_scale ? __ldg(ep.row_scale + token) * __ldg(ep.col_scale + col) : 1.f;
  const float bias = !ep.bias                       ? 0.f
                     : ep.bias_type == OZ2_TYPE_F32 ? __ldg(static_cast<const float*>(ep.bias) + col)
                                                    : load16(static_cast<const uint16_t*>(ep.bias) + col, bf16);
  z = fmaf(z, scale, bias);
  if (ep.pre) static_cast<uint16_t*>(ep.pre)[token * ep.ld_pre + col] = static_cast<uint16_t>(pack16(z, 0.f, bf16));
  switch (ep.act) {
    case OZ2_ACT_RELU: z = activate<OZ2_ACT_RELU>(z); break;
    case OZ2_ACT_GELU: z = activate<OZ2_ACT_GELU>(z); break;
    case OZ2_ACT_GELU_TANH: z = activate<OZ2_ACT_GELU_TANH>(z); break;
    case OZ2_ACT_SILU: z = activate<OZ2_ACT_SILU>(z); break;
    default: break;
  }
  if (ep.add) z += load16(static_cast<const uint16_t*>(ep.add) + token * ep.ld_add + col, bf16);
  static_cast<uint16_t*>(ep.out)[token * ep.ld_out + col] = static_cast<uint16_t>(pack16(z, 0.f, bf16));
}

template <int TYPE, int MT>
__global__ void __launch_bounds__(32 * kRowsWarps, MT == 1 ? 3 : 2) linear_rows_kernel(const __grid_constant__ RowsJob J) {
  using T = typename std::conditional<TYPE == OZ2_TYPE_E4M3, uint8_t, uint16_t>::type;
  constexpr int kVec = 16 / sizeof(T), kStep = 4 * kVec;  // of a lane; of a quad
  constexpr int kCols = kRowsCols, kTokens = 8 * MT;
  constexpr int kParts = 2 + MT;                          // rows that a lane reads
  __shared__ float sums[kRowsWarps][kTokens][kCols];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kCols;
  const T *W = static_cast<const T*>(J.w), *X = static_cast<const T*>(J.x);
  const T *w_end = W + (J.n - 1) * J.ldw + J.k, *x_end = X + (J.m - 1) * J.ldx + J.k;
  // Rows past the last are it again; what comes of them is not stored.
  const T* row[kParts];
#pragma unroll
  for (int i = 0; i < 2; ++i) row[i] = W + min(n0 + g + 8 * i, J.n - 1) * J.ldw + t * kVec;
#pragma unroll
  for (int i = 0; i < MT; ++i) row[2 + i] = X + min(g + 8 * i, J.m - 1) * J.ldx + t * kVec;
  float c[MT][4];
#pragma unroll
  for (int i = 0; i < MT; ++i) c[i][0] = c[i][1] = c[i][2] = c[i][3] = 0.f;
  auto multiply = [&](const uint4 (&v)[kParts]) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      mma_16x8<TYPE>(c[i], v[0].x, v[1].x, v[0].y, v[1].y, v[2 + i].x, v[2 + i].y);
      mma_16x8<TYPE>(c[i], v[0].z, v[1].z, v[0].w, v[1].w, v[2 + i].z, v[2 + i].w);
    }
  };
  const int64_t steps = (J.k + kStep - 1) / kStep, full = J.k / kStep;
  const int64_t stride = static_cast<int64_t>(kRowsAhead) * kRowsWarps * gridDim.y;
  for (int64_t s = kRowsAhead * (static_cast<int64_t>(blockIdx.y) * kRowsWarps + warp); s < steps; s += stride) {
    // Between the first step and the last full one, both words of every piece lie
    // inside its own row.
    if (s > 0 && s + kRowsAhead < full) {
      Words raw[kRowsAhead][kParts];
#pragma unroll
      for (int j = 0; j < kRowsAhead; ++j)
#pragma unroll
        for (int i = 0; i < kParts; ++i) raw[j][i] = load_words16(row[i] + (s + j) * kStep);
#pragma unroll
      for (int j = 0; j < kRowsAhead; ++j) {
        uint4 v[kParts];
#pragma unroll
        for (int i = 0; i < kParts; ++i) v[i] = shift_words16(row[i] + (s + j) * kStep, raw[j][i]);
        multiply(v);
      }
    } else {
#pragma unroll 1
      for (int j = 0; j < kRowsAhead && s + j < steps; ++j) {
        const int64_t left = J.k - (s + j) * kStep - t * kVec;  // elements from this lane's piece on
        const int n = static_cast<int>(max(int64_t(0), min(int64_t(kVec), left)));
        uint4 v[kParts];
        bool inside = n > 0;
#pragma unroll
        for (int i = 0; i < kParts; ++i)
          inside = inside && words_inside(row[i] + (s + j) * kStep, i < 2 ? W : X, i < 2 ? w_end : x_end);
        if (inside) {
          Words raw[kParts];
#pragma unroll
          for (int i = 0; i < kParts; ++i) raw[i] = load_words16(row[i] + (s + j) * kStep);
#pragma unroll
          for (int i = 0; i < kParts; ++i) v[i] = shift_words16(row[i] + (s + j) * kStep, raw[i]);
        } else {
#pragma unroll
          for (int i = 0; i < kParts; ++i)
            v[i] = n > 0 ? load16_any(row[i] + (s + j) * kStep, i < 2 ? W : X, i < 2 ? w_end : x_end, n)
                         : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kParts; ++i) v[i] = first_bytes(v[i], n * static_cast<int>(sizeof(T)));
        __syncwarp();
        multiply(v);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[warp][8 * i + 2 * t + (e & 1)][g + 8 * (e >> 1)] = c[i][e];
  __syncthreads();
  const int at = threadIdx.x, token = at / kCols;  // a value of D a thread
  if (MT == 1 && gridDim.y == 1 && token >= kTokens) return;
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < kRowsWarps; ++i) z += sums[i][token % kTokens][at % kCols];
  if (gridDim.y > 1) {
    __syncthreads();
    float* mine = &sums[0][0][0] + at;  // (8 warps' sums are at least one value a thread)
    *mine = z;
    cluster_sync_all();
    if (blockIdx.y == 0) {
      z = 0.f;
      for (uint32_t r = 0; r < gridDim.y; ++r) {
        float v;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(mapa_shared(smem_u32(mine), r)));
        z += v;
      }
    }
    cluster_sync_all();  // no block leaves while the first reads its sums
    if (blockIdx.y > 0) return;
  }
  if (token < J.m && n0 + at % kCols < J.n) finish_one(J.ep, token, n0 + at % kCols, z);
}

template <int TYPE>
auto rows_kernel(int64_t m) {
  return m <= 8 ? linear_rows_kernel<TYPE, 1> : linear_rows_kernel<TYPE, 2>;
}

}  // namespace

cudaError_t launch_linear_rows(const LinProduct& p, int type, cudaStream_t st) {
  const RowsJob job{p.p, p.q, p.ldp, p.ldq, p.cols, p.depth, static_cast<int>(p.rows), p.ep};
  auto kern = type == OZ2_TYPE_E4M3   ? rows_kernel<OZ2_TYPE_E4M3>(p.rows)
              : type == OZ2_TYPE_BF16 ? rows_kernel<OZ2_TYPE_BF16>(p.rows)
                                      : rows_kernel<OZ2_TYPE_F16>(p.rows);
  // Few columns: their depth over a cluster, while its warps have two turns each.
  const int64_t blocks = (p.cols + kRowsCols - 1) / kRowsCols;
  const int64_t turns = p.depth * type_bytes(type) / (64 * kRowsAhead * kRowsWarps);
  int split = 1;
  while (split < kRowsSplit && 2 * split * blocks <= 2 * num_sms() && turns >= 4 * split) split *= 2;
  count_launch();
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(split));
  cfg.blockDim = dim3(32 * kRowsWarps);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = static_cast<unsigned>(split);
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, job);
}

}  // namespace oz2
