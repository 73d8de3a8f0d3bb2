// Layer norm's gradient (norm_rows.cuh has the formulas and how rows are read).
#include "norm_rows.cuh"

namespace oz2 {
namespace {

using BackwardKernel = Kernel<void (*)(NormGradArgs, float*)>;

// ---------------------------------------------------------------------------
// Backward.  As forward, with groups that walk over rows: a thread's columns are the
// same in every row, so it adds up dw and db of them in registers; a block's groups add
// theirs in shared memory, in order, into the block's row of `parts`, and
// join_parts_kernel adds up the blocks'.
//
// Memory bounds it: 16384×4096 bf16 with a skip connection, 537 MB, take 101 µs, 5.3 TB/s (each
// row loaded when it came and the sums one value an instruction: 151), 65536×1024 f32 162 (6.6).
// A thread's 16 values of a row stay in registers between the sums and dx; the 1024 threads of
// rows over 8192 have registers for the columns' sums alone and form them a second time
// (4096×16384 bf16 184 µs, f32 244).
// ---------------------------------------------------------------------------
template <int TYPE, int TPR, int VPT, bool ALIGNED>
constexpr int backward_stages() {
  return norm_stages(3 * Pieces<TYPE, TPR, VPT, norm_block(TPR, kNormThreads), ALIGNED>::kBytes, 208 * 1024);
}

template <int TYPE, int TPR, int VPT, bool ALIGNED>
__global__ void __launch_bounds__(norm_block(TPR, kNormThreads), 1) norm_grad_kernel(NormGradArgs a, float* __restrict__ parts) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  constexpr int V = X::V, H = V / 2, kBlock = norm_block(TPR, kNormThreads), kGroups = kBlock / TPR;
  using Rows = Pieces<TYPE, TPR, VPT, kBlock, ALIGNED>;
  constexpr int STAGES = backward_stages<TYPE, TPR, VPT, ALIGNED>();
  constexpr bool KEEP = TPR < 1024;
  __shared__ float exchange[kGroups][TPR < 32 ? 1 : 4 * TPR / 32];
  // The rows' pieces, and after them the groups' columns of dw and db.
  extern __shared__ __align__(16) uint8_t norm_smem[];
  float* columns = reinterpret_cast<float*>(norm_smem);
  pdl_trigger();
  pdl_wait();
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
  const T *dy = static_cast<const T*>(a.dy), *x = static_cast<const T*>(a.x), *res = static_cast<const T*>(a.r);
  const Rows in_dy{dy, dy + (a.m - 1) * a.lddy + a.k, a.k, t}, in_x{x, x + (a.m - 1) * a.ldx + a.k, a.k, t},
      in_r{res, res + (a.m - 1) * a.ldr + a.k, a.k, t};
  const float inv_k = 1.f / static_cast<float>(a.k);
  RowSum<TPR, 2> rows{exchange[group], group, 0};
  auto col = [&](int i) { return in_x.col(i); };
  auto there = [&](int i) { return in_x.there(i); };
  const Two zero = two(0.f, 0.f), one = two(1.f, 1.f);
  Two dw[VPT][H], db[VPT][H], w[KEEP ? VPT : 1][H];
  auto weights = [&](int i, Two (&to)[H]) {
    float f[V];
    if (a.w && there(i)) load_vector<TYPE>(a.w, a.wtype, col(i), there(i), a.k, f);
#pragma unroll
    for (int e = 0; e < H; ++e) to[e] = a.w && there(i) ? two(f[2 * e], f[2 * e + 1]) : one;
  };
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    if (KEEP) weights(i, w[KEEP ? i : 0]);
#pragma unroll
    for (int e = 0; e < H; ++e) dw[i][e] = db[i][e] = zero;
  }
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kGroups, first = static_cast<int64_t>(blockIdx.x) * kGroups + group;
  auto memory = [&](int stage, int which) { return norm_smem + (stage * 3 + which) * Rows::kBytes; };
  auto fetch = [&](int64_t r, int stage) {
    if (r < a.m) {
      in_dy.fetch(memory(stage, 0), dy + r * a.lddy);
      in_x.template fetch<true>(memory(stage, 1), x + r * a.ldx);
      if (res) in_r.fetch(memory(stage, 2), res + r * a.ldr);
    }
    fetch_commit();
  };
#pragma unroll
  for (int s = 0; s < STAGES; ++s) fetch(first + s * stride, s);
  float mean = 0.f, rstd = 0.f;
  auto statistics = [&](int64_t r) {
    mean = r < a.m && a.mean ? __ldg(a.mean + r) : 0.f, rstd = r < a.m ? __ldg(a.rstd + r) : 0.f;
  };
  statistics(first);
  int stage = 0;
  for (int64_t r = first; r - groups_before<TPR>() < a.m; r += stride) {
    const bool live = TPR >= 32 || r < a.m;
    fetch_wait<STAGES - 1>();
    Rows::meet();
    const Two less = two(-mean, -mean), scale = two(rstd, rstd);
    // dy, g = dy·w and x̂ of a piece.  Past the row's end dy is zero, and x̂ counts for nothing as
    // long as it is a number: of a whole piece it is the row's first one's; of elements -mean·rstd,
    // which may be infinite (rows of one large value), and is then left out.
    const bool wild = !ALIGNED && !(fabsf(mean * rstd) < INFINITY);
    auto values = [&](int i, Two (&d)[H], Two (&g)[H], Two (&h)[H]) {
      const uint4 none = make_uint4(0, 0, 0, 0);
      unpack2<TYPE>(live ? in_dy.read(memory(stage, 0), dy + r * a.lddy, i) : none, d);
      unpack2<TYPE>(live ? in_x.read(memory(stage, 1), x + r * a.ldx, i) : none, h);
      Two own[H];
      if (!KEEP) weights(i, own);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        h[e] = (h[e] + less) * scale;
        g[e] = d[e] * (KEEP ? w[KEEP ? i : 0][e] : own[e]);
      }
      if (wild) {
        const int n = there(i);
#pragma unroll
        for (int e = 0; e < H; ++e) {
          const float2 p = both(h[e]);
          h[e] = two(2 * e < n ? p.x : 0.f, 2 * e + 1 < n ? p.y : 0.f);
        }
      }
    };
    Two s0 = zero, s1 = zero, kg[KEEP ? VPT : 1][H], kh[KEEP ? VPT : 1][H];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      Two d[H], gi[H], hi[H];
      Two(&g)[H] = KEEP ? kg[KEEP ? i : 0] : gi;
      Two(&h)[H] = KEEP ? kh[KEEP ? i : 0] : hi;
      values(i, d, g, h);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        dw[i][e] = fma(d[e], h[e], dw[i][e]);
        db[i][e] = db[i][e] + d[e];
        s0 = s0 + g[e];
        s1 = fma(g[e], h[e], s1);
      }
    }
    if (a.dx) {
      const float2 p0 = both(s0), p1 = both(s1);
      float s[2] = {p0.x + p0.y, p1.x + p1.y};
      rows.sum(s);
      const float level = a.mean ? -rstd * (s[0] * inv_k) : 0.f, along = -rstd * (s[1] * inv_k);
      const Two level2 = two(level, level), along2 = two(along, along);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int n = there(i);
        Two d[H], gi[H], hi[H];
        Two(&g)[H] = KEEP ? kg[KEEP ? i : 0] : gi;
        Two(&h)[H] = KEEP ? kh[KEEP ? i : 0] : hi;
        if (!KEEP) values(i, d, g, h);
#pragma unroll
        for (int e = 0; e < H; ++e) d[e] = fma(h[e], along2, fma(g[e], scale, level2));
        if (res) {
          Two o[H];
          unpack2<TYPE>(in_r.read(memory(stage, 2), res + r * a.ldr, i), o);
#pragma unroll
          for (int e = 0; e < H; ++e) d[e] = d[e] + o[e];
        }
        float y[V];
#pragma unroll
        for (int e = 0; e < H; ++e) {
          const float2 f = both(d[e]);
          y[2 * e] = f.x, y[2 * e + 1] = f.y;
        }
        store_piece<ALIGNED>(static_cast<T*>(a.dx) + r * a.lddx + (n ? col(i) : 0), X::pack(y), live ? n : 0);
      }
    }
    statistics(r + stride);
    Rows::meet();
    fetch(r + STAGES * stride, stage);
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
  fetch_wait<0>();
  __syncthreads();  // the pieces' memory becomes the columns'
  if (!parts) return;
  // The groups' columns in shared memory, dw's and then db's, and their sums in the groups' order.
  constexpr int kCols = TPR * VPT * V;
  auto put = [&](const Two (&v)[VPT][H], float* row) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < H; e += 2) {
        const float2 p = both(v[i][e]), q = both(v[i][e + 1]);
        *reinterpret_cast<float4*>(row + (t + i * TPR) * V + 2 * e) = make_float4(p.x, p.y, q.x, q.y);
      }
  };
  put(dw, columns + group * kCols);
  put(db, columns + (kGroups + group) * kCols);
  __syncthreads();
  float* to = parts + static_cast<int64_t>(blockIdx.x) * 2 * a.k;
  for (int c = threadIdx.x; c < a.k; c += kBlock) {
    float w_sum = columns[c], b_sum = columns[kGroups * kCols + c];
#pragma unroll
    for (int q = 1; q < kGroups; ++q) w_sum += columns[q * kCols + c], b_sum += columns[(kGroups + q) * kCols + c];
    to[c] = w_sum;
    to[a.k + c] = b_sum;
  }
}

// Long rows: dx by a block to a row, which reads it twice.
template <int TYPE>
__global__ void __launch_bounds__(kNormThreads) norm_grad_long_kernel(NormGradArgs a) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  constexpr int V = X::V;
  __shared__ float exchange[4 * kNormThreads / 32];
  pdl_trigger();
  pdl_wait();
  const T *dy = static_cast<const T*>(a.dy), *x = static_cast<const T*>(a.x), *res = static_cast<const T*>(a.r);
  const T *dy_end = dy + (a.m - 1) * a.lddy + a.k, *x_end = x + (a.m - 1) * a.ldx + a.k,
          *r_end = res + (a.m - 1) * a.ldr + a.k;
  const float inv_k = 1.f / static_cast<float>(a.k);
  RowSum<kNormThreads, 2> rows{exchange, 0, 0};
  for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
    const float mean = a.mean ? __ldg(a.mean + r) : 0.f, rstd = __ldg(a.rstd + r);
    auto each = [&](auto work) {
      for (int64_t col = static_cast<int64_t>(threadIdx.x) * V; col < a.k; col += kNormThreads * V) {
        const int n = static_cast<int>(min(int64_t(V), a.k - col));
        float g[V], h[V], w[V];
        X::unpack(load_piece<false>(dy + r * a.lddy + col, dy, dy_end, n), g);
        X::unpack(load_piece<false>(x + r * a.ldx + col, x, x_end, n), h);
        if (a.w) load_vector<TYPE>(a.w, a.wtype, col, n, a.k, w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (a.w) g[e] *= w[e];
          g[e] = e < n ? g[e] : 0.f;
          h[e] = e < n ? (h[e] - mean) * rstd : 0.f;
        }
        work(col, n, g, h);
      }
    };
    float s[2] = {0.f, 0.f};
    each([&](int64_t, int, float (&g)[V], float (&h)[V]) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s[0] += g[e];
        s[1] = fmaf(g[e], h[e], s[1]);
      }
    });
    rows.sum(s);
    const float level = a.mean ? s[0] * inv_k : 0.f, along = s[1] * inv_k;
    each([&](int64_t col, int n, float (&g)[V], float (&h)[V]) {
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = 0.f;
      if (res) X::unpack(load_piece<false, false>(res + r * a.ldr + col, res, r_end, n), o);
#pragma unroll
      for (int e = 0; e < V; ++e) g[e] = rstd * (g[e] - level - h[e] * along) + o[e];
      store16_any(static_cast<T*>(a.dx) + r * a.lddx + col, X::pack(g), n, false);
    });
  }
}
// Their dw and db: a warp's lanes are 32·V columns, a block's warps walk over a chunk of
// rows.
template <int TYPE>
__global__ void __launch_bounds__(256) norm_columns_kernel(NormGradArgs a, int64_t chunk, float* __restrict__ parts) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  constexpr int V = X::V;
  __shared__ float sums[8][2][32 * V];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const T *dy = static_cast<const T*>(a.dy), *x = static_cast<const T*>(a.x);
  const T *dy_end = dy + (a.m - 1) * a.lddy + a.k, *x_end = x + (a.m - 1) * a.ldx + a.k;
  const int64_t col = (static_cast<int64_t>(blockIdx.x) * 32 + lane) * V, r1 = min(a.m, (blockIdx.y + 1) * chunk);
  const int n = static_cast<int>(min(int64_t(V), a.k - col));
  float dw[V], db[V];
#pragma unroll
  for (int e = 0; e < V; ++e) dw[e] = db[e] = 0.f;
  if (n > 0) {
#pragma unroll 2
    for (int64_t r = blockIdx.y * chunk + warp; r < r1; r += 8) {
      float g[V], h[V];
      X::unpack(load_piece<false>(dy + r * a.lddy + col, dy, dy_end, n), g);
      X::unpack(load_piece<false>(x + r * a.ldx + col, x, x_end, n), h);
      const float mean = a.mean ? __ldg(a.mean + r) : 0.f, rstd = __ldg(a.rstd + r);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dw[e] = fmaf(g[e], (h[e] - mean) * rstd, dw[e]);
        db[e] += g[e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) sums[warp][0][lane * V + e] = dw[e], sums[warp][1][lane * V + e] = db[e];
  __syncthreads();
  for (int c = threadIdx.x; c < 64 * V; c += 256) {
    const int which = c / (32 * V), in = c % (32 * V);
    const int64_t j = static_cast<int64_t>(blockIdx.x) * 32 * V + in;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += sums[w][which][in];
    if (j < a.k) parts[static_cast<int64_t>(blockIdx.y) * 2 * a.k + which * a.k + j] = s;
  }
}

// dw and db from the blocks' rows of parts, in their order: a warp's lanes are columns,
// its 8 warps each add up every eighth row.
__global__ void __launch_bounds__(256) join_parts_kernel(int64_t k, int count, const float* __restrict__ parts,
                                                         float* __restrict__ dw, float* __restrict__ db, int accumulate) {
  __shared__ float sums[8][32];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t j = blockIdx.x * 32LL + lane;
  float* out = blockIdx.y ? db : dw;
  if (!out) return;
  const float* p = parts + blockIdx.y * k + j;
  float t = 0.f;
  if (j < k) {
#pragma unroll 8
    for (int c = warp; c < count; c += 8) t += p[c * 2 * k];
  }
  sums[warp][lane] = t;
  __syncthreads();
  if (warp == 0 && j < k) {
    t = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += sums[w][lane];
    out[j] = accumulate ? out[j] + t : t;
  }
}

template <int TYPE, bool ALIGNED>
struct Backward {
  template <int TPR, int VPT>
  struct K {
    static BackwardKernel f() {
      constexpr int kVpt = VPT * Elem<TYPE>::V <= 16 ? VPT : 2, kBlock = norm_block(TPR, kNormThreads);
      constexpr size_t columns = 2 * sizeof(float) * kBlock * kVpt * Elem<TYPE>::V;
      constexpr size_t pieces = 3 * Pieces<TYPE, TPR, kVpt, kBlock, ALIGNED>::kBytes * backward_stages<TYPE, TPR, kVpt, ALIGNED>();
      return {norm_grad_kernel<TYPE, TPR, kVpt, ALIGNED>, kBlock, pieces > columns ? pieces : columns};
    }
  };
};

constexpr int64_t kColumnRows = 64;  // rows of a long row's chunk, at least

int64_t long_chunk(int64_t m) { return std::max<int64_t>(kColumnRows, (m + 511) / 512); }
int64_t grad_blocks(const NormGradArgs& a, NormShape s) {
  if (!s.tpr) return (a.m + long_chunk(a.m) - 1) / long_chunk(a.m);
  const int groups = norm_block(s.tpr, kNormThreads) / s.tpr;
  return std::min<int64_t>((a.m + groups - 1) / groups, num_sms());
}

template <int TYPE>
cudaError_t backward(const NormGradArgs& a, float* parts, cudaStream_t st) {
  const int es = type_bytes(TYPE);
  const NormShape s = backward_shape(a.k, TYPE);
  const bool want = a.dw || a.db;
  const int64_t blocks = grad_blocks(a, s);
  cudaError_t err = cudaSuccess;
  if (!s.tpr) {
    if (a.dx) {
      count_launch();
      err = launch_dependent(norm_grad_long_kernel<TYPE>, dim3(static_cast<unsigned>(std::min<int64_t>(a.m, 4 * num_sms()))),
                             dim3(kNormThreads), 0, st, a);
    }
    if (want && err == cudaSuccess) {
      const int64_t across = (a.k + 32 * Elem<TYPE>::V - 1) / (32 * Elem<TYPE>::V);
      count_launch();
      err = launch_dependent(norm_columns_kernel<TYPE>, dim3(static_cast<unsigned>(across), static_cast<unsigned>(blocks)),
                             dim3(256), 0, st, a, long_chunk(a.m), parts);
    }
  } else {
    const bool aligned = a.k % Elem<TYPE>::V == 0 && rows_on16(a.dy, a.lddy, es) && rows_on16(a.x, a.ldx, es) && (!a.r || rows_on16(a.r, a.ldr, es)) &&
                         (!a.dx || rows_on16(a.dx, a.lddx, es));
    const BackwardKernel f = aligned ? by_shape<Backward<TYPE, true>::template K>(s) : by_shape<Backward<TYPE, false>::template K>(s);
    err = allow_smem(reinterpret_cast<const void*>(f.kernel), f.smem);
    if (err != cudaSuccess) return err;
    count_launch();
    err = launch_dependent(f.kernel, dim3(static_cast<unsigned>(blocks)), dim3(f.block), f.smem, st, a, want ? parts : nullptr);
  }
  if (err != cudaSuccess || !want) return err;
  count_launch();
  return launch_dependent(join_parts_kernel, dim3(static_cast<unsigned>((a.k + 31) / 32), 2), dim3(256), 0, st, a.k,
                          static_cast<int>(blocks), static_cast<const float*>(parts), a.dw, a.db, a.accumulate);
}

}  // namespace

size_t layer_norm_grad_scratch(const NormGradArgs& a, int type) {
  if (!a.dw && !a.db) return 0;
  return sizeof(float) * 2 * static_cast<size_t>(a.k) * grad_blocks(a, backward_shape(a.k, type));
}

cudaError_t launch_layer_norm_grad(const NormGradArgs& a, int type, void* scratch, cudaStream_t st) {
  float* parts = static_cast<float*>(scratch);
  return type == OZ2_TYPE_F32    ? backward<OZ2_TYPE_F32>(a, parts, st)
         : type == OZ2_TYPE_BF16 ? backward<OZ2_TYPE_BF16>(a, parts, st)
                                 : backward<OZ2_TYPE_F16>(a, parts, st);
}

}  // namespace oz2
