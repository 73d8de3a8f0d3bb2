// Layer norm, forward (norm_rows.cuh has the formulas and how rows are read).
#include "norm_rows.cuh"

namespace oz2 {
namespace {

using ForwardKernel = Kernel<void (*)(NormArgs)>;

// ---------------------------------------------------------------------------
// Forward.  TPR threads to a row, VPT 16-byte pieces of it to a thread: up to 16 values, two
// to an instruction.  Groups of threads walk over rows, the next ones on their way meanwhile.
//
// Memory bounds it: 65536×1024 f32 100 µs (5.4 TB/s; a block to each few rows, loaded when it came
// to them, 254), 16384×4096 bf16 58 (4.7).  Rows over 4096 wait for their two sums: one or two
// groups an SM, with their weights in shared memory (8192² bf16 62 µs, 4096×16384 62; read again for
// each row from L2, 84 and 96); rows off the grid are instructions, 2.3 times those of rows on it
// (shifts, masks and stores by single elements, five times as many): 16384×777 f16 39, at 776 20, 8 at
// the copy rate.
// ---------------------------------------------------------------------------
constexpr int kForwardThreads = 256;
// Where the weights are: in a thread's registers; of wide rows, whose threads have not enough for
// them, as FP32 in shared memory, but where those and the rows together do not fit.
enum Weights { kInRegisters, kInShared, kInMemory };
template <int TYPE, int TPR, int VPT, bool ALIGNED>
struct ForwardShape {
  static constexpr int cols = TPR * VPT * Elem<TYPE>::V;
  static constexpr Weights weights = cols <= 4096 ? kInRegisters : cols <= 8192 || TYPE != OZ2_TYPE_F32 ? kInShared : kInMemory;
  static constexpr int block = weights == kInRegisters ? norm_block(TPR, kForwardThreads) : 1024;
  static constexpr int blocks = block == 256 ? 3 : 1;  // an SM
  using Rows = Pieces<TYPE, TPR, VPT, block, ALIGNED>;
  static constexpr int weight_bytes = weights == kInShared ? 2 * 4 * cols : 0;
  static constexpr int stages = norm_stages(Rows::kBytes, 200 * 1024 / blocks - weight_bytes);
  static constexpr int smem = weight_bytes + Rows::kBytes * stages;
};

template <int TYPE, int TPR, int VPT, bool ALIGNED>
__global__ void __launch_bounds__(ForwardShape<TYPE, TPR, VPT, ALIGNED>::block, ForwardShape<TYPE, TPR, VPT, ALIGNED>::blocks)
    norm_kernel(NormArgs a) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  using Shape = ForwardShape<TYPE, TPR, VPT, ALIGNED>;
  using Rows = typename Shape::Rows;
  constexpr int V = X::V, H = V / 2, kGroups = Shape::block / TPR, STAGES = Shape::stages;
  constexpr bool KEEP = Shape::weights == kInRegisters, SHARED = Shape::weights == kInShared;
  __shared__ float exchange[kGroups][TPR < 32 ? 1 : 2 * TPR / 32];
  extern __shared__ __align__(16) uint8_t norm_all[];
  uint8_t* norm_smem = norm_all + Shape::weight_bytes;
  pdl_trigger();
  pdl_wait();
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
  const T* src = static_cast<const T*>(a.x);
  const Rows in{src, src + (a.m - 1) * a.ldx + a.k, a.k, t};
  const float inv_k = 1.f / static_cast<float>(a.k);
  RowSum<TPR, 1> rows{exchange[group], group, 0};
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kGroups, first = static_cast<int64_t>(blockIdx.x) * kGroups + group;
  auto fetch = [&](int64_t r, int stage) {
    if (r < a.m) in.fetch(norm_smem + stage * Rows::kBytes, src + r * a.ldx);
    fetch_commit();
  };
#pragma unroll
  for (int s = 0; s < STAGES; ++s) fetch(first + s * stride, s);
  const Two one = two(1.f, 1.f), zero = two(0.f, 0.f);
  auto vector = [&](const void* p, int i, Two none, Two (&to)[H]) {
    float f[V];
    if (p && in.there(i)) load_vector<TYPE>(p, a.wtype, in.col(i), in.there(i), a.k, f);
#pragma unroll
    for (int e = 0; e < H; ++e) to[e] = p && in.there(i) ? two(f[2 * e], f[2 * e + 1]) : none;
  };
  Two w[KEEP ? VPT : 1][H], b[KEEP ? VPT : 1][H];
  if (KEEP) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) vector(a.w, i, one, w[KEEP ? i : 0]), vector(a.b, i, zero, b[KEEP ? i : 0]);
  }
  // In shared memory, four values of each piece side by side: w's, then b's.
  constexpr int kPlane = TPR * VPT;
  auto plane = [&](int which, int i, int e) { return reinterpret_cast<float4*>(norm_all) + (which * (V / 4) + e / 2) * kPlane + i * TPR + t; };
  if (SHARED) {
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        Two v[H];
        if (group == 0) {
          vector(which ? a.b : a.w, i, which ? zero : one, v);
#pragma unroll
          for (int e = 0; e < H; e += 2) {
            const float2 p = both(v[e]), q = both(v[e + 1]);
            *plane(which, i, e) = make_float4(p.x, p.y, q.x, q.y);
          }
        }
      }
    __syncthreads();
  }
  auto shared_vector = [&](int which, int i, Two (&to)[H]) {
#pragma unroll
    for (int e = 0; e < H; e += 2) {
      const float4 v = *plane(which, i, e);
      to[e] = two(v.x, v.y), to[e + 1] = two(v.z, v.w);
    }
  };
  int stage = 0;
  for (int64_t r = first; r - groups_before<TPR>() < a.m; r += stride) {
    const bool live = TPR >= 32 || r < a.m;
    fetch_wait<STAGES - 1>();
    Rows::meet();
    Two x[VPT][H], s = zero;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      unpack2<TYPE>(in.read(norm_smem + stage * Rows::kBytes, src + r * a.ldx, i), x[i]);  // (zeros past the row's end)
#pragma unroll
      for (int e = 0; e < H; ++e) s = s + x[i][e];
    }
    Rows::meet();
    fetch(r + STAGES * stride, stage);
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    float mean = 0.f, sum[1];
    if (a.center) {
      const float2 p = both(s);
      sum[0] = p.x + p.y;
      rows.sum(sum);
      mean = sum[0] * inv_k;
    }
    const Two less = two(-mean, -mean);
    s = zero;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int n = in.there(i);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        x[i][e] = x[i][e] + less;
        if (n < V) {  // the row's end: what is past it deviates by nothing
          const float2 p = both(x[i][e]);
          x[i][e] = two(2 * e < n ? p.x : 0.f, 2 * e + 1 < n ? p.y : 0.f);
        }
        s = fma(x[i][e], x[i][e], s);
      }
    }
    const float2 p = both(s);
    sum[0] = p.x + p.y;
    rows.sum(sum);
    const float rstd = 1.f / sqrtf(fmaf(sum[0], inv_k, a.eps));
    if (t == 0 && live) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    const Two scale = two(rstd, rstd);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int n = in.there(i);
      float f[V];
      Two wi[H], bi[H];
      if (SHARED) {
        shared_vector(0, i, wi), shared_vector(1, i, bi);
      } else if (!KEEP) {
        vector(a.w, i, one, wi), vector(a.b, i, zero, bi);
      }
#pragma unroll
      for (int e = 0; e < H; ++e) {
        const float2 q = both(fma(x[i][e] * scale, KEEP ? w[KEEP ? i : 0][e] : wi[e], KEEP ? b[KEEP ? i : 0][e] : bi[e]));
        f[2 * e] = q.x, f[2 * e + 1] = q.y;
      }
      store_piece<ALIGNED>(static_cast<T*>(a.y) + r * a.ldy + (n ? in.col(i) : 0), X::pack(f), live ? n : 0);
    }
  }
  fetch_wait<0>();
}

// Rows too long for registers: a block to a row, which it reads again for each of the
// two sums and the result (from L2, mostly).  Not as memory that nothing writes: y may be x.
template <int TYPE>
__global__ void __launch_bounds__(kNormThreads) norm_long_kernel(NormArgs a) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  constexpr int V = X::V;
  __shared__ float exchange[2 * kNormThreads / 32];
  pdl_trigger();
  pdl_wait();
  const T* src = static_cast<const T*>(a.x);
  const T* end = src + (a.m - 1) * a.ldx + a.k;
  const float inv_k = 1.f / static_cast<float>(a.k);
  RowSum<kNormThreads, 1> rows{exchange, 0, 0};
  for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
    auto each = [&](auto work) {
      for (int64_t col = static_cast<int64_t>(threadIdx.x) * V; col < a.k; col += kNormThreads * V) {
        const int n = static_cast<int>(min(int64_t(V), a.k - col));
        float x[V];
        X::unpack(load_piece<false, false>(src + r * a.ldx + col, src, end, n), x);
        work(col, n, x);
      }
    };
    float s[1] = {0.f}, mean = 0.f;
    if (a.center) {
      each([&](int64_t, int n, float (&x)[V]) {
#pragma unroll
        for (int e = 0; e < V; ++e) s[0] += e < n ? x[e] : 0.f;
      });
      rows.sum(s);
      mean = s[0] * inv_k;
    }
    s[0] = 0.f;
    each([&](int64_t, int n, float (&x)[V]) {
#pragma unroll
      for (int e = 0; e < V; ++e) s[0] += e < n ? (x[e] - mean) * (x[e] - mean) : 0.f;
    });
    rows.sum(s);
    const float rstd = 1.f / sqrtf(fmaf(s[0], inv_k, a.eps));
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    each([&](int64_t col, int n, float (&x)[V]) {
      float w[V], b[V];
      if (a.w) load_vector<TYPE>(a.w, a.wtype, col, n, a.k, w);
      if (a.b) load_vector<TYPE>(a.b, a.wtype, col, n, a.k, b);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = (x[e] - mean) * rstd * (a.w ? w[e] : 1.f) + (a.b ? b[e] : 0.f);
      store16_any(static_cast<T*>(a.y) + r * a.ldy + col, X::pack(x), n, false);
    });
  }
}

template <int TYPE, bool ALIGNED>
struct Forward {
  template <int TPR, int VPT>
  struct K {
    static ForwardKernel f() {
      constexpr int kVpt = VPT * Elem<TYPE>::V <= 16 ? VPT : 2;
      using Shape = ForwardShape<TYPE, TPR, kVpt, ALIGNED>;
      return {norm_kernel<TYPE, TPR, kVpt, ALIGNED>, Shape::block, Shape::smem};
    }
  };
};
template <int TYPE>
cudaError_t forward(const NormArgs& a, cudaStream_t st) {
  const int es = type_bytes(TYPE);
  const NormShape s = forward_shape(a.m, a.k, TYPE);
  count_launch();
  if (!s.tpr) {
    const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(a.m, 4 * num_sms()));
    return launch_dependent(norm_long_kernel<TYPE>, dim3(blocks), dim3(kNormThreads), 0, st, a);
  }
  const bool aligned = rows_on16(a.x, a.ldx, es) && rows_on16(a.y, a.ldy, es);
  const ForwardKernel f = aligned ? by_shape<Forward<TYPE, true>::template K>(s) : by_shape<Forward<TYPE, false>::template K>(s);
  const cudaError_t err = allow_smem(reinterpret_cast<const void*>(f.kernel), f.smem);
  if (err != cudaSuccess) return err;
  const int groups = f.block / s.tpr;
  const int64_t blocks = std::min<int64_t>((a.m + groups - 1) / groups, (f.block == kForwardThreads ? 3 : 1) * static_cast<int64_t>(num_sms()));
  return launch_dependent(f.kernel, dim3(static_cast<unsigned>(blocks)), dim3(f.block), f.smem, st, a);
}

}  // namespace

cudaError_t launch_layer_norm(const NormArgs& a, int type, cudaStream_t st) {
  return type == OZ2_TYPE_F32    ? forward<OZ2_TYPE_F32>(a, st)
         : type == OZ2_TYPE_BF16 ? forward<OZ2_TYPE_BF16>(a, st)
                                 : forward<OZ2_TYPE_F16>(a, st);
}

}  // namespace oz2
