// Layer norm over a row's k features, forward and backward:
//   μ = mean x (0 where not centred)   r = 1/√(mean (x-μ)² + ε)   x̂ = (x-μ)·r
//   y  = x̂·w + b
//   dx = r·(g - mean g - x̂·mean(g·x̂)) + R   with g = dy·w (no mean g where not centred)
//   dw = Σ_t dy·x̂      db = Σ_t dy
// A row is held in registers: its mean first, then the squares of what deviates from it
// (two passes over registers, none over memory; the difference of E x² and μ² would lose
// what a large mean takes).
#include <algorithm>

#include "lm_common.cuh"

namespace oz2 {
namespace {

constexpr int kNormThreads = 512;  // of the blocks whose rows take that many threads

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The N sums over a row's TPR threads, the same bits in each of them.  Groups of more
// than one warp exchange theirs in `at` (two sets, taken in turn: a set is written again
// two barriers later) behind a barrier of their own.
template <int TPR, int N>
struct RowSum {
  static constexpr int kWarps = TPR / 32;
  float* at;
  int group, turn;
  __device__ __forceinline__ void sum(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if (kWarps == 1) return;
    float* s = at + turn * (kWarps * N);
    turn ^= 1;
    const int w = (threadIdx.x >> 5) % kWarps, lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[w * N + i] = v[i];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < kWarps ? s[lane * N + i] : 0.f);
  }
};

// V values of a vector of the rows' type or F32, from its element `col` on.
template <int TYPE>
__device__ __forceinline__ void load_vector(const void* p, int wtype, int64_t col, int n, int64_t k,
                                            float (&f)[Elem<TYPE>::V]) {
  using X = Elem<TYPE>;
  if (TYPE != OZ2_TYPE_F32 && wtype == OZ2_TYPE_F32) {
    const float* s = static_cast<const float*>(p) + col;
    if (n >= X::V && (reinterpret_cast<uintptr_t>(s) & 15) == 0) {
#pragma unroll
      for (int h = 0; h < X::V; h += 4) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(s + h));
        f[h] = v.x, f[h + 1] = v.y, f[h + 2] = v.z, f[h + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < X::V; ++e) f[e] = e < n ? __ldg(s + e) : 0.f;
    }
  } else {
    const typename X::T* s = static_cast<const typename X::T*>(p);
    if (reinterpret_cast<uintptr_t>(s) & 15) {
      X::unpack(load_piece<false>(s + col, s, s + k, n), f);
    } else {
      X::unpack(load_piece<true>(s + col, s, s + k, n), f);
    }
  }
}

template <int TYPE>
__device__ __forceinline__ void unpack2(uint4 v, Two (&t)[Elem<TYPE>::V / 2]) {
  float f[Elem<TYPE>::V];
  Elem<TYPE>::unpack(v, f);
#pragma unroll
  for (int e = 0; e < Elem<TYPE>::V / 2; ++e) t[e] = two(f[2 * e], f[2 * e + 1]);
}

// ---------------------------------------------------------------------------
// Rows on their way through shared memory (cp.async): each thread fetches its own 16-byte
// pieces of a row that is worked on later and reads them then, so no barrier is wanted.  Rows
// off the 16-byte grid come as the aligned words around them: a thread fetches the one in
// which its piece begins, and the one after it is the next lane's; the last lane of a warp,
// and of the row, fetches that too.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void fetch_async(uint32_t to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void fetch_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// A thread's pieces of one row, VPT of them, TPR pieces apart, t its number among the row's
// threads; `at` is the memory of a tensor's rows in one stage.
template <int TYPE, int TPR, int VPT, int BLOCK, bool ALIGNED>
struct Pieces {
  using X = Elem<TYPE>;
  using T = typename X::T;
  static constexpr int V = X::V, kWords = BLOCK + (ALIGNED ? 0 : BLOCK / 32), kBytes = VPT * kWords * 16;
  const T *base, *end;
  int64_t k;
  int t;
  __device__ __forceinline__ int64_t col(int i) const { return static_cast<int64_t>(t + i * TPR) * V; }
  __device__ __forceinline__ int there(int i) const {
    return static_cast<int>(max(int64_t(0), min(int64_t(V), k - col(i))));
  }
  static __device__ __forceinline__ uint8_t* slot(uint8_t* at, int i) { return at + (i * kWords + threadIdx.x) * 16; }
  static __device__ __forceinline__ uint8_t* after(uint8_t* at, int i) {
    return (threadIdx.x & 31) == 31 ? at + (i * kWords + BLOCK + (threadIdx.x >> 5)) * 16 : slot(at, i) + 16;
  }
  __device__ __forceinline__ void fetch(uint8_t* at, const T* row) const {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int n = there(i);
      if (ALIGNED) {  // (zeros past the row's end)
        fetch_async(smem_u32(slot(at, i)), row + (n ? col(i) : 0), n * sizeof(T));
      } else if (n) {
        const T* p = row + col(i);
        const int s = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15);
        const char* word = reinterpret_cast<const char*>(p) - s;
        const int64_t left = reinterpret_cast<const char*>(end) - word;
        if (word >= reinterpret_cast<const char*>(base)) {
          fetch_async(smem_u32(slot(at, i)), word, static_cast<int>(min(int64_t(16), left)));
        } else {  // the tensor's first word is not all its own
          for (int e = 0; e < n && s + e * static_cast<int>(sizeof(T)) < 16; ++e) reinterpret_cast<T*>(slot(at, i) + s)[e] = p[e];
        }
        if (s + n * static_cast<int>(sizeof(T)) > 16 && ((threadIdx.x & 31) == 31 || col(i) + V >= k))
          fetch_async(smem_u32(after(at, i)), word + 16, static_cast<int>(min(int64_t(16), left - 16)));
      }
    }
  }
  // (Other lanes' words: between the wait for them and this, and between this and the next fetch, a
  // warp barrier.)
  __device__ __forceinline__ uint4 read(uint8_t* at, const T* row, int i) const {
    if (ALIGNED) return *reinterpret_cast<const uint4*>(slot(at, i));
    const int n = there(i);
    if (n == 0) return make_uint4(0, 0, 0, 0);
    const uintptr_t s = reinterpret_cast<uintptr_t>(row + col(i)) & 15;
    Words w;
    w.a = *reinterpret_cast<const uint4*>(slot(at, i));
    w.b = s ? *reinterpret_cast<const uint4*>(after(at, i)) : w.a;
    uint4 v = shift_words16(reinterpret_cast<const void*>(s), w);
    if (n < V) {
      uint32_t* q = &v.x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int kept = n * static_cast<int>(sizeof(T)) - 4 * e;  // bytes of this word
        (&v.x)[e] = kept >= 4 ? q[e] : kept <= 0 ? 0u : q[e] & 0xFFFFu;
      }
    }
    return v;
  }
  static __device__ __forceinline__ void meet() {
    if (!ALIGNED) __syncwarp();
  }
};
constexpr int norm_block(int tpr, int least) { return tpr < least ? least : tpr; }
constexpr int norm_stages(int bytes, int room) { return room / bytes < 1 ? 1 : room / bytes > 6 ? 6 : room / bytes; }

// ---------------------------------------------------------------------------
// Forward.  TPR threads to a row, VPT 16-byte pieces of it to a thread: up to 16 values, two
// to an instruction.  Groups of threads walk over rows, the next ones on their way meanwhile.
// (A block to each few rows, loaded when it came to them, took 254 us for 65536×1024 f32.)
// ---------------------------------------------------------------------------
constexpr int kForwardThreads = 256;
constexpr int forward_room(int block) { return block == 256 ? 64 * 1024 : 200 * 1024; }  // three blocks an SM, or one
template <int TYPE, int TPR, int VPT, bool ALIGNED>
constexpr int forward_stages() {
  constexpr int block = norm_block(TPR, kForwardThreads);
  return norm_stages(Pieces<TYPE, TPR, VPT, block, ALIGNED>::kBytes, forward_room(block));
}

template <int TYPE, int TPR, int VPT, bool ALIGNED>
__global__ void __launch_bounds__(norm_block(TPR, kForwardThreads), norm_block(TPR, kForwardThreads) == 256 ? 3 : 1)
    norm_kernel(NormArgs a) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  constexpr int V = X::V, H = V / 2, kBlock = norm_block(TPR, kForwardThreads), kGroups = kBlock / TPR;
  using Rows = Pieces<TYPE, TPR, VPT, kBlock, ALIGNED>;
  constexpr int STAGES = forward_stages<TYPE, TPR, VPT, ALIGNED>();
  constexpr bool KEEP = TPR < 1024;  // weights in registers
  __shared__ float exchange[kGroups][2 * TPR / 32];
  extern __shared__ __align__(16) uint8_t norm_smem[];
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
  int stage = 0;
  for (int64_t r = first; r < a.m; r += stride) {
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
    if (t == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    const Two scale = two(rstd, rstd);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int n = in.there(i);
      float f[V];
      Two wi[H], bi[H];
      if (!KEEP) vector(a.w, i, one, wi), vector(a.b, i, zero, bi);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        const float2 q = both(fma(x[i][e] * scale, KEEP ? w[KEEP ? i : 0][e] : wi[e], KEEP ? b[KEEP ? i : 0][e] : bi[e]));
        f[2 * e] = q.x, f[2 * e + 1] = q.y;
      }
      store_piece<ALIGNED>(static_cast<T*>(a.y) + r * a.ldy + (n ? in.col(i) : 0), X::pack(f), n);
    }
  }
  fetch_wait<0>();
}

// Rows too long for registers: a block to a row, which it reads again for each of the
// two sums and the result (from L2, mostly).
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
        X::unpack(load_piece<false>(src + r * a.ldx + col, src, end, n), x);
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

// ---------------------------------------------------------------------------
// Backward.  As forward, with groups that walk over rows: a thread's columns are the
// same in every row, so it adds up dw and db of them in registers; a block's groups add
// theirs in shared memory, in order, into the block's row of `parts`, and
// join_parts_kernel adds up the blocks'.
//
// Memory bounds it.  A thread's 16 values of a row stay in registers between the sums and dx;
// the 1024 threads of rows over 8192 have registers for the columns' sums alone and form them
// a second time.
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
  __shared__ float exchange[kGroups][4 * TPR / 32];
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
      in_x.fetch(memory(stage, 1), x + r * a.ldx);
      if (res) in_r.fetch(memory(stage, 2), res + r * a.ldr);
    }
    fetch_commit();
  };
#pragma unroll
  for (int s = 0; s < STAGES; ++s) fetch(first + s * stride, s);
  float mean = 0.f, rstd = 0.f;
  auto statistics = [&](int64_t r) {
    if (r < a.m) mean = a.mean ? __ldg(a.mean + r) : 0.f, rstd = __ldg(a.rstd + r);
  };
  statistics(first);
  int stage = 0;
  for (int64_t r = first; r < a.m; r += stride) {
    fetch_wait<STAGES - 1>();
    Rows::meet();
    const Two less = two(-mean, -mean), scale = two(rstd, rstd);
    // dy, g = dy·w and x̂ of a piece.  (Past the row's end dy is zero, and whatever x̂ is there
    // counts for nothing.)
    auto values = [&](int i, Two (&d)[H], Two (&g)[H], Two (&h)[H]) {
      unpack2<TYPE>(in_dy.read(memory(stage, 0), dy + r * a.lddy, i), d);
      unpack2<TYPE>(in_x.read(memory(stage, 1), x + r * a.ldx, i), h);
      Two own[H];
      if (!KEEP) weights(i, own);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        h[e] = (h[e] + less) * scale;
        g[e] = d[e] * (KEEP ? w[KEEP ? i : 0][e] : own[e]);
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
        store_piece<ALIGNED>(static_cast<T*>(a.dx) + r * a.lddx + (n ? col(i) : 0), X::pack(y), n);
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

// ---------------------------------------------------------------------------
// Threads to a row and pieces to a thread: as few threads as hold it with 16 values to a
// thread (`least` of them at least, if it has that many pieces).  Rows of more than 16384 are
// not held.
// ---------------------------------------------------------------------------
struct NormShape {
  int tpr, vpt;  // 0: too long
};
NormShape shape_of(int64_t k, int type, int least) {
  const int v = 16 / type_bytes(type);
  const int64_t pieces = (k + v - 1) / v;
  for (int tpr : {32, 64, 128, 256, 512, 1024}) {
    if (tpr < least && pieces > tpr) continue;
    for (int vpt = 1; vpt * v <= 16; vpt *= 2)
      if (pieces <= static_cast<int64_t>(tpr) * vpt) return {tpr, vpt};
  }
  return {0, 0};
}
// Forward: few rows get more threads each.
NormShape forward_shape(int64_t m, int64_t k, int type) {
  return shape_of(k, type, m <= 2 * static_cast<int64_t>(num_sms()) ? 512 : 32);
}
NormShape backward_shape(int64_t k, int type) { return shape_of(k, type, 32); }

template <template <int, int> class K, int TPR>
auto by_pieces(int vpt) {
  return vpt == 1 ? K<TPR, 1>::f() : vpt == 2 ? K<TPR, 2>::f() : K<TPR, 4>::f();
}
template <template <int, int> class K>
auto by_shape(NormShape s) {  // the kernel K of these threads and pieces
  return s.tpr == 32    ? by_pieces<K, 32>(s.vpt)
         : s.tpr == 64  ? by_pieces<K, 64>(s.vpt)
         : s.tpr == 128 ? by_pieces<K, 128>(s.vpt)
         : s.tpr == 256 ? by_pieces<K, 256>(s.vpt)
         : s.tpr == 512 ? by_pieces<K, 512>(s.vpt)
                        : by_pieces<K, 1024>(s.vpt);
}
// (Of 4 pieces, those of 16-bit rows are never asked for.)
template <typename Args>
struct Kernel {
  Args kernel;
  int block;
  size_t smem;
};
using ForwardKernel = Kernel<void (*)(NormArgs)>;
using BackwardKernel = Kernel<void (*)(NormGradArgs, float*)>;
template <int TYPE, bool ALIGNED>
struct Forward {
  template <int TPR, int VPT>
  struct K {
    static ForwardKernel f() {
      constexpr int kVpt = VPT * Elem<TYPE>::V <= 16 ? VPT : 2, kBlock = norm_block(TPR, kForwardThreads);
      return {norm_kernel<TYPE, TPR, kVpt, ALIGNED>, kBlock,
              Pieces<TYPE, TPR, kVpt, kBlock, ALIGNED>::kBytes * forward_stages<TYPE, TPR, kVpt, ALIGNED>()};
    }
  };
};
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
  const int64_t blocks = std::min<int64_t>((a.m + groups - 1) / groups, (f.block == 256 ? 3 : 1) * static_cast<int64_t>(num_sms()));
  return launch_dependent(f.kernel, dim3(static_cast<unsigned>(blocks)), dim3(f.block), f.smem, st, a);
}

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
    const bool aligned = rows_on16(a.dy, a.lddy, es) && rows_on16(a.x, a.ldx, es) && (!a.r || rows_on16(a.r, a.ldr, es)) &&
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

cudaError_t launch_layer_norm(const NormArgs& a, int type, cudaStream_t st) {
  return type == OZ2_TYPE_F32    ? forward<OZ2_TYPE_F32>(a, st)
         : type == OZ2_TYPE_BF16 ? forward<OZ2_TYPE_BF16>(a, st)
                                 : forward<OZ2_TYPE_F16>(a, st);
}

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
