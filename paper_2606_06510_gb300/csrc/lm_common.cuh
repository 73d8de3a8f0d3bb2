// Definitions shared by the operators of a language model's ends and norms (embedding,
// layer norm, losses over a vocabulary): element types, and the launchers.
#pragma once

#include "lin_common.cuh"

namespace oz2 {

// Two FP32 values that one instruction works on.
struct Two {
  unsigned long long v;
};
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 both(Two t) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(t.v));
  return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two operator+(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
// --- 16 bytes of a row -------------------------------------------------------------
// A row's 16-byte pieces as FP32 values: V of them.
template <int TYPE>
struct Elem {
  using T = uint16_t;
  static constexpr int V = 8;
  static __device__ __forceinline__ void unpack(uint4 v, float (&f)[V]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 p = unpack16(w[e], TYPE == OZ2_TYPE_BF16);
      f[2 * e] = p.x;
      f[2 * e + 1] = p.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[V]) {
    constexpr bool b = TYPE == OZ2_TYPE_BF16;
    return make_uint4(pack16(f[0], f[1], b), pack16(f[2], f[3], b), pack16(f[4], f[5], b), pack16(f[6], f[7], b));
  }
  static __device__ __forceinline__ float one(T v) { return load16(&v, TYPE == OZ2_TYPE_BF16); }
};
template <>
struct Elem<OZ2_TYPE_F32> {
  using T = float;
  static constexpr int V = 4;
  static __device__ __forceinline__ void unpack(uint4 v, float (&f)[V]) {
    f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[V]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float one(T v) { return v; }
};

// The first n elements of a 16-byte piece to an address that need not be a multiple of
// 16 (`whole`: it is, and all of them are there).
template <typename T>
__device__ __forceinline__ void store16_any(T* p, uint4 v, int n, bool whole) {
  if (whole) {
    *reinterpret_cast<uint4*>(p) = v;
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < static_cast<int>(16 / sizeof(T)); ++e)
    if (e < n) {
      if (sizeof(T) == 4) {
        reinterpret_cast<uint32_t*>(p)[e] = w[e & 3];
      } else {
        reinterpret_cast<uint16_t*>(p)[e] = static_cast<uint16_t>(w[e >> 1 & 3] >> (16 * (e & 1)));
      }
    }
}
// The same by a whole warp whose lanes have pieces that mostly follow each other, anywhere
// (n = 0: a lane has none): a lane stores the 16-byte word that ends in its piece and begins in
// that of the lane before, and single elements only at the ends.
template <typename T>
__device__ __forceinline__ void store16_warp(T* p, uint4 v, int n) {
  constexpr int V = 16 / sizeof(T);
  const int lane = threadIdx.x & 31;
  const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p));
  const int s = at & 15, head = (16 - s) / static_cast<int>(sizeof(T));  // elements up to the next boundary
  const uint4 b = make_uint4(__shfl_up_sync(0xffffffffu, v.x, 1), __shfl_up_sync(0xffffffffu, v.y, 1),
                             __shfl_up_sync(0xffffffffu, v.z, 1), __shfl_up_sync(0xffffffffu, v.w, 1));
  const uint32_t before = __shfl_up_sync(0xffffffffu, n == V ? at + 16 : 1u, 1);  // (an odd address is no piece's)
  const bool word = n >= head && (s == 0 || (lane > 0 && before == at));
  const uint32_t words = __ballot_sync(0xffffffffu, word && s != 0);
  if (word)
    *reinterpret_cast<uint4*>(reinterpret_cast<char*>(p) - s) =
        s ? shift_words16(reinterpret_cast<const void*>(static_cast<uintptr_t>(16 - s)), Words{b, v}) : v;
  const bool tail = lane < 31 && (words >> (lane + 1) & 1);  // the next lane stores what is behind the boundary
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if (e >= n || (e < head ? word : tail)) continue;
    if (sizeof(T) == 4) {
      reinterpret_cast<uint32_t*>(p)[e] = w[e & 3];
    } else {
      reinterpret_cast<uint16_t*>(p)[e] = static_cast<uint16_t>(w[e >> 1 & 3] >> (16 * (e & 1)));
    }
  }
}
// By the warp: rows on 16-byte boundaries, of which only a row's last piece is short, or any.
template <bool ALIGNED, typename T>
__device__ __forceinline__ void store_piece(T* p, uint4 v, int n) {
  if (!ALIGNED) {
    store16_warp(p, v, n);
  } else if (n > 0) {
    store16_any(p, v, n, n >= static_cast<int>(16 / sizeof(T)));
  }
}
// A piece of which the first n elements are there; rows on 16-byte boundaries (ALIGNED)
// or anywhere.  Where n is short, the rest are zeros.
template <bool ALIGNED, bool FIXED = true, typename T>
__device__ __forceinline__ uint4 load_piece(const T* p, const T* base, const T* end, int n) {
  constexpr int V = 16 / sizeof(T);
  if (n >= V) {
    if (ALIGNED) return load_global<FIXED>(reinterpret_cast<const uint4*>(p));
    return load16_any<FIXED>(p, base, end, n);
  }
  return load16_singly<FIXED>(p, n);
}
inline bool rows_on16(const void* p, int64_t ld, int bytes) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * bytes)) & 15) == 0;
}

// Rows of a table named by tokens: 64- or 32-bit integers.
struct Ids {
  const void* p;
  int wide;
  __device__ __forceinline__ int64_t operator[](int64_t i) const {
    return wide ? __ldg(static_cast<const long long*>(p) + i) : static_cast<int64_t>(__ldg(static_cast<const int*>(p) + i));
  }
};

// --- embedding (k_embed.cu) ----------------------------------------------------------
cudaError_t launch_embedding(int64_t m, int64_t n, int64_t k, int type, Ids ids, const void* E, int64_t lde, float scale,
                             void* Y, int64_t ldy, cudaStream_t st);
// The gradient's workspace in bytes.
size_t embedding_grad_scratch(int64_t m, int64_t k, int type);
cudaError_t launch_embedding_grad(int64_t m, int64_t n, int64_t k, int type, const void* dY, int64_t lddy, Ids ids,
                                  float scale, void* dE, int64_t ldde, int de_type, bool accumulate, void* scratch,
                                  cudaStream_t st);

// --- layer norm (k_norm.cu) ------------------------------------------------------------
struct NormArgs {
  int64_t m, k;
  const void* x;
  int64_t ldx;
  const void *w, *b;       // or null
  int wtype;               // of both: the rows' type or F32
  float eps;
  int center;
  void* y;
  int64_t ldy;
  float *mean, *rstd;      // or null
};
cudaError_t launch_layer_norm(const NormArgs& a, int type, cudaStream_t st);
struct NormGradArgs {
  int64_t m, k;
  const void *dy, *x;
  int64_t lddy, ldx;
  const float *mean, *rstd;  // mean null: not centred
  const void* w;             // or null
  int wtype;
  const void* r;             // added to dx, or null
  int64_t ldr;
  void* dx;                  // or null
  int64_t lddx;
  float *dw, *db;            // or null
  int accumulate;            // dw and db are added to
};
size_t layer_norm_grad_scratch(const NormGradArgs& a, int type);
cudaError_t launch_layer_norm_grad(const NormGradArgs& a, int type, void* scratch, cudaStream_t st);

// --- losses over a vocabulary (k_head.cu) ------------------------------------------------
// The logits z = scale·x·wᵀ are formed tile by tile and used where they are.  What a
// token wants of them besides their sum of exponentials: its target, or its `top` listed
// rows of w, sorted, with their places in `picked` (forward) or their weights (gradient).
constexpr int kNoTarget = 0x7FFFFFFF;
struct HeadTargets {
  Ids ids;
  int64_t ld;          // of ids (and teacher's own)
  int top;             // a token's
  int soft;            // weights are the softmax of teacher/temperature; else top = 1 with weight 1
  const void* teacher;
  int64_t ld_teacher;
  int teacher_type;
  float temperature;
};
// A token's terms of the gradient dz_j = a·((1 + e)·exp(z_j - lse) - its targets' weights).
struct HeadRow {
  float a, lse, e;
  int live;
};
// What they come of: the losses' gradient (one a token, or one for all) and lse, and for
// listed rows, whose prepared terms are read.
struct HeadTerms {
  const HeadRow* rows;  // or null
  const float *dloss, *lse;
  int dloss_each;
  float scale, z_loss;
};
struct HeadArgs {
  int64_t m, n, k;
  const void* x;       // rows on 16-byte boundaries, like w's
  int64_t ldx;
  const void* w;       // of the piece
  int64_t ldw;
  int64_t c0, cols;    // the piece of the vocabulary
  float scale;
  Ids ids;             // targets, one a token
  const int2* entries; // or (m, top) sorted entries: row of w, place or weight's bits;
  const uint16_t* offsets;  // where those of a group of 64 rows of w begin: (groups + 1, ld_offsets)
  int64_t ld_offsets;
  int top, soft;
  // forward
  float2* stats;       // (groups of 64 columns, ld_stats): max and sum of exp2 of z·log2 e
  int64_t ld_stats;
  float* picked;       // (m, top)
  // gradient
  HeadTerms terms;
  const float* largest;  // maxima of |a|·max(1, |e|, |1 + e|), `maxima` of them, or null: dz is not scaled
  int maxima;
  float* unscale;      // dz's scale, inverted (written)
  uint16_t* dz;
  int64_t ld_dz;
};
constexpr int kHeadGroup = 64;
constexpr int kMaxTop = 1024;
// Entries and offsets (groups1 rows of ld_offsets); with `rows`, weights and the rows' terms.
struct HeadLists {
  int64_t entries, groups1, ld_offsets;
};
HeadLists head_lists(int64_t m, int64_t n, int top);
cudaError_t launch_head_targets(int64_t m, int64_t n, const HeadTargets& t, int2* entries, uint16_t* offsets, HeadRow* rows,
                                const HeadTerms& terms, cudaStream_t st);
// x's rows of live tokens to rows of ld_dst elements on 16-byte boundaries, zeros for the others; and
// with `largest` the maxima for HeadArgs, as many as live_rows_maxima(m, k).
int live_rows_maxima(int64_t m, int64_t k);
cudaError_t launch_live_rows(int64_t m, int64_t n, int64_t k, const void* x, int64_t ldx, Ids ids, const HeadTerms& terms,
                             float* largest, void* dst, int64_t ld_dst, cudaStream_t st);
cudaError_t launch_head_forward(const HeadArgs& a, int type, Oz2Device* dev, cudaStream_t st);
cudaError_t launch_head_grad(const HeadArgs& a, int type, Oz2Device* dev, cudaStream_t st);
// lse from the groups' stats; then losses, and picked where no logit is.
cudaError_t launch_head_join(int64_t m, int64_t n, const HeadTargets& t, const float2* stats, int64_t ld_stats,
                             float z_loss, float* loss, float* lse, float* picked, cudaStream_t st);
// dst = src·(*unscale, or 1) in a 16-bit type.
cudaError_t launch_round_rows(int64_t m, int64_t k, int type, const float* src, int64_t ld_src, const float* unscale,
                              void* dst, int64_t ld_dst, cudaStream_t st);

}  // namespace oz2
