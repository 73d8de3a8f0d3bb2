// Definitions shared by the layer operators' translation units (linear layer,
// its gradient, AdamW): element types, activations, and the launchers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/oz2_layers.h"
#include "oz2_gemm.cuh"

namespace oz2 {

constexpr int type_bytes(int t) { return t == OZ2_TYPE_F32 ? 4 : t == OZ2_TYPE_E4M3 ? 1 : 2; }
constexpr bool is_16bit(int t) { return t == OZ2_TYPE_BF16 || t == OZ2_TYPE_F16; }

// Two 16-bit values of either format in a word (the lower address in the low
// half), to and from FP32; the rounding is to nearest even.
__device__ __forceinline__ uint32_t pack16(float lo, float hi, bool bf16) {
  uint32_t w;
  if (bf16) {
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  } else {
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  }
  return w;
}
__device__ __forceinline__ float2 unpack16(uint32_t w, bool bf16) {
  if (bf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ float load16(const uint16_t* p, bool bf16) { return unpack16(*p, bf16).x; }

// 16 bytes from an address that need not be a multiple of 16: the two 16-byte words
// that hold them, shifted together.  `base` and `end` bound what may be read; where a
// word reaches past them, the first n elements (of T) one by one.  Past those n the
// result is of no meaning.  FIXED: nothing writes there during the kernel (a residual
// may be the result's own memory, where each value is read by the thread that then
// writes it).
template <bool FIXED, typename T>
__device__ __forceinline__ T load_global(const T* p) {
  return FIXED ? __ldg(p) : *p;
}
template <bool FIXED = true, typename T>
__device__ __noinline__ uint4 load16_singly(const T* p, int n) {
  union {
    uint4 v;
    T e[16 / sizeof(T)];
  } u;
  u.v = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < static_cast<int>(16 / sizeof(T)); ++e)
    if (e < n) u.e[e] = load_global<FIXED>(p + e);
  return u.v;
}
// The two words, and whether they lie within the bounds; the loads themselves ask for
// nothing, so that several can be under way.
struct Words {
  uint4 a, b;
};
__device__ __forceinline__ bool words_inside(const void* p, const void* base, const void* end) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p), word = at & ~static_cast<uintptr_t>(15);
  return word >= reinterpret_cast<uintptr_t>(base) && word + (at & 15 ? 32 : 16) <= reinterpret_cast<uintptr_t>(end);
}
template <bool FIXED = true>
__device__ __forceinline__ Words load_words16(const void* p) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p), word = at & ~static_cast<uintptr_t>(15);
  return Words{load_global<FIXED>(reinterpret_cast<const uint4*>(word)),
               load_global<FIXED>(reinterpret_cast<const uint4*>(word + (at & 15 ? 16 : 0)))};
}
__device__ __forceinline__ uint4 shift_words16(const void* p, const Words& x) {
  const unsigned s = static_cast<unsigned>(reinterpret_cast<uintptr_t>(p) & 15);
  uint32_t w[6] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y};
  if (s & 8) w[0] = w[2], w[1] = w[3], w[2] = w[4], w[3] = w[5], w[4] = x.b.z, w[5] = x.b.w;
  if (s & 4) w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = w[4], w[4] = w[5];
  const unsigned bits = 8 * (s & 3);
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                    __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}
template <bool FIXED = true, typename T>
__device__ __forceinline__ uint4 load16_any(const T* p, const T* base, const T* end, int n) {
  return words_inside(p, base, end) ? shift_words16(p, load_words16<FIXED>(p)) : load16_singly<FIXED>(p, n);
}

// --- activations ---------------------------------------------------------------
// exp, division and Φ are approximations of a relative error of some 2^-19, to which
// the roundings of exp's argument x add up to |x|·2^-21: results are rounded to 16 bits, and
// in db's FP32 sums such errors average out.  A factor of z below 2^-126 (of a slope: of
// either of its terms) counts as 0.
constexpr float kSqrt2OverPi = 0.79788456080286536f, kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kGeluCubic = 0.044715f, kLog2E = 1.4426950408889634f;

__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Φ(-|z|) given ex = exp(-z²/2): Φ(-x)·exp(x²/2) falls off as 1/x, so it is a polynomial
// in t = 1/(1 + c·x) without a constant term.  c and the coefficients are a minimax fit
// over 0 ≤ x ≤ 14 (a linear program on 1000 points): off by at most 6e-8, and by at most
// 1.7e-6 of the value, which the tail of gelu needs (z·Φ(z) is its result there).
// Cheaper than erff, which branches.
__device__ __forceinline__ float gauss_tail(float z, float ex) {
  const float t = reciprocal(fmaf(0.26f, fabsf(z), 1.f));
  float p = fmaf(t, -0.0731379539f, 0.229471892f);
  p = fmaf(t, p, -0.106956199f);
  p = fmaf(t, p, 0.16664277f);
  p = fmaf(t, p, 0.0732873008f);
  p = fmaf(t, p, 0.107174501f);
  p = fmaf(t, p, 0.103517644f);
  return t * ex * p;
}

template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == OZ2_ACT_RELU) return z < 0.f ? 0.f : z;  // NaN stays NaN
  if (ACT == OZ2_ACT_GELU) {
    const float h = gauss_tail(z, exp2_fast(z * z * (-0.5f * kLog2E)));
    return z * (z > 0.f ? 1.f - h : h);
  }
  if (ACT == OZ2_ACT_GELU_TANH) {
    // z(1 + tanh u)/2 = z/(1 + exp(-2u)), u = √(2/π)(z + 0.044715 z³)
    const float v = z * fmaf(-2.f * kLog2E * kSqrt2OverPi * kGeluCubic, z * z, -2.f * kLog2E * kSqrt2OverPi);
    return z * reciprocal(1.f + exp2_fast(v));
  }
  if (ACT == OZ2_ACT_SILU) return z * reciprocal(1.f + exp2_fast(-kLog2E * z));
  return z;
}

// d act(z)/dz.  Far out, where the slope is 0 or 1 to FP32, z is held (its powers
// and products with 0 would not be numbers).
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == OZ2_ACT_RELU) return z > 0.f ? 1.f : z == z ? 0.f : z;
  if (ACT == OZ2_ACT_GELU) {
    z = fabsf(z) > 16.f ? copysignf(16.f, z) : z;
    const float ex = exp2_fast(z * z * (-0.5f * kLog2E)), h = gauss_tail(z, ex);
    return fmaf(z * kInvSqrt2Pi, ex, z > 0.f ? 1.f - h : h);
  }
  if (ACT == OZ2_ACT_GELU_TANH) {
    // with g = (1 + tanh u)/2 = 1/(1 + exp(-2u)):  g + z·2g(1 - g)·u'
    z = fabsf(z) > 16.f ? copysignf(16.f, z) : z;
    const float zz = z * z;
    const float v = z * fmaf(-2.f * kLog2E * kSqrt2OverPi * kGeluCubic, zz, -2.f * kLog2E * kSqrt2OverPi);
    const float g = reciprocal(1.f + exp2_fast(v));
    const float du2 = fmaf(6.f * kGeluCubic * kSqrt2OverPi, zz, 2.f * kSqrt2OverPi);
    return fmaf(z * g * (1.f - g), du2, g);
  }
  if (ACT == OZ2_ACT_SILU) {
    z = fabsf(z) > 100.f ? copysignf(100.f, z) : z;
    const float g = reciprocal(1.f + exp2_fast(-kLog2E * z));
    return g * fmaf(z, 1.f - g, 1.f);
  }
  return 1.f;
}

// --- one product D = P·Qᵀ of the layer kernels ------------------------------------
// P has `rows` rows and Q `cols` rows of `depth` bytes' worth of elements each;
// an operand is stored with its depth contiguous ("K-major") or, 16-bit types
// only, with its rows contiguous ("MN-major").  D is row-major.
struct LinEpilogue {
  const float* row_scale;  // of D's rows, or null
  const float* col_scale;  // of D's columns, or null
  const void* bias;        // of D's columns, or null
  const void* add;         // R, like D, or null
  void* pre;               // Z, like D, or null
  void* out;               // D
  int64_t ld_add, ld_pre, ld_out;
  int bias_type;           // oz2_type
  int out_type;            // oz2_type: 16-bit, or F32 (then nothing but `accumulate` applies)
  int act;                 // oz2_act
  int accumulate;          // F32 out: D += P·Qᵀ
};
struct LinProduct {
  int64_t rows, cols;
  int64_t depth;           // elements summed over
  const void *p, *q;
  int64_t ldp, ldq;
  bool p_mn, q_mn;         // MN-major
  LinEpilogue ep;
};
constexpr int kMaxProducts = 2;

// How a launch runs: on CTA pairs (nt = 0), the depth of product i's tiles cut into
// pair_split[i] parts (`parts` of them in all, `ahead`: see LinLaunch) and the last
// product's last `halves` tiles taken as two halves each, or in tiles
// of nt rows with the depth split over `split` CTAs and `stages` of operands in
// flight.  `scratch` bytes of workspace; `cost`, an estimate in cycles.
struct LinPlan {
  int nt = 0, split = 1, stages = 0;
  int pair_split[kMaxProducts] = {1, 1}, parts = 0, ahead = 0, halves = 0;
  size_t scratch = 0;
  double cost = 0;
};
// The plan for up to two independent products in one launch (by their sizes and
// storage alone).  `type` is the operands'.
LinPlan plan_linear(const LinProduct* products, int count, int type);
// Whether two products are faster in launches of their own than together.
bool plan_apart(const LinPlan& together, const LinPlan& a, const LinPlan& b);
// Operands' base addresses and leading dimensions are multiples of 16 bytes.
cudaError_t launch_linear(const LinProduct* products, int count, int type, const LinPlan& plan, void* scratch,
                          Oz2Device* dev, cudaStream_t st);

// A product of up to kFewRows rows, both operands K-major and anywhere.
constexpr int kFewRows = 16;
cudaError_t launch_linear_rows(const LinProduct& p, int type, cudaStream_t st);

// Rows of elements of `bytes` bytes copied to rows that start on 16-byte
// boundaries (ld_dst·bytes a multiple of 16), for one or two operands at once.
struct PackJob {
  const void* src;
  int64_t ld_src, rows, cols;
  void* dst;
  int64_t ld_dst;
};
cudaError_t launch_pack_rows(const PackJob* jobs, int count, int bytes, cudaStream_t st);

// dz = dy·act'(z) in the operands' type into rows of ld_dz elements (16-byte
// rows; null: not wanted), and db = its column sums before that rounding
// (null: not wanted; `partial` holds lin_db_chunks(m, n)·n floats for them, of which
// there may be none).
int64_t lin_db_chunks(int64_t m, int64_t n);
cudaError_t launch_act_grad(int64_t m, int64_t n, int type, int act, const void* dy, int64_t ld_dy, const void* z,
                            int64_t ld_z, void* dz, int64_t ld_dz, float* db, float* partial, bool accumulate,
                            cudaStream_t st);

cudaError_t launch_adamw(const oz2_adamw_tensor* tensors, int count, int param_type, int grad_type, int state_bits,
                         const oz2_adamw_step& a, cudaStream_t st);

// From the entry points' translation unit: the library's stream-ordered pool
// and the current device's status block.
cudaError_t workspace_alloc(void** p, size_t bytes, cudaStream_t st);
Oz2Device* device_status();

}  // namespace oz2
