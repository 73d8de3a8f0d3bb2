// One AdamW step over a list of tensors in one launch (decoupled weight decay):
//
//   g' = c·g     m ← β1·m + (1-β1)·g'     v ← β2·v + (1-β2)·g'²
//   w ← w - lr·λ·w - lr·(m/(1-β1^t)) / (√(v/(1-β2^t)) + ε)
//
// w is an FP32 master beside a 16-bit copy, or the parameter itself.  m and v
// are FP32, or E4M3 values with one power-of-two scale per 256: then √v is kept
// instead of v (its range is half as many binades, and the step needs the root
// anyway), and both are rounded stochastically.  To nearest, a v that moves by
// (1-β2) of itself a step would never leave a value whose neighbours are 1/16
// to 1/8 away.  The update of w itself uses the unrounded m and v.
//
// A warp takes 256 values at a time, a lane 4 of each half, so a block's largest
// magnitude is one warp reduction and every access is 16 (FP32), 8 or 4 bytes a
// lane, consecutive over the warp.
#include <algorithm>

#include "lin_common.cuh"

namespace oz2 {
namespace {

constexpr int kAdamBlock = 256;      // values under one scale, and of a warp's turn
constexpr int kAdamWarps = 8;
constexpr int kAdamTurns = 4;        // a warp's consecutive blocks

struct AdamEntry {
  int64_t numel;
  int64_t first;                     // number of its first block in this launch
  void* param;
  const void* grad;
  float* master;
  void *m, *v;
  float *m_scale, *v_scale;
  float lr_scale, decay_scale;
  int vec;                           // every array starts where vectors may
};
template <int CAP>
struct AdamTable {
  int count;
  int param_type, grad_type;
  int64_t blocks;                    // of this launch
  int64_t base;                      // blocks of the launches before it
  float b1, c1, b2, c2;              // β1, 1-β1, β2, 1-β2
  float step, decay, root, eps;      // lr/(1-β1^t), lr·λ, 1/√(1-β2^t), ε
  uint32_t key;
  const float* grad_scale;
  AdamEntry e[CAP];
};

// 32 bits scattered: multiply and fold, with odd parts of √2 and √3.
__host__ __device__ __forceinline__ uint32_t scatter32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

struct Four {
  float v[4];
};
__device__ __forceinline__ Four load4(const void* p, int64_t at, int type, int n, bool vec) {
  Four f;
  if (type == OZ2_TYPE_F32) {
    const float* s = static_cast<const float*>(p) + at;
    if (vec && n == 4) {
      const float4 w = *reinterpret_cast<const float4*>(s);
      f.v[0] = w.x, f.v[1] = w.y, f.v[2] = w.z, f.v[3] = w.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) f.v[e] = e < n ? s[e] : 0.f;
    }
  } else {
    const uint16_t* s = static_cast<const uint16_t*>(p) + at;
    const bool bf16 = type == OZ2_TYPE_BF16;
    uint32_t w[2] = {0, 0};
    if (vec && n == 4) {
      const uint2 u = *reinterpret_cast<const uint2*>(s);
      w[0] = u.x, w[1] = u.y;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < n) w[e >> 1] |= static_cast<uint32_t>(s[e]) << (16 * (e & 1));
    }
    const float2 a = unpack16(w[0], bf16), b = unpack16(w[1], bf16);
    f.v[0] = a.x, f.v[1] = a.y, f.v[2] = b.x, f.v[3] = b.y;
  }
  return f;
}
__device__ __forceinline__ void store4(void* p, int64_t at, int type, const Four& f, int n, bool vec) {
  if (type == OZ2_TYPE_F32) {
    float* d = static_cast<float*>(p) + at;
    if (vec && n == 4) {
      *reinterpret_cast<float4*>(d) = make_float4(f.v[0], f.v[1], f.v[2], f.v[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < n) d[e] = f.v[e];
    }
  } else {
    uint16_t* d = static_cast<uint16_t*>(p) + at;
    const bool bf16 = type == OZ2_TYPE_BF16;
    const uint32_t w[2] = {pack16(f.v[0], f.v[1], bf16), pack16(f.v[2], f.v[3], bf16)};
    if (vec && n == 4) {
      *reinterpret_cast<uint2*>(d) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < n) d[e] = static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
    }
  }
}

// Four E4M3 codes in a word, and their values.
__device__ __forceinline__ uint32_t load_codes(const void* p, int64_t at, int n, bool vec) {
  const uint8_t* s = static_cast<const uint8_t*>(p) + at;
  if (vec && n == 4) return *reinterpret_cast<const uint32_t*>(s);
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) w |= static_cast<uint32_t>(s[e]) << (8 * e);
  return w;
}
__device__ __forceinline__ void store_codes(void* p, int64_t at, uint32_t w, int n, bool vec) {
  uint8_t* d = static_cast<uint8_t*>(p) + at;
  if (vec && n == 4) {
    *reinterpret_cast<uint32_t*>(d) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) d[e] = static_cast<uint8_t>(w >> (8 * e));
  }
}
__device__ __forceinline__ Four decode4(uint32_t w) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"(static_cast<uint16_t>(w)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"(static_cast<uint16_t>(w >> 16)));
  const float2 a = unpack16(lo, false), b = unpack16(hi, false);
  Four f;
  f.v[0] = a.x, f.v[1] = a.y, f.v[2] = b.x, f.v[3] = b.y;
  return f;
}

// The exponent field of a block's scale: the power of two that brings its largest
// finite magnitude (given by its bits) to (224, 448]; 1 for a block of zeros.
__device__ __forceinline__ int scale_exponent(uint32_t top) {
  if (top == 0) return 127;
  return max(1, static_cast<int>(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}

// E4M3 of y (|y| ≤ 448), away from zero with the probability of what is cut
// off, by the 16 bits of u.  Below 2^-6 the spacing is constant: 2^-6 is added,
// which leaves the value's last three bits where a normal one's are.
__device__ __forceinline__ uint32_t encode_stochastic(float y, uint32_t u) {
  const uint32_t bits = __float_as_uint(y);
  const float a = fabsf(y);
  const bool small = a < 0.015625f;
  const uint32_t b = __float_as_uint(small ? __fadd_rn(a, 0.015625f) : a);
  const uint32_t code = ((b + (u << 4)) >> 20) - (small ? 968u : 960u);
  const uint32_t sign = (bits >> 24) & 0x80u;
  return (bits & 0x7F800000u) == 0x7F800000u ? sign | 0x7Fu : sign | code;
}

__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}

template <int BITS, int CAP>
__global__ void __launch_bounds__(32 * kAdamWarps) adamw_kernel(const __grid_constant__ AdamTable<CAP> T) {
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int64_t b = (static_cast<int64_t>(blockIdx.x) * kAdamWarps + warp) * kAdamTurns;
  const int64_t end = min(b + kAdamTurns, T.blocks);
  if (b >= end) return;
  const float gscale = T.grad_scale ? __ldg(T.grad_scale) : 1.f;
  int lo = 0, hi = T.count;  // the tensor that holds block b
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (T.e[mid].first <= b) lo = mid; else hi = mid;
  }
  for (; b < end; ++b) {
    while (lo + 1 < T.count && T.e[lo + 1].first <= b) ++lo;
    const AdamEntry& x = T.e[lo];
    const int64_t in = b - x.first, at0 = in * kAdamBlock + 4 * lane;
    const bool vec = x.vec != 0;
    const int wtype = x.master ? OZ2_TYPE_F32 : T.param_type;
    void* const weight = x.master ? static_cast<void*>(x.master) : x.param;
    const float step = T.step * x.lr_scale, decay = T.decay * x.lr_scale * x.decay_scale;
    Four w[2], g[2], m[2], v[2];
    int n[2];
    float ms = 1.f, vs = 1.f;
    if (BITS == 8) {
      ms = x.m_scale[in];
      vs = x.v_scale[in];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = at0 + 128 * h;
      n[h] = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(4), x.numel - at)));
      g[h] = load4(x.grad, at, T.grad_type, n[h], vec);
      w[h] = load4(weight, at, wtype, n[h], vec);
      if (BITS == 32) {
        m[h] = load4(x.m, at, OZ2_TYPE_F32, n[h], vec);
        v[h] = load4(x.v, at, OZ2_TYPE_F32, n[h], vec);
      } else {
        m[h] = decode4(load_codes(x.m, at, n[h], vec));
        v[h] = decode4(load_codes(x.v, at, n[h], vec));
      }
    }
    uint32_t mtop = 0, vtop = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float gg = g[h].v[e] * gscale;
        float mm = m[h].v[e], vv = v[h].v[e];
        if (BITS == 8) {
          mm *= ms;
          vv *= vs;
          vv *= vv;
        }
        // Rounded one by one, so that the 8-bit states can be checked bit for bit.
        mm = __fadd_rn(__fmul_rn(mm, T.b1), __fmul_rn(gg, T.c1));
        vv = __fadd_rn(__fmul_rn(vv, T.b2), __fmul_rn(__fmul_rn(gg, gg), T.c2));
        const float root = __fsqrt_rn(vv);
        const float p = w[h].v[e];
        w[h].v[e] = fmaf(-decay, p, p) - step * __fdividef(mm, fmaf(root, T.root, T.eps));
        m[h].v[e] = mm;
        v[h].v[e] = BITS == 32 ? vv : root;
        if (BITS == 8 && e < n[h]) {
          mtop = max(mtop, finite_bits(mm));
          vtop = max(vtop, finite_bits(root));
        }
      }
    if (BITS == 8) {
      const int me = scale_exponent(__reduce_max_sync(0xffffffffu, mtop));
      const int ve = scale_exponent(__reduce_max_sync(0xffffffffu, vtop));
      const float minv = __uint_as_float(static_cast<uint32_t>(254 - me) << 23);
      const float vinv = __uint_as_float(static_cast<uint32_t>(254 - ve) << 23);
      if (lane == 0) {
        x.m_scale[in] = __uint_as_float(static_cast<uint32_t>(me) << 23);
        x.v_scale[in] = __uint_as_float(static_cast<uint32_t>(ve) << 23);
      }
      // Values are numbered through the whole list, every tensor starting a block.
      const uint64_t number = static_cast<uint64_t>(T.base + b) * kAdamBlock + 4 * lane;
      const uint32_t high = static_cast<uint32_t>(number >> 32) * 0x3C6EF372u + T.key;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t mw = 0, vw = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t r = scatter32(static_cast<uint32_t>(number + 128 * h + e) * 0x9E3779B1u + high);
          mw |= encode_stochastic(m[h].v[e] * minv, r & 0xFFFFu) << (8 * e);
          vw |= encode_stochastic(v[h].v[e] * vinv, r >> 16) << (8 * e);
        }
        store_codes(x.m, at0 + 128 * h, mw, n[h], vec);
        store_codes(x.v, at0 + 128 * h, vw, n[h], vec);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = at0 + 128 * h;
      if (BITS == 32) {
        store4(x.m, at, OZ2_TYPE_F32, m[h], n[h], vec);
        store4(x.v, at, OZ2_TYPE_F32, v[h], n[h], vec);
      }
      store4(weight, at, wtype, w[h], n[h], vec);
      if (x.master && x.param) store4(x.param, at, T.param_type, w[h], n[h], vec);
    }
  }
}

template <int BITS, int CAP>
cudaError_t launch_table(AdamTable<CAP>& T, const oz2_adamw_tensor* t, int count, cudaStream_t st) {
  T.count = 0;
  T.blocks = 0;
  for (int i = 0; i < count; ++i) {
    if (t[i].numel == 0) continue;
    AdamEntry& e = T.e[T.count++];
    e = AdamEntry{t[i].numel, T.blocks, t[i].param, t[i].grad, t[i].master, t[i].m,
                  t[i].v, t[i].m_scale, t[i].v_scale, t[i].lr_scale, t[i].decay_scale, 0};
    auto on = [](const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (4 * bytes) == 0; };
    const int state = BITS == 32 ? 4 : 1;
    e.vec = on(e.param, type_bytes(T.param_type)) && on(e.grad, type_bytes(T.grad_type)) && on(e.master, 4) &&
            on(e.m, state) && on(e.v, state);
    T.blocks += (e.numel + kAdamBlock - 1) / kAdamBlock;
  }
  if (T.blocks == 0) return cudaSuccess;
  const int64_t per = kAdamWarps * kAdamTurns, grid = (T.blocks + per - 1) / per;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  count_launch();
  const cudaError_t err = launch_dependent(adamw_kernel<BITS, CAP>, dim3(static_cast<unsigned>(grid)),
                                           dim3(32 * kAdamWarps), 0, st, T);
  T.base += T.blocks;
  return err;
}

template <int BITS, int CAP>
cudaError_t launch_list(const oz2_adamw_tensor* t, int count, int param_type, int grad_type, const oz2_adamw_step& a,
                        cudaStream_t st) {
  static thread_local AdamTable<CAP> T;  // up to 30 KB: not on the stack
  T.param_type = param_type;
  T.grad_type = grad_type;
  T.base = 0;
  T.b1 = static_cast<float>(a.beta1);
  T.c1 = static_cast<float>(1.0 - a.beta1);
  T.b2 = static_cast<float>(a.beta2);
  T.c2 = static_cast<float>(1.0 - a.beta2);
  const double t1 = 1.0 - pow(a.beta1, static_cast<double>(a.step)), t2 = 1.0 - pow(a.beta2, static_cast<double>(a.step));
  T.step = static_cast<float>(a.lr / t1);
  T.decay = static_cast<float>(a.lr * a.weight_decay);
  T.root = static_cast<float>(1.0 / sqrt(t2));
  T.eps = static_cast<float>(a.eps);
  T.key = scatter32(scatter32(a.seed) + static_cast<uint32_t>(a.step));
  T.grad_scale = a.d_grad_scale;
  for (int i = 0; i < count; i += CAP) {
    const cudaError_t err = launch_table<BITS, CAP>(T, t + i, std::min(CAP, count - i), st);
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}

}  // namespace

// A launch carries its table of tensors as a parameter, of one of two sizes:
// small lists should not pay for copying a large one.
cudaError_t launch_adamw(const oz2_adamw_tensor* t, int count, int param_type, int grad_type, int state_bits,
                         const oz2_adamw_step& a, cudaStream_t st) {
  constexpr int kSmall = 32, kLarge = 320;
  if (state_bits == 8)
    return count <= kSmall ? launch_list<8, kSmall>(t, count, param_type, grad_type, a, st)
                           : launch_list<8, kLarge>(t, count, param_type, grad_type, a, st);
  return count <= kSmall ? launch_list<32, kSmall>(t, count, param_type, grad_type, a, st)
                         : launch_list<32, kLarge>(t, count, param_type, grad_type, a, st);
}

}  // namespace oz2
