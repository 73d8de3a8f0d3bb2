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
// m and √v are rounded each for itself, so an element whose gradients are some 10^-5 of
// its block's largest may keep an m beside a √v of zero, and the next step, with only the
// new gradient in √v, would be hundreds of times lr.  A √v of zero is an element without
// history: its m counts as zero too (four instructions for four elements), and steps stay
// within what AdamW's are for any gradients.
//
// A warp takes 256 values at a time, a lane 4 of each half, so a block's largest
// magnitude is one warp reduction and every access is 16 (FP32), 8 or 4 bytes a
// lane, consecutive over the warp.
//
// With FP32 states memory bounds it: 201 M bf16 parameters with masters and bf16
// gradients, 28 bytes each, take 814 µs (6.9 TB/s, a plain copy's rate).  With 8-bit
// states there are 16 bytes and some 100 instructions a parameter (the hash and the two
// roundings are a third of them): issue bounds it (77% of the slots, integer pipe 59%),
// 648 µs at 5 TB/s.  Loading the next block ahead took it from 1209 to 826 µs, a kernel
// for each combination of types to 741, packed FP32 instructions and the weights'
// stores before the rounding, which leave room for six blocks of 128 threads an SM, to
// 648 (four: 700).  A square root without the compiler's branch cost as many
// instructions as it saved.
#include <algorithm>

#include "lin_common.cuh"

namespace oz2 {
namespace {

constexpr int kAdamBlock = 256;      // values under one scale, and of a warp's turn
constexpr int kAdamWarps = 4;
constexpr int kAdamTurns = 8;        // a warp's consecutive blocks, at most

struct AdamEntry {
  int64_t numel;
  int64_t first;                     // number of its first block in this launch
  int64_t number;                    // and in the whole list
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
  int turns;                         // a warp's consecutive blocks
  int64_t blocks;                    // of this launch
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

// Four consecutive values as they lie in memory: 16-bit types fill two words,
// E4M3 one.  A whole vector, or the first n of them one by one (the others 0).
template <typename T, int kWords = sizeof(T)>
__device__ __forceinline__ void load_words(const void* p, int64_t at, bool whole, int n, uint32_t* w) {
  constexpr int kPer = 4 / sizeof(T);
  const T* s = static_cast<const T*>(p) + at;
  if (__builtin_expect(whole, 1)) {
    if (kWords == 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(s);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else if (kWords == 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(s);
      w[0] = v.x, w[1] = v.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(s);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) w[e / kPer] |= static_cast<uint32_t>(s[e]) << (8 * sizeof(T) * (e % kPer));
  }
}
template <typename T, int kWords = sizeof(T)>
__device__ __forceinline__ void store_words(void* p, int64_t at, bool whole, int n, const uint32_t* w) {
  constexpr int kPer = 4 / sizeof(T);
  T* d = static_cast<T*>(p) + at;
  if (__builtin_expect(whole, 1)) {
    if (kWords == 4) {
      *reinterpret_cast<uint4*>(d) = make_uint4(w[0], w[1], w[2], w[3]);
    } else if (kWords == 2) {
      *reinterpret_cast<uint2*>(d) = make_uint2(w[0], w[1]);
    } else {
      *reinterpret_cast<uint32_t*>(d) = w[0];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) d[e] = static_cast<T>(w[e / kPer] >> (8 * sizeof(T) * (e % kPer)));
  }
}
template <int TYPE>
__device__ __forceinline__ void load4(const void* p, int64_t at, bool whole, int n, uint32_t* w) {
  if (TYPE == OZ2_TYPE_F32) {
    load_words<uint32_t>(p, at, whole, n, w);
  } else {
    load_words<uint16_t>(p, at, whole, n, w);
  }
}
template <int TYPE>
__device__ __forceinline__ void values4(const uint32_t* w, float* f) {
  if (TYPE == OZ2_TYPE_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(w[e]);
  } else {
    const float2 a = unpack16(w[0], TYPE == OZ2_TYPE_BF16), b = unpack16(w[1], TYPE == OZ2_TYPE_BF16);
    f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y;
  }
}
template <int TYPE>
__device__ __forceinline__ void store4(void* p, int64_t at, bool whole, int n, const float* f) {
  uint32_t w[4];
  if (TYPE == OZ2_TYPE_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(f[e]);
    store_words<uint32_t>(p, at, whole, n, w);
  } else {
    w[0] = pack16(f[0], f[1], TYPE == OZ2_TYPE_BF16);
    w[1] = pack16(f[2], f[3], TYPE == OZ2_TYPE_BF16);
    store_words<uint16_t>(p, at, whole, n, w);
  }
}
// The values of four E4M3 codes.
__device__ __forceinline__ void decode4(uint32_t w, float* f) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"(static_cast<uint16_t>(w)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"(static_cast<uint16_t>(w >> 16)));
  const float2 a = unpack16(lo, false), b = unpack16(hi, false);
  f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y;
}
// Four codes of m, 0 where √v's code is (of either sign): 0x7F and 7 bits carry into
// a byte's sign unless they are 0, and prmt spreads that sign over the byte.
__device__ __forceinline__ uint32_t with_history(uint32_t m, uint32_t v) {
  uint32_t mask;
  asm("prmt.b32 %0, %1, 0, 0xBA98;" : "=r"(mask) : "r"((v & 0x7F7F7F7Fu) + 0x7F7F7F7Fu));
  return m & mask;
}
// The codes of four values that E4M3 holds exactly (or of NaN).
__device__ __forceinline__ uint32_t encode4(const float* f) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(f[1]), "f"(f[0]));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(f[3]), "f"(f[2]));
  return static_cast<uint32_t>(lo) | static_cast<uint32_t>(hi) << 16;
}

// The exponent field of a block's scale: the power of two that brings its largest
// finite magnitude (given by its bits) to (224, 448]; 1 for a block of zeros.
__device__ __forceinline__ int scale_exponent(uint32_t top) {
  if (top == 0) return 127;
  return max(1, static_cast<int>(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}

// Two FP32 values in one 64-bit register pair, and the packed instructions on them:
// each is rounded as the single ones are, at half the issue slots.
struct Two {
  uint64_t v;
  __device__ __forceinline__ Two() {}
  __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
  __device__ __forceinline__ explicit Two(float a) : Two(a, a) {}
  __device__ __forceinline__ float x() const { return __uint_as_float(static_cast<uint32_t>(v)); }
  __device__ __forceinline__ float y() const { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
};
__device__ __forceinline__ Two mul2(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// y (|y| ≤ 448) cut to one of its two E4M3 neighbours, the one away from zero
// with the probability of what is cut off: `u` (16 bits, shifted left by 4) is
// added below the three bits that E4M3 keeps, and the rest dropped.  Below 2^-6
// the spacing is constant: 2^-6 is added first, which leaves the value's last
// three bits where a normal one's are, and taken off again (both exact but for
// what lies under 2^-29).
template <bool SIGNED>
__device__ __forceinline__ void cut_stochastic(Two y, uint32_t u0, uint32_t u1, float* out) {
  const float a = y.x(), b = y.y();
  const float ca = fabsf(a) < 0.015625f ? SIGNED ? copysignf(0.015625f, a) : 0.015625f : 0.f;
  const float cb = fabsf(b) < 0.015625f ? SIGNED ? copysignf(0.015625f, b) : 0.015625f : 0.f;
  const Two t = add2(y, Two(ca, cb));
  const Two r = add2(Two(__uint_as_float((__float_as_uint(t.x()) + u0) & 0xFFF00000u),
                         __uint_as_float((__float_as_uint(t.y()) + u1) & 0xFFF00000u)),
                     Two(-ca, -cb));
  out[0] = SIGNED ? copysignf(r.x(), a) : r.x();
  out[1] = SIGNED ? copysignf(r.y(), b) : r.y();
}

// A warp's 256 values as they were loaded.
struct AdamRaw {
  uint32_t g[2][4], w[2][4], m[2][4], v[2][4];
  float m_scale, v_scale;
};

// Elements of the four at `at` that the tensor has.
__device__ __forceinline__ int part_of(const AdamEntry& x, int64_t at) {
  return static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(4), x.numel - at)));
}

template <int BITS, int W, int G, bool MASTER>
__device__ __forceinline__ void load_raw(const AdamEntry& x, int64_t in, bool whole, int lane, AdamRaw& r) {
  const void* weight = MASTER ? x.master : x.param;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t at = in * kAdamBlock + 128 * h + 4 * lane;
    const int n = whole ? 4 : part_of(x, at);
    load4<G>(x.grad, at, whole, n, r.g[h]);
    load4<MASTER ? OZ2_TYPE_F32 : W>(weight, at, whole, n, r.w[h]);
    if (BITS == 32) {
      load_words<uint32_t>(x.m, at, whole, n, r.m[h]);
      load_words<uint32_t>(x.v, at, whole, n, r.v[h]);
    } else {
      load_words<uint8_t>(x.m, at, whole, n, r.m[h]);
      load_words<uint8_t>(x.v, at, whole, n, r.v[h]);
    }
  }
  if (BITS == 8) {
    r.m_scale = x.m_scale[in];
    r.v_scale = x.v_scale[in];
  }
}

// W: the parameters' type; G: the gradients'; MASTER: FP32 weights beside them.
template <int BITS, int W, int G, bool MASTER, int CAP>
__global__ void __launch_bounds__(32 * kAdamWarps, BITS == 8 ? 6 : 1) adamw_kernel(const __grid_constant__ AdamTable<CAP> T) {
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int64_t b = (static_cast<int64_t>(blockIdx.x) * kAdamWarps + warp) * T.turns;
  const int64_t end = min(b + T.turns, T.blocks);
  if (b >= end) return;
  const float gscale = T.grad_scale ? __ldg(T.grad_scale) : 1.f;
  int lo = 0, hi = T.count;  // the tensor that holds block b
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (T.e[mid].first <= b) lo = mid; else hi = mid;
  }
  auto is_whole = [&](const AdamEntry& x, int64_t in) { return x.vec && (in + 1) * kAdamBlock <= x.numel; };
  // The next block is on its way while one is computed: an 8-bit block is some 80
  // instructions an element and few bytes, and a load would otherwise be waited
  // for between them.
  AdamRaw next;
  bool next_whole = is_whole(T.e[lo], b - T.e[lo].first);
  load_raw<BITS, W, G, MASTER>(T.e[lo], b - T.e[lo].first, next_whole, lane, next);
  for (; b < end; ++b) {
    const AdamEntry& x = T.e[lo];
    const AdamRaw r = next;
    const bool whole = next_whole;
    const int64_t in = b - x.first, at0 = in * kAdamBlock + 4 * lane;
    if (b + 1 < end) {
      if (lo + 1 < T.count && T.e[lo + 1].first <= b + 1) ++lo;
      next_whole = is_whole(T.e[lo], b + 1 - T.e[lo].first);
      load_raw<BITS, W, G, MASTER>(T.e[lo], b + 1 - T.e[lo].first, next_whole, lane, next);
    }
    const float step = T.step * x.lr_scale, decay = T.decay * x.lr_scale * x.decay_scale;
    float w[2][4], m[2][4], v[2][4];
    float mtop = 0.f, vtop = 0.f;
    bool odd = false;  // something is not a number
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float g[4];
      values4<G>(r.g[h], g);
      values4<MASTER ? OZ2_TYPE_F32 : W>(r.w[h], w[h]);
      if (BITS == 32) {
        values4<OZ2_TYPE_F32>(r.m[h], m[h]);
        values4<OZ2_TYPE_F32>(r.v[h], v[h]);
      } else {
        decode4(with_history(r.m[h][0], r.v[h][0]), m[h]);
        decode4(r.v[h][0], v[h]);
      }
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const Two gg = mul2(Two(g[e], g[e + 1]), Two(gscale));
        Two mm(m[h][e], m[h][e + 1]), vv(v[h][e], v[h][e + 1]);
        if (BITS == 8) {
          mm = mul2(mm, Two(r.m_scale));
          vv = mul2(vv, Two(r.v_scale));
          vv = mul2(vv, vv);
        }
        // Rounded one by one, so that the 8-bit states can be checked bit for bit.
        // (The compiler joins packed products and sums; single sums it leaves alone.)
        const Two mb = mul2(mm, Two(T.b1)), mc = mul2(gg, Two(T.c1));
        const Two vb = mul2(vv, Two(T.b2)), vc = mul2(mul2(gg, gg), Two(T.c2));
        mm = Two(__fadd_rn(mb.x(), mc.x()), __fadd_rn(mb.y(), mc.y()));
        vv = Two(__fadd_rn(vb.x(), vc.x()), __fadd_rn(vb.y(), vc.y()));
        const Two root(__fsqrt_rn(vv.x()), __fsqrt_rn(vv.y()));
        const Two den = fma2(root, Two(T.root), Two(T.eps)), p(w[h][e], w[h][e + 1]);
        // The quotient by rcp.approx, 2^-23 of an update that the weight takes lr of.
        const Two u = mul2(mm, Two(reciprocal(den.x()), reciprocal(den.y())));
        const Two now = fma2(Two(-step), u, fma2(Two(-decay), p, p));
        w[h][e] = now.x(), w[h][e + 1] = now.y();
        m[h][e] = mm.x(), m[h][e + 1] = mm.y();
        const Two kept = BITS == 32 ? vv : root;
        v[h][e] = kept.x(), v[h][e + 1] = kept.y();
        if (BITS == 8) {
          mtop = fmaxf(mtop, fmaxf(fabsf(mm.x()), fabsf(mm.y())));  // drops a NaN
          vtop = fmaxf(vtop, fmaxf(root.x(), root.y()));
          odd |= !(fabsf(u.x()) < 1e38f) | !(fabsf(u.y()) < 1e38f);
        }
      }
      const int64_t at = at0 + 128 * h;
      const int n = whole ? 4 : part_of(x, at);
      if (BITS == 32) {
        store4<OZ2_TYPE_F32>(x.m, at, whole, n, m[h]);
        store4<OZ2_TYPE_F32>(x.v, at, whole, n, v[h]);
      }
      if (MASTER) {
        store4<OZ2_TYPE_F32>(x.master, at, whole, n, w[h]);
        if (x.param) store4<W>(x.param, at, whole, n, w[h]);
      } else {
        store4<W>(x.param, at, whole, n, w[h]);
      }
    }
    if (BITS == 8) {
      // Padding of a last block is zeros, which change no maximum.
      uint32_t mbits = __float_as_uint(mtop), vbits = __float_as_uint(vtop);
      odd |= !(mtop < INFINITY) || !(vtop < INFINITY);
      const bool rare = __any_sync(0xffffffffu, odd);
      if (rare) {  // the largest finite magnitudes
        mbits = vbits = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (isfinite(m[h][e])) mbits = max(mbits, __float_as_uint(fabsf(m[h][e])));
            if (isfinite(v[h][e])) vbits = max(vbits, __float_as_uint(v[h][e]));
          }
      }
      const int me = scale_exponent(__reduce_max_sync(0xffffffffu, mbits));
      const int ve = scale_exponent(__reduce_max_sync(0xffffffffu, vbits));
      const float minv = __uint_as_float(static_cast<uint32_t>(254 - me) << 23);
      const float vinv = __uint_as_float(static_cast<uint32_t>(254 - ve) << 23);
      if (lane == 0) {
        x.m_scale[in] = __uint_as_float(static_cast<uint32_t>(me) << 23);
        x.v_scale[in] = __uint_as_float(static_cast<uint32_t>(ve) << 23);
      }
      // Values are numbered through the whole list, every tensor starting a block.
      const uint64_t number = static_cast<uint64_t>(x.number + in) * kAdamBlock + 4 * lane;
      const uint32_t from = static_cast<uint32_t>(number) * 0x9E3779B1u +
                            static_cast<uint32_t>(number >> 32) * 0x3C6EF372u + T.key;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float mc[4], vc[4];
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const uint32_t u = scatter32(from + static_cast<uint32_t>(128 * h + e) * 0x9E3779B1u);
          const uint32_t w = scatter32(from + static_cast<uint32_t>(128 * h + e + 1) * 0x9E3779B1u);
          cut_stochastic<true>(mul2(Two(m[h][e], m[h][e + 1]), Two(minv)), u << 4 & 0xFFFF0u, w << 4 & 0xFFFF0u, mc + e);
          cut_stochastic<false>(mul2(Two(v[h][e], v[h][e + 1]), Two(vinv)), u >> 12 & 0xFFFF0u, w >> 12 & 0xFFFF0u, vc + e);
        }
        uint32_t mw = encode4(mc), vw = encode4(vc);
        if (rare) {  // infinities and NaN are kept as the NaN of their sign
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (!isfinite(m[h][e]))
              mw = (mw & ~(0xFFu << 8 * e)) | ((__float_as_uint(m[h][e]) >> 24 & 0x80u) | 0x7Fu) << 8 * e;
            if (!isfinite(v[h][e]))
              vw = (vw & ~(0xFFu << 8 * e)) | ((__float_as_uint(v[h][e]) >> 24 & 0x80u) | 0x7Fu) << 8 * e;
          }
        }
        const int n = whole ? 4 : part_of(x, at0 + 128 * h);
        store_words<uint8_t>(x.m, at0 + 128 * h, whole, n, &mw);
        store_words<uint8_t>(x.v, at0 + 128 * h, whole, n, &vw);
      }
    }
  }
}

template <int CAP>
using AdamKernel = void (*)(const AdamTable<CAP>);

template <int BITS, bool MASTER, int CAP>
AdamKernel<CAP> kernel_for(int w, int g) {
  if (w == OZ2_TYPE_F32) return adamw_kernel<BITS, OZ2_TYPE_F32, OZ2_TYPE_F32, false, CAP>;
  if (w == OZ2_TYPE_BF16)
    return g == OZ2_TYPE_F32 ? adamw_kernel<BITS, OZ2_TYPE_BF16, OZ2_TYPE_F32, MASTER, CAP>
                             : adamw_kernel<BITS, OZ2_TYPE_BF16, OZ2_TYPE_BF16, MASTER, CAP>;
  return g == OZ2_TYPE_F32 ? adamw_kernel<BITS, OZ2_TYPE_F16, OZ2_TYPE_F32, MASTER, CAP>
                           : adamw_kernel<BITS, OZ2_TYPE_F16, OZ2_TYPE_F16, MASTER, CAP>;
}

// The tensors of the list that have a master (or those that have none), in
// launches of up to CAP of them.
template <int CAP>
cudaError_t launch_some(AdamTable<CAP>& T, const oz2_adamw_tensor* t, int count, bool master, int w, int g, int bits,
                        cudaStream_t st) {
  T.count = 0;
  T.blocks = 0;
  int64_t number = 0;
  auto flush = [&]() -> cudaError_t {
    if (T.count == 0) return cudaSuccess;
    // A warp's turns: as many as leave every SM 24 warps.
    T.turns = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kAdamTurns, T.blocks / (24LL * num_sms()))));
    const int64_t per = static_cast<int64_t>(kAdamWarps) * T.turns, grid = (T.blocks + per - 1) / per;
    if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
    auto kern = bits == 8 ? (master ? kernel_for<8, true, CAP>(w, g) : kernel_for<8, false, CAP>(w, g))
                          : (master ? kernel_for<32, true, CAP>(w, g) : kernel_for<32, false, CAP>(w, g));
    count_launch();
    const cudaError_t err =
        launch_dependent(kern, dim3(static_cast<unsigned>(grid)), dim3(32 * kAdamWarps), 0, st, T);
    T.count = 0;
    T.blocks = 0;
    return err;
  };
  for (int i = 0; i < count; ++i) {
    const int64_t blocks = (t[i].numel + kAdamBlock - 1) / kAdamBlock;
    if (blocks && (t[i].master != nullptr) == master) {
      AdamEntry& e = T.e[T.count++];
      e = AdamEntry{t[i].numel, T.blocks, number, t[i].param, t[i].grad, t[i].master, t[i].m,
                    t[i].v, t[i].m_scale, t[i].v_scale, t[i].lr_scale, t[i].decay_scale, 0};
      auto on = [](const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (4 * bytes) == 0; };
      const int state = bits == 32 ? 4 : 1;
      e.vec = on(e.param, type_bytes(w)) && on(e.grad, type_bytes(g)) && on(e.master, 4) && on(e.m, state) &&
              on(e.v, state);
      T.blocks += blocks;
    }
    number += blocks;
    if (T.count == CAP || i + 1 == count) {
      const cudaError_t err = flush();
      if (err != cudaSuccess) return err;
    }
  }
  return cudaSuccess;
}

template <int CAP>
cudaError_t launch_list(const oz2_adamw_tensor* t, int count, int w, int g, int bits, const oz2_adamw_step& a,
                        cudaStream_t st) {
  static thread_local AdamTable<CAP> T;  // up to 30 KB: not on the stack
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
  bool some[2] = {false, false};
  for (int i = 0; i < count; ++i)
    if (t[i].numel) some[t[i].master != nullptr] = true;
  cudaError_t err = cudaSuccess;
  for (int master = 0; master < 2 && err == cudaSuccess; ++master)
    if (some[master]) err = launch_some<CAP>(T, t, count, master != 0, w, g, bits, st);
  return err;
}

}  // namespace

// A launch carries its table of tensors as a parameter, of one of two sizes:
// small lists should not pay for copying a large one.
cudaError_t launch_adamw(const oz2_adamw_tensor* t, int count, int param_type, int grad_type, int state_bits,
                         const oz2_adamw_step& a, cudaStream_t st) {
  constexpr int kSmall = 32, kLarge = 256;
  return count <= kSmall ? launch_list<kSmall>(t, count, param_type, grad_type, state_bits, a, st)
                         : launch_list<kLarge>(t, count, param_type, grad_type, state_bits, a, st);
}

}  // namespace oz2
