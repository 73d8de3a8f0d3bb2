// Layer norm over a row's k features, forward and backward:
//   μ = mean x (0 where not centred)   r = 1/√(mean (x-μ)² + ε)   x̂ = (x-μ)·r
//   y  = x̂·w + b
//   dx = r·(g - mean g - x̂·mean(g·x̂)) + R   with g = dy·w (no mean g where not centred)
//   dw = Σ_t dy·x̂      db = Σ_t dy
// A row is held in registers: its mean first, then the squares of what deviates from it
// (two passes over registers, none over memory; the difference of E x² and μ² would lose
// what a large mean takes).
#pragma once

#include <algorithm>

#include "lm_common.cuh"

namespace oz2 {

constexpr int kNormThreads = 512;  // of the blocks whose rows take that many threads

// The sum over the LANES lanes that a lane is of, a power of two.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The N sums over a row's TPR threads, the same bits in each of them.  Groups of more
// than one warp exchange theirs in `at` (two sets, taken in turn: a set is written again
// two barriers later) behind a barrier of their own.
template <int TPR, int N>
struct RowSum {
  static constexpr int kWarps = TPR < 32 ? 1 : TPR / 32;
  float* at;
  int group, turn;
  __device__ __forceinline__ void sum(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_sum<TPR < 32 ? TPR : 32>(v[i]);
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
    for (int i = 0; i < N; ++i) v[i] = lanes_sum<32>(lane < kWarps ? s[lane * N + i] : 0.f);
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
// and of the row, fetches that too.  (Short rows are 8 or 16 lanes each of one warp.)
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
  static constexpr int V = X::V, kLanes = TPR < 32 ? TPR : 32;  // of a row in a warp
  static constexpr int kWords = BLOCK + (ALIGNED ? 0 : BLOCK / kLanes), kBytes = VPT * kWords * 16;
  const T *base, *end;
  int64_t k;
  int t;
  __device__ __forceinline__ int64_t col(int i) const { return static_cast<int64_t>(t + i * TPR) * V; }
  __device__ __forceinline__ int there(int i) const {
    return static_cast<int>(max(int64_t(0), min(int64_t(V), k - col(i))));
  }
  static __device__ __forceinline__ bool last() { return threadIdx.x % kLanes == kLanes - 1; }
  static __device__ __forceinline__ uint8_t* slot(uint8_t* at, int i) { return at + (i * kWords + threadIdx.x) * 16; }
  static __device__ __forceinline__ uint8_t* after(uint8_t* at, int i) {
    return last() ? at + (i * kWords + BLOCK + threadIdx.x / kLanes) * 16 : slot(at, i) + 16;
  }
  // (REAL: what is past the row's end, by whole pieces, becomes its first piece again, not zeros.)
  template <bool REAL = false>
  __device__ __forceinline__ void fetch(uint8_t* at, const T* row) const {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int n = there(i);
      if (ALIGNED) {  // (zeros past the row's end)
        fetch_async(smem_u32(slot(at, i)), row + (n ? col(i) : 0), REAL && n == 0 ? 16 : n * static_cast<int>(sizeof(T)));
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
        if (s + n * static_cast<int>(sizeof(T)) > 16 && (last() || col(i) + V >= k))
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
// The groups of threads of a warp that come before a thread's own: a warp walks over rows while
// its first group has one.
template <int TPR>
__device__ __forceinline__ int groups_before() {
  return TPR < 32 ? (threadIdx.x & 31) / TPR : 0;
}
constexpr int norm_block(int tpr, int least) { return tpr < least ? least : tpr; }
constexpr int norm_stages(int bytes, int room) { return room / bytes < 1 ? 1 : room / bytes > 6 ? 6 : room / bytes; }

// ---------------------------------------------------------------------------
// Threads to a row and pieces to a thread: as few threads as hold it with 16 values to a
// thread (`least` of them at least, if it has that many pieces).  Rows of more than 16384 are
// not held.
// ---------------------------------------------------------------------------
struct NormShape {
  int tpr, vpt;  // 0: too long
};
inline NormShape shape_of(int64_t k, int type, int least) {
  const int v = 16 / type_bytes(type);
  const int64_t pieces = (k + v - 1) / v;
  for (int tpr : {8, 16, 32, 64, 128, 256, 512, 1024}) {
    if (tpr < least && pieces > tpr) continue;
    for (int vpt = 1; vpt * v <= (tpr < 32 ? v : 16); vpt *= 2)
      if (pieces <= static_cast<int64_t>(tpr) * vpt) return {tpr, vpt};
  }
  return {0, 0};
}
// Forward: few rows get more threads each.
inline NormShape forward_shape(int64_t m, int64_t k, int type) {
  return shape_of(k, type, m <= 2 * static_cast<int64_t>(num_sms()) ? 512 : 32);
}
inline NormShape backward_shape(int64_t k, int type) { return shape_of(k, type, 32); }

template <template <int, int> class K, int TPR>
auto by_pieces(int vpt) {
  return vpt == 1 ? K<TPR, 1>::f() : vpt == 2 ? K<TPR, 2>::f() : K<TPR, 4>::f();
}
template <template <int, int> class K>
auto by_shape(NormShape s) {  // the kernel K of these threads and pieces
  return s.tpr == 8     ? K<8, 1>::f()
         : s.tpr == 16  ? K<16, 1>::f()
         : s.tpr == 32  ? by_pieces<K, 32>(s.vpt)
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

}  // namespace oz2
