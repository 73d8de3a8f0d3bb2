// Embedding: rows of a table by tokens, and the table's gradient by sorted tokens.
//
//   forward    Y_t = s·E[id_t]           id < 0: zeros; id ≥ n: NaN
//   gradient   dE_j = s·Σ_{t: id_t = j} dY_t, or added to dE; ids outside [0, n) have no
//              row and count for nothing
#include <algorithm>

#include "lm_common.cuh"

namespace oz2 {
namespace {

// ---------------------------------------------------------------------------
// Forward: a thread takes 16-byte pieces of the result, one grid's stride apart; its
// row and place in it are found by one division and carried on.  The id is read, then
// the piece: kAhead of these chains are under way at once.  Memory bounds it (65536×2048
// bf16 72 µs: the result's 268 MB, and rows that mostly come from L2), for few tokens the
// launch (64×4096 4 µs in a graph).
// ---------------------------------------------------------------------------
constexpr int kAhead = 4, kBlocks = 8;  // pieces of a thread at once, blocks an SM

template <int TYPE, bool ALIGNED>
__global__ void __launch_bounds__(256)
    embedding_kernel(int64_t m, int64_t n, int64_t k, Ids ids, const void* E, int64_t lde, float scale, void* Y, int64_t ldy) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  pdl_trigger();
  pdl_wait();
  const T* src = static_cast<const T*>(E);
  const T* end = src + (n - 1) * lde + k;
  T* dst = static_cast<T*>(Y);
  const uint32_t per = static_cast<uint32_t>((k + X::V - 1) / X::V);
  const uint32_t first = blockIdx.x * blockDim.x + threadIdx.x, stride = gridDim.x * blockDim.x;
  const uint32_t stride_rows = stride / per, stride_pieces = stride - stride_rows * per;
  int64_t r = first / per;
  uint32_t c = first - static_cast<uint32_t>(r) * per;
  while (ALIGNED ? r < m : __any_sync(0xffffffffu, r < m) != 0) {
    int64_t row[kAhead], id[kAhead];
    int col[kAhead];
    // Rows off the 16-byte grid: the words around a piece, which are shifted when all are under way.
    uint4 v[kAhead];
    Words around[ALIGNED ? 1 : kAhead];
    bool inside[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      row[j] = r;
      col[j] = static_cast<int>(c) * X::V;
      id[j] = r < m ? ids[r] : -1;
      r += stride_rows;
      c += stride_pieces;
      if (c >= per) c -= per, ++r;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      v[j] = make_uint4(0, 0, 0, 0);
      const bool real = id[j] >= 0 && id[j] < n;
      const T* p = src + (real ? id[j] * lde + col[j] : 0);
      if (ALIGNED) {
        if (real) v[j] = load_piece<true>(p, src, end, static_cast<int>(min(int64_t(X::V), k - col[j])));
      } else {
        inside[j] = real && words_inside(p, src, end);
        if (inside[j]) around[ALIGNED ? 0 : j] = load_words16(p);
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (ALIGNED && row[j] >= m) continue;
      if (!ALIGNED && id[j] >= 0 && id[j] < n) {
        const T* p = src + id[j] * lde + col[j];
        v[j] = inside[j] ? shift_words16(p, around[ALIGNED ? 0 : j]) : load16_singly(p, static_cast<int>(min(int64_t(X::V), k - col[j])));
      }
      float f[X::V];
      X::unpack(v[j], f);
      const float by = id[j] < 0 ? 0.f : id[j] < n ? scale : __int_as_float(0x7FC00000);  // (of zeros, where there is no row)
#pragma unroll
      for (int e = 0; e < X::V; ++e) f[e] *= by;
      const int there = row[j] < m ? static_cast<int>(min(int64_t(X::V), k - col[j])) : 0;
      store_piece<ALIGNED>(dst + (there ? row[j] * ldy + col[j] : 0), X::pack(f), there);
    }
  }
}

// ---------------------------------------------------------------------------
// The gradient's tokens in the order of their rows: (row, token) pairs, sorted by row
// and within a row by token, rows that are not there (as n) last.  A radix sort of the
// rows' bits, up to 9 at a time, by one cluster: each warp has a stretch of the tokens,
// counts its digits in shared memory, and after the counts have been summed over warps
// and blocks (by distributed shared memory) gives each pair its place, which depends on
// the order of the pairs alone.
//
// One cluster, since a pass is a few exchanges between blocks: 4 µs at least (1.5 of it the
// blocks' counts, 32 KB a block by distributed shared memory), which more launches would
// not be; above some 30000 tokens its 16 SMs' instructions bound it.  16384 tokens of 50257
// rows take 14 µs, 65536 of 131072 22.
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortCluster = 16, kFillThreads = 256;
constexpr int kSortHeld = 4096;  // pairs of a block in shared memory
constexpr int kSortSmem = (kSortWarps + 3) * kDigits * 4 + kSortHeld * 8;

struct SortJob {
  Ids ids;
  int64_t m;
  uint32_t n;
  int passes, bits;    // of `bits` bits each
  uint2 *a, *b;        // the passes write a, b, a, ...
  int* long_runs;      // two counters that are set to zero
};
struct FillJob {       // `rows` rows of `bytes` bytes, `ld` bytes apart (one row: all of it)
  char* p;
  int64_t rows, bytes, ld;
  int unit;            // bytes of an element
};

// A row's zeros: 16 bytes a lane from its first boundary on, elements before and after.
__device__ __forceinline__ void zero_row(char* p, int64_t bytes, int unit, int64_t first, int64_t stride) {
  int64_t head = static_cast<int64_t>(-reinterpret_cast<uintptr_t>(p) & 15);
  head = head < bytes ? head : bytes;
  const int64_t words = (bytes - head) >> 4, tail = head + 16 * words;
  for (int64_t i = first; i < words; i += stride) reinterpret_cast<uint4*>(p + head)[i] = make_uint4(0, 0, 0, 0);
  for (int64_t i = first * unit; i < head; i += stride * unit)
    for (int b = 0; b < unit; b += 2) *reinterpret_cast<uint16_t*>(p + i + b) = 0;
  for (int64_t i = tail + first * unit; i < bytes; i += stride * unit)
    for (int b = 0; b < unit; b += 2) *reinterpret_cast<uint16_t*>(p + i + b) = 0;
}

// The zeros are written beside the sort: this kernel starts once the sort has seen the end
// of what came before the two, and ends after it, so that the kernel that follows has both
// behind it.
__global__ void __launch_bounds__(kFillThreads) fill_rows_kernel(FillJob f) {
  pdl_trigger();
  const int64_t threads = static_cast<int64_t>(gridDim.x) * kFillThreads, me = static_cast<int64_t>(blockIdx.x) * kFillThreads + threadIdx.x;
  if (f.rows == 1) {
    zero_row(f.p, f.bytes, f.unit, me, threads);
  } else {
    for (int64_t r = me >> 5; r < f.rows; r += threads >> 5) zero_row(f.p + r * f.ld, f.bytes, f.unit, threadIdx.x & 31, 32);
  }
  pdl_wait();
}

__global__ void __launch_bounds__(kSortThreads, 1) sort_tokens_kernel(SortJob s, int sorters) {
  extern __shared__ uint32_t sort_smem[];
  pdl_wait();
  pdl_trigger();  // (not before: see fill_rows_kernel)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t* mine = sort_smem + warp * kDigits;             // this warp's counts, then its next places
  uint32_t* total = sort_smem + kSortWarps * kDigits;      // the block's
  uint32_t* base = total + kDigits;                        // the first places of the block's pairs of a digit
  uint32_t* local = base + kDigits;                        // and their places among the block's own
  uint2* pairs = reinterpret_cast<uint2*>(local + kDigits);
  __shared__ uint2 sums[kSortWarps];
  const uint32_t rank = sorters > 1 ? cluster_ctarank() : 0, blocks = sorters;
  if (rank == 0 && threadIdx.x == 0) s.long_runs[0] = s.long_runs[1] = 0;
  const int64_t each = ((s.m + blocks * kSortWarps - 1) / (blocks * kSortWarps) + 31) / 32 * 32;
  const int64_t i0 = min(s.m, (static_cast<int64_t>(rank) * kSortWarps + warp) * each), i1 = min(s.m, i0 + each);
  const int64_t b0 = min(s.m, static_cast<int64_t>(rank) * kSortWarps * each);
  const int mine_all = static_cast<int>(min(s.m - b0, kSortWarps * each));
  const int digits = 1 << s.bits;
  uint2 *from = s.b, *to = s.a;
  for (int pass = 0; pass < s.passes; ++pass) {
    const int shift = pass * s.bits;
    auto pair = [&](int64_t i) {
      if (pass) return __ldcg(from + i);
      const int64_t id = s.ids[i];
      return make_uint2(id < 0 || id >= s.n ? s.n : static_cast<uint32_t>(id), static_cast<uint32_t>(i));
    };
    // A lane's pairs, eight at a time: read once where a warp's stretch is that short.
    constexpr int kHeld = 8;
    const bool once = i1 - i0 <= 32 * kHeld;
    uint2 held[kHeld];
    auto load = [&](int64_t i) {
#pragma unroll
      for (int q = 0; q < kHeld; ++q)
        if (i + 32 * q + lane < i1) held[q] = pair(i + 32 * q + lane);
    };
    for (int d = lane; d < digits; d += 32) mine[d] = 0;
    __syncwarp();
    for (int64_t i = i0; i < i1; i += 32 * kHeld) {
      load(i);
#pragma unroll
      for (int q = 0; q < kHeld; ++q)
        if (i + 32 * q + lane < i1) atomicAdd(mine + (held[q].x >> shift & (digits - 1)), 1u);
    }
    __syncthreads();
    // Places: of the pairs of smaller digits, of the blocks before, of the warps before.  (What is
    // read from shared memory, own or another block's, is all under way before the first is added.)
    const int d = threadIdx.x;
    uint32_t sum = 0;
    if (d < digits) {
      uint32_t c[kSortWarps];
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) c[w] = sort_smem[w * kDigits + d];
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) {
        sort_smem[w * kDigits + d] = sum;
        sum += c[w];
      }
      total[d] = sum;
    }
    uint32_t before = 0, all = sum;
    if (blocks > 1) {
      cluster_sync_all();
      if (d < digits) {
        uint32_t v[kSortCluster];
#pragma unroll
        for (uint32_t b = 0; b < kSortCluster; ++b) {
          v[b] = 0;
          if (b < blocks) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v[b]) : "r"(mapa_shared(smem_u32(total + d), b)));
        }
        all = 0;
#pragma unroll
        for (uint32_t b = 0; b < kSortCluster; ++b) {
          if (b < rank) before += v[b];
          all += v[b];
        }
      }
    }
    // Exclusive sums over the digits, of all pairs and of the block's.
    uint32_t inc = d < digits ? all : 0, own = d < digits ? sum : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, inc, o), u = __shfl_up_sync(0xffffffffu, own, o);
      if (lane >= o) inc += v, own += u;
    }
    if (lane == 31) sums[warp] = make_uint2(inc, own);
    __syncthreads();
    if (warp == 0) {
      const uint2 v = sums[lane];
      uint2 t = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, t.x, o), y = __shfl_up_sync(0xffffffffu, t.y, o);
        if (lane >= o) t.x += x, t.y += y;
      }
      sums[lane] = make_uint2(t.x - v.x, t.y - v.y);
    }
    __syncthreads();
    if (d < digits) {
      base[d] = sums[warp].x + inc - all + before;
      local[d] = sums[warp].y + own - sum;
    }
    __syncthreads();
    // To their places; by way of shared memory, in the block's own order, where it has so few that
    // they fit: a digit's are then written side by side.
    const bool few = mine_all <= kSortHeld;
    for (int64_t i = i0; i < i1; i += 32 * kHeld) {
      if (!once) load(i);
#pragma unroll
      for (int q = 0; q < kHeld; ++q) {
        if (i + 32 * q >= i1) break;
        const bool there = i + 32 * q + lane < i1;
        const uint32_t digit = there ? held[q].x >> shift & (digits - 1) : 0;
        // The lanes of the same digit, bit by bit: as long for any digits, where match_any takes a turn
        // for each of them (on 65536 tokens of a text, 4000 cycles less in the pass of the upper bits
        // and 2500 more in the lower ones').
        uint32_t same = __ballot_sync(0xffffffffu, there);
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {
          const uint32_t set = __ballot_sync(0xffffffffu, digit >> b & 1);
          same &= digit >> b & 1 ? set : ~set;
        }
        const uint32_t at = there ? mine[digit] : 0, ahead = __popc(same & ((1u << lane) - 1));
        __syncwarp();
        if (there) {
          if (ahead == 0) mine[digit] = at + __popc(same);
          if (few) {
            pairs[local[digit] + at + ahead] = held[q];
          } else {
            __stcg(to + base[digit] + at + ahead, held[q]);
          }
        }
        __syncwarp();
      }
    }
    if (few) {
      __syncthreads();
      for (int i = threadIdx.x; i < mine_all; i += kSortThreads) {
        const uint2 p = pairs[i];
        const uint32_t digit = p.x >> shift & (digits - 1);
        __stcg(to + base[digit] + (i - local[digit]), p);
      }
    }
    uint2* t = from;
    from = to;
    to = t;
    // (The pairs are read by other blocks, and the counts are set to zero.)
    if (blocks > 1) {
      cluster_sync_all();
    } else {
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------
// The sums over runs of equal rows.  A warp takes the runs that start in a chunk of 16
// sorted pairs, a slice of the rows' columns.  Runs of more than 16 pairs are cut
// at the chunks' ends: what of one lies in a chunk is summed into the chunk's FP32
// rows `parts` (its first one for a run that started before, its second for one that
// starts here), and join_runs_kernel adds those up in order.  So the work of a warp is
// bounded, however often a row is named, and every sum has one order.
//
// Memory bounds it where there is enough: 65536×2048 f32 added to 20000 rows 131 µs, 6.6 TB/s
// (pairs one run at a time, each waiting for its rows and for what they are added to: 230).
// 16384×1024 bf16, 33 MB, are 12 µs: one wave of warps, four to eight loads after each other.
// ---------------------------------------------------------------------------
constexpr int kChunkPairs = 16, kLongRun = 16, kSumWarps = 8;
constexpr int kFewParts = 8;  // that a warp adds up

// The rows around a chunk: the 32 pairs before it and the 64 from its first on.
struct Window {
  uint32_t before, a, b;  // rows (n where there is no pair)
  __device__ __forceinline__ void load(const uint2* sorted, int64_t m, uint32_t n, int64_t p0, int lane, uint2* pairs) {
    const int64_t p = p0 - 32 + lane;
    before = p >= 0 ? __ldg(&sorted[p].x) : 0xFFFFFFFFu;
    const uint2 none = make_uint2(n, 0), u = p0 + lane < m ? __ldg(sorted + p0 + lane) : none,
                v = p0 + 32 + lane < m ? __ldg(sorted + p0 + 32 + lane) : none;
    a = u.x, b = v.x;
    pairs[lane] = u, pairs[32 + lane] = v;
    __syncwarp();
  }
  __device__ __forceinline__ uint32_t row(int i) const { return __shfl_sync(0xffffffffu, a, i); }  // i < 32
  // Pairs of row r from place i on (of which it holds).
  __device__ __forceinline__ int count(uint32_t r, int i) const {
    return __popc(__ballot_sync(0xffffffffu, a == r) >> i) + __popc(__ballot_sync(0xffffffffu, b == r));
  }
  // Pairs of row r directly before the chunk (32: or more).
  __device__ __forceinline__ int behind(uint32_t r) const {
    const uint32_t other = ~__ballot_sync(0xffffffffu, before == r);
    return __clz(static_cast<int>(other));
  }
};

// By a warp, a piece of a row of dE from its sums: stored, or added to what is there.  Each is added
// to once, so an FP32 one can be left to the memory (a vector reduction; a result below
// 2^-126 counts as 0), which spares the way there and back; a 16-bit one is read (`old`,
// ahead) and rounded once.
template <int TYPE, int OUT, bool ADD>
__device__ __forceinline__ void finish_piece(void* dE, int64_t row, int64_t ldde, int64_t col, int n, float scale, bool vec,
                                             uint4 old, const float* sums) {
  using Y = Elem<OUT>;
  constexpr int V = Elem<TYPE>::V;
  typename Y::T* p = static_cast<typename Y::T*>(dE) + row * ldde + col;
#pragma unroll
  for (int h = 0; h < V; h += Y::V) {
    float o[Y::V];
#pragma unroll
    for (int e = 0; e < Y::V; ++e) o[e] = sums[h + e] * scale;
    if constexpr (ADD && OUT == OZ2_TYPE_F32) {
      if (vec && n >= h + 4) {
        asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p + h), "f"(o[0]), "f"(o[1]), "f"(o[2]),
                     "f"(o[3])
                     : "memory");
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (h + e < n) atomicAdd(reinterpret_cast<float*>(p) + h + e, o[e]);
      }
    } else {
      if constexpr (ADD) {
        float was[Y::V];
        Y::unpack(old, was);
#pragma unroll
        for (int e = 0; e < Y::V; ++e) o[e] = fmaf(sums[h + e], scale, was[e]);
      }
      if (vec) {
        store16_any(p + h, Y::pack(o), n - h, n >= h + Y::V);
      } else {
        store16_warp(p + h, Y::pack(o), min(max(n - h, 0), Y::V));
      }
    }
  }
}
// Pieces of a row to a lane: up to 16 FP32 sums.  (One a lane, the work on the pairs took
// longer than the rows: 65536 tokens of 2048 f32 398 µs.)
constexpr int most_pieces(int type) { return type == OZ2_TYPE_F32 ? 4 : 2; }

struct SumJob {
  int64_t m, k;
  uint32_t n;
  const void* dY;
  int64_t lddy;
  void* dE;
  int64_t ldde;
  float scale;
  int accumulate, vec;     // vec: dE's rows are on 16-byte boundaries
  const uint2* sorted;
  float* parts;            // two rows a chunk, of `slices` whole slices
  int4* runs;              // long runs of many parts: row, first chunk and how many; those of few from the end on
  int* long_runs;          // how many of either
  int most_runs;
  int slices, pieces;      // of a row, and of a slice to a lane
};

// What a piece of dE holds.  (Words around it may hold others' pieces, which are not looked at.)
template <int OUT>
__device__ __forceinline__ uint4 old_piece(const SumJob& j, int64_t row, int64_t col, int n) {
  using T = typename Elem<OUT>::T;
  const T* base = static_cast<const T*>(j.dE);
  const T* p = base + row * j.ldde + col;
  if (j.vec) return load_piece<true, false>(p, base, base, n);
  return load_piece<false, false>(p, base, base + (static_cast<int64_t>(j.n) - 1) * j.ldde + j.k, n);
}

// The next lane's word, of the last lane lane `from`'s `after`.
__device__ __forceinline__ uint4 next_lane(uint4 v, uint4 after, int from, int lane) {
  uint4 r;
  auto one = [&](uint32_t a, uint32_t b) {
    const uint32_t x = __shfl_down_sync(0xffffffffu, a, 1), y = __shfl_sync(0xffffffffu, b, from);
    return lane == 31 ? y : x;
  };
  r.x = one(v.x, after.x), r.y = one(v.y, after.y), r.z = one(v.z, after.z), r.w = one(v.w, after.w);
  return r;
}

template <int TYPE, int OUT, int P, bool ALIGNED, bool ADD>
__global__ void __launch_bounds__(32 * kSumWarps, (P == 1 ? 4 : P == 2 ? 3 : 2) - (ALIGNED || P == 4 ? 0 : 1)) sum_runs_kernel(SumJob j) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  constexpr int V = X::V;
  __shared__ uint2 pairs_s[kSumWarps][64];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kSumWarps + warp, chunk = unit / j.slices;
  const int slice = static_cast<int>(unit - chunk * j.slices);
  const int64_t p0 = chunk * kChunkPairs;
  if (p0 >= j.m) return;
  const uint2* pairs = pairs_s[warp];
  Window w;
  w.load(j.sorted, j.m, j.n, p0, lane, pairs_s[warp]);
  const int64_t col0 = (static_cast<int64_t>(slice) * P * 32 + lane) * V;
  auto col = [&](int i) { return col0 + i * 32 * V; };
  auto there = [&](int i) { return static_cast<int>(max(int64_t(0), min(int64_t(V), j.k - col(i)))); };
  const T* src = static_cast<const T*>(j.dY);
  const T* stop = src + (j.m - 1) * j.lddy + j.k;
  // What of the window is this warp's: from `begin` on (what lies before is a run's that
  // started before) to `end`, a part of such a run that is long up to `head`, and a long
  // run's first part from where the last one started.
  uint32_t r = w.row(0);
  if (r >= j.n) return;
  int begin = 0, head = 0;
  const int behind = w.behind(r);
  if (behind) {
    const int here = w.count(r, 0);
    if (behind + here > kLongRun) {
      head = min(here, kChunkPairs);
    } else {
      begin = here;
    }
  }
  if (begin >= kChunkPairs) return;
  const uint32_t valid = __ballot_sync(0xffffffffu, w.a < j.n);
  r = w.row(kChunkPairs - 1);
  int end = kChunkPairs, tail = 0;
  if (r < j.n) {  // the last run that starts here, or goes through
    const int last = __ffs(__ballot_sync(0xffffffffu, w.a == r)) - 1, here = w.count(r, last);
    if (last > 0 || !behind) {
      if (here > kLongRun) {
        tail = 1;
      } else {
        end = last + here;
      }
    }
  } else {
    end = __popc(valid);
  }
  // Places whose pair is the last of its row.
  const uint32_t after = __shfl_down_sync(0xffffffffu, w.a, 1), b0 = __shfl_sync(0xffffffffu, w.b, 0),
                 after_b = __shfl_down_sync(0xffffffffu, w.b, 1);
  const uint64_t ends = __ballot_sync(0xffffffffu, w.a != (lane < 31 ? after : b0)) |
                        static_cast<uint64_t>(__ballot_sync(0xffffffffu, lane < 31 && w.b != after_b)) << 32;
  float s[P][V];
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) s[i][e] = 0.f;
  };
  auto keep = [&](int which) {
    float* p = j.parts + ((2 * chunk + which) * j.slices + slice) * (32 * P * V) + lane * V;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int h = 0; h < V; h += 4)
        *reinterpret_cast<float4*>(p + i * 32 * V + h) = make_float4(s[i][h], s[i][h + 1], s[i][h + 2], s[i][h + 3]);
  };
  clear();
  // Several pairs at a time, whatever rows they are of: all loads are under way before the
  // first is added, and so are the old values of 16-bit rows that are added to.
  constexpr bool kOld = ADD && OUT != OZ2_TYPE_F32;
  constexpr int kAtOnce = (P == 4 ? 16 : 8) / P / (kOld ? 2 : 1);
  // Rows off the 16-byte grid: a lane loads the word in which its piece begins, the next lane's is the
  // one after it, and what comes after the last lane's are one load more, a lane's for each piece.
  // (Two words a piece, each waited for: 65536×1001 bf16 into 1000 rows 144 µs in all, so 89, and 66 at
  // 1000.  More blocks an SM spill.)
  const char* const first = reinterpret_cast<const char*>(src);
  const int64_t slice0 = static_cast<int64_t>(slice) * P * 32 * V, slice1 = min(j.k, slice0 + P * 32 * V);
  auto words_there = [&](const T* row) {  // the words around the slice are the tensor's own
    const uintptr_t from = reinterpret_cast<uintptr_t>(row + slice0) & ~static_cast<uintptr_t>(15),
                    to = (reinterpret_cast<uintptr_t>(row + slice1) + 15) & ~static_cast<uintptr_t>(15);
    return from >= reinterpret_cast<uintptr_t>(first) && to <= reinterpret_cast<uintptr_t>(stop);
  };
  for (int i = begin; i < end; i += kAtOnce) {
    uint4 v[kAtOnce][P], old[kOld ? kAtOnce : 1][P], after = make_uint4(0, 0, 0, 0);
    const char* after_at = nullptr;
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      const int at = min(i + q, end - 1);
      const uint2 pair = pairs[at];
      const T* row = src + static_cast<int64_t>(pair.y) * j.lddy;
      const bool words = !ALIGNED && words_there(row);
#pragma unroll
      for (int c = 0; c < P; ++c) {
        const int n = there(c);
        if (ALIGNED) {
          if (n > 0 && i + q < end) v[q][c] = load_piece<true>(row + col(c), src, stop, n);
        } else if (words && i + q < end) {
          const char* stops = reinterpret_cast<const char*>(row + slice1);
          const char* word = reinterpret_cast<const char*>(row + col(c)) - (reinterpret_cast<uintptr_t>(row) & 15);
          if (word < stops) v[q][c] = load_global<true>(reinterpret_cast<const uint4*>(word));
          const char* next = word + 16 * (32 - lane);  // (behind lane 31's)
          if (lane == q * P + c && next < stops) after_at = next;
        }
        if (kOld && n > 0 && i + q < end && (ends >> at & 1) && at >= head)
          old[kOld ? q : 0][c] = old_piece<OUT>(j, pair.x, col(c), n);
      }
    }
    if (!ALIGNED && after_at) after = load_global<true>(reinterpret_cast<const uint4*>(after_at));
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      const int at = i + q;
      if (at >= end) break;
#pragma unroll
      for (int c = 0; c < P; ++c) {
        if (!ALIGNED) {
          const T* row = src + static_cast<int64_t>(pairs[at].y) * j.lddy;
          if (words_there(row)) {
            const Words w{v[q][c], next_lane(v[q][c], after, q * P + c, lane)};
            v[q][c] = shift_words16(reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(row) & 15), w);
          } else if (there(c) > 0) {
            v[q][c] = load16_singly(row + col(c), there(c));
          }
        }
        float f[V];
        X::unpack(v[q][c], f);
#pragma unroll
        for (int e = 0; e < V; ++e) s[c][e] += f[e];
      }
      if (at + 1 == head) {
        keep(0);
        clear();
      } else if (ends >> at & 1) {
#pragma unroll
        for (int c = 0; c < P; ++c)
          finish_piece<TYPE, OUT, ADD>(j.dE, pairs[at].x, j.ldde, col(c), there(c), j.scale, j.vec, old[kOld ? q : 0][c], s[c]);
        clear();
      }
    }
  }
  if (!tail) return;
  keep(1);
  if (slice == 0) {  // how many chunks the run reaches: those whose first pair is its
    int64_t c = chunk + 1;
    for (;;) {
      const int64_t p = (c + lane) * kChunkPairs;
      const uint32_t in = __ballot_sync(0xffffffffu, p < j.m && __ldg(&j.sorted[p < j.m ? p : 0].x) == r);
      c += __popc(in);
      if (in != 0xFFFFFFFFu) break;
    }
    if (lane == 0) {  // (the lists' order is that of the warps: no sum depends on it)
      const int few = c - chunk <= kFewParts, at = atomicAdd(j.long_runs + few, 1);
      j.runs[few ? j.most_runs - 1 - at : at] = make_int4(static_cast<int>(r), static_cast<int>(chunk), static_cast<int>(c - chunk), 0);
    }
  }
}

// The parts of a long run, a piece of its columns at a time: by a warp, or where there are
// many of them by a block, each warp of which adds up a stretch; the warps' sums are added
// in order.
constexpr int kJoinWarps = 16;

template <int TYPE, int OUT, bool ADD>
__global__ void __launch_bounds__(32 * kJoinWarps) join_runs_kernel(SumJob j) {
  constexpr int V = Elem<TYPE>::V;
  __shared__ float sums[kJoinWarps][32 * V];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pieces = static_cast<int>((j.k + 32 * V - 1) / (32 * V));
  const int64_t row_floats = static_cast<int64_t>(j.slices) * j.pieces * 32 * V;
  float s[V];
  auto add = [&](int64_t chunk, int piece, int c0, int c1) {
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = 0.f;
#pragma unroll 8
    for (int c = c0; c < c1; ++c) {
      const float* p = j.parts + (2 * (chunk + c) + (c == 0)) * row_floats + (static_cast<int64_t>(piece) * 32 + lane) * V;
#pragma unroll
      for (int h = 0; h < V; h += 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + h);
        s[h] += v.x, s[h + 1] += v.y, s[h + 2] += v.z, s[h + 3] += v.w;
      }
    }
  };
  auto finish = [&](int row, int piece) {
    const int64_t col = (static_cast<int64_t>(piece) * 32 + lane) * V;
    const int n = static_cast<int>(max(int64_t(0), min(int64_t(V), j.k - col)));
    uint4 old = make_uint4(0, 0, 0, 0);
    if (ADD && OUT != OZ2_TYPE_F32 && n > 0) old = old_piece<OUT>(j, row, col, n);
    finish_piece<TYPE, OUT, ADD>(j.dE, row, j.ldde, col, n, j.scale, j.vec, old, s);
  };
  const int many = j.long_runs[0], few = j.long_runs[1];
  for (int64_t u = static_cast<int64_t>(warp) * gridDim.x + blockIdx.x; u < static_cast<int64_t>(few) * pieces;
       u += static_cast<int64_t>(gridDim.x) * kJoinWarps) {
    const int at = static_cast<int>(u / pieces), piece = static_cast<int>(u - static_cast<int64_t>(at) * pieces);
    const int4 run = j.runs[j.most_runs - 1 - at];
    add(run.y, piece, 0, run.z);
    finish(run.x, piece);
  }
  for (int64_t u = blockIdx.x; u < static_cast<int64_t>(many) * pieces; u += gridDim.x) {
    const int at = static_cast<int>(u / pieces), piece = static_cast<int>(u - static_cast<int64_t>(at) * pieces);
    const int4 run = j.runs[at];
    const int each = (run.z + kJoinWarps - 1) / kJoinWarps, c0 = min(run.z, warp * each);
    add(run.y, piece, c0, min(run.z, c0 + each));
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) sums[warp][lane * V + e] = s[e];
    __syncthreads();
    if (warp == 0) {
      for (int o = 1; o < kJoinWarps; ++o)
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] += sums[o][lane * V + e];
      finish(run.x, piece);
    }
  }
}

// ---------------------------------------------------------------------------
// The gradient of few tokens, in one launch without a sort.  A block takes a token and 8 × 512
// bytes of its row; where no token before it names the same row, it lists those that do and
// adds theirs up in order.  The other blocks write the zeros of a gradient that is not added
// to: of a stretch of rows, those that no token names.  (Sorted, 64 tokens of 64 f32 took 13 µs; so 4.)
// ---------------------------------------------------------------------------
constexpr int kFewTokens = 256, kFillStretch = 2048;

template <int TYPE, int OUT, bool ALIGNED, bool ADD>
__global__ void __launch_bounds__(32 * kSumWarps) few_tokens_kernel(SumJob j, Ids ids, int across, FillJob f, int stretch) {
  using X = Elem<TYPE>;
  using T = typename X::T;
  constexpr int V = X::V;
  __shared__ int rows_s[kFewTokens], list_s[kFewTokens], count_s[kSumWarps];
  __shared__ uint32_t named_s[kFillStretch / 32];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = static_cast<int>(j.m);
  const int64_t id = static_cast<int>(threadIdx.x) < m ? ids[threadIdx.x] : -1;
  const int mine = id >= 0 && id < j.n ? static_cast<int>(id) : -1;
  rows_s[threadIdx.x] = mine;
  __syncthreads();
  const int sums = m * across;
  if (static_cast<int>(blockIdx.x) >= sums) {
    const int64_t blocks = gridDim.x - sums;
    for (int64_t r0 = (blockIdx.x - sums) * static_cast<int64_t>(stretch); r0 < f.rows; r0 += blocks * stretch) {
      for (int i = threadIdx.x; i < kFillStretch / 32; i += 32 * kSumWarps) named_s[i] = 0;
      __syncthreads();
      if (mine >= r0 && mine < r0 + stretch) atomicOr(&named_s[(mine - r0) >> 5], 1u << ((mine - r0) & 31));
      __syncthreads();
      const int rows = static_cast<int>(min(static_cast<int64_t>(stretch), f.rows - r0));
      auto named = [&](int r) { return (named_s[r >> 5] >> (r & 31) & 1) != 0; };
      if (j.vec && f.bytes % 16 == 0) {  // (short rows: several to a warp)
        const int64_t words = f.bytes >> 4, all = rows * words;
        int64_t r = threadIdx.x / words, c = threadIdx.x - r * words;
        const int64_t step_rows = 32 * kSumWarps / words, step_words = 32 * kSumWarps - step_rows * words;
        for (int64_t i = threadIdx.x; i < all; i += 32 * kSumWarps) {
          if (!named(static_cast<int>(r))) *reinterpret_cast<uint4*>(f.p + (r0 + r) * f.ld + 16 * c) = make_uint4(0, 0, 0, 0);
          r += step_rows;
          c += step_words;
          if (c >= words) c -= words, ++r;
        }
      } else {
        for (int r = warp; r < rows; r += kSumWarps)
          if (!named(r)) zero_row(f.p + (r0 + r) * f.ld, f.bytes, f.unit, lane, 32);
      }
      __syncthreads();
    }
    return;
  }
  const int token = blockIdx.x / across, slice = (blockIdx.x - token * across) * kSumWarps + warp, row = rows_s[token];
  if (row < 0) return;
  const uint32_t same = __ballot_sync(0xffffffffu, mine == row);
  if (lane == 0) count_s[warp] = __popc(same);
  __syncthreads();
  int before = 0, count = 0;
#pragma unroll
  for (int w = 0; w < kSumWarps; ++w) {
    before += w < warp ? count_s[w] : 0;
    count += count_s[w];
  }
  if (mine == row) list_s[before + __popc(same & ((1u << lane) - 1))] = threadIdx.x;
  __syncthreads();
  if (list_s[0] != token) return;
  const int64_t col = (static_cast<int64_t>(slice) * 32 + lane) * V;
  const int n = static_cast<int>(max(int64_t(0), min(int64_t(V), j.k - col)));
  const T* src = static_cast<const T*>(j.dY);
  const T* stop = src + (j.m - 1) * j.lddy + j.k;
  uint4 old = make_uint4(0, 0, 0, 0);
  if (ADD && OUT != OZ2_TYPE_F32 && n > 0) old = old_piece<OUT>(j, row, col, n);
  float s[V];
#pragma unroll
  for (int e = 0; e < V; ++e) s[e] = 0.f;
  for (int i = 0; i < count; i += 8) {
    uint4 v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (i + q < count && n > 0) v[q] = load_piece<ALIGNED>(src + list_s[i + q] * j.lddy + col, src, stop, n);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if (i + q >= count) break;
      float x[V];
      X::unpack(v[q], x);
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] += x[e];
    }
  }
  finish_piece<TYPE, OUT, ADD>(j.dE, row, j.ldde, col, n, j.scale, j.vec, old, s);
}
static_assert(kFewTokens == 32 * kSumWarps, "a thread to a token");

template <int TYPE, int OUT>
cudaError_t launch_few(const SumJob& j, Ids ids, const FillJob& f, cudaStream_t st) {
  const bool aligned = rows_on16(j.dY, j.lddy, type_bytes(TYPE)), add = j.accumulate != 0;
  auto kern = aligned ? (add ? few_tokens_kernel<TYPE, OUT, true, true> : few_tokens_kernel<TYPE, OUT, true, false>)
                      : (add ? few_tokens_kernel<TYPE, OUT, false, true> : few_tokens_kernel<TYPE, OUT, false, false>);
  const int across = static_cast<int>((j.k * type_bytes(TYPE) + 512 * kSumWarps - 1) / (512 * kSumWarps));
  const int64_t most = 8 * static_cast<int64_t>(num_sms());  // blocks that write zeros, of 8 rows at least
  const int stretch = static_cast<int>(std::min<int64_t>(kFillStretch, std::max<int64_t>(8, (f.rows + most - 1) / most)));
  const int64_t fill = add ? 0 : std::min(most, (f.rows + stretch - 1) / stretch);
  const int64_t blocks = j.m * across + fill;
  if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
  count_launch();
  return launch_dependent(kern, dim3(static_cast<unsigned>(blocks)), dim3(32 * kSumWarps), 0, st, j, ids, across, f, stretch);
}

// Pieces to a lane, and the slices of a row that come of it.
// As many as leave 24 warps an SM (16384 tokens of 1024 bf16: 17 µs with two, 12 with one).
int64_t chunks_of(int64_t m) { return (m + kChunkPairs - 1) / kChunkPairs; }
int64_t slices_of(int64_t k, int type, int pieces) { return (k * type_bytes(type) + 512 * pieces - 1) / (512 * pieces); }
int pieces_of(int64_t m, int64_t k, int type) {
  int p = most_pieces(type);
  while (p > 1 && (512 * p / 2 >= k * type_bytes(type) || chunks_of(m) * slices_of(k, type, p) < 24 * static_cast<int64_t>(num_sms())))
    p /= 2;
  return p;
}
size_t up(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

using SumKernel = void (*)(SumJob);
template <int TYPE, int OUT, int P>
SumKernel sum_kernel_of(bool aligned, bool add) {
  return aligned ? (add ? sum_runs_kernel<TYPE, OUT, P, true, true> : sum_runs_kernel<TYPE, OUT, P, true, false>)
                 : (add ? sum_runs_kernel<TYPE, OUT, P, false, true> : sum_runs_kernel<TYPE, OUT, P, false, false>);
}
template <int TYPE, int OUT>
SumKernel sum_kernel(int pieces, bool aligned, bool add) {
  return pieces == 1   ? sum_kernel_of<TYPE, OUT, 1>(aligned, add)
         : pieces == 2 ? sum_kernel_of<TYPE, OUT, 2>(aligned, add)
                       : sum_kernel_of<TYPE, OUT, most_pieces(TYPE)>(aligned, add);
}
template <int TYPE>
cudaError_t launch_sums(const SumJob& j, int de_type, cudaStream_t st) {
  const bool aligned = rows_on16(j.dY, j.lddy, type_bytes(TYPE)), add = j.accumulate != 0, same = de_type == TYPE;
  const int64_t blocks = (chunks_of(j.m) * j.slices + kSumWarps - 1) / kSumWarps;
  if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
  constexpr int F32 = OZ2_TYPE_F32;
  SumKernel sum = same ? sum_kernel<TYPE, TYPE>(j.pieces, aligned, add) : sum_kernel<TYPE, F32>(j.pieces, aligned, add);
  count_launch();
  cudaError_t err = launch_dependent(sum, dim3(static_cast<unsigned>(blocks)), dim3(32 * kSumWarps), 0, st, j);
  if (err != cudaSuccess || j.m <= kLongRun) return err;
  const int64_t most = (j.m / (kLongRun + 1) * j.slices * j.pieces + 1) / 2;
  SumKernel join = same ? (add ? join_runs_kernel<TYPE, TYPE, true> : join_runs_kernel<TYPE, TYPE, false>)
                        : (add ? join_runs_kernel<TYPE, F32, true> : join_runs_kernel<TYPE, F32, false>);
  count_launch();
  return launch_dependent(join, dim3(static_cast<unsigned>(std::min<int64_t>(most, 2 * num_sms()))), dim3(32 * kJoinWarps), 0, st, j);
}

}  // namespace

cudaError_t launch_embedding(int64_t m, int64_t n, int64_t k, int type, Ids ids, const void* E, int64_t lde, float scale,
                             void* Y, int64_t ldy, cudaStream_t st) {
  const int es = type_bytes(type);
  const bool aligned = rows_on16(E, lde, es) && rows_on16(Y, ldy, es);
  const int64_t per = (k * es + 15) / 16;
  // (A grid's stride in pieces is below 2^20, so pieces count in 32 bits within a row.)
  const int64_t blocks = std::min<int64_t>((m * per + 255) / 256, kBlocks * static_cast<int64_t>(num_sms()));
  auto kern = type == OZ2_TYPE_F32    ? (aligned ? embedding_kernel<OZ2_TYPE_F32, true> : embedding_kernel<OZ2_TYPE_F32, false>)
              : type == OZ2_TYPE_BF16 ? (aligned ? embedding_kernel<OZ2_TYPE_BF16, true> : embedding_kernel<OZ2_TYPE_BF16, false>)
                                      : (aligned ? embedding_kernel<OZ2_TYPE_F16, true> : embedding_kernel<OZ2_TYPE_F16, false>);
  count_launch();
  return launch_dependent(kern, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, m, n, k, ids, E, lde, scale, Y, ldy);
}

size_t embedding_grad_scratch(int64_t m, int64_t k, int type) {
  if (m <= kFewTokens) return 0;
  const size_t chunks = static_cast<size_t>(chunks_of(m));
  const int pieces = pieces_of(m, k, type);
  const size_t values = 512 / type_bytes(type) * pieces;  // of a slice
  return 2 * up(sizeof(uint2) * m) + up(sizeof(int4) * (m / (kLongRun + 1) + 1)) + 256 +
         up(m > kLongRun ? sizeof(float) * 2 * chunks * slices_of(k, type, pieces) * values : 0);
}

cudaError_t launch_embedding_grad(int64_t m, int64_t n, int64_t k, int type, const void* dY, int64_t lddy, Ids ids,
                                  float scale, void* dE, int64_t ldde, int de_type, bool accumulate, void* scratch,
                                  cudaStream_t st) {
  const int es = type_bytes(de_type);
  if (m <= kFewTokens) {
    const SumJob j{m,     k,          static_cast<uint32_t>(n), dY,      lddy,    dE, ldde, scale,
                   accumulate, rows_on16(dE, ldde, es),  nullptr, nullptr, nullptr, nullptr, 0, 0, 0};
    const FillJob f{static_cast<char*>(dE), n, k * es, ldde * es, es};
    if (type == OZ2_TYPE_F32) return launch_few<OZ2_TYPE_F32, OZ2_TYPE_F32>(j, ids, f, st);
    if (type == OZ2_TYPE_BF16)
      return de_type == type ? launch_few<OZ2_TYPE_BF16, OZ2_TYPE_BF16>(j, ids, f, st)
                             : launch_few<OZ2_TYPE_BF16, OZ2_TYPE_F32>(j, ids, f, st);
    return de_type == type ? launch_few<OZ2_TYPE_F16, OZ2_TYPE_F16>(j, ids, f, st)
                           : launch_few<OZ2_TYPE_F16, OZ2_TYPE_F32>(j, ids, f, st);
  }
  char* at = static_cast<char*>(scratch);
  auto take = [&](size_t bytes) {
    char* p = at;
    at += up(bytes);
    return p;
  };
  uint2* a = reinterpret_cast<uint2*>(take(sizeof(uint2) * m));
  uint2* b = reinterpret_cast<uint2*>(take(sizeof(uint2) * m));
  int4* runs = reinterpret_cast<int4*>(take(sizeof(int4) * (m / (kLongRun + 1) + 1)));
  int* long_runs = reinterpret_cast<int*>(take(256));
  float* parts = reinterpret_cast<float*>(at);
  int bits = 1;
  while (n >> bits) ++bits;  // of the rows 0 to n
  const int passes = (bits + kDigitBits - 1) / kDigitBits;
  SortJob s{ids, m, static_cast<uint32_t>(n), passes, (bits + passes - 1) / passes, a, b, long_runs};
  // A block sorts up to 2048 tokens as fast as a cluster, and a cluster of 8 up to 8192 as fast as one
  // of 16 (gradients of 64 columns, 50257 rows: 2048 tokens 20.0 µs with one block, 21.1 with 8; 8192
  // 22.8 with 8, 23.5 with 16; 16384 26.0 and 24.4).  A part of a device may have room for less.
  const void* sort = reinterpret_cast<const void*>(sort_tokens_kernel);
  cudaError_t err = allow_smem(sort, kSortSmem);
  if (err != cudaSuccess) return err;
  const int sorters = m <= 2048 ? 1 : std::min(m <= 8192 ? 8 : kSortCluster, cluster_blocks(sort, kSortThreads, kSortSmem, kSortCluster));
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(sorters));
  cfg.blockDim = dim3(kSortThreads);
  cfg.dynamicSmemBytes = kSortSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(sorters);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  count_launch();
  err = cudaLaunchKernelEx(&cfg, sort_tokens_kernel, s, sorters);
  if (err != cudaSuccess) return err;
  if (!accumulate) {
    const bool whole = ldde == k || n == 1;
    const FillJob f{static_cast<char*>(dE), whole ? 1 : n, (whole ? n : 1) * k * es, ldde * es, es};
    const int64_t blocks = std::min<int64_t>(n * k * es / (64 * kFillThreads) + 1, 8 * static_cast<int64_t>(num_sms()));
    count_launch();
    err = launch_dependent(fill_rows_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kFillThreads), 0, st, f);
    if (err != cudaSuccess) return err;
  }
  const int pieces = pieces_of(m, k, type);
  SumJob j{m, k, static_cast<uint32_t>(n), dY, lddy, dE, ldde, scale, accumulate, rows_on16(dE, ldde, es),
           passes & 1 ? a : b, parts, runs, long_runs, static_cast<int>(m / (kLongRun + 1) + 1),
           static_cast<int>(slices_of(k, type, pieces)), pieces};
  return type == OZ2_TYPE_F32    ? launch_sums<OZ2_TYPE_F32>(j, de_type, st)
         : type == OZ2_TYPE_BF16 ? launch_sums<OZ2_TYPE_BF16>(j, de_type, st)
                                 : launch_sums<OZ2_TYPE_F16>(j, de_type, st);
}

}  // namespace oz2
