// The tensor cores' operands of the 16-bit and E4M3 products, and what an epilogue's
// warp does with its sums: shared by the kernels of a linear layer (k_linear.cu) and of
// a vocabulary's losses (k_head.cu).
#pragma once

#include "lin_common.cuh"

namespace oz2 {

// Instruction descriptor of kind::f16 with FP32 sums: D = F32 (bits 4-5 = 1), A
// and B BF16 (1) or F16 (0) in bits 7-9 and 10-12, MN-major A and B in bits 15
// and 16, N >> 3 in 17-22, M >> 4 in 24-28.
constexpr uint32_t idesc_16(int M, int N, bool bf16, bool a_mn, bool b_mn) {
  return (1u << 4) | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
         (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// The instruction descriptor and the operands' descriptors of the MMAs of one
// operand type and storage, constants but for the tile's address.
template <int TYPE, bool A_MN, bool B_MN, int M, int N>
struct MmaShape {
  static constexpr uint32_t idesc =
      TYPE == OZ2_TYPE_E4M3 ? idesc_f8_f32(M, N) : idesc_16(M, N, TYPE == OZ2_TYPE_BF16, A_MN, B_MN);
  // 32 bytes of depth an instruction: 32 bytes along a K-major row, 16 depth rows
  // of 128 bytes in MN-major storage (in the descriptors' units of 16 bytes).
  static constexpr uint32_t a_next = A_MN ? 128 : 2, b_next = B_MN ? 128 : 2;
};

// The descriptor of a tile in MN-major storage: 64-element (128-byte) row
// blocks kTileBytes/2 apart (leading byte offset), groups of 8 depth rows 1024
// bytes apart (stride byte offset), 128-byte swizzle.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t saddr) {
  return (smem_desc_sw128(saddr) & ~(0x3FFFull << 16)) | (static_cast<uint64_t>(kTileBytes / 2 >> 4) << 16);
}

// One lane of a whole warp, known to the compiler as one: its TMA and tensor-core
// instructions take their operands from uniform registers as they are.  Under
// `lane == 0` each is issued in a loop over the lanes that might be there (a
// producer's step of two loads took 660 cycles in place of 300).
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred P;\n elect.sync _|P, 0xffffffff;\n selp.u32 %0, 1, 0, P;\n}\n" : "=r"(p));
  return p != 0;
}

template <bool MN>
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr) {
  return MN ? smem_desc_mn(saddr) : smem_desc_sw128(saddr);
}

template <bool F8>
__device__ __forceinline__ void mma_pair(uint32_t me, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                         uint32_t accumulate) {
  if (F8) {
    mma_f8_pair(me, d_tmem, a_desc, b_desc, idesc, accumulate);
  } else {
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
        " @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(me)
        : "memory");
  }
}

// --- an epilogue warp's 32 rows × 64 bytes in shared memory ---------------------
// 16-byte piece c of row r at r·64 + (c ^ (r/2 & 3))·16: eight threads' own rows and
// two rows' eight pieces are both free of bank conflicts.
__device__ __forceinline__ uint32_t piece_at(int row, int c) { return row * 64 + ((c ^ (row >> 1 & 3)) << 4); }

__device__ __forceinline__ uint4 lds128(const uint8_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void sts128(uint8_t* p, uint4 v) { *reinterpret_cast<uint4*>(p) = v; }

__device__ __forceinline__ bool vec_ok(const void* p, int64_t ld, int bytes) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * bytes)) & 15) == 0;
}
// A warp's 32 rows × 32 columns of 16 bits from there to global memory: by 16 bytes a
// lane, eight rows at a time (`to`: this lane's place in the first eight rows), or by
// single values, and what lies past the matrix is not touched.
__device__ __forceinline__ void store_fast(uint16_t* to, int64_t ld, int lane, const uint8_t* buf) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<uint4*>(to + 8 * i * ld) = lds128(buf + piece_at(8 * i + (lane >> 2), lane & 3));
}
__device__ __forceinline__ uint8_t* value_at(uint8_t* buf, int row, int col) {
  return buf + piece_at(row, col >> 3) + 2 * (col & 7);
}
static __device__ __noinline__ void store_slow(void* dst, int64_t ld, int64_t rows, int64_t cols, int64_t row0,
                                               int64_t col0, int lane, uint8_t* buf) {
  uint16_t* d = static_cast<uint16_t*>(dst) + row0 * ld + col0 + lane;
  if (col0 + lane >= cols) return;
#pragma unroll 8
  for (int r = 0; r < 32; ++r)
    if (row0 + r < rows) d[r * ld] = *reinterpret_cast<const uint16_t*>(value_at(buf, r, lane));
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr));
}

}  // namespace oz2
