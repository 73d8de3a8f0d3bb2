// What the entry points of the layer operators share on the host: alignment, workspace,
// and operands that are copied to rows which TMA can read.
#pragma once

#include <algorithm>

#include "lin_common.cuh"

namespace oz2 {

constexpr int64_t kMaxSize = (1LL << 31) - 256;  // tile coordinates are 32-bit

inline size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
// Rows of copies: whole 128-byte lines, which TMA's pieces of a row then are too.  (On
// 16-byte boundaries alone a piece touches one 32-byte sector more, and the loads bound
// the product: 4097³ forward 135 µs, so 110; its gradient's products 256 and 210.)
inline int64_t padded_ld(int64_t cols, int bytes) { return (cols * bytes + 127) / 128 * 128 / bytes; }
inline bool on16(const void* p, int64_t ld, int bytes) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * bytes)) & 15) == 0;
}
// Rows on 16-byte boundaries that are not 32-byte ones.  Where both operands' are, TMA's
// pieces touch a fifth sector each and bound the product (9728×8192² bf16: 965 µs against
// 701, and 783 with one of them on 32 bytes), and a copy of one of them pays once its
// bytes, there and back at 6.8 TB/s, and its launch take less than a fifth of the product.
inline bool on16_only(const void* p, int64_t ld, int bytes) {
  return on16(p, ld, bytes) && ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * bytes)) & 16) != 0;
}
inline bool copy_pays(double copied_bytes, double multiplications, int bytes) {
  const double product_us = multiplications / (bytes == 1 ? 1.9e9 : 0.95e9);
  return 2 * copied_bytes / 6.8e6 + 3 < 0.2 * product_us;
}
inline bool on(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline int status_of(cudaError_t e) { return e == cudaSuccess ? OZ2_OK : OZ2_ERR_CUDA; }

// Pieces of one stream-ordered allocation; empty when nothing was asked for.
class Workspace {
 public:
  explicit Workspace(cudaStream_t st) : st_(st) {}
  ~Workspace() {
    if (base_) cudaFreeAsync(base_, st_);
  }
  Workspace(const Workspace&) = delete;
  Workspace& operator=(const Workspace&) = delete;
  size_t ask(size_t bytes) {
    const size_t at = total_;
    total_ = up256(total_ + bytes);
    return at;
  }
  bool take() {
    if (total_ == 0) return true;
    if (workspace_alloc(&base_, total_, st_) == cudaSuccess) return true;
    cudaGetLastError();
    base_ = nullptr;
    return false;
  }
  template <typename T>
  T* at(size_t off) const {
    return reinterpret_cast<T*>(static_cast<char*>(base_) + off);
  }

 private:
  cudaStream_t st_;
  void* base_ = nullptr;
  size_t total_ = 0;
};

// An operand of a product as the kernels take it: in place, or a copy whose
// rows start on 16-byte boundaries.
struct Operand {
  const void* p;
  int64_t ld, rows, cols;
  int bytes;
  bool copy;
  size_t off;
  Operand(const void* src, int64_t ld_src, int64_t r, int64_t c, int b, Workspace& ws, bool must = false)
      : p(src), ld(r > 1 ? ld_src : padded_ld(c, b)), rows(r), cols(c), bytes(b), copy(must || !on16(src, ld, b)), off(0) {
    if (copy) off = ws.ask(static_cast<size_t>(rows) * padded_ld(cols, bytes) * bytes);
  }
};

// The copies that the operands want, in one launch.
inline cudaError_t place(Operand& a, Operand& b, const Workspace& ws, cudaStream_t st) {
  PackJob jobs[2];
  int count = 0;
  for (Operand* o : {&a, &b}) {
    if (!o->copy || o->rows == 0 || o->cols == 0) continue;
    PackJob& j = jobs[count++];
    j = PackJob{o->p, o->ld, o->rows, o->cols, ws.at<void>(o->off), padded_ld(o->cols, o->bytes)};
    o->p = j.dst;
    o->ld = j.ld_dst;
  }
  return count ? launch_pack_rows(jobs, count, a.bytes, st) : cudaSuccess;
}

}  // namespace oz2
