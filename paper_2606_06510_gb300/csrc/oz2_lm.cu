// Entry points of the operators at a language model's ends (declared in
// include/oz2_lm.h): argument checks, workspace, and the order of their launches.
#include <algorithm>
#include <cmath>

#include "../../include/oz2_lm.h"
#include "lin_host.cuh"
#include "lm_common.cuh"

namespace oz2 {
namespace {

bool valid_type(int t) { return t == OZ2_TYPE_F32 || is_16bit(t); }
bool valid_ids(int bits) { return bits == 64 || bits == 32; }
bool too_large(int64_t a, int64_t b, int64_t c) { return a >= kMaxSize || b >= kMaxSize || c >= kMaxSize; }

// The bytes of dz, in 16 bits, that a piece of the vocabulary may have.  (Against no pieces,
// 8192×131072×2048 takes 1.4% longer, with 128 MB 2.7%; 4096×50257×1024 in two pieces of 256 MB 2.6%.)
constexpr int64_t kPieceBytes = 512LL << 20;

int64_t piece_columns(int64_t m, int64_t n) {
  const int64_t most = std::max<int64_t>(256, kPieceBytes / 2 / m / 256 * 256), pieces = (n + most - 1) / most;
  return std::min(n, ((n + pieces - 1) / pieces + 255) / 256 * 256);
}

struct HeadCall {
  int64_t m, n, k;
  int type;
  const void* X;
  int64_t ldx;
  const void* W;
  int64_t ldw;
  HeadTargets t;
  float scale, z_loss;
};

int check_head(const HeadCall& c, int id_bits) {
  if (c.m < 0 || c.n < 0 || c.k < 0 || !is_16bit(c.type) || !valid_ids(id_bits) || c.n < 1) return OZ2_ERR_INVALID_ARG;
  if (!std::isfinite(c.scale * kLog2E) || !std::isfinite(c.z_loss)) return OZ2_ERR_INVALID_ARG;  // (logits are powers of two)
  if (c.ldx < std::max<int64_t>(1, c.k) || c.ldw < std::max<int64_t>(1, c.k)) return OZ2_ERR_INVALID_ARG;
  if (c.t.soft && (c.t.top < 1 || c.t.top > kMaxTop || c.t.ld < c.t.top || c.t.ld_teacher < c.t.top ||
                   !valid_type(c.t.teacher_type) || !(c.t.temperature > 0)))
    return OZ2_ERR_INVALID_ARG;
  if (too_large(c.m, c.n, c.k)) return OZ2_ERR_UNSUPPORTED;
  return OZ2_OK;
}
bool head_pointers(const HeadCall& c, int id_bits) {
  return c.t.ids.p && on(c.t.ids.p, id_bits / 8) && (c.k == 0 || (c.X && c.W)) && on(c.X, 2) && on(c.W, 2) &&
         (!c.t.soft || (c.t.teacher && on(c.t.teacher, type_bytes(c.t.teacher_type))));
}

// Operands on 16-byte boundaries that are not 32-byte ones slow TMA (see oz2_linear): 4096
// tokens × 32000×1000 take 196 µs, so 142 at 1024.  The smaller one is copied where that pays,
// and w where its products (`uses` of them) gain enough by what is then left, a ninth of their time.
struct HeadCopies {
  bool x, w;
};
HeadCopies head_copies(const HeadCall& c, int uses, bool x_copied) {
  const bool slow_x = on16_only(c.X, c.ldx, 2) && !x_copied, slow_w = on16_only(c.W, c.ldw, 2);
  const double product = static_cast<double>(c.m) * c.n * c.k;
  HeadCopies r{false, false};
  if (slow_x && slow_w && copy_pays(2.0 * std::min(c.m, c.n) * c.k, product, 2)) (c.m <= c.n ? r.x : r.w) = true;
  if (slow_w && !r.w && (r.x || x_copied) && copy_pays(2.0 * c.n * c.k, 0.55 * uses * product, 2)) r.w = true;
  return r;
}

int head_forward(const HeadCall& c, float* loss, float* lse, float* picked, cudaStream_t st) {
  Oz2Device* dev = device_status();
  if (!dev) return OZ2_ERR_CUDA;
  Workspace ws(st);
  const HeadCopies copies = head_copies(c, 1, false);
  Operand X(c.X, c.ldx, c.k ? c.m : 0, c.k, 2, ws, copies.x), W(c.W, c.ldw, c.k ? c.n : 0, c.k, 2, ws, copies.w);
  const int64_t ld_stats = (c.m + 31) / 32 * 32, groups = (c.n + kHeadGroup - 1) / kHeadGroup;
  const size_t stats = ws.ask(sizeof(float2) * ld_stats * groups);
  const HeadLists lists = head_lists(c.m, c.n, c.t.top);
  const size_t entries = c.t.soft ? ws.ask(sizeof(int2) * lists.entries) : 0;
  const size_t offsets = c.t.soft ? ws.ask(sizeof(uint16_t) * lists.groups1 * lists.ld_offsets) : 0;
  if (!ws.take()) return OZ2_ERR_ALLOC;
  cudaError_t err = place(X, W, ws, st);
  if (err == cudaSuccess && c.t.soft)
    err = launch_head_targets(c.m, c.n, c.t, ws.at<int2>(entries), ws.at<uint16_t>(offsets), nullptr, HeadTerms{}, st);
  HeadArgs a{};
  a.m = c.m, a.n = c.n, a.k = c.k;
  a.x = X.p, a.ldx = X.ld, a.w = W.p, a.ldw = W.ld;
  a.cols = c.n;
  a.scale = c.scale;
  a.ids = c.t.ids;
  a.entries = ws.at<int2>(entries), a.offsets = ws.at<uint16_t>(offsets), a.ld_offsets = lists.ld_offsets;
  a.top = c.t.top, a.soft = c.t.soft;
  a.stats = ws.at<float2>(stats), a.ld_stats = ld_stats;
  a.picked = picked;
  if (err == cudaSuccess) err = launch_head_forward(a, c.type, dev, st);
  if (err == cudaSuccess) err = launch_head_join(c.m, c.n, c.t, a.stats, ld_stats, c.z_loss, loss, lse, picked, st);
  return status_of(err);
}

struct HeadGrads {
  const float *dloss, *lse;
  void* dX;
  int64_t lddx;
  void* dW;
  int64_t lddw;
  int dw_type;
  unsigned flags;
};

int head_grad(const HeadCall& c, const HeadGrads& g, int id_bits, cudaStream_t st) {
  const int bad = check_head(c, id_bits);
  if (bad == OZ2_ERR_INVALID_ARG) return bad;
  const bool accumulate = (g.flags & OZ2_GRAD_ACCUMULATE) != 0;
  if (g.flags & ~(OZ2_GRAD_ACCUMULATE | OZ2_GRAD_ONE_DLOSS)) return OZ2_ERR_INVALID_ARG;
  if (g.dW && g.dw_type != OZ2_TYPE_F32 && (g.dw_type != c.type || accumulate)) return OZ2_ERR_INVALID_ARG;
  if ((g.dX && g.lddx < std::max<int64_t>(1, c.k)) || (g.dW && g.lddw < std::max<int64_t>(1, c.k))) return OZ2_ERR_INVALID_ARG;
  if (bad) return bad;
  const int dwb = g.dw_type == OZ2_TYPE_F32 ? 4 : 2;
  if (!on(g.dX, 2) || !on(g.dW, dwb) || !on(g.dloss, 4) || !on(g.lse, 4)) return OZ2_ERR_INVALID_ARG;
  if (c.m > 0 && (!head_pointers(c, id_bits) || !g.dloss || !g.lse)) return OZ2_ERR_INVALID_ARG;
  const bool want_dx = g.dX && c.m > 0 && c.k > 0, want_dw = g.dW && c.k > 0 && !(accumulate && c.m == 0);
  if (!want_dx && !want_dw) return OZ2_OK;
  if (c.m == 0) return status_of(cudaMemset2DAsync(g.dW, g.lddw * dwb, 0, c.k * dwb, c.n, st));
  Oz2Device* dev = device_status();
  if (!dev) return OZ2_ERR_CUDA;
  const int64_t piece = piece_columns(c.m, c.n), pieces = (c.n + piece - 1) / piece;
  const bool scaled = c.type == OZ2_TYPE_F16;

  // The products of a piece, full or last: their plans depend on sizes alone.
  struct Products {
    LinProduct p[kMaxProducts] = {};
    LinPlan plan[kMaxProducts];
    int count = 0, launches = 1;
    size_t scratch[kMaxProducts] = {};
  } kinds[2];
  const int64_t ld_dz = (piece + 63) / 64 * 64, ld_sum = (c.k + 31) / 32 * 32;
  Workspace ws(st);
  const HeadLists lists = head_lists(c.m, c.n, c.t.top);
  const size_t rows = c.t.soft ? ws.ask(sizeof(HeadRow) * c.m) : 0, entries = c.t.soft ? ws.ask(sizeof(int2) * lists.entries) : 0;
  const size_t offsets = c.t.soft ? ws.ask(sizeof(uint16_t) * lists.groups1 * lists.ld_offsets) : 0;
  const size_t maxima = scaled ? ws.ask(sizeof(float) * (live_rows_maxima(c.m, c.k) + 1)) : 0;
  // (x's copy is where the largest of the terms is found, and dead tokens' x made zeros for dw.)
  const HeadCopies copies = head_copies(c, want_dx ? 2 : 1, want_dw || scaled);
  Operand X(c.X, c.ldx, c.m, c.k, 2, ws, want_dw || scaled || copies.x), W(c.W, c.ldw, c.n, c.k, 2, ws, copies.w);
  const size_t dz = ws.ask(2 * static_cast<size_t>(c.m) * ld_dz);
  const size_t sums = want_dx && pieces > 1 ? ws.ask(sizeof(float) * static_cast<size_t>(c.m) * ld_sum) : 0;
  for (int kind = 0; kind < 2; ++kind) {
    Products& q = kinds[kind];
    const int64_t cols = kind ? c.n - (pieces - 1) * piece : piece;
    if (want_dx) {
      LinProduct& p = q.p[q.count++];
      p.rows = c.m, p.cols = c.k, p.depth = cols;
      p.q_mn = true;
    }
    if (want_dw) {
      LinProduct& p = q.p[q.count++];
      p.rows = cols, p.cols = c.k, p.depth = c.m;
      p.p_mn = p.q_mn = true;
    }
    q.plan[0] = plan_linear(q.p, q.count, c.type);
    if (q.count == 2) {
      const LinPlan dx = plan_linear(q.p, 1, c.type), dw = plan_linear(q.p + 1, 1, c.type);
      if (plan_apart(q.plan[0], dx, dw)) {
        q.launches = 2;
        q.plan[0] = dx;
        q.plan[1] = dw;
      }
    }
    for (int i = 0; i < q.launches; ++i) q.scratch[i] = ws.ask(q.plan[i].scratch);
  }
  if (!ws.take()) return OZ2_ERR_ALLOC;
  float* largest = scaled ? ws.at<float>(maxima) + 1 : nullptr;
  float* unscale = scaled ? ws.at<float>(maxima) : nullptr;
  HeadTerms terms{nullptr, g.dloss, g.lse, (g.flags & OZ2_GRAD_ONE_DLOSS) == 0, c.scale, c.z_loss};
  cudaError_t err = cudaSuccess;
  if (c.t.soft) {
    err = launch_head_targets(c.m, c.n, c.t, ws.at<int2>(entries), ws.at<uint16_t>(offsets), ws.at<HeadRow>(rows), terms, st);
    terms.rows = ws.at<HeadRow>(rows);
  }
  if (err == cudaSuccess && X.copy) {
    const int64_t ld = padded_ld(c.k, 2);
    err = launch_live_rows(c.m, c.n, c.k, c.X, c.ldx, c.t.ids, terms, largest, ws.at<void>(X.off), ld, st);
    X.p = ws.at<void>(X.off);
    X.ld = ld;
    X.copy = false;
  }
  if (err == cudaSuccess) err = place(X, W, ws, st);
  for (int64_t i = 0; i < pieces && err == cudaSuccess; ++i) {
    Products q = kinds[i + 1 == pieces];
    const int64_t c0 = i * piece, cols = std::min(piece, c.n - c0);
    const uint16_t* w = static_cast<const uint16_t*>(W.p) + c0 * W.ld;
    HeadArgs a{};
    a.m = c.m, a.n = c.n, a.k = c.k;
    a.x = X.p, a.ldx = X.ld, a.w = w, a.ldw = W.ld;
    a.c0 = c0, a.cols = cols;
    a.scale = c.scale;
    a.ids = c.t.ids;
    a.entries = ws.at<int2>(entries), a.offsets = ws.at<uint16_t>(offsets), a.ld_offsets = lists.ld_offsets;
    a.top = c.t.top, a.soft = c.t.soft;
    a.terms = terms;
    a.largest = largest, a.maxima = live_rows_maxima(c.m, c.k), a.unscale = unscale;
    a.dz = ws.at<uint16_t>(dz), a.ld_dz = ld_dz;
    err = launch_head_grad(a, c.type, dev, st);
    int at = 0;
    if (want_dx) {
      LinProduct& p = q.p[at++];
      p.p = a.dz, p.ldp = ld_dz;
      p.q = w, p.ldq = W.ld;
      p.ep.out = pieces > 1 ? ws.at<void>(sums) : g.dX;
      p.ep.ld_out = pieces > 1 ? ld_sum : g.lddx;
      p.ep.out_type = pieces > 1 ? static_cast<int>(OZ2_TYPE_F32) : c.type;
      p.ep.accumulate = i > 0;
      p.ep.factor = pieces > 1 ? nullptr : unscale;
    }
    if (want_dw) {
      LinProduct& p = q.p[at++];
      p.p = a.dz, p.ldp = ld_dz;
      p.q = X.p, p.ldq = X.ld;
      p.ep.out = static_cast<char*>(g.dW) + c0 * g.lddw * dwb;
      p.ep.ld_out = g.lddw;
      p.ep.out_type = g.dw_type;
      p.ep.accumulate = accumulate;
      p.ep.factor = unscale;
    }
    for (int l = 0; l < q.launches && err == cudaSuccess; ++l)
      err = launch_linear(q.p + l, q.launches == 2 ? 1 : q.count, c.type, q.plan[l], ws.at<void>(q.scratch[l]), dev, st);
  }
  if (err == cudaSuccess && want_dx && pieces > 1)
    err = launch_round_rows(c.m, c.k, c.type, ws.at<float>(sums), ld_sum, unscale, g.dX, g.lddx, st);
  return status_of(err);
}

}  // namespace
}  // namespace oz2

using namespace oz2;

extern "C" {

int oz2_embedding(int64_t m, int64_t n, int64_t k, int type, const void* d_ids, int id_bits, const void* d_E, int64_t lde,
                  float scale, void* d_Y, int64_t ldy, void* stream) {
  if (m < 0 || n < 0 || k < 0 || !valid_type(type) || !valid_ids(id_bits)) return OZ2_ERR_INVALID_ARG;
  if (lde < std::max<int64_t>(1, k) || ldy < std::max<int64_t>(1, k)) return OZ2_ERR_INVALID_ARG;
  if (too_large(m, n, k)) return OZ2_ERR_UNSUPPORTED;
  if (m == 0 || k == 0) return OZ2_OK;
  const int es = type_bytes(type);
  if (!d_ids || !d_Y || (n > 0 && !d_E) || !on(d_ids, id_bits / 8) || !on(d_E, es) || !on(d_Y, es)) return OZ2_ERR_INVALID_ARG;
  return status_of(launch_embedding(m, n, k, type, Ids{d_ids, id_bits == 64}, d_E, lde, scale, d_Y, ldy,
                                    static_cast<cudaStream_t>(stream)));
}

int oz2_embedding_grad(int64_t m, int64_t n, int64_t k, int type, const void* d_dY, int64_t lddy, const void* d_ids,
                       int id_bits, float scale, void* d_dE, int64_t ldde, int de_type, unsigned flags, void* stream) {
  if (m < 0 || n < 0 || k < 0 || !valid_type(type) || !valid_ids(id_bits)) return OZ2_ERR_INVALID_ARG;
  if ((de_type != type && de_type != OZ2_TYPE_F32) || (flags & ~OZ2_GRAD_ACCUMULATE)) return OZ2_ERR_INVALID_ARG;
  if (lddy < std::max<int64_t>(1, k) || ldde < std::max<int64_t>(1, k)) return OZ2_ERR_INVALID_ARG;
  if (too_large(m, n, k)) return OZ2_ERR_UNSUPPORTED;
  const bool accumulate = (flags & OZ2_GRAD_ACCUMULATE) != 0;
  if (n == 0 || k == 0 || (m == 0 && accumulate)) return OZ2_OK;
  const int es = type_bytes(de_type);
  if (!d_dE || !on(d_dE, es)) return OZ2_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (m == 0) return status_of(cudaMemset2DAsync(d_dE, ldde * es, 0, k * es, n, st));
  if (!d_ids || !d_dY || !on(d_ids, id_bits / 8) || !on(d_dY, type_bytes(type))) return OZ2_ERR_INVALID_ARG;
  Workspace ws(st);
  const size_t scratch = ws.ask(embedding_grad_scratch(m, k, type));
  if (!ws.take()) return OZ2_ERR_ALLOC;
  return status_of(launch_embedding_grad(m, n, k, type, d_dY, lddy, Ids{d_ids, id_bits == 64}, scale, d_dE, ldde, de_type,
                                         accumulate, ws.at<void>(scratch), st));
}

int oz2_layer_norm(int64_t m, int64_t k, int type, const void* d_X, int64_t ldx, const void* d_w, const void* d_b,
                   int wtype, float eps, int center, void* d_Y, int64_t ldy, float* d_mean, float* d_rstd, void* stream) {
  if (m < 0 || k < 0 || !valid_type(type) || !(eps >= 0)) return OZ2_ERR_INVALID_ARG;
  if ((d_w || d_b) && wtype != type && wtype != OZ2_TYPE_F32) return OZ2_ERR_INVALID_ARG;
  if (ldx < std::max<int64_t>(1, k) || ldy < std::max<int64_t>(1, k)) return OZ2_ERR_INVALID_ARG;
  if (too_large(m, k, 0)) return OZ2_ERR_UNSUPPORTED;
  if (m == 0) return OZ2_OK;
  if (k == 0) {
    if (!on(d_mean, 4) || !on(d_rstd, 4)) return OZ2_ERR_INVALID_ARG;
    cudaError_t err = cudaSuccess;  // (all bits set: NaN; not centred, μ is 0)
    if (d_mean) err = cudaMemsetAsync(d_mean, center ? 0xFF : 0, sizeof(float) * m, static_cast<cudaStream_t>(stream));
    if (d_rstd && err == cudaSuccess) err = cudaMemsetAsync(d_rstd, 0xFF, sizeof(float) * m, static_cast<cudaStream_t>(stream));
    return status_of(err);
  }
  if (d_Y == d_X && ldy != ldx && m > 1) return OZ2_ERR_INVALID_ARG;
  const int es = type_bytes(type), wb = type_bytes(wtype);
  if (!d_X || !d_Y || !on(d_X, es) || !on(d_Y, es) || (d_w && !on(d_w, wb)) || (d_b && !on(d_b, wb)) || !on(d_mean, 4) ||
      !on(d_rstd, 4))
    return OZ2_ERR_INVALID_ARG;
  const NormArgs a{m, k, d_X, ldx, d_w, d_b, wtype, eps, center, d_Y, ldy, d_mean, d_rstd};
  return status_of(launch_layer_norm(a, type, static_cast<cudaStream_t>(stream)));
}

int oz2_layer_norm_grad(int64_t m, int64_t k, int type, const void* d_dY, int64_t lddy, const void* d_X, int64_t ldx,
                        const float* d_mean, const float* d_rstd, const void* d_w, int wtype, const void* d_R, int64_t ldr,
                        void* d_dX, int64_t lddx, float* d_dw, float* d_db, unsigned flags, void* stream) {
  if (m < 0 || k < 0 || !valid_type(type) || (flags & ~OZ2_GRAD_ACCUMULATE)) return OZ2_ERR_INVALID_ARG;
  if (d_w && wtype != type && wtype != OZ2_TYPE_F32) return OZ2_ERR_INVALID_ARG;
  if (lddy < std::max<int64_t>(1, k) || ldx < std::max<int64_t>(1, k) || (d_R && ldr < std::max<int64_t>(1, k)) ||
      (d_dX && lddx < std::max<int64_t>(1, k)))
    return OZ2_ERR_INVALID_ARG;
  if (too_large(m, k, 0)) return OZ2_ERR_UNSUPPORTED;
  const int es = type_bytes(type);
  if (!on(d_dw, 4) || !on(d_db, 4) || !on(d_dX, es)) return OZ2_ERR_INVALID_ARG;
  if (d_R && d_R == d_dX && ldr != lddx && m > 1) return OZ2_ERR_INVALID_ARG;
  if ((!d_dX && !d_dw && !d_db) || k == 0) return OZ2_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool accumulate = (flags & OZ2_GRAD_ACCUMULATE) != 0;
  if (m == 0) {
    cudaError_t err = cudaSuccess;
    if (d_dw && !accumulate) err = cudaMemsetAsync(d_dw, 0, sizeof(float) * k, st);
    if (d_db && !accumulate && err == cudaSuccess) err = cudaMemsetAsync(d_db, 0, sizeof(float) * k, st);
    return status_of(err);
  }
  if (!d_dY || !d_X || !d_rstd || !on(d_dY, es) || !on(d_X, es) || !on(d_R, es) || !on(d_mean, 4) || !on(d_rstd, 4) ||
      (d_w && !on(d_w, type_bytes(wtype))))
    return OZ2_ERR_INVALID_ARG;
  const NormGradArgs a{m,     k,   d_dY, d_X,  lddy, ldx,  d_mean, d_rstd, d_w, wtype,
                       d_R,   ldr, d_dX, lddx, d_dw, d_db, accumulate};
  Workspace ws(st);
  const size_t scratch = ws.ask(layer_norm_grad_scratch(a, type));
  if (!ws.take()) return OZ2_ERR_ALLOC;
  return status_of(launch_layer_norm_grad(a, type, ws.at<void>(scratch), st));
}

int oz2_linear_xent(int64_t m, int64_t n, int64_t k, int type, const void* d_X, int64_t ldx, const void* d_W, int64_t ldw,
                    const void* d_targets, int id_bits, float scale, float z_loss, float* d_loss, float* d_lse,
                    float* d_picked, void* stream) {
  const HeadCall c{m, n, k, type, d_X, ldx, d_W, ldw, HeadTargets{Ids{d_targets, id_bits == 64}, 1, 1, 0, nullptr, 0, 0, 1.f},
                   scale, z_loss};
  const int bad = check_head(c, id_bits);
  if (bad || m == 0) return bad;
  if (!head_pointers(c, id_bits) || !d_loss || !d_lse || !d_picked || !on(d_loss, 4) || !on(d_lse, 4) || !on(d_picked, 4))
    return OZ2_ERR_INVALID_ARG;
  return head_forward(c, d_loss, d_lse, d_picked, static_cast<cudaStream_t>(stream));
}

int oz2_linear_xent_grad(int64_t m, int64_t n, int64_t k, int type, const float* d_dloss, const void* d_X, int64_t ldx,
                         const void* d_W, int64_t ldw, const void* d_targets, int id_bits, const float* d_lse, float scale,
                         float z_loss, void* d_dX, int64_t lddx, void* d_dW, int64_t lddw, int dw_type, unsigned flags,
                         void* stream) {
  const HeadCall c{m, n, k, type, d_X, ldx, d_W, ldw, HeadTargets{Ids{d_targets, id_bits == 64}, 1, 1, 0, nullptr, 0, 0, 1.f},
                   scale, z_loss};
  return head_grad(c, HeadGrads{d_dloss, d_lse, d_dX, lddx, d_dW, lddw, dw_type, flags}, id_bits,
                   static_cast<cudaStream_t>(stream));
}

int oz2_linear_distill(int64_t m, int64_t n, int64_t k, int64_t top, int type, const void* d_X, int64_t ldx,
                       const void* d_W, int64_t ldw, const void* d_ids, int64_t ldi, int id_bits, const void* d_teacher,
                       int64_t ldt, int teacher_type, float temperature, float* d_loss, float* d_lse, float* d_picked,
                       void* stream) {
  const int listed = static_cast<int>(std::max<int64_t>(0, std::min<int64_t>(top, kMaxTop + 1)));
  const HeadCall c{m, n, k, type, d_X, ldx, d_W, ldw,
                   HeadTargets{Ids{d_ids, id_bits == 64}, ldi, listed, 1, d_teacher, ldt, teacher_type, temperature},
                   1.f / temperature, 0.f};
  const int bad = check_head(c, id_bits);
  if (bad || m == 0) return bad;
  if (!head_pointers(c, id_bits) || !d_loss || !d_lse || !d_picked || !on(d_loss, 4) || !on(d_lse, 4) || !on(d_picked, 4))
    return OZ2_ERR_INVALID_ARG;
  return head_forward(c, d_loss, d_lse, d_picked, static_cast<cudaStream_t>(stream));
}

int oz2_linear_distill_grad(int64_t m, int64_t n, int64_t k, int64_t top, int type, const float* d_dloss, const void* d_X,
                            int64_t ldx, const void* d_W, int64_t ldw, const void* d_ids, int64_t ldi, int id_bits,
                            const void* d_teacher, int64_t ldt, int teacher_type, float temperature, const float* d_lse,
                            void* d_dX, int64_t lddx, void* d_dW, int64_t lddw, int dw_type, unsigned flags, void* stream) {
  const int listed = static_cast<int>(std::max<int64_t>(0, std::min<int64_t>(top, kMaxTop + 1)));
  const HeadCall c{m, n, k, type, d_X, ldx, d_W, ldw,
                   HeadTargets{Ids{d_ids, id_bits == 64}, ldi, listed, 1, d_teacher, ldt, teacher_type, temperature},
                   1.f / temperature, 0.f};
  return head_grad(c, HeadGrads{d_dloss, d_lse, d_dX, lddx, d_dW, lddw, dw_type, flags}, id_bits,
                   static_cast<cudaStream_t>(stream));
}

}  // extern "C"
