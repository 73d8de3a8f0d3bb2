// Entry points of the layer operators (declared in include/oz2_layers.h):
// argument checks, workspace, and the order of their launches.
#include <algorithm>

#include "lin_host.cuh"

namespace oz2 {
namespace {

bool valid_act(int act) { return act >= OZ2_ACT_NONE && act <= OZ2_ACT_SILU; }

}  // namespace
}  // namespace oz2

using namespace oz2;

extern "C" {

int oz2_linear(int64_t m, int64_t n, int64_t k, int type, const void* d_X, int64_t ldx, const void* d_W, int64_t ldw,
               const float* d_x_scale, const float* d_w_scale, const void* d_bias, int bias_type, int act,
               const void* d_R, int64_t ldr, void* d_Z, int64_t ldz, void* d_Y, int64_t ldy, int out_type,
               void* stream) {
  if (m < 0 || n < 0 || k < 0 || !valid_act(act)) return OZ2_ERR_INVALID_ARG;
  if (type != OZ2_TYPE_E4M3 && !is_16bit(type)) return OZ2_ERR_INVALID_ARG;
  if (!is_16bit(out_type) || (is_16bit(type) && out_type != type)) return OZ2_ERR_INVALID_ARG;
  if ((d_x_scale || d_w_scale) && type != OZ2_TYPE_E4M3) return OZ2_ERR_INVALID_ARG;
  if (d_bias && bias_type != OZ2_TYPE_F32 && bias_type != out_type) return OZ2_ERR_INVALID_ARG;
  if (ldx < std::max<int64_t>(1, k) || ldw < std::max<int64_t>(1, k) || ldy < std::max<int64_t>(1, n) ||
      (d_R && ldr < n) || (d_Z && ldz < n))
    return OZ2_ERR_INVALID_ARG;
  if (m >= kMaxSize || n >= kMaxSize || k >= kMaxSize) return OZ2_ERR_UNSUPPORTED;
  if (m == 0 || n == 0) return OZ2_OK;  // (before the pointers: an empty array's, scales' among them, may be null)
  if (!d_x_scale != !d_w_scale) return OZ2_ERR_INVALID_ARG;
  if (!d_Y || (k > 0 && (!d_X || !d_W))) return OZ2_ERR_INVALID_ARG;
  const int es = type_bytes(type);
  if (!on(d_X, es) || !on(d_W, es) || !on(d_Y, 2) || !on(d_R, 2) || !on(d_Z, 2) ||
      (d_bias && !on(d_bias, type_bytes(bias_type))) || !on(d_x_scale, 4) || !on(d_w_scale, 4))
    return OZ2_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Oz2Device* dev = device_status();
  if (!dev) return OZ2_ERR_CUDA;
  LinProduct p{};
  p.rows = m;
  p.cols = n;
  p.depth = k;
  p.ep = LinEpilogue{d_x_scale, d_w_scale, d_bias, d_R, d_Z, d_Y, ldr, ldz, ldy, bias_type, out_type, act, 0};
  // Few tokens and weights that TMA cannot read: they are read where they lie (8 tokens ×
  // 10240×7569 bf16 47 µs, 78 with a copy).  Short rows of many weights are left to the
  // copy (16 tokens × 16384×101: 7 µs, so 14).
  if (m <= kFewRows && k > 0 && !on16(d_W, ldw, es) && (k * es >= 512 || n <= 4096)) {
    p.p = d_X;
    p.ldp = ldx;
    p.q = d_W;
    p.ldq = ldw;
    return status_of(launch_linear_rows(p, type, st));
  }
  const LinPlan plan = plan_linear(&p, 1, type);
  Workspace ws(st);
  const double product = static_cast<double>(m) * n * k;
  const bool one = on16_only(d_X, ldx, es) && on16_only(d_W, ldw, es) &&
                   copy_pays(static_cast<double>(std::min(m, n)) * k * es, product, es);
  Operand X(d_X, ldx, k ? m : 0, k, es, ws, one && m <= n), W(d_W, ldw, k ? n : 0, k, es, ws, one && m > n);
  const size_t scratch = ws.ask(plan.scratch);
  if (!ws.take()) return OZ2_ERR_ALLOC;
  const cudaError_t err = place(X, W, ws, st);
  if (err != cudaSuccess) return status_of(err);
  p.p = X.p;
  p.ldp = X.ld;
  p.q = W.p;
  p.ldq = W.ld;
  return status_of(launch_linear(&p, 1, type, plan, ws.at<void>(scratch), dev, st));
}

int oz2_linear_grad(int64_t m, int64_t n, int64_t k, int type, const void* d_dY, int64_t lddy, const void* d_Z,
                    int64_t ldz, int act, const void* d_X, int64_t ldx, const void* d_W, int64_t ldw, void* d_dX,
                    int64_t lddx, void* d_dW, int64_t lddw, int dw_type, float* d_db, unsigned flags, void* stream) {
  if (m < 0 || n < 0 || k < 0 || !valid_act(act) || !is_16bit(type)) return OZ2_ERR_INVALID_ARG;
  const bool accumulate = (flags & OZ2_GRAD_ACCUMULATE) != 0;
  if (flags & ~OZ2_GRAD_ACCUMULATE) return OZ2_ERR_INVALID_ARG;
  if (d_dW && dw_type != OZ2_TYPE_F32 && (dw_type != type || accumulate)) return OZ2_ERR_INVALID_ARG;
  if (lddy < std::max<int64_t>(1, n) || (act != OZ2_ACT_NONE && ldz < std::max<int64_t>(1, n)) ||
      (d_dX && (lddx < std::max<int64_t>(1, k) || ldw < std::max<int64_t>(1, k))) ||
      (d_dW && (lddw < std::max<int64_t>(1, k) || ldx < std::max<int64_t>(1, k))))
    return OZ2_ERR_INVALID_ARG;
  if (m >= kMaxSize || n >= kMaxSize || k >= kMaxSize) return OZ2_ERR_UNSUPPORTED;
  const bool any = m > 0 && n > 0;  // there is a dZ
  if (any && (!d_dY || (act != OZ2_ACT_NONE && !d_Z) || (k > 0 && ((d_dX && !d_W) || (d_dW && !d_X)))))
    return OZ2_ERR_INVALID_ARG;
  if (!on(d_dY, 2) || !on(d_Z, 2) || !on(d_X, 2) || !on(d_W, 2) || !on(d_dX, 2) ||
      !on(d_dW, dw_type == OZ2_TYPE_F32 ? 4 : 2) || !on(d_db, 4))
    return OZ2_ERR_INVALID_ARG;
  const bool want_dx = d_dX && m > 0 && k > 0, want_dw = d_dW && n > 0 && k > 0 && !(accumulate && m == 0);
  const bool want_db = d_db && n > 0 && !(accumulate && m == 0);
  if (!want_dx && !want_dw && !want_db) return OZ2_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Oz2Device* dev = device_status();
  if (!dev) return OZ2_ERR_CUDA;
  LinProduct p[kMaxProducts] = {};
  int count = 0;
  LinProduct* pdx = nullptr;
  LinProduct* pdw = nullptr;
  if (want_dx) {
    LinProduct& a = *(pdx = &p[count++]);
    a.rows = m;
    a.cols = k;
    a.depth = n;
    a.q_mn = true;
    a.ep.out = d_dX;
    a.ep.ld_out = lddx;
    a.ep.out_type = type;
  }
  if (want_dw) {
    LinProduct& a = *(pdw = &p[count++]);
    a.rows = n;
    a.cols = k;
    a.depth = m;
    a.p_mn = a.q_mn = true;
    a.ep.out = d_dW;
    a.ep.ld_out = lddw;
    a.ep.out_type = dw_type;
    a.ep.accumulate = accumulate;
  }
  // Both products in one launch, or each in its own.
  LinPlan plan[kMaxProducts];
  int launches = count ? 1 : 0;
  if (count) plan[0] = plan_linear(p, count, type);
  if (count == 2) {
    const LinPlan dx = plan_linear(p, 1, type), dw = plan_linear(p + 1, 1, type);
    if (plan_apart(plan[0], dx, dw)) {
      launches = 2;
      plan[0] = dx;
      plan[1] = dw;
    }
  }
  Workspace ws(st);
  // dZ is dY itself where there is no activation and TMA can read it (well).
  const bool slow = on16_only(d_dY, lddy, 2) && ((pdx && on16_only(d_W, ldw, 2)) || (pdw && on16_only(d_X, ldx, 2))) &&
                    copy_pays(2.0 * m * n, static_cast<double>(count) * m * n * k, 2);
  const bool own_dz = count && any && (act != OZ2_ACT_NONE || !on16(d_dY, lddy, 2) || slow);
  const int64_t ld_dz = padded_ld(n, 2);
  const size_t dz_off = own_dz ? ws.ask(static_cast<size_t>(m) * ld_dz * 2) : 0;
  const size_t part_off = want_db && m > 0 ? ws.ask(sizeof(float) * static_cast<size_t>(lin_db_chunks(m, n)) * n) : 0;
  Operand X(d_X, ldx, want_dw ? m : 0, k, 2, ws), W(d_W, ldw, want_dx ? n : 0, k, 2, ws);
  size_t scratch[kMaxProducts] = {};
  for (int i = 0; i < launches; ++i) scratch[i] = ws.ask(plan[i].scratch);
  if (!ws.take()) return OZ2_ERR_ALLOC;
  cudaError_t err = cudaSuccess;
  if (want_db && m == 0) err = cudaMemsetAsync(d_db, 0, sizeof(float) * n, st);
  const void* dz = d_dY;
  int64_t ldz_used = lddy;
  if (err == cudaSuccess && any && (own_dz || want_db)) {
    err = launch_act_grad(m, n, type, act, d_dY, lddy, d_Z, ldz, own_dz ? ws.at<void>(dz_off) : nullptr, ld_dz,
                          want_db ? d_db : nullptr, ws.at<float>(part_off), accumulate, st);
    if (own_dz) {
      dz = ws.at<void>(dz_off);
      ldz_used = ld_dz;
    }
  }
  if (err == cudaSuccess) err = place(X, W, ws, st);
  if (err != cudaSuccess || !count) return status_of(err);
  if (pdx) {
    pdx->p = dz;
    pdx->ldp = ldz_used;
    pdx->q = W.p;
    pdx->ldq = W.ld;
  }
  if (pdw) {
    pdw->p = dz;
    pdw->ldp = ldz_used;
    pdw->q = X.p;
    pdw->ldq = X.ld;
  }
  for (int i = 0; i < launches && err == cudaSuccess; ++i)
    err = launch_linear(p + i, launches == 2 ? 1 : count, type, plan[i], ws.at<void>(scratch[i]), dev, st);
  return status_of(err);
}

int oz2_adamw(const oz2_adamw_tensor* tensors, int count, int param_type, int grad_type, int state_bits,
              const oz2_adamw_step* args, void* stream) {
  if (count < 0 || (count > 0 && !tensors) || !args) return OZ2_ERR_INVALID_ARG;
  if (param_type != OZ2_TYPE_F32 && !is_16bit(param_type)) return OZ2_ERR_INVALID_ARG;
  if (grad_type != OZ2_TYPE_F32 && grad_type != param_type) return OZ2_ERR_INVALID_ARG;
  if (state_bits != 32 && state_bits != 8) return OZ2_ERR_INVALID_ARG;
  if (args->step < 1 || !(args->beta1 >= 0 && args->beta1 < 1) || !(args->beta2 >= 0 && args->beta2 < 1) ||
      !on(args->d_grad_scale, 4))
    return OZ2_ERR_INVALID_ARG;
  const int sb = state_bits == 32 ? 4 : 1;
  for (int i = 0; i < count; ++i) {
    const oz2_adamw_tensor& t = tensors[i];
    if (t.numel < 0) return OZ2_ERR_INVALID_ARG;
    if (t.numel == 0) continue;
    if ((!t.param && !t.master) || (t.master && param_type == OZ2_TYPE_F32) || !t.grad || !t.m || !t.v || (state_bits == 8 && (!t.m_scale || !t.v_scale)))
      return OZ2_ERR_INVALID_ARG;
    if (!on(t.param, type_bytes(param_type)) || !on(t.grad, type_bytes(grad_type)) || !on(t.master, 4) ||
        !on(t.m, sb) || !on(t.v, sb) || !on(t.m_scale, 4) || !on(t.v_scale, 4))
      return OZ2_ERR_INVALID_ARG;
  }
  return status_of(launch_adamw(tensors, count, param_type, grad_type, state_bits, *args,
                                static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
