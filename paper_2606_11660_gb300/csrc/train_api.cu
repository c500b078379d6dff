// Host side of the training-side operators' entry points: argument validation
// and error mapping.

#include <cmath>

#include "bergson.h"
#include "internal.h"
#include "train.h"

namespace bergson {
namespace {

template <typename... Args>
int fail(int code, const char* fmt, Args... args) {
  return record_error(code, fmt, args...);
}

int fail_cuda(cudaError_t e, const char* what) {
  return fail(BERGSON_ECUDA, "%s: %s (%s)", what, cudaGetErrorName(e), cudaGetErrorString(e));
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Bytes of an element, or 0.
size_t dtype_size(int dtype) {
  return dtype == BERGSON_F32 ? 4 : dtype == BERGSON_BF16 || dtype == BERGSON_F16 ? 2 : 0;
}

// A tensor of `what`: present and aligned to its elements.
int check_tensor(const void* p, size_t align, const char* what) {
  if (p == nullptr) return fail(BERGSON_EINVAL, "%s is NULL", what);
  if (!aligned(p, align))
    return fail(BERGSON_EALIGN, "%s must be %zu-byte aligned", what, align);
  return BERGSON_OK;
}

// A [rows, ld] tensor whose rows hold `cols` elements.
int check_rows(const void* p, size_t align, int64_t cols, int64_t ld, const char* what) {
  if (ld < cols)
    return fail(BERGSON_EINVAL, "the leading dimension of %s must be >= %lld (got %lld)", what,
                (long long)cols, (long long)ld);
  if (ld > (1ll << 40))
    return fail(BERGSON_EUNSUPPORTED, "the leading dimension of %s is too large", what);
  return check_tensor(p, align, what);
}

int check_workspace(const void* ws, size_t bytes, size_t need) {
  if (ws == nullptr) return fail(BERGSON_EINVAL, "workspace is NULL");
  if (!aligned(ws, 256)) return fail(BERGSON_EALIGN, "workspace must be 256-byte aligned");
  if (bytes < need)
    return fail(BERGSON_EWORKSPACE, "workspace too small: %zu < %zu bytes", bytes, need);
  return BERGSON_OK;
}

int check_logits(const void* logits, int dtype, int64_t rows, int64_t V, int64_t ld,
                 const int64_t* targets, double tau) {
  const size_t size = dtype_size(dtype);
  if (size == 0) return fail(BERGSON_EINVAL, "unknown dtype %d", dtype);
  if (rows < 0 || rows > INT32_MAX) return fail(BERGSON_EINVAL, "rows must be in [0, 2^31)");
  if (V < 1 || V > INT32_MAX) return fail(BERGSON_EINVAL, "V must be in [1, 2^31)");
  // the kernels scale by 1 / tau and log2(e) / tau in fp32
  if (!(tau > 0.0) || !std::isfinite(static_cast<float>(1.5 / tau)) ||
      !(static_cast<float>(1.0 / tau) >= 1.17549435e-38f))
    return fail(BERGSON_EINVAL, "tau must be > 0 and 1 / tau in the range of fp32");
  if (rows == 0) return BERGSON_OK;
  int st = check_rows(logits, size, V, ld, "logits");
  if (st == BERGSON_OK) st = check_tensor(targets, 8, "targets");
  return st;
}

#define BERGSON_TRY(call)               \
  do {                                  \
    const int st_ = (call);             \
    if (st_ != BERGSON_OK) return st_;  \
  } while (0)

constexpr int64_t kMaxLossTokens = 1ll << 40;
constexpr int64_t kMaxRowTokens = 1ll << 30;   // the kernels' places within a row are 32-bit

int check_policy_sizes(int64_t B, int64_t T) {
  if (B < 0 || B > INT32_MAX || T < 0 || T > INT32_MAX)
    return fail(BERGSON_EINVAL, "B and T must be in [0, 2^31)");
  if (T > kMaxRowTokens || B * T > kMaxLossTokens)
    return fail(BERGSON_EUNSUPPORTED, "T or B*T too large");
  return BERGSON_OK;
}

bool probability(double x) { return x >= 0.0 && x <= 1.0; }

}  // namespace
}  // namespace bergson

using namespace bergson;

extern "C" {

int bergson_token_logprobs(const void* logits, int dtype, int64_t rows, int64_t V, int64_t ld,
                           const int64_t* targets, double tau, float* logp, float* lse,
                           float* entropy, void* stream) {
  BERGSON_TRY(check_logits(logits, dtype, rows, V, ld, targets, tau));
  if (rows > 0) {
    BERGSON_TRY(check_tensor(logp, 4, "logp"));
    BERGSON_TRY(check_tensor(lse, 4, "lse"));
    if (entropy != nullptr) BERGSON_TRY(check_tensor(entropy, 4, "entropy"));
  }
  BERGSON_TRY(injected_status());
  if (rows == 0) return BERGSON_OK;
  DeviceGuard dg(logp);
  if (dg.err != cudaSuccess) return fail_cuda(dg.err, "output device lookup");
  int* status = device_status_word(dg.dev);
  if (status == nullptr) return fail(BERGSON_ECUDA, "device status word unavailable");
  const LogprobArgs a{logits, dtype, rows, V, ld, targets, tau, logp, lse, entropy, status};
  const cudaError_t e = launch_token_logprobs(a, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return fail_cuda(e, "token log-probability launch");
  return BERGSON_OK;
}

int bergson_token_logprobs_backward(const void* logits, int dtype, int64_t rows, int64_t V,
                                    int64_t ld, const int64_t* targets, double tau,
                                    const float* lse, const float* entropy, const float* d_logp,
                                    const float* d_entropy, void* d_logits, int64_t ld_d,
                                    void* stream) {
  BERGSON_TRY(check_logits(logits, dtype, rows, V, ld, targets, tau));
  if (rows > 0) {
    if (d_logp == nullptr && d_entropy == nullptr)
      return fail(BERGSON_EINVAL, "d_logp and d_entropy are both NULL");
    BERGSON_TRY(check_rows(d_logits, dtype_size(dtype), V, ld_d, "d_logits"));
    if (d_logits == logits && ld_d != ld)
      return fail(BERGSON_EINVAL, "d_logits in place of logits needs ld_d == ld");
    BERGSON_TRY(check_tensor(lse, 4, "lse"));
    if (d_logp != nullptr) BERGSON_TRY(check_tensor(d_logp, 4, "d_logp"));
    if (d_entropy != nullptr) {
      BERGSON_TRY(check_tensor(d_entropy, 4, "d_entropy"));
      BERGSON_TRY(check_tensor(entropy, 4, "entropy"));
    }
  }
  BERGSON_TRY(injected_status());
  if (rows == 0) return BERGSON_OK;
  DeviceGuard dg(d_logits);
  if (dg.err != cudaSuccess) return fail_cuda(dg.err, "output device lookup");
  int* status = device_status_word(dg.dev);
  if (status == nullptr) return fail(BERGSON_ECUDA, "device status word unavailable");
  const LogprobGradArgs a{logits, dtype, rows,   V,         ld,       targets, tau,
                          lse,    entropy, d_logp, d_entropy, d_logits, ld_d,  status};
  const cudaError_t e = launch_token_logprobs_backward(a, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return fail_cuda(e, "token log-probability backward launch");
  return BERGSON_OK;
}

int bergson_policy_loss_workspace(int64_t B, int64_t T, size_t* ws_bytes) {
  if (ws_bytes == nullptr) return fail(BERGSON_EINVAL, "ws_bytes is NULL");
  BERGSON_TRY(check_policy_sizes(B, T));
  *ws_bytes = policy_workspace(B, T);
  return BERGSON_OK;
}

int bergson_policy_loss(const bergson_policy_args* args, void* workspace, size_t ws_bytes,
                        void* stream) {
  if (args == nullptr) return fail(BERGSON_EINVAL, "args is NULL");
  const bergson_policy_args& a = *args;
  BERGSON_TRY(check_policy_sizes(a.B, a.T));
  if (a.reserved != 0) return fail(BERGSON_EINVAL, "reserved must be 0");
  if (a.reduction != BERGSON_POLICY_TOKEN_MEAN && a.reduction != BERGSON_POLICY_SEQ_MEAN &&
      a.reduction != BERGSON_POLICY_SUM_NORM)
    return fail(BERGSON_EINVAL, "unknown reduction %d", a.reduction);
  if (!probability(a.clip_low)) return fail(BERGSON_EINVAL, "clip_low must be in [0, 1]");
  if (!(a.clip_high >= 0.0) || !std::isfinite(a.clip_high))
    return fail(BERGSON_EINVAL, "clip_high must be >= 0 and finite");
  if (!std::isfinite(a.kl_coef) || !std::isfinite(a.entropy_coef))
    return fail(BERGSON_EINVAL, "kl_coef and entropy_coef must be finite");
  if (a.reduction == BERGSON_POLICY_SUM_NORM &&
      (!(a.norm_tokens > 0.0) || !std::isfinite(a.norm_tokens)))
    return fail(BERGSON_EINVAL, "norm_tokens must be > 0 and finite");
  if (a.ld_adv != 0 && a.ld_adv < a.T)
    return fail(BERGSON_EINVAL, "ld_adv must be 0 (one advantage a sequence) or >= T");
  if (a.B > 0 && a.T > 0) {
    if (a.kl_coef != 0.0 && a.ref_logp == nullptr)
      return fail(BERGSON_EINVAL, "kl_coef != 0 needs ref_logp");
    if (a.entropy_coef != 0.0 && a.entropy == nullptr)
      return fail(BERGSON_EINVAL, "entropy_coef != 0 needs entropy");
    BERGSON_TRY(check_rows(a.logp, 4, a.T, a.ld_logp, "logp"));
    BERGSON_TRY(check_rows(a.old_logp, 4, a.T, a.ld_old, "old_logp"));
    if (a.ref_logp != nullptr) BERGSON_TRY(check_rows(a.ref_logp, 4, a.T, a.ld_ref, "ref_logp"));
    if (a.entropy != nullptr) BERGSON_TRY(check_rows(a.entropy, 4, a.T, a.ld_entropy, "entropy"));
    BERGSON_TRY(check_tensor(a.advantages, 4, "advantages"));
    if (a.mask != nullptr) BERGSON_TRY(check_rows(a.mask, 1, a.T, a.ld_mask, "mask"));
    BERGSON_TRY(check_rows(a.d_logp, 4, a.T, a.ld_d, "d_logp"));
    if (a.d_entropy != nullptr) BERGSON_TRY(check_rows(a.d_entropy, 4, a.T, a.ld_de, "d_entropy"));
  }
  BERGSON_TRY(check_tensor(a.loss, 4, "loss"));
  if (a.seq_loss != nullptr) BERGSON_TRY(check_tensor(a.seq_loss, 4, "seq_loss"));
  if (a.stats != nullptr) BERGSON_TRY(check_tensor(a.stats, 4, "stats"));
  BERGSON_TRY(check_workspace(workspace, ws_bytes, policy_workspace(a.B, a.T)));
  BERGSON_TRY(injected_status());
  DeviceGuard dg(a.loss);
  if (dg.err != cudaSuccess) return fail_cuda(dg.err, "output device lookup");
  const cudaError_t e = launch_policy_loss(a, workspace, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return fail_cuda(e, "policy loss launch");
  return BERGSON_OK;
}

int bergson_preference_loss(const bergson_preference_args* args, void* stream) {
  if (args == nullptr) return fail(BERGSON_EINVAL, "args is NULL");
  const bergson_preference_args& a = *args;
  if (a.P < 0 || a.P >= (1ll << 30) || a.T < 0 || a.T > INT32_MAX)
    return fail(BERGSON_EINVAL, "P must be in [0, 2^30) and T in [0, 2^31)");
  if (a.T > kMaxRowTokens || 2 * a.P * a.T > kMaxLossTokens)
    return fail(BERGSON_EUNSUPPORTED, "T or 2*P*T too large");
  if (a.kind != BERGSON_PREFERENCE_SIGMOID && a.kind != BERGSON_PREFERENCE_HINGE &&
      a.kind != BERGSON_PREFERENCE_SQUARED)
    return fail(BERGSON_EINVAL, "unknown kind %d", a.kind);
  if (!(a.beta > 0.0) || !std::isfinite(a.beta))
    return fail(BERGSON_EINVAL, "beta must be > 0 and finite");
  if (!std::isfinite(a.margin)) return fail(BERGSON_EINVAL, "margin must be finite");
  if (!probability(a.label_smoothing))
    return fail(BERGSON_EINVAL, "label_smoothing must be in [0, 1]");
  if (a.P > 0) {
    if (a.T > 0) {
      BERGSON_TRY(check_rows(a.logp, 4, a.T, a.ld_logp, "logp"));
      if (a.ref_logp != nullptr) BERGSON_TRY(check_rows(a.ref_logp, 4, a.T, a.ld_ref, "ref_logp"));
      if (a.mask != nullptr) BERGSON_TRY(check_rows(a.mask, 1, a.T, a.ld_mask, "mask"));
      BERGSON_TRY(check_rows(a.d_logp, 4, a.T, a.ld_d, "d_logp"));
    }
    BERGSON_TRY(check_tensor(a.pair_loss, 4, "pair_loss"));
    if (a.rewards != nullptr) BERGSON_TRY(check_tensor(a.rewards, 4, "rewards"));
  }
  BERGSON_TRY(check_tensor(a.loss, 4, "loss"));
  BERGSON_TRY(injected_status());
  DeviceGuard dg(a.loss);
  if (dg.err != cudaSuccess) return fail_cuda(dg.err, "output device lookup");
  const cudaError_t e = launch_preference_loss(a, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return fail_cuda(e, "preference loss launch");
  return BERGSON_OK;
}

int bergson_adamw_step(const bergson_adamw_tensor* tensors, int n_tensors, double lr, double beta1,
                       double beta2, double eps, int64_t step, uint64_t seed,
                       const float* grad_scale, void* stream) {
  if (n_tensors < 0) return fail(BERGSON_EINVAL, "n_tensors must be >= 0");
  if (n_tensors > 0 && tensors == nullptr) return fail(BERGSON_EINVAL, "tensors is NULL");
  if (!std::isfinite(lr)) return fail(BERGSON_EINVAL, "lr must be finite");
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
    return fail(BERGSON_EINVAL, "beta1 and beta2 must be in [0, 1)");
  if (!(eps >= 0.0) || !std::isfinite(eps))
    return fail(BERGSON_EINVAL, "eps must be >= 0 and finite");
  if (step < 1) return fail(BERGSON_EINVAL, "step must be >= 1");
  if (grad_scale != nullptr) BERGSON_TRY(check_tensor(grad_scale, 4, "grad_scale"));
  const void* any = nullptr;
  for (int i = 0; i < n_tensors; ++i) {
    const bergson_adamw_tensor& t = tensors[i];
    const size_t ps = dtype_size(t.param_dtype), gs = dtype_size(t.grad_dtype);
    if (ps == 0 || gs == 0)
      return fail(BERGSON_EINVAL, "tensor %d: unknown dtype (param %d, grad %d)", i, t.param_dtype,
                  t.grad_dtype);
    if (t.state_kind != BERGSON_STATE_F32 && t.state_kind != BERGSON_STATE_8BIT)
      return fail(BERGSON_EINVAL, "tensor %d: unknown state_kind %d", i, t.state_kind);
    if (t.reserved != 0) return fail(BERGSON_EINVAL, "tensor %d: reserved must be 0", i);
    if (t.n < 0) return fail(BERGSON_EINVAL, "tensor %d: n must be >= 0", i);
    if (t.n > (1ll << 38)) return fail(BERGSON_EUNSUPPORTED, "tensor %d: n too large", i);
    if (!std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay))
      return fail(BERGSON_EINVAL, "tensor %d: lr_scale and weight_decay must be finite", i);
    if (t.n == 0) continue;
    const bool eight = t.state_kind == BERGSON_STATE_8BIT;
    if (t.param == nullptr || t.grad == nullptr || t.m == nullptr || t.v == nullptr ||
        (eight && (t.m_scale == nullptr || t.v_scale == nullptr)))
      return fail(BERGSON_EINVAL, "tensor %d: a pointer is NULL", i);
    if (!aligned(t.param, ps) || !aligned(t.grad, gs) || !aligned(t.master, 4) ||
        (!eight && (!aligned(t.m, 4) || !aligned(t.v, 4))) ||
        (eight && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))))
      return fail(BERGSON_EALIGN, "tensor %d: a pointer is not aligned to its elements", i);
    if (any == nullptr) any = t.param;
  }
  BERGSON_TRY(injected_status());
  if (any == nullptr) return BERGSON_OK;
  DeviceGuard dg(any);
  if (dg.err != cudaSuccess) return fail_cuda(dg.err, "parameter device lookup");
  const AdamwScalars a{lr, beta1, beta2, eps, step, seed, grad_scale};
  const cudaError_t e = launch_adamw(tensors, n_tensors, a, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return fail_cuda(e, "AdamW launch");
  return BERGSON_OK;
}

int bergson_adamw_state_values(const uint8_t* codes, const float* scale, int64_t n, int moment,
                               float* out, void* stream) {
  if (n < 0) return fail(BERGSON_EINVAL, "n must be >= 0");
  if (n > (1ll << 38)) return fail(BERGSON_EUNSUPPORTED, "n too large");
  if (moment != BERGSON_MOMENT_FIRST && moment != BERGSON_MOMENT_SECOND)
    return fail(BERGSON_EINVAL, "unknown moment %d", moment);
  if (n > 0) {
    BERGSON_TRY(check_tensor(codes, 1, "codes"));
    BERGSON_TRY(check_tensor(scale, 4, "scale"));
    BERGSON_TRY(check_tensor(out, 4, "out"));
  }
  BERGSON_TRY(injected_status());
  if (n == 0) return BERGSON_OK;
  DeviceGuard dg(out);
  if (dg.err != cudaSuccess) return fail_cuda(dg.err, "output device lookup");
  const cudaError_t e =
      launch_state_values(codes, scale, n, moment, out, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return fail_cuda(e, "state value launch");
  return BERGSON_OK;
}

static int check_moment_matrices(const bergson_moment_matrix* mats, int n_mats, bool pointers) {
  if (n_mats < 0) return fail(BERGSON_EINVAL, "n_mats must be >= 0");
  if (n_mats > 0 && mats == nullptr) return fail(BERGSON_EINVAL, "mats is NULL");
  for (int i = 0; i < n_mats; ++i) {
    const bergson_moment_matrix& m = mats[i];
    if (m.d_out < 1 || m.d_in < 1 || m.d_out > (1 << 24) || m.d_in > (1 << 24))
      return fail(BERGSON_EINVAL, "matrix %d: d_out and d_in must be in [1, 2^24]", i);
    if (m.d_out * m.d_in > (1ll << 38))
      return fail(BERGSON_EUNSUPPORTED, "matrix %d: d_out*d_in too large", i);
    if (m.state_kind != BERGSON_STATE_F32 && m.state_kind != BERGSON_STATE_8BIT)
      return fail(BERGSON_EINVAL, "matrix %d: unknown state_kind %d", i, m.state_kind);
    if (m.reserved != 0) return fail(BERGSON_EINVAL, "matrix %d: reserved must be 0", i);
    if (!pointers) continue;
    const bool eight = m.state_kind == BERGSON_STATE_8BIT;
    if (m.v == nullptr || m.r == nullptr || m.c == nullptr || (eight && m.v_scale == nullptr))
      return fail(BERGSON_EINVAL, "matrix %d: a pointer is NULL", i);
    if ((!eight && !aligned(m.v, 4)) || (eight && !aligned(m.v_scale, 4)) || !aligned(m.r, 4) ||
        !aligned(m.c, 4))
      return fail(BERGSON_EALIGN, "matrix %d: a pointer is not aligned to its elements", i);
  }
  return BERGSON_OK;
}

int bergson_factor_moments_workspace(const bergson_moment_matrix* mats, int n_mats,
                                     size_t* ws_bytes) {
  if (ws_bytes == nullptr) return fail(BERGSON_EINVAL, "ws_bytes is NULL");
  BERGSON_TRY(check_moment_matrices(mats, n_mats, false));
  *ws_bytes = moments_workspace(mats, n_mats);
  return BERGSON_OK;
}

int bergson_factor_moments(const bergson_moment_matrix* mats, int n_mats, double correction,
                           double floor, void* workspace, size_t ws_bytes, void* stream) {
  BERGSON_TRY(check_moment_matrices(mats, n_mats, true));
  if (!(correction > 0.0) || !std::isfinite(correction))
    return fail(BERGSON_EINVAL, "correction must be > 0 and finite");
  if (!(floor > 0.0) || !std::isfinite(floor) || !(static_cast<float>(floor) > 0.0f))
    return fail(BERGSON_EINVAL, "floor must be > 0 (in fp32) and finite");
  BERGSON_TRY(check_workspace(workspace, ws_bytes, moments_workspace(mats, n_mats)));
  BERGSON_TRY(injected_status());
  if (n_mats == 0) return BERGSON_OK;
  DeviceGuard dg(workspace);
  if (dg.err != cudaSuccess) return fail_cuda(dg.err, "workspace device lookup");
  const cudaError_t e = launch_factor_moments(mats, n_mats, correction, floor, workspace,
                                              static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return fail_cuda(e, "factored moment launch");
  return BERGSON_OK;
}

}  // extern "C"
