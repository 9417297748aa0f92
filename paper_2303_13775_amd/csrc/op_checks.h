// What the losses over rows of logits and the update accept: checks of plain values and addresses, without the HIP runtime
// (host programs include this header too).  Each returns what is wrong, or nullptr.
#pragma once

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "gsplit.h"

inline int op_elem_size(int32_t dtype) { return dtype == GSPLIT_F32 ? 4 : dtype == GSPLIT_BF16 ? 2 : 0; }
inline bool op_misaligned(const void *p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }
inline bool op_not_negative(double x) { return std::isfinite(x) && x >= 0.0; }

// rows of logits and of their gradient (may be absent)
inline const char *op_check_rows(int32_t dtype, const void *d_logits, int64_t n_rows, int32_t n_classes, int64_t logits_stride,
                                 const int64_t *d_actions, const void *d_grad, int64_t grad_stride) {
    const int size = op_elem_size(dtype);
    if (!size) return "unknown dtype";
    if (n_rows < 0 || n_rows > (int64_t)1 << 40) return "n_rows out of range";
    if (n_classes < 1 || n_classes > 1 << 30) return "n_classes out of range";
    const int64_t stride_max = (int64_t)1 << 40;
    if (logits_stride < n_classes || logits_stride > stride_max || (d_grad && (grad_stride < n_classes || grad_stride > stride_max)))
        return "stride below n_classes or out of range";
    if (n_rows == 0) return nullptr;
    if (!d_logits || !d_actions) return "NULL buffer";
    if (op_misaligned(d_logits, size) || op_misaligned(d_grad, size) || op_misaligned(d_actions, 8)) return "misaligned buffer";
    if (d_grad == d_logits && grad_stride != logits_stride) return "gradient in place needs the stride of the logits";
    return nullptr;
}

inline const char *op_check_policy(const gsplit_policy_config *c, const void *d_logits, int64_t n_rows, int32_t n_classes,
                                   int64_t logits_stride, const int64_t *d_actions, const float *d_old_logp, const float *d_ref_logp,
                                   const float *d_advantages, const float *d_row_weight, const void *d_grad, int64_t grad_stride,
                                   const float *d_row_loss, const float *d_row_logp, const float *d_row_kl) {
    if (!c) return "NULL config";
    if (const char *e = op_check_rows(c->dtype, d_logits, n_rows, n_classes, logits_stride, d_actions, d_grad, grad_stride)) return e;
    if (!(c->clip_low >= 0.f && c->clip_low <= 1.f)) return "clip_low outside [0, 1]";
    if (!op_not_negative(c->clip_high)) return "clip_high negative or not finite";
    if (!op_not_negative(c->kl_coef)) return "kl_coef negative or not finite";
    if (n_rows == 0) return nullptr;
    if (!d_old_logp || !d_advantages) return "NULL buffer";
    if (c->kl_coef > 0.f && !d_ref_logp) return "kl_coef needs d_ref_logp";
    for (const float *p : {d_old_logp, d_ref_logp, d_advantages, d_row_weight, d_row_loss, d_row_logp, d_row_kl})
        if (op_misaligned(p, 4)) return "misaligned buffer";
    return nullptr;
}

inline const char *op_check_preference(const gsplit_preference_config *c, const void *d_logits, int64_t n_rows, int32_t n_classes,
                                       int64_t logits_stride, const int64_t *d_actions, const int64_t *d_seq_ptr, int64_t n_pairs,
                                       const float *d_ref_logp, const float *d_pair_weight, const void *d_grad, int64_t grad_stride,
                                       const float *d_row_logp, const float *d_pair_loss, const float *d_pair_margin,
                                       const float *d_row_work) {
    if (!c) return "NULL config";
    if (const char *e = op_check_rows(c->dtype, d_logits, n_rows, n_classes, logits_stride, d_actions, d_grad, grad_stride)) return e;
    if (!std::isfinite(c->beta)) return "beta not finite";
    if (!(c->label_smoothing >= 0.f && c->label_smoothing <= 1.f)) return "label_smoothing outside [0, 1]";
    if (n_pairs < 0 || n_pairs > (int64_t)1 << 40) return "n_pairs out of range";
    if (n_pairs == 0) return nullptr;
    if (!d_seq_ptr || (n_rows > 0 && !d_row_work)) return "NULL buffer";
    if (op_misaligned(d_seq_ptr, 8) || op_misaligned(d_row_work, 16)) return "misaligned buffer";
    for (const float *p : {d_ref_logp, d_pair_weight, d_row_logp, d_pair_loss, d_pair_margin})
        if (op_misaligned(p, 4)) return "misaligned buffer";
    return nullptr;
}

inline const char *op_check_run(const void *p, int64_t n, int size) {
    if (!size) return "unknown dtype";
    if (n < 0 || n > (int64_t)1 << 46) return "number of elements out of range";
    if (n > 0 && !p) return "NULL buffer";
    return op_misaligned(p, size) ? "misaligned buffer" : nullptr;
}

inline const char *op_check_grads(const gsplit_grad_tensor *t, int64_t n_tensors, double max_norm, bool clip) {
    if (n_tensors < 0 || (n_tensors > 0 && !t)) return "bad tensor list";
    if (clip && !(max_norm > 0.0)) return "max_norm not above 0";
    for (int64_t i = 0; i < n_tensors; ++i) {
        const int size = op_elem_size(t[i].dtype);
        if (const char *e = op_check_run(t[i].d_grad, t[i].n, size)) return e;
        if (clip && op_misaligned(t[i].d_out, size)) return "misaligned buffer";
    }
    return nullptr;
}

inline const char *op_check_adamw(const gsplit_adamw_config *c, const gsplit_adamw_tensor *t, int64_t n_tensors) {
    if (!c) return "NULL config";
    if (n_tensors < 0 || (n_tensors > 0 && !t)) return "bad tensor list";
    if (!(c->beta1 >= 0.0 && c->beta1 < 1.0 && c->beta2 >= 0.0 && c->beta2 < 1.0)) return "beta outside [0, 1)";
    if (!(c->d_lr || op_not_negative(c->lr)) || !op_not_negative(c->eps) || !op_not_negative(c->weight_decay))
        return "lr, eps or weight_decay negative or not finite";
    if (!(c->max_norm >= 0.0)) return "max_norm below 0";
    if (!c->d_step && c->step < 1) return "step below 1";
    if (op_misaligned(c->d_step, 8) || op_misaligned(c->d_lr, 4)) return "misaligned buffer";
    for (int64_t i = 0; i < n_tensors; ++i) {
        const gsplit_adamw_tensor &x = t[i];
        if (const char *e = op_check_run(x.d_param, x.n, op_elem_size(x.param_dtype))) return e;
        if (const char *e = op_check_run(x.d_grad, x.n, op_elem_size(x.grad_dtype))) return e;
        if (const char *e = op_check_run(x.d_m, x.n, 4)) return e;
        if (const char *e = op_check_run(x.d_v, x.n, 4)) return e;
        if (x.param_dtype == GSPLIT_F32 && x.d_master) return "a float parameter has no d_master";
        if (x.param_dtype == GSPLIT_BF16)
            if (const char *e = op_check_run(x.d_master, x.n, 4)) return e;
    }
    return nullptr;
}
