// What the losses over rows of logits and the update accept: checks of plain values and addresses, without the HIP runtime
// (host programs include this header too).  Each returns what is wrong, or nullptr.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <numeric>

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

// Memory of a call: `rows` runs of `width` bytes, `stride` bytes from one to the next (at least `width`)
struct OpArea {
    const void *p;
    int64_t rows, width, stride;
    bool empty() const { return !p || rows <= 0 || width <= 0; }
    int64_t first() const { return (int64_t)(uintptr_t)p; }
    int64_t end() const {           // INT64_MAX: no memory reaches so far
        const int64_t left = first() < 0 ? 0 : INT64_MAX - first(), more = rows - 1;
        return left < width || (more && more > (left - width) / stride) ? INT64_MAX : first() + more * stride + width;
    }
};
inline OpArea op_run(const void *p, int64_t bytes) { return {p, 1, bytes, bytes}; }
inline OpArea op_matrix(const void *p, int64_t n_rows, int64_t width, int64_t stride, int size) { return {p, n_rows, width * size, stride * size}; }
inline int64_t op_floor_div(int64_t a, int64_t b) { return a / b - (a % b != 0 && (a < 0) != (b < 0)); }

// Whether two areas have a byte in common; columns of one buffer side by side have none.
inline bool op_meet(const OpArea &a, const OpArea &b) {
    if (a.empty() || b.empty() || a.first() >= b.end() || b.first() >= a.end() || a.end() == INT64_MAX || b.end() == INT64_MAX) return false;
    if (a.rows == 1 && b.rows == 1) return true;
    // rows i of a and j of b meet where low < j * b.stride - i * a.stride < high
    const int64_t d = b.first() - a.first(), low = -b.width - d, high = a.width - d;
    if (a.rows > 1 && b.rows > 1 && a.stride == b.stride) {
        const int64_t k = std::max(op_floor_div(low, a.stride) + 1, 1 - a.rows);         // j - i
        return k < b.rows && k * a.stride < high;
    }
    if (a.rows > 1 && b.rows > 1) {         // the difference is a multiple of what divides both strides
        const int64_t g = std::gcd(a.stride, b.stride);
        if ((op_floor_div(low, g) + 1) * g >= high) return false;
    }
    if (a.rows > b.rows) return op_meet(b, a);
    // from the first row of a that ends behind b's start on: the first row of b that ends behind this one's start
    for (int64_t i = std::max<int64_t>(op_floor_div(d - a.width, a.stride) + 1, 0); i < a.rows; ++i) {
        const int64_t at = i * a.stride, j = std::max<int64_t>(op_floor_div(low + at, b.stride) + 1, 0);
        if (j >= b.rows) return false;
        if (j * b.stride - at < high) return true;
    }
    return false;
}
// The first `written` areas overlap no other one.
inline const char *op_check_apart(std::initializer_list<OpArea> areas, int written) {
    const OpArea *p = areas.begin();
    for (int i = 0; i < written; ++i)
        for (int j = i + 1; j < (int)areas.size(); ++j)
            if (op_meet(p[i], p[j])) return "what is written overlaps another buffer";
    return nullptr;
}

inline const char *op_check_group_rows(const int32_t *d_group, int64_t n_rows, int32_t n_groups, const int32_t *d_group_ptr,
                                       const int32_t *d_rows) {
    if (n_rows < 0 || n_rows > INT32_MAX) return "n_rows out of range";
    if (n_groups < 1 || n_groups > GSPLIT_MAX_GROUPS) return "n_groups out of range";
    if (!d_group_ptr || (n_rows > 0 && (!d_group || !d_rows))) return "NULL buffer";
    if (op_misaligned(d_group, 4) || op_misaligned(d_group_ptr, 4) || op_misaligned(d_rows, 4)) return "misaligned buffer";
    return nullptr;
}

inline const char *op_check_grouped(const gsplit_grouped_config *c, int64_t n_rows) {
    if (!c) return "NULL config";
    if (!op_elem_size(c->dtype)) return "unknown dtype";
    if (c->n_groups < 1 || c->n_groups > GSPLIT_MAX_GROUPS) return "n_groups out of range";
    if (c->n_in < 1 || c->n_in > 1 << 20 || c->n_out < 1 || c->n_out > 1 << 20) return "width out of range";
    if (n_rows < 0 || n_rows > INT32_MAX) return "n_rows out of range";
    return nullptr;
}
// a matrix of the rows, `needed` if there are any
inline const char *op_check_grouped_rows(const void *p, int64_t n_rows, int64_t width, int64_t stride, int size, bool needed) {
    if (!p) return needed && n_rows > 0 ? "NULL buffer" : nullptr;
    if (op_misaligned(p, size)) return "misaligned buffer";
    return stride < width || stride > INT32_MAX ? "stride below its width or out of range" : nullptr;
}
inline const char *op_check_grouped_lists(const gsplit_grouped_config *c, const int32_t *d_group_ptr, const int32_t *d_rows) {
    if (!d_group_ptr) return "NULL buffer";
    return op_misaligned(d_group_ptr, 4) || op_misaligned(d_rows, 4) ? "misaligned buffer" : nullptr;
}

inline const char *op_check_grouped_fwd(const gsplit_grouped_config *c, const void *d_x, int64_t n_rows, int64_t x_stride,
                                        const int32_t *d_group_ptr, const int32_t *d_rows, const void *d_w, const float *d_bias,
                                        const void *d_y, int64_t y_stride) {
    if (const char *e = op_check_grouped(c, n_rows)) return e;
    const int size = op_elem_size(c->dtype);
    if (const char *e = op_check_grouped_rows(d_x, n_rows, c->n_in, x_stride, size, true)) return e;
    if (const char *e = op_check_grouped_rows(d_y, n_rows, c->n_out, y_stride, size, true)) return e;
    if (n_rows == 0) return nullptr;
    if (const char *e = op_check_grouped_lists(c, d_group_ptr, d_rows)) return e;
    if (!d_w) return "NULL buffer";
    return op_misaligned(d_w, size) || op_misaligned(d_bias, 4) ? "misaligned buffer" : nullptr;
}

inline const char *op_check_grouped_bwd(const gsplit_grouped_config *c, const void *d_x, int64_t n_rows, int64_t x_stride,
                                        const int32_t *d_group_ptr, const int32_t *d_rows, const void *d_w, const void *d_dy,
                                        int64_t dy_stride, const void *d_dx, int64_t dx_stride, const float *d_dw, const float *d_dbias,
                                        const void *d_work) {
    if (const char *e = op_check_grouped(c, n_rows)) return e;
    const int size = op_elem_size(c->dtype);
    if (const char *e = op_check_grouped_rows(d_x, n_rows, c->n_in, x_stride, size, d_dw)) return e;
    if (const char *e = op_check_grouped_rows(d_dy, n_rows, c->n_out, dy_stride, size, true)) return e;
    if (const char *e = op_check_grouped_rows(d_dx, n_rows, c->n_in, dx_stride, size, false)) return e;
    if (d_dbias && !d_dw) return "d_dbias needs d_dw";
    if (!d_dx && !d_dw) return "nothing to compute";
    if (const char *e = op_check_grouped_lists(c, d_group_ptr, d_rows)) return e;
    if (d_dx && n_rows > 0 && !d_w) return "NULL buffer";
    return op_misaligned(d_w, size) || op_misaligned(d_dw, 4) || op_misaligned(d_dbias, 4) || op_misaligned(d_work, 16) ? "misaligned buffer"
                                                                                                                        : nullptr;
}

// (of arguments that are right by themselves)
inline const char *op_apart_group_rows(const int32_t *d_group, int64_t n_rows, int32_t n_groups, const int32_t *d_group_ptr, const int32_t *d_rows) {
    return op_check_apart({op_run(d_group_ptr, 4 * ((int64_t)n_groups + 1)), op_run(d_rows, 4 * n_rows), op_run(d_group, 4 * n_rows)}, 2);
}
inline const char *op_apart_grouped_fwd(const gsplit_grouped_config *c, const void *d_x, int64_t n_rows, int64_t x_stride,
                                        const int32_t *d_group_ptr, const int32_t *d_rows, const void *d_w, const float *d_bias,
                                        const void *d_y, int64_t y_stride) {
    const int size = op_elem_size(c->dtype);
    const int64_t b = (int64_t)c->n_groups * c->n_out;
    return op_check_apart({op_matrix(d_y, n_rows, c->n_out, y_stride, size), op_matrix(d_x, n_rows, c->n_in, x_stride, size), op_run(d_w, b * c->n_in * size),
                           op_run(d_bias, 4 * b), op_run(d_group_ptr, 4 * ((int64_t)c->n_groups + 1)), op_run(d_rows, 4 * n_rows)}, 1);
}
inline const char *op_apart_grouped_bwd(const gsplit_grouped_config *c, const void *d_x, int64_t n_rows, int64_t x_stride,
                                        const int32_t *d_group_ptr, const int32_t *d_rows, const void *d_w, const void *d_dy,
                                        int64_t dy_stride, const void *d_dx, int64_t dx_stride, const float *d_dw, const float *d_dbias,
                                        const void *d_work, int64_t work_bytes) {
    const int size = op_elem_size(c->dtype);
    const int64_t b = (int64_t)c->n_groups * c->n_out;
    return op_check_apart({op_matrix(d_dx, n_rows, c->n_in, dx_stride, size), op_run(d_dw, b * c->n_in * 4), op_run(d_dbias, 4 * b),
                           op_run(d_dw ? d_work : nullptr, work_bytes), op_matrix(d_x, n_rows, c->n_in, x_stride, size),
                           op_matrix(d_dy, n_rows, c->n_out, dy_stride, size), op_run(d_w, b * c->n_in * size),
                           op_run(d_group_ptr, 4 * ((int64_t)c->n_groups + 1)), op_run(d_rows, 4 * n_rows)}, 4);
}

// Singular values s of [0, 1] under s -> |s (a + b s^2 + c s^4)|: the bounds of what the halves hold (newton.hip).
inline bool op_newton_bounded(double a, double b, double c, int steps) {
    double top = 1.0;           // of the values in front of a step
    for (int k = 0; k < steps; ++k) {
        // largest |s (a + b s^2 + c s^4)| and |a + b x + c x^2| (x = s^2) on [0, top]: at an end or where a derivative is 0
        const auto p = [&](double s) { const double x = s * s; return s * (a + x * (b + x * c)); };
        const auto q = [&](double x) { return std::fabs(a + x * (b + x * c)); };
        double next = std::fabs(p(top)), most = std::fmax(q(0.0), q(top * top));
        if (c != 0.0) {
            const double turn = -b / (2.0 * c), root = 9.0 * b * b - 20.0 * a * c;
            if (turn > 0.0 && turn < top * top) most = std::fmax(most, q(turn));
            if (root >= 0.0) {          // of 5 c x^2 + 3 b x + a: the sum that does not cancel gives either root
                const double q0 = -0.5 * (3.0 * b + std::copysign(std::sqrt(root), b));
                for (const double x : {q0 / (5.0 * c), a / q0})
                    if (x > 0.0 && x < top * top) next = std::fmax(next, std::fabs(p(std::sqrt(x))));
            }
        } else if (b != 0.0 && -a / (3.0 * b) > 0.0 && -a / (3.0 * b) < top * top) {
            next = std::fmax(next, std::fabs(p(std::sqrt(-a / (3.0 * b)))));
        }
        if (!(next <= 1.99 && most <= 15.0)) return false;
        top = std::fmax(next, 1e-300);
    }
    return true;
}

inline const char *op_check_newton(const gsplit_newton_config *c) {
    if (!c) return "NULL config";
    if (c->steps < 1 || c->steps > 64) return "steps out of range";
    if (!op_not_negative(c->eps)) return "eps negative or not finite";
    if (!std::isfinite(c->a) || !std::isfinite(c->b) || !std::isfinite(c->c) || !op_newton_bounded(c->a, c->b, c->c, c->steps))
        return "coefficients that do not keep singular values in bounds";
    return nullptr;
}
inline const char *op_check_shape(int64_t count, int32_t rows, int32_t cols) {
    if (rows < 0 || rows > 65536 || cols < 0 || cols > 65536) return "rows or cols out of range";
    return count < 0 || count > (int64_t)1 << 31 || count * rows > (int64_t)1 << 40 || count * rows * cols > (int64_t)1 << 46
               ? "number of matrices out of range" : nullptr;
}
inline const char *op_check_matrices(const gsplit_matrix_tensor *t, int64_t n_tensors) {
    if (n_tensors < 0 || (n_tensors > 0 && !t)) return "bad tensor list";
    for (int64_t i = 0; i < n_tensors; ++i) {
        if (const char *e = op_check_shape(t[i].count, t[i].rows, t[i].cols)) return e;
        const int64_t n = t[i].count * t[i].rows * t[i].cols;
        if (const char *e = op_check_run(t[i].d_in, n, op_elem_size(t[i].in_dtype))) return e;
        if (const char *e = op_check_run(t[i].d_out, n, op_elem_size(t[i].out_dtype))) return e;
        if (n > 0 && t[i].d_in == t[i].d_out && t[i].in_dtype != t[i].out_dtype) return "in place needs one type";
    }
    return nullptr;
}
inline const char *op_check_muon(const gsplit_muon_config *c) {
    if (!c) return "NULL config";
    if (const char *e = op_check_newton(&c->newton)) return e;
    if (!(c->momentum >= 0.0 && c->momentum < 1.0)) return "momentum outside [0, 1)";
    if (!(c->d_lr || op_not_negative(c->lr)) || !op_not_negative(c->weight_decay)) return "lr or weight_decay negative or not finite";
    if (c->scaling < GSPLIT_MUON_PLAIN || c->scaling > GSPLIT_MUON_RMS) return "unknown scaling";
    return op_misaligned(c->d_lr, 4) ? "misaligned buffer" : nullptr;
}
inline const char *op_check_muon_tensors(const gsplit_muon_tensor *t, int64_t n_tensors) {
    if (n_tensors < 0 || (n_tensors > 0 && !t)) return "bad tensor list";
    for (int64_t i = 0; i < n_tensors; ++i) {
        const gsplit_muon_tensor &x = t[i];
        if (const char *e = op_check_shape(x.count, x.rows, x.cols)) return e;
        const int64_t n = x.count * x.rows * x.cols;
        if (const char *e = op_check_run(x.d_param, n, op_elem_size(x.param_dtype))) return e;
        if (const char *e = op_check_run(x.d_grad, n, op_elem_size(x.grad_dtype))) return e;
        if (const char *e = op_check_run(x.d_momentum, n, 4)) return e;
        if (x.param_dtype == GSPLIT_F32 && x.d_master) return "a float parameter has no d_master";
        if (x.param_dtype == GSPLIT_BF16)
            if (const char *e = op_check_run(x.d_master, n, 4)) return e;
    }
    return nullptr;
}
inline const char *op_check_work(const void *d_work, int64_t bytes) {
    if (bytes > 0 && !d_work) return "NULL d_work";
    return op_misaligned(d_work, 16) ? "misaligned buffer" : nullptr;
}
