// Host side of the operators declared in include/hapmoe.h: argument checks and
// the launches.  Nothing here allocates, waits or throws.
#include <cmath>

#include "internal.h"
#include "operators.h"

using namespace hapmoe;

namespace {

constexpr int64_t kMaxRows = INT32_MAX;                // rows, tokens * top_k: 32-bit indices
constexpr int64_t kMaxSide = INT32_MAX / 2;            // columns of a matrix
constexpr int64_t kMaxElements = int64_t(1) << 46;     // of a tensor

bool any_type(int32_t t) { return t == HAPMOE_F32 || t == HAPMOE_BF16 || t == HAPMOE_F16; }
bool half_type(int32_t t) { return t == HAPMOE_BF16 || t == HAPMOE_F16; }
bool element_aligned(const void *p, int32_t t) { return aligned(p, type_bytes(t)); }

bool bad_route(int64_t tokens, int32_t experts, int32_t top_k)
{
    return tokens < 0 || experts < 1 || experts > HAPMOE_MAX_EXPERTS || top_k < 1 || top_k > HAPMOE_MAX_TOP_K ||
           top_k > experts || tokens > kMaxRows / top_k;
}

bool bad_combine(int32_t type, int64_t tokens, int32_t top_k, int64_t hidden)
{
    return !any_type(type) || tokens < 0 || top_k < 1 || top_k > HAPMOE_MAX_TOP_K || hidden < 1 || hidden > (1 << 24) ||
           tokens > kMaxRows / top_k;
}

// the fields that the three products share; x, w, d_y: whether they are read
bool bad_product(const ExpertProduct &a, bool x, bool w, bool d_y)
{
    if (!half_type(a.type) || a.rows < 0 || a.rows > kMaxRows - 256 || a.experts < 1 ||
        a.experts > HAPMOE_MAX_EXPERTS || a.outputs < 1 || a.outputs > kMaxSide || a.inputs < 1 || a.inputs > kMaxSide ||
        a.outputs > kMaxElements / a.inputs)
        return true;
    if (!a.offset || (!a.out && (a.rows > 0 || !w))) return true;   // without rows only d_w has elements
    if (x) {
        if (a.x_rows < 0 || a.x_rows > kMaxRows || a.x_stride < a.inputs || a.x_stride > kMaxElements) return true;
        if (a.slot ? a.top_k < 1 : a.x_rows < a.rows) return true;
        if (a.rows > 0 && a.x_rows > 0 && !a.x) return true;
        if (!element_aligned(a.x, a.type)) return true;
    }
    if (w && (!a.w || !element_aligned(a.w, a.type))) return true;
    if (d_y && (a.d_y_stride < a.outputs || a.d_y_stride > kMaxElements || (a.rows > 0 && !a.d_y) ||
                !element_aligned(a.d_y, a.type)))
        return true;
    return !element_aligned(a.out, a.out_type) || !aligned(a.offset, 4) || !aligned(a.slot, 4);
}

bool bad_balanced(int64_t stride, int32_t experts, int32_t type, int32_t scores, float scale)
{
    return !any_type(type) || stride < experts || stride > kMaxElements ||
           (scores != HAPMOE_SOFTMAX && scores != HAPMOE_SIGMOID) || !(std::isfinite(scale) && scale > 0.0f);
}

// rows of `columns` elements, `stride` apart
bool bad_rows(int64_t rows, int64_t columns, int64_t stride)
{
    return rows < 0 || rows > kMaxRows || columns < 1 || columns > (1 << 24) || stride < columns || stride > kMaxElements ||
           rows > kMaxElements / stride;
}

bool bad_weight_type(int32_t type, int32_t weight_type)
{
    return !any_type(type) || (weight_type != type && weight_type != HAPMOE_F32);
}

int32_t status(hipError_t e) { return e == hipSuccess ? HAPMOE_OK : HAPMOE_E_HIP; }

}  // namespace

extern "C" {

int32_t hapmoe_route_ws_bytes(int64_t tokens, int32_t experts, int32_t top_k, int64_t *bytes)
{
    if (bad_route(tokens, experts, top_k) || !bytes) return HAPMOE_E_INVAL;
    *bytes = route_ws_bytes(tokens, experts, top_k);
    return HAPMOE_OK;
}

int32_t hapmoe_route(const void *d_logits, int32_t type, int64_t stride, int64_t tokens, int32_t experts,
                     int32_t top_k, const uint8_t *d_keep, int32_t renormalize, float *d_weight, int32_t *d_expert,
                     int32_t *d_count, int32_t *d_offset, int32_t *d_slot, int32_t *d_place, void *d_ws,
                     int64_t ws_bytes, void *stream)
{
    if (bad_route(tokens, experts, top_k) || !any_type(type) || stride < experts || stride > kMaxElements)
        return HAPMOE_E_INVAL;
    if (!d_count || !d_offset || (tokens > 0 && (!d_logits || !d_weight || !d_expert || !d_slot || !d_place)))
        return HAPMOE_E_INVAL;
    if (!element_aligned(d_logits, type)) return HAPMOE_E_INVAL;
    const int64_t need = route_ws_bytes(tokens, experts, top_k);
    if (need > 0 && (!d_ws || !aligned(d_ws, 4))) return HAPMOE_E_INVAL;
    if (ws_bytes < need) return HAPMOE_E_WORKSPACE;
    if (const int e = check_arch()) return e;
    return status(launch_route(d_logits, type, stride, tokens, experts, top_k, d_keep, renormalize != 0, d_weight,
                               d_expert, d_count, d_offset, d_slot, d_place, d_ws, (hipStream_t)stream));
}

int32_t hapmoe_route_backward(const void *d_logits, int32_t type, int64_t stride, int64_t tokens, int32_t experts,
                              int32_t top_k, const uint8_t *d_keep, int32_t renormalize, const int32_t *d_expert,
                              const float *d_weight, const float *d_d_weight, void *d_d_logits, void *stream)
{
    if (bad_route(tokens, experts, top_k) || !any_type(type) || stride < experts || stride > kMaxElements)
        return HAPMOE_E_INVAL;
    if (tokens > 0 && (!d_logits || !d_expert || !d_weight || !d_d_weight || !d_d_logits)) return HAPMOE_E_INVAL;
    if (!element_aligned(d_logits, type) || !element_aligned(d_d_logits, type)) return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (tokens == 0) return HAPMOE_OK;
    return status(launch_route_backward(d_logits, type, stride, tokens, experts, top_k, d_keep, renormalize != 0,
                                        d_expert, d_weight, d_d_weight, d_d_logits, (hipStream_t)stream));
}

int32_t hapmoe_combine(const void *d_y, int32_t type, int64_t rows, int64_t tokens, int32_t top_k, int64_t hidden,
                       const int32_t *d_place, const float *d_weight, void *d_out, void *stream)
{
    if (bad_combine(type, tokens, top_k, hidden) || rows < 0 || rows > kMaxRows) return HAPMOE_E_INVAL;
    if (tokens > 0 && (!d_place || !d_out || (rows > 0 && !d_y))) return HAPMOE_E_INVAL;
    if (!element_aligned(d_y, type) || !element_aligned(d_out, type)) return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (tokens == 0) return HAPMOE_OK;
    return status(launch_combine(d_y, type, rows, tokens, top_k, hidden, d_place, d_weight, d_out,
                                 (hipStream_t)stream));
}

int32_t hapmoe_combine_backward(const void *d_d_out, const void *d_y, int32_t type, int64_t tokens, int32_t top_k,
                                int64_t hidden, const int32_t *d_slot, const int32_t *d_place, const float *d_weight,
                                void *d_d_y, float *d_d_weight, void *stream)
{
    if (bad_combine(type, tokens, top_k, hidden)) return HAPMOE_E_INVAL;
    if (tokens > 0 && (!d_d_out || !d_y || !d_slot || !d_place || !d_weight || !d_d_y || !d_d_weight))
        return HAPMOE_E_INVAL;
    if (!element_aligned(d_y, type) || !element_aligned(d_d_out, type) || !element_aligned(d_d_y, type))
        return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (tokens == 0) return HAPMOE_OK;
    return status(launch_combine_backward(d_d_out, d_y, type, tokens, top_k, hidden, d_slot, d_place, d_weight, d_d_y,
                                          d_d_weight, (hipStream_t)stream));
}

int32_t hapmoe_expert_matmul(const void *d_x, int64_t x_rows, int64_t x_stride, const void *d_w, int32_t type,
                             int64_t rows, int32_t experts, int64_t outputs, int64_t inputs, const int32_t *d_offset,
                             const int32_t *d_slot, int32_t top_k, void *d_y, void *stream)
{
    const ExpertProduct a = {d_x,  d_w,     nullptr, d_y,     d_offset, d_slot, x_rows, x_stride, outputs,
                             rows, outputs, inputs,  experts, top_k,    type,   type};
    if (bad_product(a, true, true, false)) return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (rows == 0) return HAPMOE_OK;
    return status(launch_expert_matmul(a, (hipStream_t)stream));
}

int32_t hapmoe_expert_matmul_grad_x(const void *d_d_y, int64_t d_y_stride, const void *d_w, int32_t type,
                                    int64_t rows, int32_t experts, int64_t outputs, int64_t inputs,
                                    const int32_t *d_offset, void *d_d_x, void *stream)
{
    const ExpertProduct a = {nullptr, d_w,     d_d_y,  d_d_x,   d_offset, nullptr, rows, inputs, d_y_stride,
                             rows,    outputs, inputs, experts, 1,        type,    type};
    if (bad_product(a, false, true, true)) return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (rows == 0) return HAPMOE_OK;
    return status(launch_expert_matmul_grad_x(a, (hipStream_t)stream));
}

int32_t hapmoe_expert_matmul_grad_w(const void *d_d_y, int64_t d_y_stride, const void *d_x, int64_t x_rows,
                                    int64_t x_stride, int32_t type, int64_t rows, int32_t experts, int64_t outputs,
                                    int64_t inputs, const int32_t *d_offset, const int32_t *d_slot, int32_t top_k,
                                    int32_t out_type, void *d_d_w, void *stream)
{
    const ExpertProduct a = {d_x,  nullptr, d_d_y,  d_d_w,   d_offset, d_slot, x_rows, x_stride, d_y_stride,
                             rows, outputs, inputs, experts, top_k,    type,   out_type};
    if (out_type != HAPMOE_F32 && out_type != type) return HAPMOE_E_INVAL;
    if (bad_product(a, true, false, true)) return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    return status(launch_expert_matmul_grad_w(a, (hipStream_t)stream));
}

int32_t hapmoe_adamw(const hapmoe_adamw_tensor *tensors, const void *const *grads, int32_t n_tensors,
                     const hapmoe_adamw_args *args, void *stream)
{
    if (n_tensors < 0 || (n_tensors > 0 && (!tensors || !grads)) || !args) return HAPMOE_E_INVAL;
    const hapmoe_adamw_args &a = *args;
    if (!any_type(a.grad_type) || (a.state_bits != 32 && a.state_bits != 8) || a.step < 1) return HAPMOE_E_INVAL;
    if (!(std::isfinite(a.lr) && a.lr >= 0.0) || !(a.beta1 >= 0.0 && a.beta1 < 1.0) ||
        !(a.beta2 >= 0.0 && a.beta2 < 1.0) || !(std::isfinite(a.eps) && a.eps >= 0.0) || !std::isfinite(a.grad_scale) ||
        !aligned(a.d_skip, 4))
        return HAPMOE_E_INVAL;
    int64_t total = 0;
    int copies = -1;   // whether there are any: as the first tensor that has elements
    for (int i = 0; i < n_tensors; ++i) {
        const hapmoe_adamw_tensor &t = tensors[i];
        if (t.n < 0 || t.n > kMaxElements || (total += t.n) > kMaxElements) return HAPMOE_E_INVAL;
        if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.0f) return HAPMOE_E_INVAL;
        if (t.n == 0) continue;
        if (copies < 0) copies = t.copy != nullptr;
        if ((t.copy != nullptr) != (copies == 1) || (t.copy && !half_type(a.copy_type))) return HAPMOE_E_INVAL;
        if (!t.param || !grads[i] || !t.m || !t.v || (a.state_bits == 8 && (!t.m_exp || !t.v_exp))) return HAPMOE_E_INVAL;
        if (!aligned(t.param, 4) || !element_aligned(grads[i], a.grad_type) || !aligned(t.copy, 2)) return HAPMOE_E_INVAL;
        if (a.state_bits == 32 && (!aligned(t.m, 4) || !aligned(t.v, 4))) return HAPMOE_E_INVAL;
    }
    if (const int e = check_arch()) return e;
    return status(launch_adamw(tensors, grads, n_tensors, a, (hipStream_t)stream));
}

int32_t hapmoe_adamw_moments(const hapmoe_adamw_tensor *tensors, void *const *d_m, void *const *d_v, int32_t n_tensors,
                             int32_t out_type, void *stream)
{
    if (n_tensors < 0 || (n_tensors > 0 && (!tensors || !d_m || !d_v))) return HAPMOE_E_INVAL;
    if (out_type != HAPMOE_F32 && out_type != HAPMOE_BF16) return HAPMOE_E_INVAL;
    int64_t total = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const hapmoe_adamw_tensor &t = tensors[i];
        if (t.n < 0 || t.n > kMaxElements || (total += t.n) > kMaxElements) return HAPMOE_E_INVAL;
        if (t.n == 0) continue;
        if (!t.m || !t.v || !t.m_exp || !t.v_exp || !d_m[i] || !d_v[i]) return HAPMOE_E_INVAL;
        if (!element_aligned(d_m[i], out_type) || !element_aligned(d_v[i], out_type)) return HAPMOE_E_INVAL;
    }
    if (const int e = check_arch()) return e;
    return status(launch_adamw_moments(tensors, d_m, d_v, n_tensors, out_type, (hipStream_t)stream));
}

int32_t hapmoe_route_balanced(const void *d_logits, int32_t type, int64_t stride, int64_t tokens, int32_t experts,
                              int32_t top_k, const float *d_bias, int32_t scores, int32_t groups, int32_t top_groups,
                              int32_t group_best, const uint8_t *d_keep, int32_t renormalize, float scale,
                              float *d_weight, int32_t *d_expert, int32_t *d_count, int32_t *d_offset, int32_t *d_slot,
                              int32_t *d_place, void *d_ws, int64_t ws_bytes, void *stream)
{
    if (bad_route(tokens, experts, top_k) || bad_balanced(stride, experts, type, scores, scale)) return HAPMOE_E_INVAL;
    if (groups < 1 || groups > HAPMOE_MAX_GROUPS || experts % groups != 0 || top_groups < 1 || top_groups > groups ||
        group_best < 1 || group_best > 2 || !aligned(d_bias, 4))
        return HAPMOE_E_INVAL;
    if (!d_count || !d_offset || (tokens > 0 && (!d_logits || !d_weight || !d_expert || !d_slot || !d_place)))
        return HAPMOE_E_INVAL;
    if (!element_aligned(d_logits, type)) return HAPMOE_E_INVAL;
    const int64_t need = route_ws_bytes(tokens, experts, top_k);
    if (need > 0 && (!d_ws || !aligned(d_ws, 4))) return HAPMOE_E_INVAL;
    if (ws_bytes < need) return HAPMOE_E_WORKSPACE;
    if (const int e = check_arch()) return e;
    const BalancedRoute a = {d_logits, d_bias, d_keep,  d_weight, d_expert, d_count,    d_offset,   d_slot, d_place,
                             d_ws,     stride, tokens,  type,     experts,  top_k,      groups,     top_groups,
                             group_best, scale, scores == HAPMOE_SIGMOID, renormalize != 0};
    return status(launch_route_balanced(a, (hipStream_t)stream));
}

int32_t hapmoe_route_balanced_backward(const void *d_logits, int32_t type, int64_t stride, int64_t tokens,
                                       int32_t experts, int32_t top_k, int32_t scores, const uint8_t *d_keep,
                                       int32_t renormalize, float scale, const int32_t *d_expert, const float *d_weight,
                                       const float *d_d_weight, void *d_d_logits, void *stream)
{
    if (bad_route(tokens, experts, top_k) || bad_balanced(stride, experts, type, scores, scale)) return HAPMOE_E_INVAL;
    if (tokens > 0 && (!d_logits || !d_expert || !d_weight || !d_d_weight || !d_d_logits)) return HAPMOE_E_INVAL;
    if (!element_aligned(d_logits, type) || !element_aligned(d_d_logits, type)) return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (tokens == 0) return HAPMOE_OK;
    return status(launch_route_balanced_backward(d_logits, type, stride, tokens, experts, top_k, scores == HAPMOE_SIGMOID,
                                                 d_keep, renormalize != 0, scale, d_expert, d_weight, d_d_weight,
                                                 d_d_logits, (hipStream_t)stream));
}

int32_t hapmoe_layer_norm(const void *d_x, int32_t type, int64_t x_stride, int64_t rows, int64_t hidden,
                          const void *d_weight, const void *d_bias, int32_t weight_type, float eps, float *d_mean,
                          float *d_rstd, void *d_y, void *stream)
{
    if (bad_weight_type(type, weight_type) || bad_rows(rows, hidden, x_stride)) return HAPMOE_E_INVAL;
    if (!(std::isfinite(eps) && eps >= 0.0f) || !d_weight) return HAPMOE_E_INVAL;
    if (rows > 0 && (!d_x || !d_rstd || !d_y)) return HAPMOE_E_INVAL;
    if (!element_aligned(d_x, type) || !element_aligned(d_y, type) || !element_aligned(d_weight, weight_type) ||
        !element_aligned(d_bias, weight_type) || !aligned(d_mean, 4) || !aligned(d_rstd, 4))
        return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (rows == 0) return HAPMOE_OK;
    LayerNorm a = {};
    a.x = d_x, a.weight = d_weight, a.bias = d_bias, a.out = d_y, a.mean = d_mean, a.rstd = d_rstd;
    a.x_stride = x_stride, a.rows = rows, a.hidden = hidden, a.type = type, a.weight_type = weight_type, a.eps = eps;
    return status(launch_layer_norm(a, (hipStream_t)stream));
}

int32_t hapmoe_layer_norm_ws_bytes(int64_t rows, int64_t hidden, int64_t *bytes)
{
    if (bad_rows(rows, hidden, hidden) || !bytes) return HAPMOE_E_INVAL;
    *bytes = layer_norm_ws_bytes(rows, hidden);
    return HAPMOE_OK;
}

int32_t hapmoe_layer_norm_backward(const void *d_d_y, int64_t d_y_stride, const void *d_x, int32_t type,
                                   int64_t x_stride, int64_t rows, int64_t hidden, const void *d_weight,
                                   int32_t weight_type, const float *d_mean, const float *d_rstd, const void *d_add,
                                   int64_t add_stride, void *d_d_x, float *d_d_weight, float *d_d_bias, void *d_ws,
                                   int64_t ws_bytes, void *stream)
{
    if (bad_weight_type(type, weight_type) || bad_rows(rows, hidden, x_stride) || bad_rows(rows, hidden, d_y_stride) ||
        (d_add && bad_rows(rows, hidden, add_stride)))
        return HAPMOE_E_INVAL;
    if (!d_weight || !d_d_weight || (rows > 0 && (!d_d_y || !d_x || !d_rstd || !d_d_x))) return HAPMOE_E_INVAL;
    if (!element_aligned(d_d_y, type) || !element_aligned(d_x, type) || !element_aligned(d_add, type) ||
        !element_aligned(d_d_x, type) || !element_aligned(d_weight, weight_type) || !aligned(d_mean, 4) ||
        !aligned(d_rstd, 4) || !aligned(d_d_weight, 4) || !aligned(d_d_bias, 4))
        return HAPMOE_E_INVAL;
    const int64_t need = layer_norm_ws_bytes(rows, hidden);
    if (need > 0 && (!d_ws || !aligned(d_ws, 16))) return HAPMOE_E_INVAL;
    if (ws_bytes < need) return HAPMOE_E_WORKSPACE;
    if (const int e = check_arch()) return e;
    LayerNorm a = {};
    a.x = d_x, a.weight = d_weight, a.d_y = d_d_y, a.add = d_add, a.out = d_d_x;
    a.mean = const_cast<float *>(d_mean), a.rstd = const_cast<float *>(d_rstd);
    a.d_weight = d_d_weight, a.d_bias = d_d_bias, a.ws = d_ws;
    a.x_stride = x_stride, a.d_y_stride = d_y_stride, a.add_stride = add_stride, a.rows = rows, a.hidden = hidden;
    a.type = type, a.weight_type = weight_type;
    return status(launch_layer_norm_backward(a, (hipStream_t)stream));
}

int32_t hapmoe_embed(const void *d_token, int32_t token_bits, int64_t tokens, const void *d_table, int32_t type,
                     int64_t stride, int64_t vocab, int64_t hidden, float scale, void *d_out, void *stream)
{
    if (!any_type(type) || bad_rows(vocab, hidden, stride) || bad_rows(tokens, hidden, hidden) || vocab < 1 ||
        (token_bits != 32 && token_bits != 64) || !std::isfinite(scale))
        return HAPMOE_E_INVAL;
    if (!d_table || (tokens > 0 && (!d_token || !d_out))) return HAPMOE_E_INVAL;
    if (!element_aligned(d_table, type) || !element_aligned(d_out, type) || !aligned(d_token, token_bits / 8))
        return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (tokens == 0) return HAPMOE_OK;
    return status(launch_embed(d_token, token_bits == 64, tokens, d_table, type, stride, vocab, hidden, scale, d_out,
                               (hipStream_t)stream));
}

int32_t hapmoe_embed_ws_bytes(int64_t tokens, int64_t hidden, int64_t *bytes)
{
    if (bad_rows(tokens, hidden, hidden) || !bytes) return HAPMOE_E_INVAL;
    *bytes = embed_ws_bytes(tokens, hidden);
    return HAPMOE_OK;
}

int32_t hapmoe_embed_backward(const void *d_d_out, int32_t type, int64_t stride, int64_t tokens, int64_t hidden,
                              const void *d_token, int32_t token_bits, int64_t vocab, float scale, int32_t add,
                              float *d_d_table, void *d_ws, int64_t ws_bytes, void *stream)
{
    if (!any_type(type) || bad_rows(tokens, hidden, stride) || bad_rows(vocab, hidden, hidden) || vocab < 1 ||
        vocab > INT32_MAX - 1 ||   // a token that is none of the table's sorts as vocab, before the end's mark
        (token_bits != 32 && token_bits != 64) || !std::isfinite(scale))
        return HAPMOE_E_INVAL;
    if (!d_d_table || !aligned(d_d_table, 4) || (tokens > 0 && (!d_d_out || !d_token))) return HAPMOE_E_INVAL;
    if (!element_aligned(d_d_out, type) || !aligned(d_token, token_bits / 8)) return HAPMOE_E_INVAL;
    const int64_t need = embed_ws_bytes(tokens, hidden);
    if (need > 0 && (!d_ws || !aligned(d_ws, 16))) return HAPMOE_E_INVAL;
    if (ws_bytes < need) return HAPMOE_E_WORKSPACE;
    if (const int e = check_arch()) return e;
    return status(launch_embed_backward(d_d_out, type, stride, tokens, hidden, d_token, token_bits == 64, vocab, scale,
                                        add != 0, d_d_table, d_ws, (hipStream_t)stream));
}

int32_t hapmoe_dropout(const void *d_x, int32_t type, int64_t x_stride, int64_t rows, int64_t columns,
                       const void *d_residual, int64_t residual_stride, double p, uint64_t seed, uint64_t offset,
                       const int64_t *d_counter, void *d_out, void *stream)
{
    if (!any_type(type) || bad_rows(rows, columns, x_stride) || (d_residual && bad_rows(rows, columns, residual_stride)) ||
        !(p >= 0.0 && p <= 1.0))
        return HAPMOE_E_INVAL;
    if (rows > 0 && (!d_x || !d_out)) return HAPMOE_E_INVAL;
    if (!element_aligned(d_x, type) || !element_aligned(d_residual, type) || !element_aligned(d_out, type) ||
        !aligned(d_counter, 8))
        return HAPMOE_E_INVAL;
    if (const int e = check_arch()) return e;
    if (rows == 0) return HAPMOE_OK;
    return status(launch_dropout(d_x, type, x_stride, rows, columns, d_residual, residual_stride, p, seed, offset,
                                 d_counter, d_out, (hipStream_t)stream));
}

}  // extern "C"
