// layer_api.cpp -- host side of the layer operators: the C ABI declared in include/ep_layer.h.
// Argument checks only; the launchers choose kernels and grids.
#include "ep_layer.h"
#include "layer.h"
#include "staging.h"

using ep::aligned16;
using ep::fail;
using ep::hip_fail;

namespace {

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

ep_status check_norm(const char *who, int64_t T, int32_t H, float eps) {
    if (T < 0 || H < 8 || H % 8 != 0 || H > EP_NORM_MAX_HIDDEN || !(eps >= 0.f))
        return fail(EP_ERR_INVALID_ARG, "%s: need T >= 0, H a multiple of 8 in [8, %d], eps >= 0 (T=%lld H=%d eps=%g)", who,
                    EP_NORM_MAX_HIDDEN, (long long)T, H, (double)eps);
    return EP_OK;
}

ep_status check_route(const char *who, int64_t T, int32_t E, int32_t k) {
    if (T < 0 || E < 1 || E > EP_MAX_EXPERTS || k < 1 || k > E || T > INT32_MAX / k)
        return fail(EP_ERR_INVALID_ARG, "%s: need T >= 0, 1 <= k <= E <= %d, T*k < 2^31 (T=%lld k=%d E=%d)", who,
                    EP_MAX_EXPERTS, (long long)T, k, E);
    return EP_OK;
}

ep_status check_product(const char *who, int64_t rows, int32_t E, int32_t K, int32_t N, int32_t kind, int32_t act) {
    if (kind != EP_ROWS_BF16 && kind != EP_ROWS_8BIT)
        return fail(EP_ERR_INVALID_ARG, "%s: unknown kind of rows %d", who, kind);
    if (act < EP_ACT_NONE || act > EP_ACT_SWIGLU)
        return fail(EP_ERR_INVALID_ARG, "%s: unknown activation %d", who, act);
    const int32_t unit = kind == EP_ROWS_8BIT ? 16 : 8;
    const int64_t Nw = act == EP_ACT_SWIGLU ? 2 * (int64_t)N : N;
    if (rows < 0 || rows > INT32_MAX || E < 1 || E > EP_MAX_EXPERTS || K < unit || K % unit != 0 || N < 8 || N % 8 != 0 ||
        K > EP_PRODUCT_MAX_LENGTH || Nw > EP_PRODUCT_MAX_LENGTH)
        return fail(EP_ERR_INVALID_ARG,
                    "%s: need 0 <= rows < 2^31, 1 <= E <= %d, K a multiple of %d and N of 8, both positive, K and the weight "
                    "rows at most %d (rows=%lld E=%d K=%d N=%d)",
                    who, EP_MAX_EXPERTS, unit, EP_PRODUCT_MAX_LENGTH, (long long)rows, E, K, N);
    if (Nw * K * (kind == EP_ROWS_8BIT ? 1 : 2) > INT32_MAX)
        return fail(EP_ERR_INVALID_ARG, "%s: an expert's weights take 2^31 bytes or more", who);
    return EP_OK;
}

}  // namespace

extern "C" ep_status ep_rmsnorm(const void *x_dev, const void *residual_dev, const void *weight_dev, int64_t num_tokens,
                                int32_t hidden, float eps, void *total_dev, void *out_dev, void *rows8_dev,
                                hipStream_t stream) {
    const ep_status st = check_norm("ep_rmsnorm", num_tokens, hidden, eps);
    if (st != EP_OK)
        return st;
    if (num_tokens > 0 && !total_dev && !out_dev && !rows8_dev)
        return fail(EP_ERR_INVALID_ARG, "ep_rmsnorm: no output");
    if (rows8_dev && hidden % 16 != 0)
        return fail(EP_ERR_INVALID_ARG, "ep_rmsnorm: 8-bit rows need H %% 16 == 0 (H=%d)", hidden);
    if (num_tokens > 0 && (!x_dev || !aligned16(x_dev) || !aligned16(residual_dev) || !aligned16(weight_dev) ||
                           !aligned16(total_dev) || !aligned16(out_dev) || !aligned16(rows8_dev)))
        return fail(EP_ERR_INVALID_ARG, "ep_rmsnorm: x is required, every array 16-byte aligned");
    ep::NormArgs a{};
    a.x = static_cast<const ep::u32x4 *>(x_dev);
    a.residual = static_cast<const ep::u32x4 *>(residual_dev);
    a.weight = static_cast<const ep::u32x4 *>(weight_dev);
    a.total = static_cast<ep::u32x4 *>(total_dev);
    a.out = static_cast<ep::u32x4 *>(out_dev);
    a.rows8 = static_cast<uint8_t *>(rows8_dev);
    a.T = num_tokens;
    a.H = hidden;
    a.eps = eps;
    EP_HIP(ep::launch_rmsnorm(a, stream));
    return EP_OK;
}

extern "C" ep_status ep_rmsnorm_grad_workspace_bytes(int64_t num_tokens, int32_t hidden, size_t *bytes) {
    const ep_status st = check_norm("ep_rmsnorm_grad_workspace_bytes", num_tokens, hidden, 0.f);
    if (st != EP_OK)
        return st;
    if (!bytes)
        return fail(EP_ERR_INVALID_ARG, "ep_rmsnorm_grad_workspace_bytes: bytes is NULL");
    *bytes = (size_t)ep::rmsnorm_grad_groups(num_tokens, hidden) * hidden * sizeof(float);
    return EP_OK;
}

extern "C" ep_status ep_rmsnorm_grad(const void *total_dev, const void *weight_dev, const void *d_out_dev,
                                     const void *d_total_dev, int64_t num_tokens, int32_t hidden, float eps, void *dx_dev,
                                     float *d_weight, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const ep_status st = check_norm("ep_rmsnorm_grad", num_tokens, hidden, eps);
    if (st != EP_OK)
        return st;
    if (num_tokens > 0 && (!total_dev || !d_out_dev || !dx_dev || !aligned16(total_dev) || !aligned16(weight_dev) ||
                           !aligned16(d_out_dev) || !aligned16(d_total_dev) || !aligned16(dx_dev)))
        return fail(EP_ERR_INVALID_ARG, "ep_rmsnorm_grad: total, d_out and dx are required, every array 16-byte aligned");
    const size_t need = d_weight ? (size_t)ep::rmsnorm_grad_groups(num_tokens, hidden) * hidden * sizeof(float) : 0;
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need))
        return fail(EP_ERR_INVALID_ARG, "ep_rmsnorm_grad: workspace of %zu bytes, need %zu, 16-byte aligned",
                    workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned(d_weight, 4))
        return fail(EP_ERR_INVALID_ARG, "ep_rmsnorm_grad: d_weight is not 4-byte aligned");
    ep::NormGradArgs a{};
    a.total = static_cast<const ep::u32x4 *>(total_dev);
    a.weight = static_cast<const ep::u32x4 *>(weight_dev);
    a.d_out = static_cast<const ep::u32x4 *>(d_out_dev);
    a.d_total = static_cast<const ep::u32x4 *>(d_total_dev);
    a.dx = static_cast<ep::u32x4 *>(dx_dev);
    a.d_weight = d_weight;
    a.partial = static_cast<float *>(workspace);
    a.T = num_tokens;
    a.H = hidden;
    a.eps = eps;
    EP_HIP(ep::launch_rmsnorm_grad(a, stream));
    return EP_OK;
}

extern "C" ep_status ep_route_workspace_bytes(int64_t num_tokens, int32_t num_experts, size_t *bytes) {
    const ep_status st = check_route("ep_route_workspace_bytes", num_tokens, num_experts, 1);
    if (st != EP_OK)
        return st;
    if (!bytes)
        return fail(EP_ERR_INVALID_ARG, "ep_route_workspace_bytes: bytes is NULL");
    *bytes = ep::route_workspace_bytes(num_tokens, num_experts);
    return EP_OK;
}

extern "C" ep_status ep_route(const void *logits_dev, int32_t logits_bf16, const uint8_t *mask, int64_t num_tokens,
                              int32_t num_experts, int32_t topk, int32_t normalize, float balance, int32_t *topk_idx,
                              float *topk_w, int32_t *counts, float *prob_sums, float *loss, void *workspace,
                              size_t workspace_bytes, hipStream_t stream) {
    const ep_status st = check_route("ep_route", num_tokens, num_experts, topk);
    if (st != EP_OK)
        return st;
    if (num_tokens > 0 && (!logits_dev || !topk_idx || !topk_w || !aligned16(logits_dev) || !aligned(topk_idx, 4) ||
                           !aligned(topk_w, 4)))
        return fail(EP_ERR_INVALID_ARG, "ep_route: 16-byte aligned logits, topk_idx and topk_w are required");
    if ((counts || prob_sums || loss) && !(counts && prob_sums && loss))
        return fail(EP_ERR_INVALID_ARG, "ep_route: counts, prob_sums and loss come together");
    if (!aligned(counts, 4) || !aligned(prob_sums, 4) || !aligned(loss, 4))
        return fail(EP_ERR_INVALID_ARG, "ep_route: counts, prob_sums and loss are not 4-byte aligned");
    const size_t need = counts ? ep::route_workspace_bytes(num_tokens, num_experts) : 0;
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need))
        return fail(EP_ERR_INVALID_ARG, "ep_route: workspace of %zu bytes, need %zu, 16-byte aligned",
                    workspace ? workspace_bytes : (size_t)0, need);
    ep::RouteArgs a{};
    a.logits = logits_dev;
    a.bf16 = logits_bf16 != 0;
    a.mask = mask;
    a.T = num_tokens;
    a.E = num_experts;
    a.k = topk;
    a.normalize = normalize != 0;
    a.balance = balance;
    a.topk_idx = topk_idx;
    a.topk_w = topk_w;
    a.counts = counts;
    a.prob_sums = prob_sums;
    a.loss = loss;
    a.workspace = workspace;
    EP_HIP(ep::launch_route(a, stream));
    return EP_OK;
}

extern "C" ep_status ep_route_grad(const void *logits_dev, int32_t logits_bf16, const uint8_t *mask,
                                   const int32_t *topk_idx, const int32_t *counts, const float *d_topk_w,
                                   const float *d_loss, int64_t num_tokens, int32_t num_experts, int32_t topk,
                                   int32_t normalize, float balance, void *d_logits_dev, hipStream_t stream) {
    const ep_status st = check_route("ep_route_grad", num_tokens, num_experts, topk);
    if (st != EP_OK)
        return st;
    if (num_tokens > 0 && (!logits_dev || !d_logits_dev || !aligned16(logits_dev) || !aligned16(d_logits_dev)))
        return fail(EP_ERR_INVALID_ARG, "ep_route_grad: 16-byte aligned logits and d_logits are required");
    if (num_tokens > 0 && d_topk_w && (!topk_idx || !aligned(topk_idx, 4) || !aligned(d_topk_w, 4)))
        return fail(EP_ERR_INVALID_ARG, "ep_route_grad: the gates' gradient needs topk_idx, both 4-byte aligned");
    if (num_tokens > 0 && d_loss && (!counts || !aligned(counts, 4) || !aligned(d_loss, 4)))
        return fail(EP_ERR_INVALID_ARG, "ep_route_grad: the loss's gradient needs counts, both 4-byte aligned");
    ep::RouteGradArgs a{};
    a.logits = logits_dev;
    a.bf16 = logits_bf16 != 0;
    a.mask = mask;
    a.topk_idx = topk_idx;
    a.counts = counts;
    a.d_topk_w = d_topk_w;
    a.d_loss = d_loss;
    a.T = num_tokens;
    a.E = num_experts;
    a.k = topk;
    a.normalize = normalize != 0;
    a.balance = balance;
    a.d_logits = d_logits_dev;
    EP_HIP(ep::launch_route_grad(a, stream));
    return EP_OK;
}

extern "C" ep_status ep_combine_grad(const void *d_out_dev, const void *y_dev, int64_t max_rows, const int32_t *slot_pos,
                                     const float *topk_w, int64_t num_tokens, int32_t hidden, int32_t topk, void *dy_dev,
                                     float *d_topk_w, hipStream_t stream) {
    if (num_tokens < 0 || topk < 1 || hidden < 8 || hidden % 8 != 0 || max_rows < 0 || num_tokens > INT32_MAX / topk)
        return fail(EP_ERR_INVALID_ARG,
                    "ep_combine_grad: need T >= 0, k >= 1, T*k < 2^31, H a positive multiple of 8, max_rows >= 0 "
                    "(T=%lld k=%d H=%d max_rows=%lld)",
                    (long long)num_tokens, topk, hidden, (long long)max_rows);
    if (num_tokens > 0 && !dy_dev && !d_topk_w)
        return fail(EP_ERR_INVALID_ARG, "ep_combine_grad: no output");
    if (num_tokens > 0 && (!d_out_dev || !slot_pos || !topk_w || !aligned16(d_out_dev) || !aligned16(y_dev) ||
                           !aligned16(dy_dev) || !aligned(slot_pos, 4) || !aligned(topk_w, 4) || !aligned(d_topk_w, 4) ||
                           (max_rows > 0 && d_topk_w && !y_dev)))
        return fail(EP_ERR_INVALID_ARG, "ep_combine_grad: 16-byte aligned d_out and y, slot_pos and topk_w are required");
    EP_HIP(ep::launch_combine_grad(d_out_dev, y_dev, max_rows, slot_pos, topk_w, num_tokens, hidden, topk, dy_dev, d_topk_w,
                                   stream));
    return EP_OK;
}

extern "C" ep_status ep_expert_product_workspace_bytes(int64_t rows, int32_t num_experts, int32_t in_length,
                                                       int32_t out_length, ep_rows_kind kind, ep_activation act,
                                                       size_t *bytes) {
    const ep_status st = check_product("ep_expert_product_workspace_bytes", rows, num_experts, in_length, out_length, kind, act);
    if (st != EP_OK)
        return st;
    if (!bytes)
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product_workspace_bytes: bytes is NULL");
    *bytes = ep::product_workspace_bytes(rows, num_experts, in_length, out_length, kind == EP_ROWS_8BIT, act);
    return EP_OK;
}

extern "C" ep_status ep_expert_product(const void *x_dev, ep_rows_kind kind, int64_t rows, const int32_t *offsets,
                                       int32_t num_experts, const void *w_dev, const float *w_scale, int32_t in_length,
                                       int32_t out_length, const void *bias_dev, ep_activation act,
                                       const void *residual_dev, void *pre_dev, void *y_dev, ep_out_dtype out_dtype,
                                       void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const ep_status st = check_product("ep_expert_product", rows, num_experts, in_length, out_length, kind, act);
    if (st != EP_OK)
        return st;
    if (out_dtype != EP_OUT_BF16 && out_dtype != EP_OUT_F32)
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product: unknown out_dtype %d", (int)out_dtype);
    if (!offsets && num_experts != 1)
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product: more than one expert needs offsets");
    if ((kind == EP_ROWS_8BIT) != (w_scale != nullptr))
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product: w_scale goes with 8-bit rows, and with them only");
    if (rows > 0 && (!x_dev || !w_dev || !y_dev || !aligned16(x_dev) || !aligned16(w_dev) || !aligned16(y_dev) ||
                     !aligned16(w_scale) || !aligned16(bias_dev) || !aligned16(residual_dev) || !aligned16(pre_dev) ||
                     !aligned(offsets, 4)))
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product: x, w and y are required, every array 16-byte aligned");
    const size_t need = ep::product_workspace_bytes(rows, num_experts, in_length, out_length, kind == EP_ROWS_8BIT, act);
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need))
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product: workspace of %zu bytes, need %zu, 16-byte aligned",
                    workspace ? workspace_bytes : (size_t)0, need);
    ep::ProductArgs a{};
    a.x = x_dev;
    a.bits8 = kind == EP_ROWS_8BIT;
    a.rows = rows;
    a.offsets = offsets;
    a.E = num_experts;
    a.w = w_dev;
    a.w_scale = w_scale;
    a.K = in_length;
    a.N = out_length;
    a.Nw = act == EP_ACT_SWIGLU ? 2 * out_length : out_length;
    a.bias = bias_dev;
    a.act = act;
    a.residual = residual_dev;
    a.pre = pre_dev;
    a.y = y_dev;
    a.f32 = out_dtype == EP_OUT_F32;
    a.partial = static_cast<float *>(workspace);
    EP_HIP(ep::launch_product(a, stream));
    return EP_OK;
}

extern "C" ep_status ep_expert_product_grad_workspace_bytes(int64_t rows, int32_t num_experts, int32_t in_length,
                                                            int32_t out_length, ep_activation act, int32_t results,
                                                            size_t *bytes) {
    const ep_status st = check_product("ep_expert_product_grad_workspace_bytes", rows, num_experts, in_length, out_length,
                                       EP_ROWS_BF16, act);
    if (st != EP_OK)
        return st;
    if (!bytes)
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product_grad_workspace_bytes: bytes is NULL");
    if (results < 0 || results > (EP_GRAD_DBIAS | EP_GRAD_WITHOUT_DX | EP_GRAD_WITHOUT_DW))
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product_grad_workspace_bytes: unknown results %d", results);
    *bytes = ep::product_grad_workspace_bytes(rows, num_experts, in_length, out_length, act, !(results & EP_GRAD_WITHOUT_DX),
                                              !(results & EP_GRAD_WITHOUT_DW), (results & EP_GRAD_DBIAS) != 0);
    return EP_OK;
}

extern "C" ep_status ep_expert_product_grad(const void *x_dev, int64_t rows, const int32_t *offsets, int32_t num_experts,
                                            const void *w_dev, int32_t in_length, int32_t out_length, ep_activation act,
                                            const void *pre_dev, const void *d_y_dev, void *dx_dev, void *dw_dev,
                                            float *dbias, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const ep_status st = check_product("ep_expert_product_grad", rows, num_experts, in_length, out_length, EP_ROWS_BF16, act);
    if (st != EP_OK)
        return st;
    if (rows > 0 && !dx_dev && !dw_dev && !dbias)
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product_grad: no output");
    if (!offsets && num_experts != 1)
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product_grad: more than one expert needs offsets");
    if (rows > 0 && (!d_y_dev || (act != EP_ACT_NONE && !pre_dev) || (dx_dev && !w_dev) || (dw_dev && !x_dev) ||
                     !aligned16(d_y_dev) || !aligned16(pre_dev) || !aligned16(x_dev) || !aligned16(w_dev)))
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product_grad: d_y, pre (with an activation), w (for dx) and x (for dw) "
                                        "are required, every array 16-byte aligned");
    if (!aligned16(dx_dev) || !aligned16(dw_dev) || !aligned16(dbias) || !aligned(offsets, 4))
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product_grad: an output is not 16-byte aligned");
    const size_t need = ep::product_grad_workspace_bytes(rows, num_experts, in_length, out_length, act, dx_dev != nullptr,
                                                         dw_dev != nullptr, dbias != nullptr);
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need))
        return fail(EP_ERR_INVALID_ARG, "ep_expert_product_grad: workspace of %zu bytes, need %zu, 16-byte aligned",
                    workspace ? workspace_bytes : (size_t)0, need);
    ep::ProductGradArgs a{};
    a.x = x_dev;
    a.rows = rows;
    a.offsets = offsets;
    a.E = num_experts;
    a.w = w_dev;
    a.K = in_length;
    a.N = out_length;
    a.Nw = act == EP_ACT_SWIGLU ? 2 * out_length : out_length;
    a.act = act;
    a.pre = pre_dev;
    a.d_y = d_y_dev;
    a.dx = dx_dev;
    a.dw = dw_dev;
    a.dbias = dbias;
    a.workspace = workspace;
    EP_HIP(ep::launch_product_grad(a, stream));
    return EP_OK;
}
