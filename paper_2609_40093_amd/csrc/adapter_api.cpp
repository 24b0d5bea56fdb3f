// adapter_api.cpp -- host side of the low-rank adapters: their part of the C ABI declared in
// include/ep_layer.h.  Argument checks only; the launchers choose kernels and grids.
#include "ep_layer.h"
#include "layer.h"
#include "staging.h"

using ep::aligned16;
using ep::fail;
using ep::hip_fail;

namespace {

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

ep_status check_sizes(const char *who, int64_t rows, int32_t A, int32_t R, int32_t K, int32_t N, int32_t act) {
    if (act < EP_ACT_NONE || act > EP_ACT_SWIGLU)
        return fail(EP_ERR_INVALID_ARG, "%s: unknown activation %d", who, act);
    const int64_t Nw = act == EP_ACT_SWIGLU ? 2 * (int64_t)N : N;
    if (rows < 0 || rows > INT32_MAX || A < 1 || A > EP_ADAPTER_MAX || R < 8 || R % 8 != 0 || R > EP_ADAPTER_MAX_RANK ||
        K < 8 || K % 8 != 0 || N < 8 || N % 8 != 0 || K > EP_PRODUCT_MAX_LENGTH || Nw > EP_PRODUCT_MAX_LENGTH)
        return fail(EP_ERR_INVALID_ARG,
                    "%s: need 0 <= rows < 2^31, 1 <= A <= %d, the rank a multiple of 8 up to %d, K and N positive multiples "
                    "of 8, K and the weight rows at most %d (rows=%lld A=%d R=%d K=%d N=%d)",
                    who, EP_ADAPTER_MAX, EP_ADAPTER_MAX_RANK, EP_PRODUCT_MAX_LENGTH, (long long)rows, A, R, K, N);
    // A launch has fewer than 2^32 threads.  The low-rank pass takes the most: 4 per row and 64 ranks (128 for 32 rows, 512 for
    // 128), and the 2^21 rows less than 2^30 leave room for each adapter's last tile.  The products take 2 to 4 per row and
    // column of tiles; with more than two columns so many rows would be results of 2^39 bytes.
    if (rows * ((R + 63) / 64) > EP_ADAPTER_MAX_ROWS)
        return fail(EP_ERR_INVALID_ARG, "%s: rows * ceil(rank / 64) must be at most %d (rows=%lld R=%d)", who,
                    EP_ADAPTER_MAX_ROWS, (long long)rows, R);
    if (Nw * K * 2 > INT32_MAX || (int64_t)A * R * K * 2 > INT32_MAX || A * R * Nw * 2 > INT32_MAX)
        return fail(EP_ERR_INVALID_ARG, "%s: w, a or b takes 2^31 bytes or more", who);
    return EP_OK;
}

}  // namespace

extern "C" ep_status ep_adapter_rows(const int32_t *row_adapter, int64_t rows, int32_t num_adapters, int32_t *order,
                                     int32_t *offsets, hipStream_t stream) {
    if (rows < 0 || rows > INT32_MAX || num_adapters < 1 || num_adapters > EP_ADAPTER_MAX)
        return fail(EP_ERR_INVALID_ARG, "ep_adapter_rows: need 0 <= rows < 2^31, 1 <= A <= %d (rows=%lld A=%d)",
                    EP_ADAPTER_MAX, (long long)rows, num_adapters);
    if (!offsets || !aligned4(offsets) || (rows > 0 && (!row_adapter || !order || !aligned4(row_adapter) || !aligned4(order))))
        return fail(EP_ERR_INVALID_ARG, "ep_adapter_rows: row_adapter, order and offsets are required, 4-byte aligned");
    EP_HIP(ep::launch_adapter_rows(row_adapter, rows, num_adapters, order, offsets, stream));
    return EP_OK;
}

extern "C" ep_status ep_adapter_product_workspace_bytes(int64_t rows, int32_t num_adapters, int32_t rank, int32_t in_length,
                                                        int32_t out_length, int32_t with_w, ep_activation act,
                                                        size_t *bytes) {
    const ep_status st =
        check_sizes("ep_adapter_product_workspace_bytes", rows, num_adapters, rank, in_length, out_length, act);
    if (st != EP_OK)
        return st;
    if (!bytes)
        return fail(EP_ERR_INVALID_ARG, "ep_adapter_product_workspace_bytes: bytes is NULL");
    *bytes = ep::adapter_product_workspace_bytes(rows, num_adapters, rank, in_length, out_length, with_w != 0, act);
    return EP_OK;
}

extern "C" ep_status ep_adapter_product(const void *x_dev, int64_t rows, const int32_t *order, const int32_t *offsets,
                                        int32_t num_adapters, int32_t rank, const void *a_dev, const void *b_dev,
                                        const float *scale, const void *w_dev, int32_t in_length, int32_t out_length,
                                        const void *bias_dev, ep_activation act, const void *residual_dev, void *pre_dev,
                                        void *low_dev, void *y_dev, void *workspace, size_t workspace_bytes,
                                        hipStream_t stream) {
    const ep_status st = check_sizes("ep_adapter_product", rows, num_adapters, rank, in_length, out_length, act);
    if (st != EP_OK)
        return st;
    if (!offsets && num_adapters != 1)
        return fail(EP_ERR_INVALID_ARG, "ep_adapter_product: more than one adapter needs offsets");
    if (order && w_dev && rows * in_length * 2 > INT32_MAX)
        return fail(EP_ERR_INVALID_ARG, "ep_adapter_product: with an order and w, x must be smaller than 2^31 bytes");
    if (order && rows * in_length * 2 > INT32_MAX && rows * ((rank + 15) / 16) > EP_ADAPTER_MAX_GATHERED)
        return fail(EP_ERR_INVALID_ARG, "ep_adapter_product: with an order over x of 2^31 bytes and more, rows * ceil(rank / 16) "
                                        "must be at most %d (rows=%lld R=%d)",
                    EP_ADAPTER_MAX_GATHERED, (long long)rows, rank);
    if (rows > 0 && (!x_dev || !a_dev || !b_dev || !y_dev || !aligned16(x_dev) || !aligned16(a_dev) || !aligned16(b_dev) ||
                     !aligned16(y_dev) || !aligned16(w_dev) || !aligned16(bias_dev) || !aligned16(residual_dev) ||
                     !aligned16(pre_dev) || !aligned16(low_dev) || !aligned4(order) || !aligned4(offsets) || !aligned4(scale)))
        return fail(EP_ERR_INVALID_ARG,
                    "ep_adapter_product: x, a, b and y are required, every array 16-byte aligned (order, offsets, scale 4)");
    const size_t need =
        ep::adapter_product_workspace_bytes(rows, num_adapters, rank, in_length, out_length, w_dev != nullptr, act);
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need))
        return fail(EP_ERR_INVALID_ARG, "ep_adapter_product: workspace of %zu bytes, need %zu, 16-byte aligned",
                    workspace ? workspace_bytes : (size_t)0, need);
    ep::AdapterArgs a{};
    a.x = x_dev;
    a.rows = rows;
    a.order = order;
    a.offsets = offsets;
    a.A = num_adapters;
    a.R = rank;
    a.K = in_length;
    a.N = out_length;
    a.a = a_dev;
    a.b = b_dev;
    a.scale = scale;
    a.w = w_dev;
    a.bias = bias_dev;
    a.act = act;
    a.residual = residual_dev;
    a.pre = pre_dev;
    a.low = low_dev;
    a.y = y_dev;
    a.workspace = workspace;
    EP_HIP(ep::launch_adapter_product(a, stream));
    return EP_OK;
}

extern "C" ep_status ep_adapter_product_grad_workspace_bytes(int64_t rows, int32_t num_adapters, int32_t rank,
                                                             int32_t in_length, int32_t out_length, int32_t with_w,
                                                             ep_activation act, int32_t with_order, int32_t results,
                                                             size_t *bytes) {
    const char *who = "ep_adapter_product_grad_workspace_bytes";
    const ep_status st = check_sizes(who, rows, num_adapters, rank, in_length, out_length, act);
    if (st != EP_OK)
        return st;
    if (!bytes)
        return fail(EP_ERR_INVALID_ARG, "%s: bytes is NULL", who);
    if (results < 0 || results > (EP_ADAPTER_DX | EP_ADAPTER_DA | EP_ADAPTER_DB))
        return fail(EP_ERR_INVALID_ARG, "%s: unknown results %d", who, results);
    *bytes = ep::adapter_grad_workspace_bytes(rows, num_adapters, rank, in_length, out_length, act, with_w != 0, with_order != 0,
                                              (results & EP_ADAPTER_DX) != 0, (results & EP_ADAPTER_DA) != 0,
                                              (results & EP_ADAPTER_DB) != 0);
    return EP_OK;
}

extern "C" ep_status ep_adapter_product_grad(const void *x_dev, int64_t rows, const int32_t *order, const int32_t *offsets,
                                             int32_t num_adapters, int32_t rank, const void *a_dev, const void *b_dev,
                                             const float *scale, const void *w_dev, int32_t in_length, int32_t out_length,
                                             const void *low_dev, ep_activation act, const void *pre_dev,
                                             const void *d_y_dev, void *dx_dev, void *da_dev, void *db_dev, void *workspace,
                                             size_t workspace_bytes, hipStream_t stream) {
    const char *who = "ep_adapter_product_grad";
    const ep_status st = check_sizes(who, rows, num_adapters, rank, in_length, out_length, act);
    if (st != EP_OK)
        return st;
    if (rows > 0 && !dx_dev && !da_dev && !db_dev)
        return fail(EP_ERR_INVALID_ARG, "%s: no output", who);
    if (!offsets && num_adapters != 1)
        return fail(EP_ERR_INVALID_ARG, "%s: more than one adapter needs offsets", who);
    if (rows > 0 && (!d_y_dev || (act != EP_ACT_NONE && !pre_dev) || (dx_dev && !a_dev) || ((dx_dev || da_dev) && !b_dev) ||
                     (da_dev && !x_dev) || (db_dev && !low_dev)))
        return fail(EP_ERR_INVALID_ARG, "%s: d_y, pre (with an activation), a (for dx), b (for dx and da), x (for da) and low "
                                        "(for db) are required", who);
    if (!aligned16(x_dev) || !aligned16(a_dev) || !aligned16(b_dev) || !aligned16(w_dev) || !aligned16(low_dev) ||
        !aligned16(pre_dev) || !aligned16(d_y_dev) || !aligned16(dx_dev) || !aligned16(da_dev) || !aligned16(db_dev) ||
        !aligned4(order) || !aligned4(offsets) || !aligned4(scale))
        return fail(EP_ERR_INVALID_ARG, "%s: an array is not 16-byte aligned (order, offsets, scale: 4)", who);
    const size_t need = ep::adapter_grad_workspace_bytes(rows, num_adapters, rank, in_length, out_length, act,
                                                         w_dev != nullptr, order != nullptr, dx_dev != nullptr, da_dev != nullptr,
                                                         db_dev != nullptr);
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need))
        return fail(EP_ERR_INVALID_ARG, "%s: workspace of %zu bytes, need %zu, 16-byte aligned", who,
                    workspace ? workspace_bytes : (size_t)0, need);
    ep::AdapterGradArgs a{};
    a.x = x_dev;
    a.rows = rows;
    a.order = order;
    a.offsets = offsets;
    a.A = num_adapters;
    a.R = rank;
    a.K = in_length;
    a.N = out_length;
    a.a = a_dev;
    a.b = b_dev;
    a.low = low_dev;
    a.scale = scale;
    a.w = w_dev;
    a.act = act;
    a.pre = pre_dev;
    a.d_y = d_y_dev;
    a.dx = dx_dev;
    a.da = da_dev;
    a.db = db_dev;
    a.workspace = workspace;
    EP_HIP(ep::launch_adapter_grad(a, stream));
    return EP_OK;
}
