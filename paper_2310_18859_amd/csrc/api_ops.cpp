// Host side of the C ABI: the operators that need no context (experts in 4 bits, the router, plain bf16 experts).
#include <hip/hip_runtime_api.h>

#include <climits>

#include "expert_rule.h"
#include "kernels.h"
#include "sida_moe.h"

using namespace sida;

namespace {

bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t up(size_t v, size_t n) { return (v + n - 1) / n * n; }

constexpr int64_t kMostWorkgroups = (1 << 24) - 1;        // of 256 threads: a launch has fewer than 2^32
constexpr int64_t kMostPitch = 1 << 24;                   // values between two rows: 32-bit byte offsets within a tile of rows

bool mx_cols_ok(int32_t cols) { return cols >= 32 && cols <= SIDA_MX_MAX_COLS && cols % 32 == 0; }
bool mx_matrix_ok(int64_t rows, int32_t cols, int32_t layout)
{
    return rows >= 0 && mx_cols_ok(cols) && (layout == SIDA_MX_ROWS || layout == SIDA_MX_TILES) && rows <= (int64_t)1 << 40;
}
int status(int hip) { return hip == 0 ? SIDA_OK : SIDA_EHIP; }

bool route_cfg_ok(const sida_route_config *c)
{
    return c && c->E >= 1 && c->E <= SIDA_MAX_E && c->top_k >= 1 && c->top_k <= SIDA_MAX_TOP_K && c->top_k <= c->E &&
           (c->logits_type == SIDA_BF16 || c->logits_type == SIDA_FP32);
}
bool route_rows_ok(const sida_route_config *c, int32_t T, int64_t ld)
{
    return T >= 0 && T <= 1 << 26 && ld >= c->E && ld < kMostPitch;
}
RouteShape route_shape(const sida_route_config *c) { return RouteShape{c->E, c->top_k, c->logits_type == SIDA_FP32, c->normalize != 0}; }

bool pairs_ok(int32_t E, int32_t top_k, int32_t T)
{
    return E >= 1 && E <= SIDA_MAX_E && top_k >= 1 && top_k <= SIDA_MAX_TOP_K && T >= 0 &&
           (int64_t)T * top_k < 1 << 26;                      // 64 lanes each: a launch has fewer than 2^32
}
bool rows_cfg_ok(const sida_expert_rows_config *c)
{
    return c && pairs_ok(1, c->top_k, c->T) && c->M >= 0 && c->d >= 1 && c->d <= 65536 && (c->type == SIDA_BF16 || c->type == SIDA_FP32);
}
bool row_ok(const sida_expert_rows_config *c, const void *p, int64_t ld) { return p && aligned(p, c->type == SIDA_FP32 ? 4 : 2) && ld >= c->d && ld < kMostPitch; }
ExpertRowsShape rows_shape(const sida_expert_rows_config *c) { return ExpertRowsShape{c->T, c->top_k, c->M, c->d, c->type == SIDA_FP32}; }

bool expert_cfg_ok(const sida_expert_gemm_config *c, int32_t M)
{
    return c && c->groups >= 1 && c->groups <= SIDA_MAX_E && c->N >= 8 && c->N <= 65536 && c->N % 8 == 0 && c->K >= 8 && c->K <= 65536 &&
           c->K % 8 == 0 && (int64_t)c->N * c->K <= 1 << 30 &&
           (int64_t)c->groups * c->N * c->K <= (int64_t)1 << 36 && (c->out_type == SIDA_BF16 || c->out_type == SIDA_FP32) &&
           c->activation >= SIDA_ACT_NONE && c->activation <= SIDA_ACT_SILU && M >= 0 && M <= 1 << 24 &&
           (int64_t)M * c->N <= (int64_t)1 << 35 && (int64_t)M * c->K <= (int64_t)1 << 35;
}
bool matrix_ok(const void *p, int64_t ld, int32_t cols, int32_t type)
{
    return p && aligned(p, 16) && ld >= cols && ld < kMostPitch && ld * (type == SIDA_FP32 ? 4 : 2) <= kMostExpertPitch &&
           ld % (type == SIDA_FP32 ? 4 : 8) == 0;
}
ExpertGemmShape expert_shape(const sida_expert_gemm_config *c)
{
    return ExpertGemmShape{c->groups, c->N, c->K, c->out_type == SIDA_FP32, c->activation};
}

}  // namespace

extern "C" {

size_t sida_mx_codes_bytes(int64_t rows, int32_t cols, int32_t layout)
{
    if (!mx_matrix_ok(rows, cols, layout)) return 0;
    return layout == SIDA_MX_ROWS ? (size_t)rows * (cols / 2) : up(rows, 32) * (up(cols, 64) / 2);
}

size_t sida_mx_scales_bytes(int64_t rows, int32_t cols, int32_t layout)
{
    if (!mx_matrix_ok(rows, cols, layout)) return 0;
    return (layout == SIDA_MX_ROWS ? (size_t)rows : up(rows, 32)) * (up(cols, 256) / 32);
}

int sida_mx_quantize(const void *x_dev, int32_t x_type, int64_t rows, int32_t cols, int64_t ld, int32_t layout, void *codes_dev,
                     void *scales_dev, void *values_dev, void *stream)
{
    if (!mx_matrix_ok(rows, cols, layout) || (x_type != SIDA_BF16 && x_type != SIDA_FP32) || ld < cols || ld > (int64_t)1 << 40) return SIDA_EINVAL;
    if (rows == 0) return SIDA_OK;
    if (!x_dev || !codes_dev || !scales_dev) return SIDA_EINVAL;
    if (!aligned(x_dev, x_type == SIDA_FP32 ? 4 : 2) || !aligned(codes_dev, 16) || !aligned(scales_dev, layout == SIDA_MX_TILES ? 16 : 8) ||
        !aligned(values_dev, 16))
        return SIDA_EINVAL;
    if ((rows + 31) / 32 * ((cols + 255) / 256) > kMostWorkgroups) return SIDA_EINVAL;
    return status(launch_mx_quantize(x_dev, x_type == SIDA_FP32, rows, cols, ld, layout == SIDA_MX_TILES, codes_dev, scales_dev, values_dev,
                                     static_cast<hipStream_t>(stream)));
}

int sida_mx_gemm(const sida_mx_gemm_config *c, const void *x_dev, const void *x_scales_dev, int64_t ldx, int32_t M, const void *codes_dev,
                 const void *scales_dev, const int32_t *offsets_dev, void *y_dev, int64_t ldy, void *stream)
{
    if (!c || c->groups < 1 || c->groups > SIDA_MAX_E || c->N < 1 || c->N > 65536 || !mx_cols_ok(c->K) ||
        (c->x_type != SIDA_BF16 && c->x_type != SIDA_MXFP4) || (c->y_type != SIDA_BF16 && c->y_type != SIDA_FP32))
        return SIDA_EINVAL;
    const bool x4 = c->x_type == SIDA_MXFP4, y32 = c->y_type == SIDA_FP32;
    if (M < 0 || M > 1 << 24 || ldx < c->K || ldx >= kMostPitch || ldy < c->N || ldy >= kMostPitch) return SIDA_EINVAL;
    if (x4 ? ldx != c->K : ldx % 8 != 0) return SIDA_EINVAL;
    if ((int64_t)M * c->N > (int64_t)1 << 35) return SIDA_EINVAL;      // tiles of 32 x 128 at least: a launch's workgroups
    if (M == 0) return SIDA_OK;
    if (!x_dev || !codes_dev || !scales_dev || !y_dev || (x4 && !x_scales_dev) || (!offsets_dev && c->groups != 1)) return SIDA_EINVAL;
    if (!aligned(x_dev, 16) || !aligned(codes_dev, 16) || !aligned(scales_dev, 4) || !aligned(y_dev, y32 ? 4 : 2) || !aligned(offsets_dev, 4) ||
        (x4 && !aligned(x_scales_dev, 8)))
        return SIDA_EINVAL;
    const MxShape sh{c->groups, c->N, c->K, x4, y32, c->relu != 0};
    return status(launch_mx_gemm(sh, x_dev, x_scales_dev, ldx, M, codes_dev, scales_dev, offsets_dev, y_dev, ldy, static_cast<hipStream_t>(stream)));
}

size_t sida_route_workspace_bytes(const sida_route_config *c, int32_t T)
{
    if (!route_cfg_ok(c) || !route_rows_ok(c, T, c->E)) return 0;
    return up(kRouteTailBytes + (size_t)route_workgroups(T) * up(c->E, 4) * 8, 256);
}

int sida_route(const sida_route_config *c, const void *logits_dev, int64_t ld, int32_t T, const uint8_t *mask_dev, int32_t *ids_dev,
               float *gates_dev, int32_t *counts_dev, float *loss_dev, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    if (!route_cfg_ok(c) || !route_rows_ok(c, T, ld)) return SIDA_EINVAL;
    if (!counts_dev || !loss_dev || !workspace_dev || (T > 0 && (!logits_dev || !ids_dev || !gates_dev))) return SIDA_EINVAL;
    if (!aligned(logits_dev, c->logits_type == SIDA_FP32 ? 4 : 2) || !aligned(ids_dev, 4) || !aligned(gates_dev, 4) || !aligned(counts_dev, 4) ||
        !aligned(loss_dev, 4) || !aligned(workspace_dev, 16))
        return SIDA_EINVAL;
    if (workspace_bytes < sida_route_workspace_bytes(c, T)) return SIDA_ENOSPC;
    return status(launch_route(route_shape(c), logits_dev, ld, T, mask_dev, ids_dev, gates_dev, counts_dev, loss_dev, workspace_dev,
                               static_cast<hipStream_t>(stream)));
}

int sida_route_backward(const sida_route_config *c, const void *logits_dev, int64_t ld, int32_t T, const uint8_t *mask_dev,
                        const int32_t *ids_dev, const int32_t *counts_dev, const float *d_gates_dev, const float *d_loss_dev,
                        void *d_logits_dev, int64_t ld_d, void *stream)
{
    if (!route_cfg_ok(c) || !route_rows_ok(c, T, ld) || !route_rows_ok(c, T, ld_d)) return SIDA_EINVAL;
    if (T == 0) return SIDA_OK;
    if (!logits_dev || !counts_dev || !d_logits_dev || (d_gates_dev && !ids_dev)) return SIDA_EINVAL;
    const uintptr_t size = c->logits_type == SIDA_FP32 ? 4 : 2;
    if (!aligned(logits_dev, size) || !aligned(d_logits_dev, size) || !aligned(ids_dev, 4) || !aligned(counts_dev, 4) ||
        !aligned(d_gates_dev, 4) || !aligned(d_loss_dev, 4))
        return SIDA_EINVAL;
    if (logits_dev == d_logits_dev && ld != ld_d) return SIDA_EINVAL;     // a row would be written where another is still to be read
    return status(launch_route_backward(route_shape(c), logits_dev, ld, T, mask_dev, ids_dev, counts_dev, d_gates_dev, d_loss_dev, d_logits_dev,
                                        ld_d, static_cast<hipStream_t>(stream)));
}

size_t sida_expert_sort_workspace_bytes(int32_t E, int32_t top_k, int32_t T)
{
    if (!pairs_ok(E, top_k, T)) return 0;
    return up((size_t)expert_sort_most((int64_t)T * top_k) * E * 4, 256);
}

int sida_expert_sort(int32_t E, int32_t top_k, const int32_t *ids_dev, const float *gates_dev, int32_t T, int32_t *offsets_dev,
                     int32_t *places_dev, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    if (!pairs_ok(E, top_k, T)) return SIDA_EINVAL;
    if (!offsets_dev || !workspace_dev || (T > 0 && (!ids_dev || !places_dev))) return SIDA_EINVAL;
    if (!aligned(ids_dev, 4) || !aligned(gates_dev, 4) || !aligned(offsets_dev, 4) || !aligned(places_dev, 4) || !aligned(workspace_dev, 4)) return SIDA_EINVAL;
    if (workspace_bytes < sida_expert_sort_workspace_bytes(E, top_k, T)) return SIDA_ENOSPC;
    return status(launch_expert_sort(ids_dev, gates_dev, (int64_t)T * top_k, E, offsets_dev, places_dev, workspace_dev, static_cast<hipStream_t>(stream)));
}

int sida_expert_rows(const sida_expert_rows_config *c, const void *x_dev, int64_t ld_x, const int32_t *places_dev, void *rows_dev, int64_t ld_rows, void *stream)
{
    if (!rows_cfg_ok(c)) return SIDA_EINVAL;
    if (c->T == 0 || c->M == 0) return SIDA_OK;
    if (!row_ok(c, x_dev, ld_x) || !row_ok(c, rows_dev, ld_rows) || !places_dev || !aligned(places_dev, 4)) return SIDA_EINVAL;
    return status(launch_expert_rows(rows_shape(c), x_dev, ld_x, places_dev, rows_dev, ld_rows, static_cast<hipStream_t>(stream)));
}

int sida_expert_sum(const sida_expert_rows_config *c, const void *rows_dev, int64_t ld_rows, const int32_t *places_dev, const float *gates_dev,
                    const void *residual_dev, int64_t ld_res, void *y_dev, int64_t ld_y, void *stream)
{
    if (!rows_cfg_ok(c)) return SIDA_EINVAL;
    if (c->T == 0) return SIDA_OK;
    if ((c->M > 0 && !row_ok(c, rows_dev, ld_rows)) || !row_ok(c, y_dev, ld_y) || (residual_dev && !row_ok(c, residual_dev, ld_res)) || !places_dev ||
        !aligned(places_dev, 4) || !aligned(gates_dev, 4))
        return SIDA_EINVAL;
    if (residual_dev == y_dev && ld_res != ld_y) return SIDA_EINVAL;       // a row would be written where another is still to be read
    return status(launch_expert_sum(rows_shape(c), rows_dev, ld_rows, places_dev, gates_dev, residual_dev, ld_res, y_dev, ld_y,
                                    static_cast<hipStream_t>(stream)));
}

int sida_expert_sum_backward(const sida_expert_rows_config *c, const void *dy_dev, int64_t ld_dy, const void *rows_dev, int64_t ld_rows,
                             const int32_t *places_dev, const float *gates_dev, void *d_rows_dev, int64_t ld_d, float *d_gates_dev, void *stream)
{
    if (!rows_cfg_ok(c)) return SIDA_EINVAL;
    if (c->T == 0) return SIDA_OK;
    if (!row_ok(c, dy_dev, ld_dy) || !places_dev || !aligned(places_dev, 4) || !aligned(gates_dev, 4) || !aligned(d_gates_dev, 4)) return SIDA_EINVAL;
    if (c->M > 0 && (!row_ok(c, d_rows_dev, ld_d) || (d_gates_dev && !row_ok(c, rows_dev, ld_rows)))) return SIDA_EINVAL;
    if (d_gates_dev && rows_dev == d_rows_dev && ld_rows != ld_d) return SIDA_EINVAL;
    return status(launch_expert_sum_backward(rows_shape(c), dy_dev, ld_dy, rows_dev, ld_rows, places_dev, gates_dev, d_rows_dev, ld_d, d_gates_dev,
                                             static_cast<hipStream_t>(stream)));
}

int sida_expert_gemm(const sida_expert_gemm_config *c, const void *x_dev, int64_t ldx, int32_t M, const void *w_dev, const int32_t *offsets_dev,
                     const float *bias_dev, void *pre_dev, int64_t ld_pre, const void *residual_dev, int64_t ld_res, void *y_dev, int64_t ldy, void *stream)
{
    if (!expert_cfg_ok(c, M)) return SIDA_EINVAL;
    if (M == 0) return SIDA_OK;
    if (!matrix_ok(x_dev, ldx, c->K, SIDA_BF16) || !w_dev || !aligned(w_dev, 16) || !matrix_ok(y_dev, ldy, c->N, c->out_type) || !aligned(bias_dev, 16) ||
        !aligned(offsets_dev, 4) || (!offsets_dev && c->groups != 1))
        return SIDA_EINVAL;
    if ((pre_dev && !matrix_ok(pre_dev, ld_pre, c->N, SIDA_BF16)) || (residual_dev && !matrix_ok(residual_dev, ld_res, c->N, c->out_type))) return SIDA_EINVAL;
    if (residual_dev == y_dev && ld_res != ldy) return SIDA_EINVAL;
    return status(launch_expert_gemm(expert_shape(c), x_dev, ldx, M, w_dev, offsets_dev, bias_dev, pre_dev, ld_pre, residual_dev, ld_res, y_dev, ldy,
                                     static_cast<hipStream_t>(stream)));
}

int sida_expert_gemm_input(const sida_expert_gemm_config *c, const void *dy_dev, int64_t ld_dy, int32_t M, const void *w_dev, const int32_t *offsets_dev,
                           const void *pre_dev, int64_t ld_pre, void *dx_dev, int64_t ld_dx, void *stream)
{
    if (!expert_cfg_ok(c, M)) return SIDA_EINVAL;
    if (M == 0) return SIDA_OK;
    if (!matrix_ok(dy_dev, ld_dy, c->N, SIDA_BF16) || !w_dev || !aligned(w_dev, 16) || !matrix_ok(dx_dev, ld_dx, c->K, c->out_type) ||
        !aligned(offsets_dev, 4) || (!offsets_dev && c->groups != 1))
        return SIDA_EINVAL;
    if (pre_dev ? !matrix_ok(pre_dev, ld_pre, c->K, SIDA_BF16) : c->activation != SIDA_ACT_NONE) return SIDA_EINVAL;
    if (pre_dev == dx_dev && (ld_pre != ld_dx || c->out_type != SIDA_BF16)) return SIDA_EINVAL;
    return status(launch_expert_gemm_input(expert_shape(c), dy_dev, ld_dy, M, w_dev, offsets_dev, pre_dev, ld_pre, dx_dev, ld_dx,
                                           static_cast<hipStream_t>(stream)));
}

size_t sida_expert_gemm_weights_workspace_bytes(const sida_expert_gemm_config *c, int32_t M)
{
    if (!expert_cfg_ok(c, M)) return 0;
    if (!expert_weights_chunk(M, c->groups, c->N, c->K)) return 0;
    return up((size_t)(expert_weights_most(c->groups, c->N, c->K) + c->groups) * c->N * (c->K + 1) * 4, 256);
}

int sida_expert_gemm_weights(const sida_expert_gemm_config *c, const void *dy_dev, int64_t ld_dy, const void *x_dev, int64_t ldx, int32_t M,
                             const int32_t *offsets_dev, void *dw_dev, float *d_bias_dev, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    if (!expert_cfg_ok(c, M) || c->activation != SIDA_ACT_NONE) return SIDA_EINVAL;
    if (M > 0 && (!matrix_ok(dy_dev, ld_dy, c->N, SIDA_BF16) || !matrix_ok(x_dev, ldx, c->K, SIDA_BF16))) return SIDA_EINVAL;
    if (!dw_dev || !aligned(dw_dev, 16) || !aligned(d_bias_dev, 16) || !aligned(offsets_dev, 4) || (!offsets_dev && c->groups != 1) || !aligned(workspace_dev, 16))
        return SIDA_EINVAL;
    const size_t need = sida_expert_gemm_weights_workspace_bytes(c, M);
    if (need && !workspace_dev) return SIDA_EINVAL;
    if (workspace_bytes < need) return SIDA_ENOSPC;
    return status(launch_expert_gemm_weights(expert_shape(c), dy_dev, ld_dy, x_dev, ldx, M, offsets_dev, dw_dev, d_bias_dev, workspace_dev,
                                             static_cast<hipStream_t>(stream)));
}

}  // extern "C"
