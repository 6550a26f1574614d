// Host side of the layer norm, of the 8-bit checkpoints of activations and of the weight gradients from them: part of slope_lib.cu,
// whose argument checks, plans and launches it uses.
#pragma once
#include "norm_kernels.cuh"

namespace slope {
static bool plain_type(int t) { return t == SLOPE_BF16 || t == SLOPE_F32; }
static bool checkpoint_dims_ok(int rows, int cols) { return rows > 0 && cols > 0 && cols % kQBlock == 0; }

// How the rows of a layer norm are laid over warps: `chunks` times eight columns per lane.
struct NormPlan {
    int row_warps, chunks, groups, blocks;
    int threads() const { return 32 * row_warps * groups; }
};
static NormPlan norm_fwd_plan(int b, int d) {
    const int units = (d + 255) / 256;                        // warps that a row fills with one chunk per lane
    NormPlan p;
    p.row_warps = (units + 3) / 4;
    p.chunks = (units + p.row_warps - 1) / p.row_warps;
    p.groups = std::max(1, 8 / p.row_warps);
    p.blocks = (b + p.groups - 1) / p.groups;
    return p;
}
// (the caller's workspace follows from the blocks and is asked for with no device at hand: the SM count is the B200's)
static NormPlan norm_bwd_plan(int b, int d) {
    constexpr int kSms = 148;
    const int units = (d + 255) / 256;
    NormPlan p;
    p.chunks = units > 16 ? 2 : 1;
    p.row_warps = (units + p.chunks - 1) / p.chunks;
    p.groups = std::max(1, std::min(kNormMaxGroups, 16 / p.row_warps));
    const int resident = p.row_warps > 16 ? 1 : 2;
    p.blocks = std::min((b + p.groups - 1) / p.groups, resident * kSms);
    return p;
}

template <typename... KArgs, typename... Args>
static slope_status_t launch_rows(void (*kern)(KArgs...), int blocks, int threads, int smem_bytes, cudaStream_t stream, Args&&... args) {
    return launch_cluster_ex(kern, blocks, 1, threads, smem_bytes, /*overlap_prologue=*/true, stream, std::forward<Args>(args)...);
}
template <int TYPE>
static slope_status_t launch_norm_fwd(const NormPlan& plan, const NormFwdParams& p, cudaStream_t stream) {
    auto kern = plan.chunks == 1   ? layer_norm_fwd_kernel<TYPE, 1>
                : plan.chunks == 2 ? layer_norm_fwd_kernel<TYPE, 2>
                : plan.chunks == 3 ? layer_norm_fwd_kernel<TYPE, 3>
                                   : layer_norm_fwd_kernel<TYPE, 4>;
    return launch_rows(kern, plan.blocks, plan.threads(), 0, stream, p);
}
template <int TYPE, int DX_TYPE>
static slope_status_t launch_norm_bwd(const NormPlan& plan, const NormBwdParams& p, cudaStream_t stream) {
    auto kern = plan.row_warps > 16 ? layer_norm_bwd_kernel<TYPE, DX_TYPE, 2, 1024>
                : plan.chunks == 2  ? layer_norm_bwd_kernel<TYPE, DX_TYPE, 2, 512>
                                    : layer_norm_bwd_kernel<TYPE, DX_TYPE, 1, 512>;
    return launch_rows(kern, plan.blocks, plan.threads(), plan.groups > 1 ? 8 * p.d : 0, stream, p);
}

}  // namespace slope

extern "C" {

size_t slope_checkpoint_bytes(int rows, int cols) {
    if (!checkpoint_dims_ok(rows, cols)) return 0;
    return static_cast<size_t>(rows) * cols + static_cast<size_t>(rows) * cols / kQBlock;
}

slope_status_t slope_checkpoint_store(const void* X, int x_type, int rows, int cols, void* checkpoint, void* stream) {
    if (!X || !checkpoint || !plain_type(x_type)) return SLOPE_ERR_INVALID_ARG;
    if (!checkpoint_dims_ok(rows, cols)) return SLOPE_ERR_SHAPE;
    if (!aligned16(X) || !aligned16(checkpoint)) return SLOPE_ERR_ALIGNMENT;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    const size_t n8 = static_cast<size_t>(rows) * cols / 8;
    return launch_stream(x_type == SLOPE_F32 ? checkpoint_store_kernel<kTypeF32> : checkpoint_store_kernel<kTypeBf16>,
                         dim3(stream_grid(n8, info)), static_cast<cudaStream_t>(stream), X, n8, checkpoint);
}

slope_status_t slope_checkpoint_load(const void* checkpoint, int rows, int cols, void* X, int x_type, void* stream) {
    if (!X || !checkpoint || !plain_type(x_type)) return SLOPE_ERR_INVALID_ARG;
    if (!checkpoint_dims_ok(rows, cols)) return SLOPE_ERR_SHAPE;
    if (!aligned16(X) || !aligned16(checkpoint)) return SLOPE_ERR_ALIGNMENT;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    const size_t n8 = static_cast<size_t>(rows) * cols / 8;
    return launch_stream(x_type == SLOPE_F32 ? checkpoint_load_kernel<kTypeF32> : checkpoint_load_kernel<kTypeBf16>,
                         dim3(stream_grid(n8, info)), static_cast<cudaStream_t>(stream), checkpoint, n8, X);
}

slope_status_t slope_layer_norm_fwd(const void* X, int x_type, const void* residual, const void* gamma, const void* beta, int p_type,
                                    int b, int d, float eps, void* H, void* Y, void* mean, void* rstd, void* H_ckpt, void* Y_ckpt,
                                    void* stream_) {
    if (!X || !Y || !plain_type(x_type) || !plain_type(p_type) || !(eps >= 0.0f)) return SLOPE_ERR_INVALID_ARG;
    if ((H && !residual) || !mean != !rstd) return SLOPE_ERR_INVALID_ARG;
    if (b < 1 || d < 1 || d % 8 != 0 || d > kNormMaxWidth) return SLOPE_ERR_SHAPE;
    if ((H_ckpt || Y_ckpt) && !checkpoint_dims_ok(b, d)) return SLOPE_ERR_SHAPE;
    for (const void* p : {X, residual, gamma, beta, static_cast<const void*>(H), static_cast<const void*>(Y), static_cast<const void*>(mean),
                          static_cast<const void*>(rstd), static_cast<const void*>(H_ckpt), static_cast<const void*>(Y_ckpt)})
        if (!aligned16(p)) return SLOPE_ERR_ALIGNMENT;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    const NormPlan plan = norm_fwd_plan(b, d);
    const NormFwdParams p{X, residual, gamma, beta, H, Y, H_ckpt, Y_ckpt, static_cast<float*>(mean), static_cast<float*>(rstd),
                          b, d, plan.row_warps, p_type == SLOPE_F32, eps};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return x_type == SLOPE_F32 ? launch_norm_fwd<kTypeF32>(plan, p, stream) : launch_norm_fwd<kTypeBf16>(plan, p, stream);
}

size_t slope_layer_norm_bwd_workspace_bytes(int b, int d) {
    if (b < 1 || d < 1 || d > kNormMaxWidth) return 0;
    const int blocks = norm_bwd_plan(b, d).blocks;
    return blocks > 1 ? static_cast<size_t>(blocks) * 2 * d * sizeof(float) : 0;
}

slope_status_t slope_layer_norm_bwd(const void* dY, const void* H, int h_type, const void* mean, const void* rstd, const void* gamma,
                                    int p_type, const void* dH, int b, int d, void* dX, int dx_type, void* dgamma, void* dbeta,
                                    void* workspace, size_t workspace_bytes, void* stream_) {
    if (!dY || !H || !mean || !rstd || !dX || !plain_type(dx_type) || !plain_type(p_type)) return SLOPE_ERR_INVALID_ARG;
    if (!plain_type(h_type) && h_type != SLOPE_Q8) return SLOPE_ERR_INVALID_ARG;
    if (b < 1 || d < 1 || d % 8 != 0 || d > kNormMaxWidth || (h_type == SLOPE_Q8 && !checkpoint_dims_ok(b, d))) return SLOPE_ERR_SHAPE;
    for (const void* p : {dY, H, mean, rstd, gamma, dH, static_cast<const void*>(dX), static_cast<const void*>(dgamma),
                          static_cast<const void*>(dbeta), static_cast<const void*>(workspace)})
        if (!aligned16(p)) return SLOPE_ERR_ALIGNMENT;
    const size_t need = slope_layer_norm_bwd_workspace_bytes(b, d);
    const bool params = dgamma || dbeta;
    if (params && need && (!workspace || workspace_bytes < need)) return SLOPE_ERR_INVALID_ARG;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    const NormPlan plan = norm_bwd_plan(b, d);
    const NormBwdParams p{dY, H, gamma, dH, static_cast<const float*>(mean), static_cast<const float*>(rstd), dX, dgamma, dbeta,
                          static_cast<float*>(workspace), b, d, plan.row_warps, p_type == SLOPE_F32};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const bool wide = dx_type == SLOPE_F32;
    slope_status_t st;
    if (h_type == SLOPE_BF16) st = wide ? launch_norm_bwd<kTypeBf16, kTypeF32>(plan, p, stream) : launch_norm_bwd<kTypeBf16, kTypeBf16>(plan, p, stream);
    else if (h_type == SLOPE_F32) st = wide ? launch_norm_bwd<kTypeF32, kTypeF32>(plan, p, stream) : launch_norm_bwd<kTypeF32, kTypeBf16>(plan, p, stream);
    else st = wide ? launch_norm_bwd<kTypeQ8, kTypeF32>(plan, p, stream) : launch_norm_bwd<kTypeQ8, kTypeBf16>(plan, p, stream);
    if (st != SLOPE_OK || !params || plan.blocks == 1) return st;
    return launch_rows(layer_norm_params_kernel, (2 * d + 127) / 128, 256, 0, stream, p.partial, plan.blocks, d, dgamma, dbeta, p.p_f32);
}

// ------------------------------------------------------------------ weight gradients from a checkpoint
size_t slope_bwd_dw_q8_workspace_bytes(int b, int d_out, int d_in, int r) {
    if (b <= 0 || d_out <= 0 || d_in <= 0 || r < 0) return 0;
    return align256(static_cast<size_t>(b) * d_in * 2) + slope_bwd_dw_adapter_workspace_bytes(b, d_out, d_in, r);
}

slope_status_t slope_linear_bwd_dw_masked_q8(const void* dY, const void* X_ckpt, int b, int d_out, int d_in, const void* mask1_bits,
                                             void* dWc_vals, void* workspace, size_t workspace_bytes, void* stream) {
    if (!dY || !X_ckpt || !mask1_bits || !dWc_vals || !workspace) return SLOPE_ERR_INVALID_ARG;
    if (!dims_ok(d_out, d_in) || b < 1) return SLOPE_ERR_SHAPE;
    if (!aligned16(dY) || !aligned16(X_ckpt) || !aligned16(mask1_bits) || !aligned16(dWc_vals) || !aligned16(workspace)) return SLOPE_ERR_ALIGNMENT;
    if (workspace_bytes < slope_bwd_dw_q8_workspace_bytes(b, d_out, d_in, 0)) return SLOPE_ERR_INVALID_ARG;
    if (slope_status_t st = slope_checkpoint_load(X_ckpt, b, d_in, workspace, SLOPE_BF16, stream)) return st;
    return slope_linear_bwd_dw_masked(dY, workspace, b, d_out, d_in, mask1_bits, dWc_vals, stream);
}

slope_status_t slope_linear_bwd_dw_adapter_q8(const void* dY, const void* X_ckpt, const void* T, const void* dT, int b, int d_out, int d_in,
                                              int r, const void* mask1_bits, void* dWc_vals, void* dL, void* dR, void* workspace,
                                              size_t workspace_bytes, void* stream) {
    if (!dY || !X_ckpt || !T || !dT || !mask1_bits || !dWc_vals || !dL || !dR || !workspace) return SLOPE_ERR_INVALID_ARG;
    if (!dims_ok(d_out, d_in) || b < 1 || !rank_ok(r) || r == 0) return SLOPE_ERR_SHAPE;
    if (!aligned16(dY) || !aligned16(X_ckpt) || !aligned16(T) || !aligned16(dT) || !aligned16(mask1_bits) || !aligned16(dWc_vals) ||
        !aligned16(dL) || !aligned16(dR) || !aligned16(workspace))
        return SLOPE_ERR_ALIGNMENT;
    if (workspace_bytes < slope_bwd_dw_q8_workspace_bytes(b, d_out, d_in, r)) return SLOPE_ERR_INVALID_ARG;
    if (slope_status_t st = slope_checkpoint_load(X_ckpt, b, d_in, workspace, SLOPE_BF16, stream)) return st;
    const size_t x_bytes = align256(static_cast<size_t>(b) * d_in * 2);
    return slope_linear_bwd_dw_adapter(dY, workspace, T, dT, b, d_out, d_in, r, mask1_bits, dWc_vals, dL, dR,
                                       static_cast<uint8_t*>(workspace) + x_bytes, workspace_bytes - x_bytes, stream);
}

slope_status_t slope_dense_linear_bwd_dw_q8(const void* dY, const void* X_ckpt, int b, int d_out, int d_in, void* dW, void* workspace,
                                            size_t workspace_bytes, void* stream) {
    if (!workspace) return SLOPE_ERR_INVALID_ARG;
    if (slope_status_t st = dense_args(dY, X_ckpt, dW, b, d_out, d_in)) return st;
    if (!aligned16(workspace)) return SLOPE_ERR_ALIGNMENT;
    if (workspace_bytes < slope_bwd_dw_q8_workspace_bytes(b, d_out, d_in, 0)) return SLOPE_ERR_INVALID_ARG;
    if (slope_status_t st = slope_checkpoint_load(X_ckpt, b, d_in, workspace, SLOPE_BF16, stream)) return st;
    return slope_dense_linear_bwd_dw(dY, workspace, b, d_out, d_in, dW, stream);
}

}  // extern "C"
