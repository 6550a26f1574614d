// Host side of the layer norm, of the 8-bit checkpoints of activations and of the weight gradients from them: part of slope_lib.cu,
// whose argument checks, plans and launches it uses.
#pragma once
#include "norm_kernels.cuh"

namespace slope {
static bool plain_type(int t) { return t == SLOPE_BF16 || t == SLOPE_F32; }
static bool checkpoint_dims_ok(int rows, int cols) { return rows > 0 && cols > 0 && cols % kQBlock == 0; }

// How the rows of a layer norm are laid over a block: `chunks` times eight columns per lane, `row_warps` warps per row, `groups` rows at a time.
struct NormPlan {
    int row_warps, chunks, groups, batch, blocks, shared_bytes;
    int threads() const { return 32 * row_warps * groups; }
};
// Four chunks and few warps per row as far as that goes: what a row costs beside its columns (two sums over its warps, its place in the
// ring) is shared by more of them.  us, two / three / four chunks: backward 8192 x 5120 from 8 bits 98 / 82 / 76, 16384 x 4096 94 / 123 /
// 94, forward 8192 x 5120 48 / 42 / 37.
// `most`, `warps`, `per_sm`: chunks of a lane, warps of a block and blocks of an SM.
static NormPlan norm_plan(int b, int d, int most, int warps, int per_sm, int sms) {
    const int units = (d + 255) / 256;                        // warps that a row fills with one chunk per lane
    NormPlan p{(units + most - 1) / most, 0, 0, 1, 0, 0};
    p.chunks = (units + p.row_warps - 1) / p.row_warps;
    p.groups = std::max(1, warps / p.row_warps);
    if (p.row_warps > 1) p.groups = std::min(p.groups, 15);   // (named barriers)
    // adjacent rows that travel together: up to 2 KB of bf16, as long as every group of the GPU gets two such batches.  us, where that is
    // one batch for the groups of two blocks per SM / so: 10000 x 512 11.5 / 9.8, 16384 x 256 10.3 / 9.7, 20000 x 128 10.1 / 8.7, 40000 x
    // 64 16.7 / 13.6, but 14000 x 128 6.5 / 7.3; 4 % less on average.
    while (p.batch < 8 && 8 * p.batch * d <= 4096 && 4ll * p.batch * p.groups * sms * per_sm <= b) p.batch *= 2;
    p.blocks = std::min((b - 1) / (p.groups * p.batch) + 1, sms * per_sm);
    p.shared_bytes = per_sm > 1 ? kNormSharedBytes / 2 - 2048 : kNormSharedBytes;
    return p;
}
// Two blocks of 12 warps, so that one of them works while the other begins or ends, or one of 16, whose ring has two stages where those of
// two blocks have one: for rows of which two do not fit in half the memory beside gamma and beta, and, with checkpoints, from 4096 on.  us,
// one block of 24 / two of 12: 8192 x 768 with both checkpoints 25.6 / 22.2, 2039 x 5120 14.7 / 13.1, 4096 x 8192 49 / 53; one of 16 / two
// of 12: 4096 x 8192 50 / 53, with a checkpoint of Y 16384 x 4096 140 / 144, 8192 x 5120 90.5 / 92.5, 4096 x 3584 34.9 / 34.2, 8192 x 768
// 18.8 / 16.8.  Up to 6144 one block of 24, which has four rows at a time and not two: 4096 x 6144 with a checkpoint 61 / 42; 4096 x 8192
// with residual and checkpoint 70 / 75.
// An fp32 stream with a residual and without checkpoints moves 12 bytes per value and has little else to do: two chunks a lane, so that
// fewer rows are under way at a time (two per SM at 4096), and rows that leave L2 like others.  us, as above / so: 8192 x 3584 63.8 / 57.8,
// 16384 x 4096 139 / 127 (98 % of a copy), 8192 x 5120 91.5 / 83, 8192 x 6144 110 / 103, 8192 x 8192 139.5 / 127, 8192 x 2304 41.6 / 39.4,
// but 16384 x 2048 70 / 72.6; bf16 16384 x 4096 90 / 92, 8192 x 5120 59 / 82.
static bool norm_fwd_heavy(int d, int x_type, bool residual, bool ckpt) {
    return x_type == SLOPE_F32 && residual && !ckpt && d > 2048 && d <= 8192;
}
// Wider than 8192: three chunks on up to 24 warps, two rows at a time up to 9216 (what a block's memory holds of an fp32 row with its
// residual, gamma and beta). 4096 rows, us, four chunks on 16 warps / so: 8448 bf16 55 / 31, with residual and checkpoint 104 / 75, in fp32
// 114 / 97; 11008 57 / 55, 113 / 107, 133 / 128; 13824 65 / 56.5, 130 / 116, 165 / 162; 16384 62 / 70, 142 / 143, 192 / 188.
static NormPlan norm_fwd_plan(int b, int d, bool heavy, bool ckpt, const DeviceInfo& info) {
    if (heavy) return norm_plan(b, d, 2, d <= 4096 ? 16 : kNormFwdWarps, 1, info.sm_count);
    if (d > 8192 && d <= 15 * 1024) return norm_plan(b, d, 3, kNormFwdWarps, 1, info.sm_count);
    const bool two = ckpt ? d < 4096 : d <= 5 * 1024;
    return norm_plan(b, d, 4, two ? kNormFwdWarps / 2 : d > 5120 && d <= 6144 ? kNormFwdWarps : 16, two ? 2 : 1, info.sm_count);
}
// One block of 16 warps per SM, or two of 8 where a row is one warp's: they begin and end apart.  Not for up to 16 rows, which one block
// takes without a second launch, nor for many rows of at most 512.  us, one / two: 256 x 512 6.3 / 5.5, 2048 x 512 7.3 / 7.6, 8192 x 512
// 13.4 / 14.9, 100 x 768 7.5 / 6.3, 2048 x 768 8.6 / 8.9, 16384 x 768 27.6 / 25.8, 32768 x 1024 55.3 / 54.8, 16 x 512 4.6 / 5.2.
// Three chunks where four would have no more rows at a time: us, four / three, 4096 rows from 8 bits: 5376 48 / 44.5, 6144 55 / 48, 8448 83
// / 70, 11008 90 / 86, 12288 104 / 91; bf16 8448 75 / 65, 11008 82 / 83; fp32 12288 184 / 160.
// (The caller's workspace follows from the blocks and is asked for with no device at hand: the SM count is the B200's.)
static NormPlan norm_bwd_plan(int b, int d) {
    const bool two = d <= 1024 && b > kNormBwdWarps && (d > 512 || b <= 1024);
    const int units = (d + 255) / 256, w3 = (units + 2) / 3, w4 = (units + 3) / 4;
    const int most = w3 <= kNormBwdWarps && kNormBwdWarps / w3 == kNormBwdWarps / w4 ? 3 : 4;
    return norm_plan(b, d, most, two ? kNormBwdWarps / 2 : kNormBwdWarps, two ? 2 : 1, 148);
}

// The ring of a launch, gamma and beta behind it.  `leave_first`: us, rows leave L2 first / like others: forward 16384 x 4096 90 / 95, in
// fp32 139 / 147; but with a checkpoint of Y (written and then read back) 140 / 136, in fp32 189 / 181.
static NormRing norm_ring(const NormPlan& plan, int b, int d, bool leave_first, const void* gamma, const void* beta, int params, int p_type,
                          const void* s0, int bytes0, const void* s1, int bytes1, const void* s2, int bytes2) {
    NormRing r{{static_cast<const uint8_t*>(s0), static_cast<const uint8_t*>(s1), static_cast<const uint8_t*>(s2)},
               {bytes0, s1 ? bytes1 : 0, s2 ? bytes2 : 0}, plan.batch, 0, plan.groups, plan.row_warps, b, d, leave_first, {gamma, beta},
               p_type == SLOPE_F32, params};
    r.stages = std::max(1, std::min(kNormMaxStages, (plan.shared_bytes - r.param_bytes()) / (r.groups * r.stage_bytes())));
    return r;
}
template <typename Params>
static slope_status_t launch_norm(void (*kern)(const Params), const NormPlan& plan, int least_bytes, cudaStream_t stream, const Params& p) {
    const int smem = std::max(p.ring.bytes() + p.ring.param_bytes(), least_bytes);
    if (!set_smem(kern, kNormSharedBytes)) return SLOPE_ERR_CUDA;
    return launch_cluster_ex(kern, plan.blocks, 1, plan.threads(), smem, /*overlap_prologue=*/true, stream, p);
}
template <int TYPE, int CHUNKS>
static slope_status_t launch_norm_fwd_of(const NormPlan& plan, const NormFwdParams& p, cudaStream_t stream) {
    const bool full = p.ring.d == 256 * plan.row_warps * CHUNKS, residual = p.ring.src[1], ckpt = p.H_ckpt || p.Y_ckpt;
    const auto pick = [&](auto r, auto c) {
        return full ? layer_norm_fwd_kernel<TYPE, CHUNKS, true, r.value, c.value> : layer_norm_fwd_kernel<TYPE, CHUNKS, false, r.value, c.value>;
    };
    using Yes = std::true_type;
    using No = std::false_type;
    return launch_norm(residual ? (ckpt ? pick(Yes{}, Yes{}) : pick(Yes{}, No{})) : ckpt ? pick(No{}, Yes{}) : pick(No{}, No{}), plan, 0, stream, p);
}
template <int TYPE>
static slope_status_t launch_norm_fwd(const NormPlan& plan, const NormFwdParams& p, cudaStream_t stream) {
    return plan.chunks == 1   ? launch_norm_fwd_of<TYPE, 1>(plan, p, stream)
           : plan.chunks == 2 ? launch_norm_fwd_of<TYPE, 2>(plan, p, stream)
           : plan.chunks == 3 ? launch_norm_fwd_of<TYPE, 3>(plan, p, stream)
                              : launch_norm_fwd_of<TYPE, 4>(plan, p, stream);
}
template <int TYPE, int DX_TYPE, int CHUNKS>
static slope_status_t launch_norm_bwd_of(const NormPlan& plan, const NormBwdParams& p, cudaStream_t stream) {
    const bool full = p.ring.d == 256 * plan.row_warps * CHUNKS, side = p.ring.src[2];
    // (the groups' sums of the parameters' gradients take the place of the ring in the end)
    return launch_norm(full ? (side ? layer_norm_bwd_kernel<TYPE, DX_TYPE, CHUNKS, true, true>
                                    : layer_norm_bwd_kernel<TYPE, DX_TYPE, CHUNKS, true, false>)
                            : side ? layer_norm_bwd_kernel<TYPE, DX_TYPE, CHUNKS, false, true>
                                   : layer_norm_bwd_kernel<TYPE, DX_TYPE, CHUNKS, false, false>,
                       plan, plan.groups * 8 * p.ring.d, stream, p);
}
template <int TYPE, int DX_TYPE>
static slope_status_t launch_norm_bwd(const NormPlan& plan, const NormBwdParams& p, cudaStream_t stream) {
    return plan.chunks == 1   ? launch_norm_bwd_of<TYPE, DX_TYPE, 1>(plan, p, stream)
           : plan.chunks == 2 ? launch_norm_bwd_of<TYPE, DX_TYPE, 2>(plan, p, stream)
           : plan.chunks == 3 ? launch_norm_bwd_of<TYPE, DX_TYPE, 3>(plan, p, stream)
                              : launch_norm_bwd_of<TYPE, DX_TYPE, 4>(plan, p, stream);
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
                         dim3(stream_grid(n8 / 2 + 1, info)), static_cast<cudaStream_t>(stream), X, n8, checkpoint);
}

slope_status_t slope_checkpoint_load(const void* checkpoint, int rows, int cols, void* X, int x_type, void* stream) {
    if (!X || !checkpoint || !plain_type(x_type)) return SLOPE_ERR_INVALID_ARG;
    if (!checkpoint_dims_ok(rows, cols)) return SLOPE_ERR_SHAPE;
    if (!aligned16(X) || !aligned16(checkpoint)) return SLOPE_ERR_ALIGNMENT;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    const size_t n8 = static_cast<size_t>(rows) * cols / 8;
    return launch_stream(x_type == SLOPE_F32 ? checkpoint_load_kernel<kTypeF32> : checkpoint_load_kernel<kTypeBf16>,
                         dim3(stream_grid(n8 / 2 + 1, info)), static_cast<cudaStream_t>(stream), checkpoint, n8, X);
}

slope_status_t slope_layer_norm_fwd(const void* X, int x_type, const void* residual, const void* gamma, const void* beta, int p_type,
                                    int b, int d, float eps, void* H, void* Y, void* mean, void* rstd, void* H_ckpt, void* Y_ckpt,
                                    void* stream_) {
    if (!X || !Y || !plain_type(x_type) || !plain_type(p_type) || !(eps >= 0.0f && eps <= FLT_MAX)) return SLOPE_ERR_INVALID_ARG;
    if ((H && !residual) || !mean != !rstd) return SLOPE_ERR_INVALID_ARG;
    if (b < 1 || d < 1 || d % 8 != 0 || d > kNormMaxWidth) return SLOPE_ERR_SHAPE;
    if ((H_ckpt || Y_ckpt) && !checkpoint_dims_ok(b, d)) return SLOPE_ERR_SHAPE;
    for (const void* p : {X, residual, gamma, beta, static_cast<const void*>(H), static_cast<const void*>(Y), static_cast<const void*>(mean),
                          static_cast<const void*>(rstd), static_cast<const void*>(H_ckpt), static_cast<const void*>(Y_ckpt)})
        if (!aligned16(p)) return SLOPE_ERR_ALIGNMENT;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    const bool ckpt = H_ckpt || Y_ckpt, heavy = norm_fwd_heavy(d, x_type, residual, ckpt);
    const NormPlan plan = norm_fwd_plan(b, d, heavy, ckpt, info);
    const int x_bytes = x_type == SLOPE_F32 ? 4 * d : 2 * d;
    const NormFwdParams p{norm_ring(plan, b, d, !ckpt && !heavy, gamma, beta, 2, p_type, X, x_bytes, residual, 2 * d, nullptr, 0), H, Y,
                          H_ckpt, Y_ckpt, static_cast<float*>(mean), static_cast<float*>(rstd), eps};
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
    const int h_bytes = h_type == SLOPE_F32 ? 4 * d : h_type == SLOPE_Q8 ? d : 2 * d;
    const int dx_bytes = dx_type == SLOPE_F32 ? 4 * d : 2 * d;
    const NormBwdParams p{norm_ring(plan, b, d, true, gamma, nullptr, plan.chunks > 2, p_type, H, h_bytes, dY, 2 * d, dH, dx_bytes),
                          static_cast<const uint8_t*>(H) + static_cast<size_t>(b) * d, static_cast<const float*>(mean),
                          static_cast<const float*>(rstd), dX, dgamma, dbeta, static_cast<float*>(workspace)};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const bool wide = dx_type == SLOPE_F32;
    slope_status_t st;
    if (h_type == SLOPE_BF16)
        st = wide ? launch_norm_bwd<kTypeBf16, kTypeF32>(plan, p, stream) : launch_norm_bwd<kTypeBf16, kTypeBf16>(plan, p, stream);
    else if (h_type == SLOPE_F32)
        st = wide ? launch_norm_bwd<kTypeF32, kTypeF32>(plan, p, stream) : launch_norm_bwd<kTypeF32, kTypeBf16>(plan, p, stream);
    else st = wide ? launch_norm_bwd<kTypeQ8, kTypeF32>(plan, p, stream) : launch_norm_bwd<kTypeQ8, kTypeBf16>(plan, p, stream);
    if (st != SLOPE_OK || !params || plan.blocks == 1) return st;
    return launch_cluster_ex(layer_norm_params_kernel, (2 * d + 31) / 32, 1, 256, 0, /*overlap_prologue=*/true, stream, p.partial, plan.blocks, d,
                             dgamma, dbeta, p.ring.p_f32);
}

// ------------------------------------------------------------------ weight gradients from a checkpoint
// X is read back into the workspace and multiplied by the bf16 kernels: 3.03 bytes of HBM traffic per value in front of a product that the tensor
// cores bound (16384 tokens 11008 -> 4096: 84 of 1080 us).  Converting inside the product instead, codes by TMA into a ring, eight warps that
// write the operand tile, gave the same bits at 1256 us: a k-block of 256 x 256 x 64 keeps an SM's shared memory busy for 512 clocks as
// it is (what TMA brings, what the MMAs read), the time that the MMAs take, and the conversion adds 350.
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
