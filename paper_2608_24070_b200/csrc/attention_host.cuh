// Host side of attention and of the rotation by positions: part of slope_lib.cu, whose argument checks and launches it uses.
#pragma once
#include <climits>
#include <cmath>

#include "attention_kernels.cuh"

namespace slope {
// A matrix [b x heads * head_dim] of row stride `ld` as columns, heads, rows; boxes of 64 columns of a head and 128 rows, 128-byte swizzle.
// Columns past the head and rows past the matrix read as zeros.
static bool make_tmap_heads(CUtensorMap* tm, const void* base, int b, int heads, int head_dim, int ld) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t gdim[3] = {static_cast<cuuint64_t>(head_dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(b)};
    const cuuint64_t gstride[2] = {static_cast<cuuint64_t>(head_dim) * 2, static_cast<cuuint64_t>(ld) * 2};
    const cuuint32_t box[3] = {64, 1, kAttnRows};
    const cuuint32_t estr[3] = {1, 1, 1};
    return tmap_memo(tm, TmapKey{base, b, ld, heads, head_dim, 4}, [&](CUtensorMap* out) {
        return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), gdim, gstride, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    });
}

static bool heads_ok(int b, int heads, int kv_heads, int head_dim) {
    return b > 0 && b <= 1 << 30 && heads > 0 && kv_heads > 0 && heads % kv_heads == 0 && head_dim > 0 && head_dim % 8 == 0 && head_dim <= 128 &&
           static_cast<long long>(heads) * head_dim <= INT_MAX;
}
static bool ld_ok(int ld, int heads, int head_dim) { return ld >= heads * head_dim && ld % 8 == 0; }
// CTAs of a launch that takes `rows` rows of a sequence each: with starts, which only the device knows, every sequence may end inside a tile.
static long long attn_units(int b, int sequences, bool starts, int rows) {
    if (starts) return static_cast<long long>(b) / rows + sequences;
    return static_cast<long long>((b / sequences - 1) / rows + 1) * sequences;
}
static slope_status_t attn_batch(AttnShape* s, int b, int heads, int kv_heads, int head_dim, int sequences, const void* starts, const void* lengths,
                                 int causal, int window, float scale) {
    if (!(scale > 0.0f && scale * kLog2e <= FLT_MAX) || window < 0 || (window && !causal)) return SLOPE_ERR_INVALID_ARG;
    if (!heads_ok(b, heads, kv_heads, head_dim) || sequences < 1 || (!starts && b % sequences != 0)) return SLOPE_ERR_SHAPE;
    if (attn_units(b, sequences, starts, kAttnRows) * (heads + kv_heads) > INT_MAX) return SLOPE_ERR_SHAPE;
    *s = AttnShape{b, heads, kv_heads, head_dim, sequences, static_cast<const int*>(starts), static_cast<const int*>(lengths), causal != 0,
                   window < b ? window : 0, scale * kLog2e, heads / kv_heads, b / sequences, 1.0f / heads, 1.0f / kv_heads,
                   static_cast<float>(kv_heads) / heads};
    return SLOPE_OK;
}
// Keys that a query of a sequence sees, in the mean; with starts or lengths, which only the device knows, as if the sequences shared the rows evenly.
// (Causal, window w of n tokens: w - w^2 / 2 n, and n / 2 without a window or with one that leaves nothing out.)
static double attn_reach(const AttnShape& s) {
    const double n = s.part;
    if (!s.causal || s.part == 0) return n;
    const double w = s.window ? std::min<double>(s.window, n) : n;
    return w * (1.0 - w / (2.0 * n));
}
template <typename Kernel, typename... Args>
static slope_status_t launch_attn(Kernel kern, long long grid, int threads, int smem, cudaStream_t stream, const Args&... args) {
    if (!set_smem(kern, smem)) return SLOPE_ERR_CUDA;
    return launch_cluster_ex(kern, static_cast<int>(grid), 1, threads, smem, /*overlap_prologue=*/true, stream, args...);
}
template <int HD, int TILES>
static slope_status_t attn_fwd(const AttnFwdParams& p, const CUtensorMap (&tm)[3], cudaStream_t stream) {
    using Cfg = AttnFwdCfg<HD, TILES>;
    return launch_attn(attention_fwd_kernel<HD, TILES>, attn_units(p.s.b, p.s.sequences, p.s.starts, TILES * kAttnRows) * p.s.heads, Cfg::kThreads,
                       Cfg::kSmem, stream, tm[0], tm[1], tm[2], p);
}
template <int HD>
static slope_status_t attn_bwd(AttnBwdParams p, const AttnDeltaParams& d, const CUtensorMap (&tm)[4], cudaStream_t stream) {
    const long long units = attn_units(p.s.b, p.s.sequences, p.s.starts, kAttnRows);
    p.key_blocks = static_cast<int>(units * p.s.kv_heads);
    const long long blocks = static_cast<long long>((p.s.b - 1) / 32 + 1) * ((p.s.heads + 7) / 8);
    if (slope_status_t st = launch_cluster_ex(attention_delta_kernel<HD>, static_cast<int>(blocks), 1, 256, 0, /*overlap_prologue=*/true, stream, d)) return st;
    // tiles begin on a multiple of 1 KB behind what has a fixed place (which ends on a multiple of 128 bytes, as dynamic shared memory begins)
    constexpr int kFixed = sizeof(AttnBwdShared<HD>), kSmem = (2 + AttnCfg<HD>::kStages) * AttnCfg<HD>::kTile + (kFixed + 1023) / 1024 * 1024 - kFixed;
    static_assert(kFixed % 128 == 0 && kFixed + kSmem <= 227 * 1024, "shared memory of a block");
    return launch_attn(attention_bwd_kernel<HD>, p.key_blocks + units * p.s.heads, kAttnThreads, kSmem, stream, tm[0], tm[1], tm[2], tm[3], p);
}
template <int TYPE, bool PAIRS>
static slope_status_t launch_rotary(const RotaryParams& p, int wide, cudaStream_t stream) {
    const auto kern = PAIRS || wide == 8 ? rotary_kernel<TYPE, PAIRS, 8>
                      : wide == 4        ? rotary_kernel<TYPE, false, 4>
                      : wide == 2        ? rotary_kernel<TYPE, false, 2>
                                         : rotary_kernel<TYPE, false, 1>;
    return launch_cluster_ex(kern, (p.b - 1) / p.tokens + 1, 1, kRotaryThreads, 0, /*overlap_prologue=*/true, stream, p);
}
}  // namespace slope

extern "C" {

slope_status_t slope_attention_fwd(const void* Q, int q_ld, const void* K, int k_ld, const void* V, int v_ld, int b, int heads, int kv_heads,
                                   int head_dim, int sequences, const void* starts, const void* lengths, int causal, int window, float scale,
                                   void* O, int o_ld, void* lse, void* stream_) {
    if (!Q || !K || !V || !O) return SLOPE_ERR_INVALID_ARG;
    AttnShape s;
    if (slope_status_t st = attn_batch(&s, b, heads, kv_heads, head_dim, sequences, starts, lengths, causal, window, scale)) return st;
    if (!ld_ok(q_ld, heads, head_dim) || !ld_ok(o_ld, heads, head_dim) || !ld_ok(k_ld, kv_heads, head_dim) || !ld_ok(v_ld, kv_heads, head_dim))
        return SLOPE_ERR_SHAPE;
    for (const void* p : {Q, K, V, starts, lengths, static_cast<const void*>(O), static_cast<const void*>(lse)})
        if (!aligned16(p)) return SLOPE_ERR_ALIGNMENT;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    CUtensorMap tm[3];
    if (!make_tmap_heads(&tm[0], Q, b, heads, head_dim, q_ld) || !make_tmap_heads(&tm[1], K, b, kv_heads, head_dim, k_ld) ||
        !make_tmap_heads(&tm[2], V, b, kv_heads, head_dim, v_ld))
        return SLOPE_ERR_CUDA;
    const AttnFwdParams p{s, static_cast<uint16_t*>(O), static_cast<float*>(lse), o_ld};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    // One tile of queries a block, two blocks on an SM, where few keys make loading and storing a large part of a block's time, or where blocks of two
    // tiles would not even give every SM one; else two tiles, which share the keys' tiles. Measured, us, one / two:
    //   heads of 64, 16384 tokens, 16 heads: 16 x 1024 causal 82 / 94, 4 x 4096 causal 206 / 211, 8 x 2048 full 196 / 196, 4 x 4096 full 386 / 372
    //   heads of 128, 16384 tokens, 8 heads: 64 x 256 causal 36 / 42, 16 x 1024 causal 59 / 60, 8 x 2048 causal 90 / 89, 4 x 4096 full 300 / 282
    //   1024 tokens alone, causal: 16 heads of 64 16.5 / 19.3, 8 heads of 128 21.7 / 24.9
    //   windows of 4096 tokens' sequences, 64 columns: 3000 (reach 1901) 193 / 204, 1024 (896) 113 / 127; 128 columns: 3000 148 / 145, 1024 86 / 90,
    //   512 (480) 65 / 69; of 1024 tokens' sequences, 128 columns: 700 (461) 59 / 62
    const double reach = attn_reach(p.s);
    const bool one = reach <= (head_dim <= 64 ? 2048 : 512) || attn_units(b, sequences, p.s.starts, 2 * kAttnRows) * heads <= info.sm_count;
    if (head_dim <= 64) return one ? attn_fwd<64, 1>(p, tm, stream) : attn_fwd<64, 2>(p, tm, stream);
    return one ? attn_fwd<128, 1>(p, tm, stream) : attn_fwd<128, 2>(p, tm, stream);
}

size_t slope_attention_bwd_workspace_bytes(int b, int heads, int kv_heads, int head_dim) {
    return heads_ok(b, heads, kv_heads, head_dim) ? static_cast<size_t>(b) * heads * sizeof(float) : 0;
}

slope_status_t slope_attention_bwd(const void* dO, int do_ld, const void* Q, int q_ld, const void* K, int k_ld, const void* V, int v_ld,
                                   const void* O, int o_ld, const void* lse, int b, int heads, int kv_heads, int head_dim, int sequences,
                                   const void* starts, const void* lengths, int causal, int window, float scale, void* dQ, int dq_ld, void* dK,
                                   int dk_ld, void* dV, int dv_ld, void* workspace, size_t workspace_bytes, void* stream_) {
    if (!dO || !Q || !K || !V || !O || !lse || !dQ || !dK || !dV || !workspace) return SLOPE_ERR_INVALID_ARG;
    AttnShape s;
    if (slope_status_t st = attn_batch(&s, b, heads, kv_heads, head_dim, sequences, starts, lengths, causal, window, scale)) return st;
    for (int ld : {do_ld, q_ld, o_ld, dq_ld})
        if (!ld_ok(ld, heads, head_dim)) return SLOPE_ERR_SHAPE;
    for (int ld : {k_ld, v_ld, dk_ld, dv_ld})
        if (!ld_ok(ld, kv_heads, head_dim)) return SLOPE_ERR_SHAPE;
    for (const void* p : {dO, Q, K, V, O, lse, starts, lengths, static_cast<const void*>(dQ), static_cast<const void*>(dK),
                          static_cast<const void*>(dV), static_cast<const void*>(workspace)})
        if (!aligned16(p)) return SLOPE_ERR_ALIGNMENT;
    if (workspace_bytes < slope_attention_bwd_workspace_bytes(b, heads, kv_heads, head_dim)) return SLOPE_ERR_INVALID_ARG;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    CUtensorMap tm[4];
    if (!make_tmap_heads(&tm[0], Q, b, heads, head_dim, q_ld) || !make_tmap_heads(&tm[1], K, b, kv_heads, head_dim, k_ld) ||
        !make_tmap_heads(&tm[2], V, b, kv_heads, head_dim, v_ld) || !make_tmap_heads(&tm[3], dO, b, heads, head_dim, do_ld))
        return SLOPE_ERR_CUDA;
    float* delta = static_cast<float*>(workspace);
    const AttnBwdParams p{s,    static_cast<const float*>(lse), delta, static_cast<uint16_t*>(dQ), static_cast<uint16_t*>(dK), static_cast<uint16_t*>(dV),
                          dq_ld, dk_ld, dv_ld, scale, 0};
    const AttnDeltaParams d{static_cast<const uint16_t*>(O), static_cast<const uint16_t*>(dO), o_ld, do_ld, b, heads, head_dim, delta};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return head_dim <= 64 ? attn_bwd<64>(p, d, tm, stream) : attn_bwd<128>(p, d, tm, stream);
}

slope_status_t slope_rotary(const void* Q, int q_ld, const void* K, int k_ld, int type, int b, int heads, int kv_heads, int head_dim, int rot_dim,
                            int interleaved, int backward, const void* positions, const void* frequencies, float factor, void* Qr, int qr_ld,
                            void* Kr, int kr_ld, void* stream) {
    if (!Q || !Qr || !positions || !frequencies || !K != !Kr || !plain_type(type) || !std::isfinite(factor)) return SLOPE_ERR_INVALID_ARG;
    if ((K && Q == Qr) != (K && K == Kr) || (Q == Qr && q_ld != qr_ld) || (K && K == Kr && k_ld != kr_ld)) return SLOPE_ERR_INVALID_ARG;
    if (b < 1 || heads < 1 || (K && kv_heads < 1) || head_dim < 8 || head_dim % 8 != 0 || head_dim > 2 * kRotaryTable) return SLOPE_ERR_SHAPE;
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > head_dim) return SLOPE_ERR_SHAPE;
    const auto ld_fits = [&](int ld, int n) { return ld % 8 == 0 && static_cast<long long>(n) * head_dim <= ld; };
    if (!ld_fits(q_ld, heads) || !ld_fits(qr_ld, heads) || (K && (!ld_fits(k_ld, kv_heads) || !ld_fits(kr_ld, kv_heads)))) return SLOPE_ERR_SHAPE;
    for (const void* p : {Q, K, positions, frequencies, static_cast<const void*>(Qr), static_cast<const void*>(Kr)})
        if (!aligned16(p)) return SLOPE_ERR_ALIGNMENT;
    DeviceInfo info;
    if (slope_status_t st = check_arch(info)) return st;
    // as many values at a time as the rotated part is a multiple of; columns behind it are copied where the output is not the input
    const int n = rot_dim / 2, wide = interleaved || n % 8 == 0 ? 8 : n % 4 == 0 ? 4 : n % 2 == 0 ? 2 : 1;
    const int turned = interleaved ? (rot_dim + 7) / 8 : n / wide;
    const int per_head = turned + (Q == Qr ? 0 : interleaved ? head_dim / 8 - turned : (head_dim - rot_dim) / wide);
    const long long per_token = (static_cast<long long>(heads) + (K ? kv_heads : 0)) * per_head;
    // Tokens of a block: an angle for every thread, if that leaves four blocks for every SM and a thread two batches of tasks at most (us, rotating 20 of 80
    // columns of 64 heads, 2039 tokens: neighbouring pairs, 25 tokens a block 47, 3 as by the rule 11.0, 1 12.6; halves 116, 28.4, 1 by the rule 23.4;
    // all of 64 heads of 128, 16384 tokens, halves, 25 tokens 107, 4 by the rule 83.3, 1 92)
    const long long most = std::min<long long>({kRotaryThreads / n, b / (4ll * info.sm_count), 8 * kRotaryThreads / per_token, 64});
    const int tokens = static_cast<int>(std::max(1ll, most));
    if (tokens * per_token > INT_MAX / 2) return SLOPE_ERR_SHAPE;
    const RotaryParams p{{Q, K}, {Qr, Kr}, {q_ld, k_ld}, {qr_ld, kr_ld}, {heads, K ? kv_heads : 0}, b, head_dim, n, tokens, turned, per_head,
                         static_cast<int>(per_token), 1.0f / per_head, 1.0f / per_token, factor, backward ? -1.0f : 1.0f,
                         static_cast<const int*>(positions), static_cast<const double*>(frequencies)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == SLOPE_F32) return interleaved ? launch_rotary<kTypeF32, true>(p, wide, s) : launch_rotary<kTypeF32, false>(p, wide, s);
    return interleaved ? launch_rotary<kTypeBf16, true>(p, wide, s) : launch_rotary<kTypeBf16, false>(p, wide, s);
}

}  // extern "C"
