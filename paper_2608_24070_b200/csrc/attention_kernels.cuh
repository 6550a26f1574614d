// Softmax attention between the linear layers, forward and backward, and the rotation of queries and keys by their positions.
#pragma once
#include <cfloat>

#include "norm_kernels.cuh"

namespace slope {

// ---------------------------------------------------------------- instructions
// 3-D tiled load: columns of a head, head, row.
__device__ __forceinline__ void tma_load_3d(void* smem_dst, const CUtensorMap* tmap, uint64_t* bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_u32(smem_dst)), "l"(tmap), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: A in bf16, two values of a row per 32-bit column
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// 32 consecutive 32-bit columns of this warp's 32 lanes (one row per thread)
__device__ __forceinline__ void tmem_ld_32(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
          "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
          "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_32(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]),
        "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]),
        "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}

// ---------------------------------------------------------------- a call's sequences
// Sequences lie one behind the other in `b` rows: at starts[i] ... starts[i + 1], or (starts NULL) in `sequences` equal parts; lengths[i], if
// there, says how many rows of the part there are.  Starts and lengths are read on the device and held to [0, b] there.
struct AttnShape {
    int b, heads, kv_heads, head_dim, sequences;
    const int *starts, *lengths;
    int causal, window;
    float scale;                          // of the products, times log2(e): probabilities are powers of two here
};
struct AttnTile {
    int first, len, tile;                 // the sequence's first row, its length, number of the tile of `rows` rows; len 0: nothing to do
};
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr int kAttnRows = 128;            // rows of a tile of queries or keys
constexpr int kAttnThreads = 384;         // two groups of four warps that compute, one that feeds them
// registers of a thread that computes / that feeds; with 168 at launch the three groups come to 384 x 168
constexpr int kAttnRegsUp = 208, kAttnRegsDown = 88;
static_assert(2 * kAttnRegsUp + kAttnRegsDown == 3 * 168, "shares of the launch's registers");

// Tile number `unit` of the call, the last tile of a sequence first where later rows see more keys.  By one whole warp.
__device__ __forceinline__ AttnTile attn_locate(const AttnShape& s, int unit, int rows, bool last_first) {
    const int lane = threadIdx.x & 31;
    AttnTile t{0, 0, 0};
    int n = 0, rank = 0;
    if (!s.starts) {
        const int part = s.b / s.sequences, tiles = (part - 1) / rows + 1, seq = unit / tiles;
        rank = unit - seq * tiles;
        t.first = seq * part;
        t.len = s.lengths ? min(max(s.lengths[seq], 0), part) : part;
        n = (t.len + rows - 1) / rows;
        if (rank >= n) t.len = 0;
    } else {
        int before = 0;
        for (int i0 = 0; i0 < s.sequences; i0 += 32) {
            const int i = i0 + lane;
            int first = 0, len = 0;
            if (i < s.sequences) {
                first = min(max(s.starts[i], 0), s.b);
                len = max(min(s.starts[i + 1], s.b) - first, 0);
                if (s.lengths) len = min(len, max(s.lengths[i], 0));
            }
            const int own = (len + rows - 1) / rows;
            int sum = own;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int o = __shfl_up_sync(0xFFFFFFFFu, sum, d);
                if (lane >= d) sum += o;
            }
            const unsigned hit = __ballot_sync(0xFFFFFFFFu, before + sum > unit);
            if (hit) {
                const int src = __ffs(hit) - 1;
                t.first = __shfl_sync(0xFFFFFFFFu, first, src);
                t.len = __shfl_sync(0xFFFFFFFFu, len, src);
                n = __shfl_sync(0xFFFFFFFFu, own, src);
                rank = unit - before - (__shfl_sync(0xFFFFFFFFu, sum, src) - n);
                break;
            }
            before += __shfl_sync(0xFFFFFFFFu, sum, 31);
        }
    }
    t.tile = !t.len ? 0 : last_first ? n - 1 - rank : rank;
    return t;
}
// Tiles of keys that queries [a, a + 128) of a sequence see, and the other way round.
__device__ __forceinline__ int attn_first_key_tile(const AttnShape& s, int a) { return s.window ? max(0, a - s.window + 1) / kAttnRows : 0; }
__device__ __forceinline__ int attn_end_key_tile(const AttnShape& s, int a, int len) {
    return (min(s.causal ? a + kAttnRows : len, len) + kAttnRows - 1) / kAttnRows;
}
__device__ __forceinline__ int attn_first_query_tile(const AttnShape& s, int a) { return s.causal ? a / kAttnRows : 0; }
__device__ __forceinline__ int attn_end_query_tile(const AttnShape& s, int a, int len) {
    const int all = (len + kAttnRows - 1) / kAttnRows;
    return s.window && s.window < len ? min(all, (a + kAttnRows - 2 + s.window) / kAttnRows + 1) : all;
}

// ---------------------------------------------------------------- tiles
// A tile of 128 rows x HD columns (64 or 128; columns past the head read as zeros) lies in shared memory as chunks of 64 columns, 128 bytes a
// row, in the 128-byte swizzle.  As an operand it is read with its columns as the reduction (K contiguous) or with its
// rows (the other index contiguous).
constexpr int kAttnChunk = kAttnRows * 128;
template <int HD>
struct AttnCfg {
    static constexpr int kChunks = HD / 64, kTile = kChunks * kAttnChunk;
    static constexpr int kStages = HD == 128 ? 5 : 8;           // of the ring, beside two tiles that stay
    static constexpr int kSmem = (2 + kStages) * kTile + 1024;
    // the kernel of dK and dV keeps 2 KB beside its tiles
    static constexpr int kKvStages = HD == 128 ? 4 : 8, kKvSmem = (2 + kKvStages) * kTile + 1024;
};
template <int HD>
__device__ __forceinline__ void attn_load(uint8_t* tile, const CUtensorMap* tm, uint64_t* bar, int head, int row) {
    mbar_expect_tx(bar, AttnCfg<HD>::kTile);
#pragma unroll
    for (int c = 0; c < AttnCfg<HD>::kChunks; ++c) tma_load_3d(tile + c * kAttnChunk, tm, bar, 64 * c, head, row);
}
// D[128 x 128] = A B^T over the columns of a head, `steps` of 16
template <int HD>
__device__ __forceinline__ void attn_mma_columns(uint32_t d, uint32_t a, uint32_t b, int steps) {
    constexpr uint32_t idesc = make_idesc_bf16(kAttnRows, kAttnRows, false, false, false);
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
        const uint32_t off = (k >> 2) * kAttnChunk + (k & 3) * 32;
        if (k < steps)
            umma_bf16(d, make_smem_desc(a + off, 16, 1024, kSwizzle128B), make_smem_desc(b + off, 16, 1024, kSwizzle128B), idesc, k != 0);
    }
}
// D[128 x head] (+)= A B over the tile's rows, `steps` of 16; A from tensor memory: its first 64 values at `a0`, the others at `a1`
__device__ __forceinline__ void attn_mma_rows(uint32_t d, uint32_t a0, uint32_t a1, uint32_t b, uint32_t idesc, int steps, bool accumulate) {
#pragma unroll
    for (int k = 0; k < kAttnRows / 16; ++k) {
        if (k < steps)
            umma_bf16_ts(d, k < 4 ? a0 + 8 * k : a1 + 8 * (k - 4), make_smem_desc(b + k * 2048, kAttnChunk, 1024, kSwizzle128B), idesc,
                         accumulate || k != 0);
    }
}
// Rows [valid, 16-multiple) of a tile to zero: they belong to other sequences or to none, and what stands there may be an infinity or a NaN,
// which a probability of zero does not take out of a product.  Such a tile's copies complete on a barrier of its own, for one warp that zeroes the
// rows and then completes the barrier that the tile's readers wait for.
template <int HD>
__device__ __forceinline__ void attn_zero_rows(uint8_t* tile, int valid) {
    const int lane = threadIdx.x & 31, units = (((valid + 15) & ~15) - valid) * 8;
    for (int c = 0; c < AttnCfg<HD>::kChunks; ++c)
        for (int u = lane; u < units; u += 32) *reinterpret_cast<uint4*>(tile + c * kAttnChunk + valid * 128 + u * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
}
// This warp's 32 rows of an accumulator, columns [c0, c1) of the head, times `mul`, to bf16 rows in global memory; `stage` is shared memory of
// 128 rows x HD columns.  Straight from the lanes a store would touch a row per lane.
template <int HD>
__device__ __forceinline__ void attn_store(uint32_t t_row, int c0, int c1, float mul, uint8_t* stage, uint16_t* out, int ld, int rows, int head_dim) {
    const int lane = threadIdx.x & 31, row0 = 32 * ((threadIdx.x >> 5) & 3);
    const uint32_t base = smem_u32(stage) + row0 * HD * 2;
    c1 = min(c1, head_dim);
#pragma unroll 1
    for (int c = c0; c < c1; c += 32) {
        uint32_t v[32];
        tmem_ld_32(t_row + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(__uint_as_float(v[8 * u + 2 * i]) * mul, __uint_as_float(v[8 * u + 2 * i + 1]) * mul);
            st_shared_v4(base + lane * HD * 2 + (((c >> 3) + u) ^ (lane & 7)) * 16, make_uint4(w[0], w[1], w[2], w[3]));
        }
    }
    __syncwarp();
    const int first = c0 >> 3, units = (c1 >> 3) - first;
    if (units <= 0) return;
    for (int i = lane; i < 32 * units; i += 32) {
        const int r = i / units, u = first + i - r * units;
        if (row0 + r < rows) {
            const uint4 v = lds_v4(base + r * HD * 2 + (u ^ (r & 7)) * 16);
            *reinterpret_cast<uint4*>(out + static_cast<size_t>(row0 + r) * ld + 8 * u) = v;
        }
    }
}
// A wait whose outcome all lanes share: what follows it is done by whole warps.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag));
}
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// =====================================================================================
// Forward.  One CTA takes 256 queries of a head as two tiles of 128, one per group of four warps, and walks the tiles of keys once:
//   S = Q K^T (tensor memory) -> the group that owns the tile takes a row per thread: running maximum m, P = 2^(S - m), its sum l,
//   P as bf16 over S -> O += P V (A from tensor memory).
// While one group forms its P the tensor cores work for the other.  m follows the true maximum only where that is more than 2^8 ahead, when the
// thread rescales O and l itself: O / l does not depend on m, P up to 2^8 has the same relative precision, and O is not touched in most
// steps.  P is rounded to bf16 as an operand (2^-9 relative, as any operand of these products); l sums the unrounded values in fp32.
// Warps 0-3, 4-7: queries 0-127, 128-255; warp 8: MMAs; 9: loads; 10: zeros behind the sequence's last row of V.
// =====================================================================================
constexpr float kAttnSlack = 8.0f;
struct AttnFwdParams {
    AttnShape s;
    uint16_t* O;
    float* lse;
    int o_ld;
};
template <int HD>
__global__ void __launch_bounds__(kAttnThreads, 1)
attention_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const AttnFwdParams p) {
    using Cfg = AttnCfg<HD>;
    __shared__ uint64_t q_full[2], s_full[2], p_full[2], o_full[2], full_bar[Cfg::kStages], empty_bar[Cfg::kStages], ragged_bar;
    __shared__ uint32_t tmem_slot[1];
    __shared__ int abort_word;
    __shared__ AttnTile work;
    volatile int* abort_flag = &abort_word;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* ring = smem + 2 * Cfg::kTile;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = threadIdx.x >> 7;

    griddep_launch_dependents();
    if (threadIdx.x == 0) {
        for (int t = 0; t < 2; ++t) {
            mbar_init(&q_full[t], 1);
            mbar_init(&s_full[t], 1);
            mbar_init(&p_full[t], 4);
            mbar_init(&o_full[t], 1);
        }
        for (int i = 0; i < Cfg::kStages; ++i) { mbar_init(&full_bar[i], 1); mbar_init(&empty_bar[i], 1); }
        mbar_init(&ragged_bar, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 8) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    griddep_wait();
    const int head = blockIdx.x % p.s.heads, kv_head = head / (p.s.heads / p.s.kv_heads);
    if (warp == 0) {
        const AttnTile t = attn_locate(p.s, blockIdx.x / p.s.heads, 2 * kAttnRows, p.s.causal);
        if (lane == 0) work = t;
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;                      // S of either tile, then O of either
    const int len = work.len, first = work.first, q0 = work.tile * 2 * kAttnRows;
    const int tiles = !len ? 0 : len - q0 > kAttnRows ? 2 : 1;
    // tiles of keys [lo, hi) of the two tiles of queries and of both
    int lo[2], hi[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        lo[t] = attn_first_key_tile(p.s, q0 + t * kAttnRows);
        hi[t] = t < tiles ? attn_end_key_tile(p.s, q0 + t * kAttnRows, len) : lo[t];
    }
    const int begin = lo[0], end = tiles ? max(hi[0], hi[1]) : begin;
    // the sequence's last tile of keys, if it is not full and among these
    const int last = (len - 1) / kAttnRows, last_rows = len - last * kAttnRows, ragged = last_rows < kAttnRows && end == last + 1 ? last : -1;

    if (group == 2) {
        registers_down<kAttnRegsDown>();
        if (warp == 9) {
            if (elect_one()) {
                PipeState ps;
                bool ok = true;
                for (int t = 0; t < tiles; ++t) attn_load<HD>(smem + t * Cfg::kTile, &tmQ, &q_full[t], head, first + q0 + t * kAttnRows);
                for (int j = begin; j < end && ok; ++j) {
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        if (!mbar_wait(&empty_bar[ps.stage], ps.phase ^ 1u, abort_flag)) { ok = false; break; }
                        attn_load<HD>(ring + ps.stage * Cfg::kTile, v ? &tmV : &tmK, v && j == ragged ? &ragged_bar : &full_bar[ps.stage], kv_head, first + j * kAttnRows);
                        ps.advance(Cfg::kStages);
                    }
                }
            }
        } else if (warp == 8) {
            if (elect_one()) {
                const int steps = (p.s.head_dim + 15) / 16;
                const uint32_t idesc = make_idesc_bf16(kAttnRows, 16 * steps, false, true, false);
                PipeState ps;                             // of the next tile of the ring to be waited for
                uint32_t p_phase[2] = {0, 0};
                bool ok = true;
                const auto scores = [&](int t, int stage) {
                    attn_mma_columns<HD>(tmem + t * kAttnRows, smem_u32(smem + t * Cfg::kTile), smem_u32(ring + stage * Cfg::kTile), steps);
                    umma_commit(&s_full[t]);
                };
                for (int j = begin; j < end && ok; ++j) {
                    // the first scores; behind them each step leaves those of the next
                    if (j == begin) {
                        if (!(ok = mbar_wait(&full_bar[ps.stage], ps.phase, abort_flag))) break;
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            if (t >= tiles || !ok) continue;
                            if (!(ok = mbar_wait(&q_full[t], 0, abort_flag))) continue;
                            tc_fence_after_sync();
                            if (lo[t] <= j && j < hi[t]) scores(t, ps.stage);
                        }
                        umma_commit(&empty_bar[ps.stage]);
                        ps.advance(Cfg::kStages);
                        if (!ok) break;
                    }
                    const int v_stage = ps.stage;
                    if (!(ok = mbar_wait(&full_bar[ps.stage], ps.phase, abort_flag))) break;
                    const int rows = j == ragged ? last_rows : kAttnRows;
                    ps.advance(Cfg::kStages);
                    const int k_stage = ps.stage;
                    if (j + 1 < end) {
                        if (!(ok = mbar_wait(&full_bar[ps.stage], ps.phase, abort_flag))) break;
                        ps.advance(Cfg::kStages);
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (lo[t] <= j && j < hi[t]) {
                            if (!(ok = ok && mbar_wait(&p_full[t], p_phase[t], abort_flag))) continue;
                            p_phase[t] ^= 1u;
                            tc_fence_after_sync();
                            const uint32_t s = tmem + t * kAttnRows;
                            attn_mma_rows(tmem + 2 * kAttnRows + t * HD, s, s + 32, smem_u32(ring + v_stage * Cfg::kTile), idesc, (rows + 15) / 16,
                                          j != lo[t]);
                            if (j + 1 == hi[t]) umma_commit(&o_full[t]);
                        }
                        if (lo[t] <= j + 1 && j + 1 < hi[t]) scores(t, k_stage);
                    }
                    if (!ok) break;
                    umma_commit(&empty_bar[v_stage]);
                    if (j + 1 < end) umma_commit(&empty_bar[k_stage]);
                }
            }
        } else if (warp == 10 && ragged >= 0) {
            const int stage = (2 * (last - begin) + 1) % Cfg::kStages;
            if (warp_wait(&ragged_bar, 0, abort_flag)) {
                attn_zero_rows<HD>(ring + stage * Cfg::kTile, last_rows);
                warp_arrive(&full_bar[stage]);
            }
        }
    } else {
        registers_up<kAttnRegsUp>();
        const int t = group, row = threadIdx.x & 127, i = q0 + t * kAttnRows + row;       // the query's place in its sequence
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_row = tmem + lanes + t * kAttnRows, o_row = tmem + lanes + 2 * kAttnRows + t * HD;
        float m = -INFINITY, l = 0.0f;
        uint32_t phase = 0;
        bool ok = t < tiles;
        const int j_lo = t ? lo[1] : lo[0], j_hi = t ? hi[1] : hi[0];
        for (int j = j_lo; j < j_hi; ++j) {
            if (!(ok = warp_wait(&s_full[t], phase, abort_flag))) break;
            phase ^= 1u;
            tc_fence_after_sync();
            uint32_t v[kAttnRows];
#pragma unroll
            for (int c = 0; c < kAttnRows; c += 32) tmem_ld_32(s_row + c, v + c);
            tmem_ld_wait();
            // columns [c_lo, c_hi) of the tile are seen
            const int c0 = j * kAttnRows, t0 = q0 + t * kAttnRows;
            if ((p.s.causal ? c0 + kAttnRows - 1 > t0 : c0 + kAttnRows > len) || (p.s.window && t0 + kAttnRows - 1 - c0 >= p.s.window)) {
                const int c_hi = (p.s.causal ? min(i + 1, len) : len) - c0, c_lo = p.s.window ? i - p.s.window + 1 - c0 : 0;
#pragma unroll
                for (int c = 0; c < kAttnRows; ++c)
                    if (c < c_lo || c >= c_hi) v[c] = 0xFF800000u;
            }
            float top[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) top[c] = __uint_as_float(v[c]);
#pragma unroll
            for (int c = 4; c < kAttnRows; c += 8) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    top[k] = c + 4 + k < kAttnRows ? max3(top[k], __uint_as_float(v[c + k]), __uint_as_float(v[c + 4 + k])) : fmaxf(top[k], __uint_as_float(v[c + k]));
            }
            const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.s.scale;
            if (j == j_lo) {
                m = now;
            } else if (__any_sync(0xFFFFFFFFu, now > m + kAttnSlack)) {
                const float next = fmaxf(m, now), by = next == m ? 1.0f : exp2_fast(m - next);
                m = next;
                l *= by;
#pragma unroll 1
                for (int c = 0; c < p.s.head_dim; c += 32) {
                    uint32_t o[32];
                    tmem_ld_32(o_row + c, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * by);
                    tmem_st_32(o_row + c, o);
                }
            }
            const Pair by = both(p.s.scale), less = both(m == -INFINITY ? 0.0f : -m);
            Pair sum[2] = {0, 0};
#pragma unroll
            for (int c = 0; c < kAttnRows; c += 2) {
                const Pair x = fma2(pair(v[c], v[c + 1]), by, less);
                const float e0 = exp2_fast(low(x)), e1 = exp2_fast(high(x));
                sum[(c >> 1) & 1] = add2(sum[(c >> 1) & 1], pair(e0, e1));
                v[c >> 1] = pack_bf16x2(e0, e1);
            }
            tmem_st_32(s_row, v);
            tmem_st_32(s_row + 32, v + 32);
            const Pair all = add2(sum[0], sum[1]);
            l += low(all) + high(all);
            tmem_st_wait();
            tc_fence_before_sync();
            warp_arrive(&p_full[t]);
        }
        if (ok && (ok = warp_wait(&o_full[t], 0, abort_flag))) {
            tc_fence_after_sync();
            const size_t at = static_cast<size_t>(first) + q0 + t * kAttnRows;
            if (p.lse && i < len) p.lse[static_cast<size_t>(head) * p.s.b + at + row] = m * kLn2 + logf(l);
            // (a row that has seen none but infinitely small scores: 0 / 0)
            const float inv = 1.0f / l;
            // every lane's own row: `mul` differs between lanes
            attn_store<HD>(o_row, 0, HD, inv, smem + t * Cfg::kTile, p.O + at * p.o_ld + head * p.s.head_dim, p.o_ld, len - q0 - t * kAttnRows,
                           p.s.head_dim);
        }
        tc_fence_before_sync();
    }
    if (*abort_flag) drain_after_abort();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

// =====================================================================================
// Backward.  With D = rowsum(dO O), P = 2^(scale S - lse) and dS = P (dO V^T - D):
//   dV = P^T dO,   dK = scale dS^T Q (sums over queries and over the heads that share a key head),   dQ = scale dS K (a sum over keys).
// Two kernels form S and dP = dO V^T once each: with a third more products nothing is added up in memory, so that every sum has a fixed order.
// =====================================================================================
// D of every row and head, [heads x b].  A group of HD / 8 lanes takes a head of a row; 32 rows of a block go out together.
struct AttnDeltaParams {
    const uint16_t *O, *dO;
    int o_ld, do_ld, b, heads, head_dim;
    float* delta;
};
template <int HD>
__global__ void __launch_bounds__(256)
attention_delta_kernel(const AttnDeltaParams p) {
    constexpr int kLanes = HD / 8, kAtOnce = 256 / kLanes;
    __shared__ float out[8][33];
    griddep_launch_dependents();
    griddep_wait();
    const int row0 = (blockIdx.x / ((p.heads + 7) / 8)) * 32, head0 = (blockIdx.x % ((p.heads + 7) / 8)) * 8;
    const int part = threadIdx.x % kLanes, col = 8 * part;
#pragma unroll 4
    for (int i = threadIdx.x / kLanes; i < 256; i += kAtOnce) {
        const int r = i >> 3, h = i & 7, row = row0 + r;
        float sum = 0.0f;
        if (row < p.b && head0 + h < p.heads && col < p.head_dim) {
            const size_t at = (head0 + h) * p.head_dim + col;
            const V8 a = from_bf16(ld_v4(p.O + static_cast<size_t>(row) * p.o_ld + at)), g = from_bf16(ld_v4(p.dO + static_cast<size_t>(row) * p.do_ld + at));
            Pair s = mul2(a.p[0], g.p[0]);
#pragma unroll
            for (int k = 1; k < 4; ++k) s = fma2(a.p[k], g.p[k], s);
            sum = low(s) + high(s);
        }
#pragma unroll
        for (int d = kLanes / 2; d > 0; d /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (part == 0) out[h][r] = sum;
    }
    __syncthreads();
    const int h = threadIdx.x >> 5, r = threadIdx.x & 31;
    if (head0 + h < p.heads && row0 + r < p.b) p.delta[static_cast<size_t>(head0 + h) * p.b + row0 + r] = out[h][r];
}

struct AttnBwdParams {
    AttnShape s;
    const float *lse, *delta;
    uint16_t *dQ, *dK, *dV;
    int dq_ld, dk_ld, dv_ld;
    float grad_scale;                     // the products' factor itself
};

// dK and dV of 128 keys.  Keys lie on the lanes: S^T = K Q^T, dP^T = V dO^T, so that P^T and dS^T are where the next products
// want them as A.  Both groups work on every tile, 64 queries each; what belongs to a query (lse, D) comes from shared memory.
// The tensor cores' order is dV(i), S(i + 1), dK(i), dP(i + 1): P(i + 1) is formed beside dK(i) and dP(i + 1), dS(i) beside dV(i) and S(i + 1).
// Warp 8: MMAs; 9: loads; 10: lse and D, zeros behind the sequence's last row.
template <int HD>
__global__ void __launch_bounds__(kAttnThreads, 1)
attention_bwd_kv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                        const __grid_constant__ CUtensorMap tmdO, const AttnBwdParams p) {
    using Cfg = AttnCfg<HD>;
    __shared__ uint64_t k_full, v_full, s_full, dp_full, p_ready, ds_ready, acc_full, vec_full[2], vec_empty[2];
    __shared__ uint64_t full_bar[Cfg::kKvStages], empty_bar[Cfg::kKvStages], ragged_bar[Cfg::kKvStages];
    __shared__ __align__(16) float vec[2][2][kAttnRows];       // lse (in powers of two) and D of a tile's queries
    __shared__ uint32_t tmem_slot[1];
    __shared__ int abort_word;
    __shared__ AttnTile work;
    volatile int* abort_flag = &abort_word;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *sK = smem, *sV = smem + Cfg::kTile, *ring = smem + 2 * Cfg::kTile;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = threadIdx.x >> 7;

    griddep_launch_dependents();
    if (threadIdx.x == 0) {
        for (uint64_t* bar : {&k_full, &v_full, &s_full, &dp_full, &acc_full}) mbar_init(bar, 1);
        mbar_init(&p_ready, 8);
        mbar_init(&ds_ready, 8);
        for (int i = 0; i < 2; ++i) { mbar_init(&vec_full[i], 1); mbar_init(&vec_empty[i], 8); }
        for (int i = 0; i < Cfg::kKvStages; ++i) { mbar_init(&full_bar[i], 1); mbar_init(&empty_bar[i], 1); mbar_init(&ragged_bar[i], 1); }
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 8) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    griddep_wait();
    const int kv_head = blockIdx.x % p.s.kv_heads, share = p.s.heads / p.s.kv_heads;
    if (warp == 0) {
        const AttnTile t = attn_locate(p.s, blockIdx.x / p.s.kv_heads, kAttnRows, false);
        if (lane == 0) work = t;
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot, t_s = tmem, t_dp = tmem + kAttnRows, t_dv = tmem + 2 * kAttnRows, t_dk = t_dv + HD;
    const int len = work.len, first = work.first, k0 = work.tile * kAttnRows;
    const int lo = attn_first_query_tile(p.s, k0), per_head = len ? attn_end_query_tile(p.s, k0, len) - lo : 0, items = per_head * share;
    const int last = (len - 1) / kAttnRows, last_rows = len - last * kAttnRows;
    const auto tile_of = [&](int it) { return lo + it % per_head; };
    const auto rows_of = [&](int tile) { return tile == last ? last_rows : kAttnRows; };

    if (group == 2) {
        registers_down<kAttnRegsDown>();
        if (warp == 9) {
            if (items && elect_one()) {
                PipeState ps;
                bool ok = true;
                attn_load<HD>(sK, &tmK, &k_full, kv_head, first + k0);
                for (int it = 0; it < items && ok; ++it) {
                    const int head = kv_head * share + it / per_head, row = first + tile_of(it) * kAttnRows;
                    uint64_t* bars = rows_of(tile_of(it)) < kAttnRows ? ragged_bar : full_bar;
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        if (!mbar_wait(&empty_bar[ps.stage], ps.phase ^ 1u, abort_flag)) { ok = false; break; }
                        attn_load<HD>(ring + ps.stage * Cfg::kTile, g ? &tmdO : &tmQ, &bars[ps.stage], head, row);
                        ps.advance(Cfg::kKvStages);
                        if (it == 0 && g == 0) attn_load<HD>(sV, &tmV, &v_full, kv_head, first + k0);
                    }
                }
            }
        } else if (warp == 8) {
            if (items && elect_one()) {
                const int steps = (p.s.head_dim + 15) / 16;
                const uint32_t idesc = make_idesc_bf16(kAttnRows, 16 * steps, false, true, false);
                PipeState ps;
                int q_stage = 0, o_stage = 0, q_next = 0, o_next = 0;
                bool ok = true;
                const auto ready = [&](int& stage) {
                    stage = ps.stage;
                    const bool got = mbar_wait(&full_bar[ps.stage], ps.phase, abort_flag);
                    ps.advance(Cfg::kKvStages);
                    return got;
                };
                const auto at = [&](int stage) { return smem_u32(ring + stage * Cfg::kTile); };
                ok = mbar_wait(&k_full, 0, abort_flag) && ready(q_stage);
                if (ok) {
                    tc_fence_after_sync();
                    attn_mma_columns<HD>(t_s, smem_u32(sK), at(q_stage), steps);
                    umma_commit(&s_full);
                    ok = mbar_wait(&v_full, 0, abort_flag) && ready(o_stage);
                }
                if (ok) {
                    tc_fence_after_sync();
                    attn_mma_columns<HD>(t_dp, smem_u32(sV), at(o_stage), steps);
                    umma_commit(&dp_full);
                }
                for (int it = 0; it < items && ok; ++it) {
                    const int row_steps = (rows_of(tile_of(it)) + 15) / 16;
                    if (!(ok = mbar_wait(&p_ready, it & 1, abort_flag))) break;
                    tc_fence_after_sync();
                    attn_mma_rows(t_dv, t_s, t_s + 64, at(o_stage), idesc, row_steps, it != 0);
                    umma_commit(&empty_bar[o_stage]);
                    if (it + 1 < items) {
                        if (!(ok = ready(q_next))) break;
                        tc_fence_after_sync();
                        attn_mma_columns<HD>(t_s, smem_u32(sK), at(q_next), steps);
                        umma_commit(&s_full);
                    }
                    if (!(ok = mbar_wait(&ds_ready, it & 1, abort_flag))) break;
                    tc_fence_after_sync();
                    attn_mma_rows(t_dk, t_dp, t_dp + 64, at(q_stage), idesc, row_steps, it != 0);
                    umma_commit(it + 1 < items ? &empty_bar[q_stage] : &acc_full);
                    if (it + 1 < items) {
                        if (!(ok = ready(o_next))) break;
                        tc_fence_after_sync();
                        attn_mma_columns<HD>(t_dp, smem_u32(sV), at(o_next), steps);
                        umma_commit(&dp_full);
                    }
                    q_stage = q_next;
                    o_stage = o_next;
                }
            }
        } else if (warp == 10) {
            uint32_t phases = 0;                             // of the stages' ragged barriers
            for (int it = 0; it < items; ++it) {
                const int head = kv_head * share + it / per_head, tile = tile_of(it), rows = rows_of(tile), slot = it & 1;
                const size_t at = static_cast<size_t>(head) * p.s.b + first + tile * kAttnRows;
                if (it > 1 && !warp_wait(&vec_empty[slot], ((it >> 1) & 1) ^ 1u, abort_flag)) break;
#pragma unroll
                for (int i = lane; i < kAttnRows; i += 32) {
                    vec[slot][0][i] = i < rows ? __uint_as_float(ld_u32(p.lse + at + i)) * kLog2e : 0.0f;
                    vec[slot][1][i] = i < rows ? __uint_as_float(ld_u32(p.delta + at + i)) : 0.0f;
                }
                warp_arrive(&vec_full[slot]);
                if (rows < kAttnRows) {
                    bool ok = true;
                    for (int g = 0; g < 2 && ok; ++g) {
                        const int stage = (2 * it + g) % Cfg::kKvStages;
                        if (!(ok = warp_wait(&ragged_bar[stage], (phases >> stage) & 1, abort_flag))) break;
                        phases ^= 1u << stage;
                        attn_zero_rows<HD>(ring + stage * Cfg::kTile, rows);
                        warp_arrive(&full_bar[stage]);
                    }
                    if (!ok) break;
                }
            }
        }
    } else {
        registers_up<kAttnRegsUp>();
        const int key = k0 + (threadIdx.x & 127);
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16, half = 64 * group;
        const uint32_t s_row = t_s + lanes + half, dp_row = t_dp + lanes + half;
        bool ok = items > 0;
        for (int it = 0; it < items; ++it) {
            const int q0 = tile_of(it) * kAttnRows, slot = it & 1;
            const bool edge = (p.s.causal && q0 == k0) || q0 + kAttnRows > len || (p.s.window && q0 + kAttnRows - 1 - k0 >= p.s.window);
            // queries [c_lo, c_hi) of this group's 64 see the key
            const int c_lo = p.s.causal ? key - q0 - static_cast<int>(half) : 0;
            const int c_hi = min(len, p.s.window ? min(key, len) + p.s.window : len) - q0 - static_cast<int>(half);
            if (!(ok = warp_wait(&vec_full[slot], (it >> 1) & 1, abort_flag) && warp_wait(&s_full, it & 1, abort_flag))) break;
            tc_fence_after_sync();
            uint32_t v[64], w[32];
            tmem_ld_32(s_row, v);
            tmem_ld_32(s_row + 32, v + 32);
            tmem_ld_wait();
            const uint32_t vec_lse = smem_u32(&vec[slot][0][half]), vec_delta = smem_u32(&vec[slot][1][half]);
            const Pair by = both(p.s.scale);
#pragma unroll
            for (int c = 0; c < 64; c += 4) {
                const float4 e = ld_shared_v4(vec_lse + 4 * c);
                const Pair x0 = fma2(pair(v[c], v[c + 1]), by, pair(-e.x, -e.y)), x1 = fma2(pair(v[c + 2], v[c + 3]), by, pair(-e.z, -e.w));
                v[c] = __float_as_uint(exp2_fast(low(x0)));
                v[c + 1] = __float_as_uint(exp2_fast(high(x0)));
                v[c + 2] = __float_as_uint(exp2_fast(low(x1)));
                v[c + 3] = __float_as_uint(exp2_fast(high(x1)));
            }
            if (edge) {
#pragma unroll
                for (int c = 0; c < 64; ++c)
                    if (c < c_lo || c >= c_hi) v[c] = 0u;
            }
#pragma unroll
            for (int c = 0; c < 64; c += 2) w[c >> 1] = pack_bf16x2(__uint_as_float(v[c]), __uint_as_float(v[c + 1]));
            tmem_st_32(s_row, w);
            tmem_st_wait();
            tc_fence_before_sync();
            warp_arrive(&p_ready);
            if (!(ok = warp_wait(&dp_full, it & 1, abort_flag))) break;
            tc_fence_after_sync();
            uint32_t g[64];
            tmem_ld_32(dp_row, g);
            tmem_ld_32(dp_row + 32, g + 32);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 64; c += 4) {
                const float4 d = ld_shared_v4(vec_delta + 4 * c);
                const Pair y0 = mul2(pair(v[c], v[c + 1]), add2(pair(g[c], g[c + 1]), pair(-d.x, -d.y)));
                const Pair y1 = mul2(pair(v[c + 2], v[c + 3]), add2(pair(g[c + 2], g[c + 3]), pair(-d.z, -d.w)));
                w[c >> 1] = pack_bf16x2(low(y0), high(y0));
                w[(c >> 1) + 1] = pack_bf16x2(low(y1), high(y1));
            }
            if (edge) {                                     // (zero times what a row of no sequence holds)
#pragma unroll
                for (int c = 0; c < 64; ++c)
                    if (c < c_lo || c >= c_hi) w[c >> 1] &= c & 1 ? 0x0000FFFFu : 0xFFFF0000u;
            }
            tmem_st_32(dp_row, w);
            tmem_st_wait();
            tc_fence_before_sync();
            warp_arrive(&ds_ready);
            warp_arrive(&vec_empty[slot]);
        }
        if (ok && warp_wait(&acc_full, 0, abort_flag)) {
            tc_fence_after_sync();
            const size_t row = static_cast<size_t>(first) + k0;
            uint16_t* out = group ? p.dK + row * p.dk_ld : p.dV + row * p.dv_ld;
            attn_store<HD>((group ? t_dk : t_dv) + lanes, 0, HD, group ? p.grad_scale : 1.0f, group ? sK : sV, out + kv_head * p.s.head_dim,
                           group ? p.dk_ld : p.dv_ld, len - k0, p.s.head_dim);
        }
        tc_fence_before_sync();
    }
    if (*abort_flag) drain_after_abort();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

// dQ of 128 queries, which lie on the lanes; both groups work on every tile of keys, 64 keys each.  S is formed a tile ahead in the other of
// two places; dS takes the place of S.
template <int HD>
__global__ void __launch_bounds__(kAttnThreads, 1)
attention_bwd_q_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                       const __grid_constant__ CUtensorMap tmdO, const AttnBwdParams p) {
    using Cfg = AttnCfg<HD>;
    __shared__ uint64_t q_full, do_full, s_full[2], dp_full, ds_ready, acc_full, ragged_bar;
    __shared__ uint64_t full_bar[Cfg::kStages], empty_bar[Cfg::kStages];
    __shared__ uint32_t tmem_slot[1];
    __shared__ int abort_word;
    __shared__ AttnTile work;
    volatile int* abort_flag = &abort_word;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *sQ = smem, *sdO = smem + Cfg::kTile, *ring = smem + 2 * Cfg::kTile;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = threadIdx.x >> 7;

    griddep_launch_dependents();
    if (threadIdx.x == 0) {
        for (uint64_t* bar : {&q_full, &do_full, &s_full[0], &s_full[1], &dp_full, &acc_full, &ragged_bar}) mbar_init(bar, 1);
        mbar_init(&ds_ready, 8);
        for (int i = 0; i < Cfg::kStages; ++i) { mbar_init(&full_bar[i], 1); mbar_init(&empty_bar[i], 1); }
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 8) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    griddep_wait();
    const int head = blockIdx.x % p.s.heads, kv_head = head / (p.s.heads / p.s.kv_heads);
    if (warp == 0) {
        const AttnTile t = attn_locate(p.s, blockIdx.x / p.s.heads, kAttnRows, p.s.causal);
        if (lane == 0) work = t;
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot, t_dp = tmem + 2 * kAttnRows, t_dq = tmem + 3 * kAttnRows;
    const int len = work.len, first = work.first, q0 = work.tile * kAttnRows;
    const int lo = attn_first_key_tile(p.s, q0), items = len ? attn_end_key_tile(p.s, q0, len) - lo : 0;
    const int last = (len - 1) / kAttnRows, last_rows = len - last * kAttnRows;
    const bool ragged = items && lo + items == last + 1 && last_rows < kAttnRows;     // the last item is the sequence's ragged end

    if (group == 2) {
        registers_down<kAttnRegsDown>();
        if (warp == 9) {
            if (items && elect_one()) {
                PipeState ps;
                bool ok = true;
                attn_load<HD>(sQ, &tmQ, &q_full, head, first + q0);
                for (int it = 0; it < items && ok; ++it) {
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        if (!mbar_wait(&empty_bar[ps.stage], ps.phase ^ 1u, abort_flag)) { ok = false; break; }
                        attn_load<HD>(ring + ps.stage * Cfg::kTile, g ? &tmV : &tmK, ragged && g == 0 && it + 1 == items ? &ragged_bar : &full_bar[ps.stage], kv_head, first + (lo + it) * kAttnRows);
                        ps.advance(Cfg::kStages);
                        if (it == 0 && g == 0) attn_load<HD>(sdO, &tmdO, &do_full, head, first + q0);
                    }
                }
            }
        } else if (warp == 8) {
            if (items && elect_one()) {
                const int steps = (p.s.head_dim + 15) / 16;
                const uint32_t idesc = make_idesc_bf16(kAttnRows, 16 * steps, false, true, false);
                PipeState ps;
                int k_stage = 0, k_next = 0, v_stage = 0;
                const auto ready = [&](int& stage) {
                    stage = ps.stage;
                    const bool got = mbar_wait(&full_bar[ps.stage], ps.phase, abort_flag);
                    ps.advance(Cfg::kStages);
                    return got;
                };
                const auto at = [&](int stage) { return smem_u32(ring + stage * Cfg::kTile); };
                bool ok = mbar_wait(&q_full, 0, abort_flag) && ready(k_stage);
                if (ok) {
                    tc_fence_after_sync();
                    attn_mma_columns<HD>(tmem, smem_u32(sQ), at(k_stage), steps);
                    umma_commit(&s_full[0]);
                    ok = mbar_wait(&do_full, 0, abort_flag) && ready(v_stage);
                }
                if (ok) {
                    tc_fence_after_sync();
                    attn_mma_columns<HD>(t_dp, smem_u32(sdO), at(v_stage), steps);
                    umma_commit(&dp_full);
                    umma_commit(&empty_bar[v_stage]);
                }
                for (int it = 0; it < items && ok; ++it) {
                    const uint32_t t_s = tmem + (it & 1) * kAttnRows;
                    const int rows = ragged && it + 1 == items ? last_rows : kAttnRows;
                    if (it + 1 < items) {
                        if (!(ok = ready(k_next))) break;
                        tc_fence_after_sync();
                        attn_mma_columns<HD>(tmem + ((it + 1) & 1) * kAttnRows, smem_u32(sQ), at(k_next), steps);
                        umma_commit(&s_full[(it + 1) & 1]);
                    }
                    if (!(ok = mbar_wait(&ds_ready, it & 1, abort_flag))) break;
                    tc_fence_after_sync();
                    attn_mma_rows(t_dq, t_s, t_s + 64, at(k_stage), idesc, (rows + 15) / 16, it != 0);
                    umma_commit(it + 1 < items ? &empty_bar[k_stage] : &acc_full);
                    if (it + 1 < items) {
                        if (!(ok = ready(v_stage))) break;
                        tc_fence_after_sync();
                        attn_mma_columns<HD>(t_dp, smem_u32(sdO), at(v_stage), steps);
                        umma_commit(&dp_full);
                        umma_commit(&empty_bar[v_stage]);
                    }
                    k_stage = k_next;
                }
            }
        } else if (warp == 10 && ragged) {
            const int stage = 2 * (items - 1) % Cfg::kStages;
            if (warp_wait(&ragged_bar, 0, abort_flag)) {
                attn_zero_rows<HD>(ring + stage * Cfg::kTile, last_rows);
                warp_arrive(&full_bar[stage]);
            }
        }
    } else {
        registers_up<kAttnRegsUp>();
        const int row = threadIdx.x & 127, i = q0 + row;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16, half = 64 * group;
        float lse = 0.0f, delta = 0.0f;
        if (items && i < len) {
            const size_t at = static_cast<size_t>(head) * p.s.b + first + i;
            lse = __uint_as_float(ld_u32(p.lse + at)) * kLog2e;
            delta = __uint_as_float(ld_u32(p.delta + at));
        }
        const Pair by = both(p.s.scale), less = both(-lse), minus = both(-delta);
        bool ok = items > 0;
        for (int it = 0; it < items; ++it) {
            const int c0 = (lo + it) * kAttnRows;
            const bool edge = (p.s.causal ? c0 + kAttnRows - 1 > q0 : c0 + kAttnRows > len) || (p.s.window && q0 + kAttnRows - 1 - c0 >= p.s.window);
            const int c_hi = (p.s.causal ? min(i + 1, len) : len) - c0 - static_cast<int>(half);
            const int c_lo = p.s.window ? i - p.s.window + 1 - c0 - static_cast<int>(half) : 0;
            const uint32_t s_row = tmem + (it & 1) * kAttnRows + lanes + half, dp_row = t_dp + lanes + half;
            if (!(ok = warp_wait(&s_full[it & 1], (it >> 1) & 1, abort_flag))) break;
            tc_fence_after_sync();
            uint32_t v[64], g[64];
            tmem_ld_32(s_row, v);
            tmem_ld_32(s_row + 32, v + 32);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 64; c += 2) {
                const Pair x = fma2(pair(v[c], v[c + 1]), by, less);
                v[c] = __float_as_uint(exp2_fast(low(x)));
                v[c + 1] = __float_as_uint(exp2_fast(high(x)));
            }
            if (!(ok = warp_wait(&dp_full, it & 1, abort_flag))) break;
            tc_fence_after_sync();
            tmem_ld_32(dp_row, g);
            tmem_ld_32(dp_row + 32, g + 32);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 64; c += 2) {
                const Pair y = mul2(pair(v[c], v[c + 1]), add2(pair(g[c], g[c + 1]), minus));
                v[c >> 1] = pack_bf16x2(low(y), high(y));
            }
            if (edge) {
#pragma unroll
                for (int c = 0; c < 64; ++c)
                    if (c < c_lo || c >= c_hi) v[c >> 1] &= c & 1 ? 0x0000FFFFu : 0xFFFF0000u;
            }
            tmem_st_32(s_row, v);
            tmem_st_wait();
            tc_fence_before_sync();
            warp_arrive(&ds_ready);
        }
        if (ok && warp_wait(&acc_full, 0, abort_flag)) {
            tc_fence_after_sync();
            const size_t at = static_cast<size_t>(first) + q0;
            attn_store<HD>(t_dq + lanes, group * HD / 2, (group + 1) * HD / 2, p.grad_scale, group ? sdO : sQ,
                           p.dQ + at * p.dq_ld + head * p.s.head_dim, p.dq_ld, len - q0, p.s.head_dim);
        }
        tc_fence_before_sync();
    }
    if (*abort_flag) drain_after_abort();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

// =====================================================================================
// Rotation by positions: of the first 2 n columns of every head, the pairs (u_i, v_i) become
//   factor (u cos a - v sin a, v cos a + u sin a),   a = position frequency_i
// (backward: the transposed map, sin negated).  Pairs are columns i and n + i, or (PAIRS) 2 i and 2 i + 1.
// What bounds it is HBM; an angle is formed once per token and pair, by one thread of the block that has the token, for all heads.  Angles are
// taken in whole turns in fp64, of which the nearest whole number is left out: in fp32 a position of 10^6 would be 0.06 rad off.
// =====================================================================================
struct RotaryParams {
    const void *src[2];
    void* dst[2];
    int src_ld[2], dst_ld[2], heads[2];
    int b, head_dim, n, tokens;           // n: pairs of a head; tokens of a block
    int copy;                             // columns behind the rotated ones are copied (not where the output is the input)
    float factor, sign;
    const int* positions;
    const double* frequencies;
};
// `N` values of a row, as fp32
template <int TYPE, int N>
__device__ __forceinline__ void load_n(const void* base, size_t at, float (&x)[N]) {
    if constexpr (N == 8) {
        const V8 v = load8<TYPE>(base, at, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = low(v.p[i]); x[2 * i + 1] = high(v.p[i]); }
    } else if constexpr (TYPE == kTypeBf16) {
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
        uint32_t w[(N + 1) / 2];
        if constexpr (N == 4) { const uint2 v = ld_v2(p); w[0] = v.x; w[1] = v.y; }
        else if constexpr (N == 2) w[0] = ld_u32(p);
        else w[0] = ld_u16(p);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    } else {
        const float* p = static_cast<const float*>(base) + at;
        if constexpr (N == 4) {
            const uint4 v = ld_v4(p);
            x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
        } else if constexpr (N == 2) {
            const uint2 v = ld_v2(p);
            x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y);
        } else x[0] = __uint_as_float(ld_u32(p));
    }
}
template <int TYPE, int N>
__device__ __forceinline__ void store_n(void* base, size_t at, const float (&x)[N]) {
    if constexpr (N == 8) {
        store8<TYPE>(base, at, V8{{pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7])}});
    } else if constexpr (TYPE == kTypeBf16) {
        uint16_t* p = static_cast<uint16_t*>(base) + at;
        if constexpr (N == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
        else if constexpr (N == 2) *reinterpret_cast<uint32_t*>(p) = pack_bf16x2(x[0], x[1]);
        else *p = to_bf16(x[0]);
    } else {
        float* p = static_cast<float*>(base) + at;
        if constexpr (N == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
        else if constexpr (N == 2) *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
        else *p = x[0];
    }
}
constexpr int kRotaryThreads = 256, kRotaryTable = 2048;       // angles of a block
// A thread takes N values at a time: N pairs' two halves, or N / 2 neighbouring pairs.
template <int TYPE, bool PAIRS, int N>
__global__ void __launch_bounds__(kRotaryThreads)
rotary_kernel(const RotaryParams p) {
    __shared__ float cosine[kRotaryTable], sine[kRotaryTable];
    griddep_launch_dependents();
    griddep_wait();
    const int token0 = blockIdx.x * p.tokens, tokens = min(p.tokens, p.b - token0);
    for (int i = threadIdx.x; i < tokens * p.n; i += kRotaryThreads) {
        const int t = i / p.n;
        const uint2 f = ld_v2(p.frequencies + (i - t * p.n));
        const double turns = static_cast<double>(static_cast<int>(ld_u32(p.positions + token0 + t))) *
                             (__hiloint2double(static_cast<int>(f.y), static_cast<int>(f.x)) * 0.15915494309189535);
        float s, c;
        sincospif(2.0f * static_cast<float>(turns - rint(turns)), &s, &c);
        cosine[i] = c * p.factor;
        sine[i] = s * p.factor * p.sign;
    }
    __syncthreads();
    constexpr int kPairs = PAIRS ? N / 2 : N;                  // of a task
    const int turned = p.n / kPairs, rest = p.copy ? (p.head_dim - 2 * p.n) / N : 0, per_head = turned + rest;
    const int per_token = (p.heads[0] + p.heads[1]) * per_head;
    for (int task = threadIdx.x; task < tokens * per_token; task += kRotaryThreads) {
        const int t = task / per_token, in_token = task - t * per_token;
        int head = in_token / per_head;
        const int u = in_token - head * per_head, which = head >= p.heads[0];
        if (which) head -= p.heads[0];
        const size_t row = static_cast<size_t>(token0 + t);
        const void* src = which ? p.src[1] : p.src[0];
        void* dst = which ? p.dst[1] : p.dst[0];
        const size_t from = row * (which ? p.src_ld[1] : p.src_ld[0]) + head * p.head_dim, to = row * (which ? p.dst_ld[1] : p.dst_ld[0]) + head * p.head_dim;
        float x[N], y[N];
        if (u >= turned) {
            const int col = 2 * p.n + (u - turned) * N;
            load_n<TYPE, N>(src, from + col, x);
            store_n<TYPE, N>(dst, to + col, x);
            continue;
        }
        const float *c = cosine + t * p.n + u * kPairs, *s = sine + t * p.n + u * kPairs;
        if (PAIRS) {
            load_n<TYPE, N>(src, from + u * N, x);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                y[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * s[i];
                y[2 * i + 1] = x[2 * i + 1] * c[i] + x[2 * i] * s[i];
            }
            store_n<TYPE, N>(dst, to + u * N, y);
        } else {
            float z[N];
            load_n<TYPE, N>(src, from + u * N, x);
            load_n<TYPE, N>(src, from + p.n + u * N, z);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                y[i] = x[i] * c[i] - z[i] * s[i];
                z[i] = z[i] * c[i] + x[i] * s[i];
            }
            store_n<TYPE, N>(dst, to + u * N, y);
            store_n<TYPE, N>(dst, to + p.n + u * N, z);
        }
    }
}

}  // namespace slope
