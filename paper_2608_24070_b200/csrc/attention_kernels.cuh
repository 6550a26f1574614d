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
__device__ __forceinline__ void tmem_st_16(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
// The wait for loads from tensor memory, tied to the registers that they fill, so that nothing that uses these is moved in front of it.
#define SLOPE_TIE8(v, i) "+r"((v)[i]), "+r"((v)[i + 1]), "+r"((v)[i + 2]), "+r"((v)[i + 3]), "+r"((v)[i + 4]), "+r"((v)[i + 5]), "+r"((v)[i + 6]), "+r"((v)[i + 7])
__device__ __forceinline__ void tmem_ld_wait_32(uint32_t* v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : SLOPE_TIE8(v, 0), SLOPE_TIE8(v, 8), SLOPE_TIE8(v, 16), SLOPE_TIE8(v, 24)::"memory");
}
// Nothing but the tie.
__device__ __forceinline__ void tie_32(uint32_t* v) {
    asm volatile("" : SLOPE_TIE8(v, 0), SLOPE_TIE8(v, 8), SLOPE_TIE8(v, 16), SLOPE_TIE8(v, 24)::"memory");
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
    int share, part;                      // query heads of a key head; rows of a sequence, where all are equal
    float per_heads, per_kv_heads, per_share;      // reciprocals
};
struct AttnTile {
    int first, len, tile;                 // the sequence's first row, its length, number of the tile of `rows` rows; len 0: nothing to do
};
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr int kAttnRows = 128;            // rows of a tile of queries or keys
constexpr int kAttnThreads = 384;         // two groups of four warps that compute, one that feeds them
// backward: registers of a thread that computes / that feeds; with 168 at launch the three groups come to 384 x 168.  (us, 4 x 2048 tokens, 40 heads of
// 128, causal: 200 768, 208 747, 216 740; 224, where the warps that feed run out of theirs, 744)
constexpr int kAttnRegsUp = 216, kAttnRegsDown = 72;
static_assert(2 * kAttnRegsUp + kAttnRegsDown == 3 * 168, "shares of the launch's registers");

// x / d and what is left, x >= 0, with the reciprocal at hand (a division takes 100 clocks, and a block has four in front of its first load).
struct AttnQuotient {
    int quotient, rest;
};
__device__ __forceinline__ AttnQuotient attn_divide(int x, int d, float per_d) {
    AttnQuotient r;
    r.quotient = static_cast<int>(static_cast<float>(x) * per_d);
    r.rest = x - r.quotient * d;                                     // (2^-23 of the quotient off, at most, and one)
    while (r.rest < 0) { --r.quotient; r.rest += d; }
    while (r.rest >= d) { ++r.quotient; r.rest -= d; }
    return r;
}
// Tile number `unit` of the call, the last tile of a sequence first where later rows see more keys.  By one whole warp.
template <int ROWS>
__device__ __forceinline__ AttnTile attn_locate(const AttnShape& s, int unit, bool last_first) {
    constexpr int rows = ROWS;
    const int lane = threadIdx.x & 31;
    AttnTile t{0, 0, 0};
    int n = 0, rank = 0;
    if (!s.starts) {
        const int tiles = (s.part - 1) / rows + 1;
        const AttnQuotient q = attn_divide(unit, tiles, 1.0f / static_cast<float>(tiles));
        rank = q.rest;
        t.first = q.quotient * s.part;
        t.len = s.lengths ? min(max(s.lengths[q.quotient], 0), s.part) : s.part;
        n = (t.len + rows - 1) / rows;
        if (rank >= n) t.len = 0;
    } else {
        int before = 0;
        for (int i0 = 0; i0 < s.sequences; i0 += 32) {
            const int i = i0 + lane;
            int first = 0, len = 0;
            if (i < s.sequences) {
                first = min(max(s.starts[i], 0), s.b);
                len = max(min(max(s.starts[i + 1], 0), s.b) - first, 0);      // (both ends held first: the difference of any two ints need not be one)
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
    // of a block of dQ: places for K, which stay until dQ has them, and for V
    static constexpr int kKeys = HD == 128 ? 3 : 4, kValues = kStages - kKeys;
};
// What a block of dK and dV has beside its tiles ...
template <int HD, int STAGES>
struct alignas(128) AttnKvShared {
    static constexpr int kLse = HD == 64 ? 2 : 1;
    uint4 minus_d[kAttnRows];             // of a tile's queries: -D / 2 as a sum of three bf16 values, zeros behind them
    uint4 ones[8];                        // eight rows of three ones
    float lse[kLse][kAttnRows];           // in powers of two; with two places (which 64 columns leave room for) the groups' powers need not wait for one another:
                                          // 4 x 4096 tokens, 16 heads, full, 1160 -> 1110 us
    // completed by one arrival, by two (the scores, and what belongs to their queries), by a group's four warps
    uint64_t k_full, v_full, acc_full, d_full, dp_full[2], full[STAGES], empty[STAGES], ragged[STAGES];
    uint64_t s_full[2];
    uint64_t s_read[2], pairs_full[2][2], powers_done[kLse];
    uint32_t tmem;
    int abort_word;
    AttnTile work;
};
// ... and that of dQ
template <int KEYS, int VALUES>
struct alignas(128) AttnQShared {
    // completed by one arrival, by a group's four warps
    uint64_t q_full, do_full, s_full[2], dp_full[2], acc_full, ragged_bar, k_full[KEYS], k_empty[KEYS], v_full[VALUES], v_empty[VALUES];
    uint64_t dp_read[2], ds_ready[2];
    uint32_t tmem;
    int abort_word;
    AttnTile work;
};
template <int HD>
union AttnBwdShared {
    AttnKvShared<HD, AttnCfg<HD>::kStages> keys;
    AttnQShared<AttnCfg<HD>::kKeys, AttnCfg<HD>::kValues> queries;
};
// The forward pass: TILES tiles of queries a block; with one, two blocks share an SM.
template <int HD, int TILES>
struct AttnFwdCfg {
    static constexpr int kTile = AttnCfg<HD>::kTile, kBlocks = 3 - TILES, kThreads = 128 * (TILES + 1);
    static constexpr int kStages = TILES == 2 ? AttnCfg<HD>::kStages : HD == 128 ? 2 : 5, kSmem = (TILES + kStages) * kTile + 1024;
    // registers of a thread that computes / that feeds, out of 168 or 128 a thread at launch
    static constexpr int kUp = 208, kDown = TILES == 2 ? 88 : 48;
    static_assert(TILES * kUp + kDown == (TILES + 1) * (TILES == 2 ? 168 : 128), "shares of the launch's registers");
};
template <int HD>
__device__ __forceinline__ void attn_load(uint8_t* tile, const CUtensorMap* tm, uint64_t* bar, int head, int row) {
    mbar_expect_tx(bar, AttnCfg<HD>::kTile);
#pragma unroll
    for (int c = 0; c < AttnCfg<HD>::kChunks; ++c) tma_load_3d(tile + c * kAttnChunk, tm, bar, 64 * c, head, row);
}
// Descriptors of a tile read with its columns as the reduction, and with its rows; a step of 16 along either is a constant further on in the
// address field.  (What the one thread computes per product it cannot issue meanwhile: with descriptors made from addresses each time, 8 products took it
// 450 to 600 clocks, the time that they run.)
__device__ __forceinline__ uint64_t attn_column_desc(const uint8_t* tile) { return make_smem_desc(smem_u32(tile), 16, 1024, kSwizzle128B); }
__device__ __forceinline__ uint64_t attn_row_desc(const uint8_t* tile) { return make_smem_desc(smem_u32(tile), kAttnChunk, 1024, kSwizzle128B); }
// D[128 x 128] (+)= A B^T over the columns of a head, `steps` of 16
template <int HD>
__device__ __forceinline__ void attn_mma_columns(uint32_t d, uint64_t a, uint64_t b, int steps, bool accumulate = false) {
    constexpr uint32_t idesc = make_idesc_bf16(kAttnRows, kAttnRows, false, false, false);
    const auto product = [&](int k) {
        const uint32_t off = ((k >> 2) * kAttnChunk + (k & 3) * 32) >> 4;
        umma_bf16(d, a + off, b + off, idesc, accumulate || k != 0);
    };
    if (steps == HD / 16) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) product(k);
    } else {
#pragma unroll 1
        for (int k = 0; k < steps; ++k) product(k);
    }
}
// D[128 x head] (+)= A B over 64 of a tile's rows, `steps` of 16; A from tensor memory, 32 values every CHUNK columns
template <int CHUNK = 16>
__device__ __forceinline__ void attn_mma_rows(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, int steps, bool accumulate) {
    const auto product = [&](int k) { umma_bf16_ts(d, a + CHUNK * (k >> 1) + 8 * (k & 1), b + k * (2048 >> 4), idesc, accumulate || k != 0); };
    if (steps >= 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) product(k);
    } else {
#pragma unroll 1
        for (int k = 0; k < steps; ++k) product(k);
    }
}
// ... over all of its rows: the first 64 values of A at `a0`, the others at `a1`
__device__ __forceinline__ void attn_mma_rows(uint32_t d, uint32_t a0, uint32_t a1, uint64_t b, uint32_t idesc, int steps, bool accumulate) {
    attn_mma_rows(d, a0, b, idesc, steps, accumulate);
    attn_mma_rows(d, a1, b + (64 * 128 >> 4), idesc, steps - 4, true);
}
// of a product whose B is [rows x head]
__device__ __forceinline__ uint32_t attn_row_idesc(int head_dim) { return make_idesc_bf16(kAttnRows, (head_dim + 15) & ~15, false, true, false); }
// Bits [lo, hi) of 32: which of 32 columns are seen.  (A bit of a register as a condition is half of what two comparisons cost.)
__device__ __forceinline__ uint32_t attn_bits(int lo, int hi) {
    const uint32_t below_hi = hi >= 32 ? 0xFFFFFFFFu : hi <= 0 ? 0u : (1u << hi) - 1u, below_lo = lo >= 32 ? 0xFFFFFFFFu : lo <= 0 ? 0u : (1u << lo) - 1u;
    return below_hi & ~below_lo;
}
// Barriers [begin, end), by a warp
__device__ __forceinline__ void attn_barriers(uint64_t* begin, uint64_t* end, uint32_t count) {
    for (uint64_t* bar = begin + (threadIdx.x & 31); bar < end; bar += 32) mbar_init(bar, count);
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
// This warp's 32 rows of an accumulator, COLS columns of the head from `c0` on, times `mul`, to bf16 rows in global memory; `stage` is shared memory of
// 128 rows x HD columns.  Straight from the lanes a store would touch a row per lane.
template <int HD, int COLS>
__device__ __forceinline__ void attn_store(uint32_t t_row, int c0, float mul, uint8_t* stage, uint16_t* out, int ld, int rows, int head_dim) {
    const int lane = threadIdx.x & 31, row0 = 32 * ((threadIdx.x >> 5) & 3);
    const uint32_t base = smem_u32(stage) + row0 * HD * 2;
    const int c1 = min(c0 + COLS, head_dim);
#pragma unroll 1
    for (int c = c0; c < c1; c += 32) {
        uint32_t v[32];
        tmem_ld_32(t_row + c, v);
        tmem_ld_wait_32(v);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(__uint_as_float(v[8 * u + 2 * i]) * mul, __uint_as_float(v[8 * u + 2 * i + 1]) * mul);
            st_shared_v4(base + lane * HD * 2 + (((c >> 3) + u) ^ (lane & 7)) * 16, make_uint4(w[0], w[1], w[2], w[3]));
        }
    }
    __syncwarp();
    // `kUnits` lanes take 16 bytes each of a row
    constexpr int kUnits = COLS / 8, kRows = 32 / kUnits;
    const int u = (c0 >> 3) + lane % kUnits, r0 = lane / kUnits;
    if (8 * u >= c1) return;
    uint16_t* to = out + static_cast<size_t>(row0 + r0) * ld + 8 * u;
#pragma unroll 4
    for (int r = r0; r < min(32, rows - row0); r += kRows, to += static_cast<size_t>(kRows) * ld)
        *reinterpret_cast<uint4*>(to) = lds_v4(base + r * HD * 2 + (u ^ (r & 7)) * 16);
}
// Waits that are often over when they begin: a test takes 40 clocks, a try with a limit of its own 75.
__device__ __forceinline__ bool attn_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return mbar_test(bar, parity) || mbar_wait(bar, parity, abort_flag);
}
// The outcome is the same for all lanes: what follows is done by whole warps.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xFFFFFFFFu, attn_wait(bar, parity, abort_flag));
}
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// =====================================================================================
// Forward.  One CTA takes a tile of 128 queries of a head, or two, one per group of four warps, and walks the tiles of keys once:
//   S = Q K^T (tensor memory) -> the group that owns the tile takes a row per thread: P = 2^(S - m) and its sum l, m a reference for the
//   row's maximum -> P as bf16 over S -> O += P V (A from tensor memory).
// While one group (of this block or of the other on its SM) forms its P the tensor cores work for the other; one warp issues the products of both in turn, which keeps the groups half a period
// apart, so that each has the special-function unit for itself.  P is handed over in two halves: the first is multiplied while the second is formed.
// m follows the true maximum only where that is more than 2^16 ahead, when the thread rescales O and l itself: O / l does not depend on m, a value up
// to 2^16 is as exact as one up to 1 in fp32 and bf16, and O is not touched in most steps.
// P is rounded to bf16 as an operand (2^-9 relative on average, as any operand of these products); l sums the unrounded values in fp32.
// Warps 0-3 (4-7): queries 0-127 (128-255); of the four behind them the first: MMAs; the second: barriers and loads; the third: zeros behind the
// sequence's last row of V.  Measured: 4 x 2048 tokens, 40 heads of 128, causal, 190 us = 909 TFLOP/s in bursts, 217 in long runs (the same number of
// cycles, at the power limiter's clock); 4 x 4096, 16 heads, all tokens, 513 us = 1072; 8 x 1024, 12 heads of 64 35.2 us = 366.
// =====================================================================================
constexpr float kAttnSlack = 16.0f;
// A row's 128 scores from tensor memory and their maximum.  EDGE: those outside [lo, hi) are minus infinity.  (Two instances: as a condition inside,
// the comparisons were carried out for every tile and cost a third of what the powers of two do.)
template <bool EDGE>
__device__ __forceinline__ float attn_scores(uint32_t s_row, uint32_t (&v)[kAttnRows], int lo, int hi) {
#pragma unroll
    for (int c = 0; c < kAttnRows; c += 32) tmem_ld_32(s_row + c, v + c);
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int c = 0; c < kAttnRows; c += 32) {
        if (c == 0) tmem_ld_wait_32(v);
        else tie_32(v + c);
        if (EDGE) {
            const uint32_t bits = attn_bits(lo - c, hi - c);
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (!(bits >> k & 1u)) v[c + k] = 0xFF800000u;
        }
#pragma unroll
        for (int k = c; k < c + 32; k += 2) top[(k >> 1) & 3] = max3(top[(k >> 1) & 3], __uint_as_float(v[k]), __uint_as_float(v[k + 1]));
    }
    return fmaxf(max3(top[0], top[1], top[2]), top[3]);
}
// 64 scores -> 2^(v by + less) in bf16 pairs; what they were before the rounding is added to `sum`
__device__ __forceinline__ void attn_probabilities(const uint32_t* v, uint32_t (&w)[32], float by, float less, Pair (&sum)[2]) {
#pragma unroll
    for (int c = 0; c < 64; c += 2) {
        const Pair x = fma2(pair(v[c], v[c + 1]), both(by), both(less));
        const Pair e = pair(exp2_fast(low(x)), exp2_fast(high(x)));
        sum[(c >> 1) & 1] = add2(sum[(c >> 1) & 1], e);
        w[c >> 1] = pack_bf16x2(low(e), high(e));
    }
}

struct AttnFwdParams {
    AttnShape s;
    uint16_t* O;
    float* lse;
    int o_ld;
};
template <int HD, int TILES>
__global__ void __launch_bounds__(AttnFwdCfg<HD, TILES>::kThreads, AttnFwdCfg<HD, TILES>::kBlocks)
attention_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const AttnFwdParams p) {
    using Cfg = AttnFwdCfg<HD, TILES>;
    // barriers completed by one arrival, by a group's four warps
    __shared__ struct {
        uint64_t q_full[TILES], s_full[TILES], pv_done[TILES], o_full[TILES], full_bar[Cfg::kStages], empty_bar[Cfg::kStages], ragged_bar;
        uint64_t s_read[TILES], p_full[TILES][2], end[1];
    } sh;
    auto &q_full = sh.q_full, &s_full = sh.s_full, &pv_done = sh.pv_done, &o_full = sh.o_full, &s_read = sh.s_read;
    auto &full_bar = sh.full_bar, &empty_bar = sh.empty_bar;
    auto& p_full = sh.p_full;
    uint64_t& ragged_bar = sh.ragged_bar;
    __shared__ uint32_t tmem_slot[1];
    __shared__ int abort_word;
    __shared__ AttnTile work;
    volatile int* abort_flag = &abort_word;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* ring = smem + TILES * Cfg::kTile;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = threadIdx.x >> 7;

    // (behind the allocation: a dependent block that took the tensor memory first would wait for this grid, and this block for the memory)
    if (warp == 4 * TILES) {
        tmem_alloc(tmem_slot, 256 * TILES);
        tmem_relinquish();
        griddep_launch_dependents();
    }
    const AttnQuotient unit = attn_divide(blockIdx.x, p.s.heads, p.s.per_heads);
    const int head = unit.rest, kv_head = attn_divide(head, p.s.share, p.s.per_share).quotient;
    // the warp that loads sets the barriers up, a lane each, and has the first tiles on their way before the others go on
    if (warp == 4 * TILES + 1) {
        attn_barriers(sh.q_full, sh.s_read, 1);
        attn_barriers(sh.s_read, sh.end, 4);
        if (lane == 0) *abort_flag = 0;
        fence_mbar_init();
        griddep_wait();
        const AttnTile t = attn_locate<TILES * kAttnRows>(p.s, unit.quotient, p.s.causal);
        if (lane == 0) work = t;
        __syncwarp();
        if (t.len && elect_one()) {
            const int q0 = t.tile * TILES * kAttnRows, c0 = attn_first_key_tile(p.s, q0) * kAttnRows;
#pragma unroll
            for (int v = 0; v < TILES; ++v)
                if (q0 + v * kAttnRows < t.len) attn_load<HD>(smem + v * Cfg::kTile, &tmQ, &q_full[v], head, t.first + q0 + v * kAttnRows);
            attn_load<HD>(ring, &tmK, &full_bar[0], kv_head, t.first + c0);
            attn_load<HD>(ring + Cfg::kTile, &tmV, c0 + kAttnRows > t.len ? &ragged_bar : &full_bar[1], kv_head, t.first + c0);
        }
        __syncwarp();
    }
    griddep_wait();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    // S of either tile, then O of either.  P: over the first and third quarter of S; where a head has 64 columns, behind O, so that the next scores wait
    // for these ones to be read only (us, 4 x 4096 tokens, 16 heads, all tokens: over / apart 400 / 376)
    constexpr bool kApart = HD == 64;
    const uint32_t tmem = *tmem_slot;
    const uint32_t o_at = tmem + TILES * kAttnRows;
    const auto p_at = [&](int t, int h) { return kApart ? o_at + TILES * HD + 64 * t + 32 * h : tmem + kAttnRows * t + 64 * h; };
    const int len = work.len, first = work.first, q0 = work.tile * TILES * kAttnRows;
    const int tiles = !len ? 0 : min(TILES, (len - q0 - 1) / kAttnRows + 1);
    // tiles of keys [lo, hi) of each tile of queries and of all
    int lo[TILES], hi[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        lo[t] = attn_first_key_tile(p.s, q0 + t * kAttnRows);
        hi[t] = t < tiles ? attn_end_key_tile(p.s, q0 + t * kAttnRows, len) : lo[t];
    }
    const int begin = lo[0], end = tiles ? max(hi[0], hi[TILES - 1]) : begin;
    // the sequence's last tile of keys, if it is not full and among these
    const int last = (len - 1) / kAttnRows, last_rows = len - last * kAttnRows, ragged = last_rows < kAttnRows && end == last + 1 ? last : -1;

    if (group == TILES) {
        registers_down<Cfg::kDown>();
        if (warp == 4 * TILES + 1) {
            if (elect_one()) {
                PipeState ps;
                bool ok = true;
                for (int j = begin; j < end && ok; ++j) {
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        // (the first are on their way, and may be used and free again by now: nothing to wait for)
                        if (j != begin) {
                            if (!attn_wait(&empty_bar[ps.stage], ps.phase ^ 1u, abort_flag)) { ok = false; break; }
                            attn_load<HD>(ring + ps.stage * Cfg::kTile, v ? &tmV : &tmK, v && j == ragged ? &ragged_bar : &full_bar[ps.stage], kv_head,
                                          first + j * kAttnRows);
                        }
                        ps.advance(Cfg::kStages);
                    }
                }
            }
        } else if (warp == 4 * TILES) {
            if (elect_one()) {
                const int steps = (p.s.head_dim + 15) / 16;
                PipeState ps;                             // of the next tile of the ring to be waited for
                const uint32_t idesc = attn_row_idesc(p.s.head_dim);
                const uint64_t q_desc = attn_column_desc(smem), column_desc = attn_column_desc(ring), row_desc = attn_row_desc(ring);
                uint32_t phase[TILES] = {};
                bool ok = true;
                const auto scores = [&](int t, int stage) {
                    attn_mma_columns<HD>(tmem + t * kAttnRows, q_desc + t * (Cfg::kTile >> 4), column_desc + stage * (Cfg::kTile >> 4), steps);
                    umma_commit(&s_full[t]);
                };
                // the first scores; behind them each step leaves those of the next
                if (begin < end && (ok = attn_wait(&full_bar[ps.stage], ps.phase, abort_flag))) {
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        if (t >= tiles || !(ok = ok && attn_wait(&q_full[t], 0, abort_flag))) continue;
                        tc_fence_after_sync();
                        if (lo[t] <= begin && begin < hi[t]) scores(t, ps.stage);
                    }
                    umma_commit(&empty_bar[ps.stage]);
                    ps.advance(Cfg::kStages);
                }
                for (int j = begin; j < end && ok; ++j) {
                    const int rows = j == ragged ? last_rows : kAttnRows, v_stage = ps.stage;
                    if (!(ok = attn_wait(&full_bar[ps.stage], ps.phase, abort_flag))) break;
                    ps.advance(Cfg::kStages);
                    const int k_stage = ps.stage;
                    if (j + 1 < end) {
                        if (!(ok = attn_wait(&full_bar[ps.stage], ps.phase, abort_flag))) break;
                        ps.advance(Cfg::kStages);
                    }
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        const bool next = lo[t] <= j + 1 && j + 1 < hi[t];
                        if (kApart && next) {
                            if (lo[t] <= j && !(ok = ok && attn_wait(&s_read[t], phase[t], abort_flag))) continue;
                            tc_fence_after_sync();
                            scores(t, k_stage);
                        }
                        if (lo[t] <= j && j < hi[t]) {
                            const uint32_t o = o_at + t * HD;
                            const uint64_t v = row_desc + v_stage * (Cfg::kTile >> 4);
                            if (!(ok = ok && attn_wait(&p_full[t][0], phase[t], abort_flag))) continue;
                            tc_fence_after_sync();
                            attn_mma_rows(o, p_at(t, 0), v, idesc, (rows + 15) / 16, j != lo[t]);
                            if (!(ok = attn_wait(&p_full[t][1], phase[t], abort_flag))) continue;
                            tc_fence_after_sync();
                            attn_mma_rows(o, p_at(t, 1), v + (64 * 128 >> 4), idesc, (rows + 15) / 16 - 4, true);
                            if (kApart) umma_commit(&pv_done[t]);
                            phase[t] ^= 1u;
                            if (j + 1 == hi[t]) umma_commit(&o_full[t]);
                        }
                        if (!kApart && next) scores(t, k_stage);
                    }
                    if (!ok) break;
                    umma_commit(&empty_bar[v_stage]);
                    if (j + 1 < end) umma_commit(&empty_bar[k_stage]);
                }
            }
        } else if (warp == 4 * TILES + 2 && ragged >= 0) {
            const int stage = (2 * (last - begin) + 1) % Cfg::kStages;
            if (warp_wait(&ragged_bar, 0, abort_flag)) {
                attn_zero_rows<HD>(ring + stage * Cfg::kTile, last_rows);
                warp_arrive(&full_bar[stage]);
            }
        }
    } else {
        registers_up<Cfg::kUp>();
        const int t = group, row = threadIdx.x & 127, t0 = q0 + t * kAttnRows, i = t0 + row;       // the query's place in its sequence
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_row = tmem + lanes + t * kAttnRows, o_row = o_at + lanes + t * HD;
        float m = -INFINITY, l = 0.0f;
        uint32_t phase = 0;
        bool ok = t < tiles;
        const float by = p.s.scale;
        const int j_lo = t ? lo[TILES - 1] : lo[0], j_hi = t ? hi[TILES - 1] : hi[0];
        for (int j = j_lo; j < j_hi; ++j) {
            if (!(ok = warp_wait(&s_full[t], phase, abort_flag))) break;
            phase ^= 1u;
            tc_fence_after_sync();
            const int c0 = j * kAttnRows;
            uint32_t v[kAttnRows];
            float now;
            if ((p.s.causal ? c0 + kAttnRows - 1 > t0 : c0 + kAttnRows > len) || (p.s.window && t0 + kAttnRows - 1 - c0 >= p.s.window))
                now = attn_scores<true>(s_row, v, p.s.window ? i - p.s.window + 1 - c0 : 0, (p.s.causal ? min(i + 1, len) : len) - c0) * by;
            else
                now = attn_scores<false>(s_row, v, 0, kAttnRows) * by;
            if (kApart) {
                tc_fence_before_sync();
                warp_arrive(&s_read[t]);
                // the last P V: P is free, O may be rescaled.  (Otherwise it has completed with these scores.)
                if (j != j_lo && !(ok = warp_wait(&pv_done[t], phase, abort_flag))) break;
                tc_fence_after_sync();
            }
            // (a row moves its own m alone: its bits depend on no other row, be it of another sequence or of none; the vote is for the collective loads)
            const bool ahead = now > m + kAttnSlack;
            if (__any_sync(0xFFFFFFFFu, ahead)) {
                const float part = ahead ? exp2_fast(m - now) : 1.0f;
                m = ahead ? now : m;
                l *= part;
#pragma unroll 1
                for (int c = 0; c < (j == j_lo ? 0 : p.s.head_dim); c += 32) {
                    uint32_t o[32];
                    tmem_ld_32(o_row + c, o);
                    tmem_ld_wait_32(o);
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * part);
                    tmem_st_32(o_row + c, o);
                }
            }
            const float less = m == -INFINITY ? 0.0f : -m;
            Pair sum[2] = {0, 0};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t w[32];
                attn_probabilities(v + 64 * h, w, by, less, sum);
                tmem_st_32(p_at(t, h) + lanes, w);
                tmem_st_wait();
                tc_fence_before_sync();
                warp_arrive(&p_full[t][h]);
            }
            const Pair all = add2(sum[0], sum[1]);
            l += low(all) + high(all);
        }
        if (ok && (ok = warp_wait(&o_full[t], 0, abort_flag))) {
            tc_fence_after_sync();
            const size_t at = static_cast<size_t>(first) + t0;
            if (p.lse && i < len) p.lse[static_cast<size_t>(head) * p.s.b + at + row] = m * kLn2 + logf(l);
            // (a row that has seen none but infinitely small scores: 0 / 0)
            attn_store<HD, HD>(o_row, 0, 1.0f / l, smem + t * Cfg::kTile, p.O + at * p.o_ld + head * p.s.head_dim, p.o_ld, len - t0, p.s.head_dim);
        }
        tc_fence_before_sync();
    }
    if (*abort_flag) drain_after_abort();
    __syncthreads();
    if (warp == 4 * TILES) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 256 * TILES);
    }
}

// =====================================================================================
// Backward.  With D = rowsum(dO O), P = 2^(scale S - lse) and dS = P (dO V^T - D):
//   dV = P^T dO,   dK = scale dS^T Q (sums over queries and over the heads that share a key head),   dQ = scale dS K (a sum over keys).
// Blocks of keys and blocks of queries form S and dP = dO V^T once each: with two fifths more products nothing is added up in memory, and every sum has
// a fixed order.
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
    constexpr int kBatch = 4;
    for (int i0 = threadIdx.x / kLanes; i0 < 256; i0 += kBatch * kAtOnce) {
        uint4 a[kBatch], g[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = i0 + j * kAtOnce, row = row0 + (i >> 3), head = head0 + (i & 7);
            a[j] = g[j] = make_uint4(0u, 0u, 0u, 0u);
            if (row < p.b && head < p.heads && col < p.head_dim) {
                const size_t at = static_cast<size_t>(head) * p.head_dim + col;
                a[j] = ld_v4(p.O + static_cast<size_t>(row) * p.o_ld + at);
                g[j] = ld_v4(p.dO + static_cast<size_t>(row) * p.do_ld + at);
            }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const V8 x = from_bf16(a[j]), y = from_bf16(g[j]);
            Pair s = mul2(x.p[0], y.p[0]);
#pragma unroll
            for (int k = 1; k < 4; ++k) s = fma2(x.p[k], y.p[k], s);
            float sum = low(s) + high(s);
#pragma unroll
            for (int d = kLanes / 2; d > 0; d /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
            const int i = i0 + j * kAtOnce;
            if (part == 0) out[i & 7][i >> 3] = sum;
        }
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
    int key_blocks;                       // blocks of dK and dV
};

// A key's 128 scores -> 2^(v by - lse): lse belongs to the query, the column, and lies in shared memory ...  EDGE: those outside [lo, hi) are 0 (two
// instances, as in the forward pass)
template <bool EDGE>
__device__ __forceinline__ void attn_column_powers(uint32_t (&v)[kAttnRows], float by, uint32_t lse, int lo, int hi) {
#pragma unroll
    for (int c = 0; c < kAttnRows; c += 4) {
        const float4 e = ld_shared_v4(lse + 4 * c);
        const Pair x0 = fma2(pair(v[c], v[c + 1]), both(by), pair(-e.x, -e.y)), x1 = fma2(pair(v[c + 2], v[c + 3]), both(by), pair(-e.z, -e.w));
        v[c] = __float_as_uint(exp2_fast(low(x0)));
        v[c + 1] = __float_as_uint(exp2_fast(high(x0)));
        v[c + 2] = __float_as_uint(exp2_fast(low(x1)));
        v[c + 3] = __float_as_uint(exp2_fast(high(x1)));
    }
    if (EDGE) {
#pragma unroll
        for (int c = 0; c < kAttnRows; c += 32) {
            const uint32_t bits = attn_bits(lo - c, hi - c);
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (!(bits >> k & 1u)) v[c + k] = 0u;
        }
    }
}
// ... and, with dP - D from tensor memory, to bf16 pairs: 32 values of P and behind them 32 of dS = P (dP - D) at a time, in the place of dP; the
// barriers say that either half is there.
template <bool EDGE>
__device__ __forceinline__ void attn_column_pairs(uint32_t dp_row, uint32_t (&v)[kAttnRows], uint64_t (&half_full)[2], int lo, int hi) {
    uint32_t g[32];
    tmem_ld_32(dp_row, g);
#pragma unroll
    for (int c = 0; c < kAttnRows; c += 32) {
        tmem_ld_wait_32(g);
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
            const Pair p = pair(v[c + k], v[c + k + 1]), y = mul2(p, pair(g[k], g[k + 1]));
            v[c + (k >> 1)] = pack_bf16x2(low(p), high(p));       // (in the registers that they came in)
            g[k >> 1] = pack_bf16x2(low(y), high(y));
        }
        if (EDGE) {                                         // (zero times what a row of no sequence holds)
            const uint32_t bits = attn_bits(lo - c, hi - c);
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (!(bits >> k & 1u)) g[k >> 1] &= k & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        }
        tmem_st_16(dp_row + c, v + c);
        tmem_st_16(dp_row + c + 16, g);
        if (c + 32 < kAttnRows) tmem_ld_32(dp_row + c + 32, g);
        if (c & 32) {
            tmem_st_wait();
            tc_fence_before_sync();
            warp_arrive(&half_full[c >> 6]);
        }
    }
}
// x as a sum of three bf16 values, exact to 2^-24 of it, in the first three eighths of a row of 16
__device__ __forceinline__ uint4 attn_split(float x) {
    const float h = __uint_as_float(pack_bf16x2(0.0f, x) & 0xFFFF0000u), m = __uint_as_float(pack_bf16x2(0.0f, x - h) & 0xFFFF0000u);
    return make_uint4(pack_bf16x2(h, m), pack_bf16x2(x - h - m, 0.0f), 0u, 0u);
}

// dK and dV of 128 keys.  Keys lie on the lanes: S^T = K Q^T, dP^T = V dO^T, so that P^T and dS^T are where the next products
// want them as A.  The groups take the tiles of queries in turn, a key per thread.  What belongs to a query: lse comes from shared memory; -D is one
// more step of 16 of the product dP^T, of rows of three ones and rows with -D / 2 in three parts (read twice: a step has two eighths), since the
// products leave other reads of shared memory little room (16 of them per 64 values of dS: 1300 of 3700 clocks a tile).
// A thread reads its scores at once, so that the next tile's are formed, and keeps P in registers until dP is there; P and dS then take the
// place of dP, 32 queries at a time.  So while one group has dP and the products dV, dK and the next dP run, the other has its powers of two.
// What bounds it is the way dP - dS - dV, dK - next dP, 2000 of whose clocks at 128 columns are the products' (2048 with S).
// (Both kernels, as 10 operations a pair and column: 16384 tokens, 32 / 8 heads of 128, 6600 us = 833 TFLOP/s; 8 x 1024, 12 heads of 64 129 us = 250.)
// Warp 11: the MMAs of S; 8: the others; 9: loads; 10: lse and D, zeros behind the sequence's last row.
template <int HD>
__device__ __forceinline__ void attn_bwd_keys(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const CUtensorMap& tmdO,
                                              const AttnBwdParams& p, int block, AttnKvShared<HD, AttnCfg<HD>::kStages>& sh, uint8_t* smem) {
    using Cfg = AttnCfg<HD>;
    volatile int* abort_flag = &sh.abort_word;
    uint8_t *sK = smem, *sV = smem + Cfg::kTile, *ring = smem + 2 * Cfg::kTile;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = threadIdx.x >> 7;

    if (threadIdx.x < 8) {
        sh.ones[threadIdx.x] = make_uint4(0x3F803F80u, 0x00003F80u, 0u, 0u);
        fence_proxy_async_smem();
    }
    if (warp == 8) {
        tmem_alloc(&sh.tmem, 512);
        tmem_relinquish();
        griddep_launch_dependents();          // (behind the allocation, as in the forward pass)
    }
    const AttnQuotient unit = attn_divide(block, p.s.kv_heads, p.s.per_kv_heads);
    const int kv_head = unit.rest, share = p.s.share;
    // The warp that loads sets the barriers up, a lane each, and has the first item's tiles on their way before the others go on.
    if (warp == 9) {
        attn_barriers(&sh.k_full, sh.s_full, 1);
        attn_barriers(sh.s_full, sh.s_read, 2);
        attn_barriers(sh.s_read, reinterpret_cast<uint64_t*>(&sh.tmem), 4);
        if (lane == 0) *abort_flag = 0;
        fence_mbar_init();
        griddep_wait();
        const AttnTile t = attn_locate<kAttnRows>(p.s, unit.quotient, false);
        if (lane == 0) sh.work = t;
        __syncwarp();
        if (t.len && elect_one()) {
            const int k0 = t.tile * kAttnRows, tile = attn_first_query_tile(p.s, k0);
            uint64_t* bars = (tile + 1) * kAttnRows > t.len ? sh.ragged : sh.full;
            attn_load<HD>(sK, &tmK, &sh.k_full, kv_head, t.first + k0);
            attn_load<HD>(ring, &tmQ, &bars[0], kv_head * share, t.first + tile * kAttnRows);
            attn_load<HD>(sV, &tmV, &sh.v_full, kv_head, t.first + k0);
            attn_load<HD>(ring + Cfg::kTile, &tmdO, &bars[1], kv_head * share, t.first + tile * kAttnRows);
        }
        __syncwarp();
    }
    griddep_wait();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    // S, dP, dV, dK; where a head has 64 columns another place for dP, which then waits for nothing of the item before
    constexpr bool kTwo = HD == 64;
    const uint32_t tmem = sh.tmem, t_s = tmem, t_dv = tmem + 2 * kAttnRows, t_dk = t_dv + HD;
    const auto dp_at = [&](int it) { return tmem + (kTwo && (it & 1) ? 3 * kAttnRows : kAttnRows); };
    const int len = sh.work.len, first = sh.work.first, k0 = sh.work.tile * kAttnRows;
    // an item: a tile of queries of one of the heads that share the key head
    const int lo = attn_first_query_tile(p.s, k0), hi = len ? attn_end_query_tile(p.s, k0, len) : lo, items = (hi - lo) * share;
    const int last = (len - 1) / kAttnRows, last_rows = len - last * kAttnRows;
    const auto rows_of = [&](int tile) { return tile == last ? last_rows : kAttnRows; };

    if (group == 2) {
        registers_down<kAttnRegsDown>();
        if (warp == 9) {
            if (items && elect_one()) {
                PipeState ps;
                bool ok = true;
                for (int it = 0, tile = lo, head = kv_head * share; it < items && ok; ++it) {
                    uint64_t* bars = rows_of(tile) < kAttnRows ? sh.ragged : sh.full;
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        // (the first are on their way, and may be used and free again by now: nothing to wait for)
                        if (it) {
                            if (!attn_wait(&sh.empty[ps.stage], ps.phase ^ 1u, abort_flag)) { ok = false; break; }
                            attn_load<HD>(ring + ps.stage * Cfg::kTile, g ? &tmdO : &tmQ, &bars[ps.stage], head, first + tile * kAttnRows);
                        }
                        ps.advance(Cfg::kStages);
                    }
                    if (++tile == hi) { tile = lo; ++head; }
                }
            }
        } else if (warp == 11) {
            // the scores, by a warp of its own: what they wait for does not hold the other products up
            if (items && elect_one()) {
                const int steps = (p.s.head_dim + 15) / 16;
                const uint64_t k_desc = attn_column_desc(sK), column_desc = attn_column_desc(ring);
                PipeState ps;
                bool ok = attn_wait(&sh.k_full, 0, abort_flag);
                for (int it = 0; it < items && ok; ++it) {
                    if (!(ok = attn_wait(&sh.full[ps.stage], ps.phase, abort_flag) &&
                               (it == 0 || attn_wait(&sh.s_read[(it - 1) & 1], ((it - 1) >> 1) & 1, abort_flag))))
                        break;
                    tc_fence_after_sync();
                    attn_mma_columns<HD>(t_s, k_desc, column_desc + ps.stage * (Cfg::kTile >> 4), steps);
                    umma_commit(&sh.s_full[it & 1]);
                    ps.advance(Cfg::kStages);
                    ps.advance(Cfg::kStages);
                }
            }
        } else if (warp == 8) {
            if (items && elect_one()) {
                const int steps = (p.s.head_dim + 15) / 16;
                const uint32_t idesc = attn_row_idesc(p.s.head_dim);
                const uint64_t v_desc = attn_column_desc(sV), column_desc = attn_column_desc(ring), row_desc = attn_row_desc(ring);
                // rows of eight values without a swizzle, the same eight for both eighths of the step; the same eight rows of ones throughout
                const uint64_t ones_desc = make_smem_desc(smem_u32(sh.ones), 0, 0, kSwizzleNone), d_desc = make_smem_desc(smem_u32(sh.minus_d), 0, 128, kSwizzleNone);
                PipeState qs, os;                         // places of an item's Q, and of the next products' dO
                os.advance(Cfg::kStages);
                // (behind `d_full` dO is there, too)
                const auto products = [&](int it) {
                    if (!attn_wait(&sh.d_full, it & 1, abort_flag)) return false;
                    tc_fence_after_sync();
                    umma_bf16(dp_at(it), ones_desc, d_desc, make_idesc_bf16(kAttnRows, kAttnRows, false, false, false), 0);
                    attn_mma_columns<HD>(dp_at(it), v_desc, column_desc + os.stage * (Cfg::kTile >> 4), steps, true);
                    umma_commit(&sh.dp_full[it & 1]);
                    os.advance(Cfg::kStages);
                    os.advance(Cfg::kStages);
                    return true;
                };
                bool ok = attn_wait(&sh.v_full, 0, abort_flag) && products(0);
                for (int it = 0, tile = lo; it < items && ok; ++it) {
                    const int row_steps = (rows_of(tile) + 15) / 16, o_stage = qs.stage + 1 < Cfg::kStages ? qs.stage + 1 : 0;
                    if (++tile == hi) tile = lo;
                    if (kTwo && it + 1 < items && !(ok = products(it + 1))) break;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (!(ok = ok && attn_wait(&sh.pairs_full[it & 1][h], (it >> 1) & 1, abort_flag))) continue;
                        tc_fence_after_sync();
                        const uint32_t a = dp_at(it) + 64 * h, b = h * (64 * 128 >> 4);
                        attn_mma_rows<32>(t_dv, a, row_desc + o_stage * (Cfg::kTile >> 4) + b, idesc, row_steps - 4 * h, it != 0 || h);
                        attn_mma_rows<32>(t_dk, a + 16, row_desc + qs.stage * (Cfg::kTile >> 4) + b, idesc, row_steps - 4 * h, it != 0 || h);
                    }
                    if (!ok) break;
                    umma_commit(&sh.empty[qs.stage]);
                    umma_commit(&sh.empty[o_stage]);
                    qs.advance(Cfg::kStages);
                    qs.advance(Cfg::kStages);
                    if (it + 1 == items) umma_commit(&sh.acc_full);
                    else if (!kTwo) ok = products(it + 1);
                }
            }
        } else if (warp == 10) {
            uint32_t phases = 0;                             // of the stages' ragged barriers
            for (int it = 0, tile = lo, head = kv_head * share; it < items; ++it) {
                const int rows = rows_of(tile);
                const size_t at = static_cast<size_t>(head) * p.s.b + first + tile * kAttnRows;
                uint32_t e[4], d[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool in = lane + 32 * k < rows;
                    e[k] = in ? ld_u32(p.lse + at + lane + 32 * k) : 0u;
                    d[k] = in ? ld_u32(p.delta + at + lane + 32 * k) : 0u;
                }
                if (rows < kAttnRows) {
                    bool ok = true;
                    for (int g = 0; g < 2 && ok; ++g) {
                        const int stage = (2 * it + g) % Cfg::kStages;
                        if (!(ok = warp_wait(&sh.ragged[stage], (phases >> stage) & 1, abort_flag))) break;
                        phases ^= 1u << stage;
                        attn_zero_rows<HD>(ring + stage * Cfg::kTile, rows);
                        warp_arrive(&sh.full[stage]);
                    }
                    if (!ok) break;
                }
                // the powers of two of the tile that had the place are done, and the last tile's dP
                constexpr int kLse = sh.kLse;
                if (it >= kLse && !warp_wait(&sh.powers_done[it % kLse], (it / kLse - 1) & 1, abort_flag)) break;
#pragma unroll
                for (int k = 0; k < 4; ++k) sh.lse[it % kLse][lane + 32 * k] = __uint_as_float(e[k]) * kLog2e;
                warp_arrive(&sh.s_full[it & 1]);
                if (it && !warp_wait(&sh.dp_full[(it - 1) & 1], ((it - 1) >> 1) & 1, abort_flag)) break;
#pragma unroll
                for (int k = 0; k < 4; ++k) sh.minus_d[lane + 32 * k] = attn_split(-0.5f * __uint_as_float(d[k]));
                fence_proxy_async_smem();
                if (!warp_wait(&sh.full[(2 * it + 1) % Cfg::kStages], ((2 * it + 1) / Cfg::kStages) & 1, abort_flag)) break;
                warp_arrive(&sh.d_full);
                if (++tile == hi) { tile = lo; ++head; }
            }
        }
    } else {
        registers_up<kAttnRegsUp>();
        const int key = k0 + (threadIdx.x & 127);
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_row = t_s + lanes, dp_row = dp_at(group) + lanes;
        bool ok = items > 0;
        for (int it = group, tile = lo + group; it < items; it += 2, tile += 2) {
            while (tile >= hi) tile -= hi - lo;
            const int q0 = tile * kAttnRows;
            const uint32_t phase = (it >> 1) & 1;
            const bool edge = (p.s.causal && q0 == k0) || q0 + kAttnRows > len || (p.s.window && q0 + kAttnRows - 1 - k0 >= p.s.window);
            // queries [c_lo, c_hi) of the tile's see the key
            const int c_lo = p.s.causal ? key - q0 : 0, c_hi = min(len, p.s.window ? min(key, len) + p.s.window : len) - q0;
            if (!(ok = warp_wait(&sh.s_full[group], phase, abort_flag))) break;
            tc_fence_after_sync();
            uint32_t v[kAttnRows];
#pragma unroll
            for (int c = 0; c < kAttnRows; c += 32) tmem_ld_32(s_row + c, v + c);
            tmem_ld_wait_32(v);
            tie_32(v + 32);
            tie_32(v + 64);
            tie_32(v + 96);
            tc_fence_before_sync();
            warp_arrive(&sh.s_read[group]);
            if (edge) attn_column_powers<true>(v, p.s.scale, smem_u32(sh.lse[group % sh.kLse]), c_lo, c_hi);
            else attn_column_powers<false>(v, p.s.scale, smem_u32(sh.lse[group % sh.kLse]), 0, kAttnRows);
            warp_arrive(&sh.powers_done[group % sh.kLse]);
            if (!(ok = warp_wait(&sh.dp_full[group], phase, abort_flag))) break;
            tc_fence_after_sync();
            if (edge) attn_column_pairs<true>(dp_row, v, sh.pairs_full[group], c_lo, c_hi);
            else attn_column_pairs<false>(dp_row, v, sh.pairs_full[group], 0, kAttnRows);
        }
        if (ok && warp_wait(&sh.acc_full, 0, abort_flag)) {
            tc_fence_after_sync();
            const size_t row = static_cast<size_t>(first) + k0;
            uint16_t* out = group ? p.dK + row * p.dk_ld : p.dV + row * p.dv_ld;
            attn_store<HD, HD>((group ? t_dk : t_dv) + lanes, 0, group ? p.grad_scale : 1.0f, group ? sK : sV, out + kv_head * p.s.head_dim,
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

// A row's 128 scores from tensor memory -> 2^(v by - lse); EDGE: those outside [lo, hi) are 0
template <bool EDGE>
__device__ __forceinline__ void attn_row_powers(uint32_t s_row, uint32_t (&v)[kAttnRows], float by, float lse, int lo, int hi) {
#pragma unroll
    for (int c = 0; c < kAttnRows; c += 32) tmem_ld_32(s_row + c, v + c);
#pragma unroll
    for (int c = 0; c < kAttnRows; c += 32) {
        if (c == 0) tmem_ld_wait_32(v);
        else tie_32(v + c);
#pragma unroll
        for (int k = c; k < c + 32; k += 2) {
            const Pair x = fma2(pair(v[k], v[k + 1]), both(by), both(-lse));
            v[k] = __float_as_uint(exp2_fast(low(x)));
            v[k + 1] = __float_as_uint(exp2_fast(high(x)));
        }
        if (EDGE) {
#pragma unroll
            for (int k = c; k < c + 32; ++k)
                if (k < lo || k >= hi) v[k] = 0u;
        }
    }
}
// ... and, with dP from tensor memory, to dS = P (dP - D) in bf16 pairs; the barrier says that dP has been read
template <bool EDGE>
__device__ __forceinline__ void attn_row_gradients(uint32_t dp_row, uint32_t (&v)[kAttnRows], float d, uint64_t* dp_read, int lo, int hi) {
    uint32_t g[2][32];
    tmem_ld_32(dp_row, g[0]);
#pragma unroll
    for (int c = 0; c < kAttnRows; c += 32) {
        uint32_t(&now)[32] = g[(c >> 5) & 1];
        tmem_ld_wait_32(now);
        if (c + 32 < kAttnRows) {
            tmem_ld_32(dp_row + c + 32, g[((c >> 5) + 1) & 1]);
        } else {
            tc_fence_before_sync();
            warp_arrive(dp_read);
        }
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
            const Pair y = mul2(pair(v[c + k], v[c + k + 1]), add2(pair(now[k], now[k + 1]), both(-d)));
            v[(c + k) >> 1] = pack_bf16x2(low(y), high(y));
        }
        if (EDGE) {                                         // (zero times what a row of no sequence holds)
#pragma unroll
            for (int k = c; k < c + 32; ++k)
                if (k < lo || k >= hi) v[k >> 1] &= k & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        }
    }
}
// dQ of 128 queries, which lie on the lanes.  The groups take the tiles of keys in turn, a row per thread: while one forms its powers of two the other has
// its dS.  S has a place for either group and is formed two tiles ahead; dS takes the place of S; dP is read as soon as it is there, so that the
// next one is formed beside dS.  (Both groups on every tile, 64 keys each: 2400 clocks a tile.)
template <int HD>
__device__ __forceinline__ void attn_bwd_queries(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const CUtensorMap& tmdO,
                                                 const AttnBwdParams& p, int block, AttnQShared<AttnCfg<HD>::kKeys, AttnCfg<HD>::kValues>& sh, uint8_t* smem) {
    using Cfg = AttnCfg<HD>;
    volatile int* abort_flag = &sh.abort_word;
    uint8_t *sQ = smem, *sdO = smem + Cfg::kTile, *keys = smem + 2 * Cfg::kTile, *values = keys + Cfg::kKeys * Cfg::kTile;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = threadIdx.x >> 7;

    if (warp == 8) {
        tmem_alloc(&sh.tmem, 512);
        tmem_relinquish();
        griddep_launch_dependents();          // (behind the allocation, as in the forward pass)
    }
    const AttnQuotient unit = attn_divide(block, p.s.heads, p.s.per_heads);
    const int head = unit.rest, kv_head = attn_divide(head, p.s.share, p.s.per_share).quotient;
    if (warp == 9) {
        attn_barriers(&sh.q_full, sh.dp_read, 1);
        attn_barriers(sh.dp_read, reinterpret_cast<uint64_t*>(&sh.tmem), 4);
        if (lane == 0) *abort_flag = 0;
        fence_mbar_init();
        griddep_wait();
        const AttnTile t = attn_locate<kAttnRows>(p.s, unit.quotient, p.s.causal);
        if (lane == 0) sh.work = t;
        __syncwarp();
        if (t.len && elect_one()) {
            const int q0 = t.tile * kAttnRows, c0 = attn_first_key_tile(p.s, q0) * kAttnRows;
            attn_load<HD>(sQ, &tmQ, &sh.q_full, head, t.first + q0);
            // (ragged: the sequence's end, and with it the only item)
            attn_load<HD>(keys, &tmK, c0 + kAttnRows > t.len ? &sh.ragged_bar : &sh.k_full[0], kv_head, t.first + c0);
            attn_load<HD>(sdO, &tmdO, &sh.do_full, head, t.first + q0);
            attn_load<HD>(values, &tmV, &sh.v_full[0], kv_head, t.first + c0);
        }
        __syncwarp();
    }
    griddep_wait();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem, t_dp = tmem + 2 * kAttnRows, t_dq = tmem + 3 * kAttnRows;
    const int len = sh.work.len, first = sh.work.first, q0 = sh.work.tile * kAttnRows;
    const int lo = attn_first_key_tile(p.s, q0), items = len ? attn_end_key_tile(p.s, q0, len) - lo : 0;
    const int last = (len - 1) / kAttnRows, last_rows = len - last * kAttnRows;
    const bool ragged = items && lo + items == last + 1 && last_rows < kAttnRows;     // the last item is the sequence's ragged end

    if (group == 2) {
        registers_down<kAttnRegsDown>();
        if (warp == 9) {
            if (items && elect_one()) {
                PipeState ks, vs;
                ks.advance(Cfg::kKeys);
                vs.advance(Cfg::kValues);
                for (int it = 1; it < items; ++it) {
                    const int row = first + (lo + it) * kAttnRows;
                    if (!attn_wait(&sh.k_empty[ks.stage], ks.phase ^ 1u, abort_flag)) break;
                    attn_load<HD>(keys + ks.stage * Cfg::kTile, &tmK, ragged && it + 1 == items ? &sh.ragged_bar : &sh.k_full[ks.stage], kv_head, row);
                    ks.advance(Cfg::kKeys);
                    if (!attn_wait(&sh.v_empty[vs.stage], vs.phase ^ 1u, abort_flag)) break;
                    attn_load<HD>(values + vs.stage * Cfg::kTile, &tmV, &sh.v_full[vs.stage], kv_head, row);
                    vs.advance(Cfg::kValues);
                }
            }
        } else if (warp == 8) {
            if (items && elect_one()) {
                const int steps = (p.s.head_dim + 15) / 16;
                const uint32_t idesc = attn_row_idesc(p.s.head_dim);
                const uint64_t q_desc = attn_column_desc(sQ), do_desc = attn_column_desc(sdO), key_desc = attn_column_desc(keys),
                               key_rows = attn_row_desc(keys), value_desc = attn_column_desc(values);
                PipeState ks, vs;                         // of the next scores and of the next products
                const auto scores = [&](int it) {
                    if (!attn_wait(&sh.k_full[ks.stage], ks.phase, abort_flag)) return false;
                    tc_fence_after_sync();
                    attn_mma_columns<HD>(tmem + (it & 1) * kAttnRows, q_desc, key_desc + ks.stage * (Cfg::kTile >> 4), steps);
                    umma_commit(&sh.s_full[it & 1]);
                    ks.advance(Cfg::kKeys);
                    return true;
                };
                const auto products = [&](int it) {
                    if (!attn_wait(&sh.v_full[vs.stage], vs.phase, abort_flag)) return false;
                    tc_fence_after_sync();
                    attn_mma_columns<HD>(t_dp, do_desc, value_desc + vs.stage * (Cfg::kTile >> 4), steps);
                    umma_commit(&sh.dp_full[it & 1]);
                    umma_commit(&sh.v_empty[vs.stage]);
                    vs.advance(Cfg::kValues);
                    return true;
                };
                bool ok = attn_wait(&sh.q_full, 0, abort_flag) && scores(0) && attn_wait(&sh.do_full, 0, abort_flag) && products(0) && (items < 2 || scores(1));
                for (int it = 0; it < items && ok; ++it) {
                    const int rows = ragged && it + 1 == items ? last_rows : kAttnRows, g = it & 1, stage = it % Cfg::kKeys;
                    const uint32_t t_s = tmem + g * kAttnRows, phase = (it >> 1) & 1;
                    if (!(ok = attn_wait(&sh.dp_read[g], phase, abort_flag) && (it + 1 >= items || products(it + 1)) && attn_wait(&sh.ds_ready[g], phase, abort_flag)))
                        break;
                    tc_fence_after_sync();
                    attn_mma_rows(t_dq, t_s, t_s + 64, key_rows + stage * (Cfg::kTile >> 4), idesc, (rows + 15) / 16, it != 0);
                    umma_commit(it + 1 < items ? &sh.k_empty[stage] : &sh.acc_full);
                    if (it + 2 < items) ok = scores(it + 2);
                }
            }
        } else if (warp == 10 && ragged) {
            const int stage = (items - 1) % Cfg::kKeys;
            if (warp_wait(&sh.ragged_bar, 0, abort_flag)) {
                attn_zero_rows<HD>(keys + stage * Cfg::kTile, last_rows);
                warp_arrive(&sh.k_full[stage]);
            }
        }
    } else {
        registers_up<kAttnRegsUp>();
        const int row = threadIdx.x & 127, i = q0 + row;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        float lse = 0.0f, delta = 0.0f;
        if (items && i < len) {
            const size_t at = static_cast<size_t>(head) * p.s.b + first + i;
            lse = __uint_as_float(ld_u32(p.lse + at)) * kLog2e;
            delta = __uint_as_float(ld_u32(p.delta + at));
        }
        bool ok = items > 0;
        for (int it = group; it < items; it += 2) {
            const int c0 = (lo + it) * kAttnRows;
            const bool edge = (p.s.causal ? c0 + kAttnRows - 1 > q0 : c0 + kAttnRows > len) || (p.s.window && q0 + kAttnRows - 1 - c0 >= p.s.window);
            const int c_hi = (p.s.causal ? min(i + 1, len) : len) - c0, c_lo = p.s.window ? i - p.s.window + 1 - c0 : 0;
            const uint32_t s_row = tmem + group * kAttnRows + lanes, dp_row = t_dp + lanes, phase = (it >> 1) & 1;
            if (!(ok = warp_wait(&sh.s_full[group], phase, abort_flag))) break;
            tc_fence_after_sync();
            uint32_t v[kAttnRows];
            if (edge) attn_row_powers<true>(s_row, v, p.s.scale, lse, c_lo, c_hi);
            else attn_row_powers<false>(s_row, v, p.s.scale, lse, 0, kAttnRows);
            if (!(ok = warp_wait(&sh.dp_full[group], phase, abort_flag))) break;
            tc_fence_after_sync();
            if (edge) attn_row_gradients<true>(dp_row, v, delta, &sh.dp_read[group], c_lo, c_hi);
            else attn_row_gradients<false>(dp_row, v, delta, &sh.dp_read[group], 0, kAttnRows);
            tmem_st_32(s_row, v);
            tmem_st_32(s_row + 64, v + 32);
            tmem_st_wait();
            tc_fence_before_sync();
            warp_arrive(&sh.ds_ready[group]);
        }
        if (ok && warp_wait(&sh.acc_full, 0, abort_flag)) {
            tc_fence_after_sync();
            const size_t at = static_cast<size_t>(first) + q0;
            attn_store<HD, HD / 2>(t_dq + lanes, group * HD / 2, p.grad_scale, group ? sdO : sQ,
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

// Both in one launch, the keys' blocks first: the queries' fill the machine while the last of these run.
template <int HD>
__global__ void __launch_bounds__(kAttnThreads, 1)
attention_bwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const __grid_constant__ CUtensorMap tmdO, const AttnBwdParams p) {
    using Cfg = AttnCfg<HD>;
    // (one object, whose size the host knows: beside seven tiles of 128 columns there are 3 KB)
    __shared__ AttnBwdShared<HD> sh;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int block = static_cast<int>(blockIdx.x) - p.key_blocks;
    if (block < 0) attn_bwd_keys<HD>(tmQ, tmK, tmV, tmdO, p, blockIdx.x, sh.keys, smem);
    else attn_bwd_queries<HD>(tmQ, tmK, tmV, tmdO, p, block, sh.queries, smem);
}

// =====================================================================================
// Rotation by positions: of the first 2 n columns of every head, the pairs (u_i, v_i) become
//   factor (u cos a - v sin a, v cos a + u sin a),   a = position frequency_i
// (backward: the transposed map, sin negated).  Pairs are columns i and n + i, or (PAIRS) 2 i and 2 i + 1.
// What bounds it is HBM; an angle is formed once per token and pair, by one thread of the block that has the token, for all heads.  Angles are
// taken in whole turns in fp64, of which the nearest whole number is left out: in fp32 a position of 10^6 would be 0.06 rad off.  (At 2^31 and a
// frequency of 1 the two fp64 roundings and the one to fp32 come to 8e-8 of a turn; they grow with the frequency.)
// =====================================================================================
struct RotaryParams {
    const void *src[2];
    void* dst[2];
    int src_ld[2], dst_ld[2], heads[2];
    int b, head_dim, n, tokens;           // n: pairs of a head; tokens of a block
    int turned, per_head, per_token;      // tasks of a head that rotate; all of a head's, with those that copy the columns behind; a token's
    float per_per_head, per_per_token;    // their reciprocals
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
// A thread takes N values at a time: N pairs' two halves, or N / 2 neighbouring pairs; kBatch of these are in flight, the first while the block's
// angles are formed.  Measured on the same buffers each time, us, one at a time behind the angles / two / four: 20 of 80 columns of 64 heads turned, 2039 tokens, neighbouring pairs
// 17.2 / 9.2 / 10.2, halves 41.8 / 20.8 / 23.9; all of 64 heads of 128, 16384 tokens, bf16, halves 84.7 / 83.2 / 100; fp32, where a task of eight
// has four loads of its own and goes alone, 40 heads of 128, 8191 tokens, 55.1 / 55.6 / -, one in flight 54.9.
template <int TYPE, bool PAIRS, int N>
__global__ void __launch_bounds__(kRotaryThreads)
rotary_kernel(const RotaryParams p) {
    __shared__ float cosine[kRotaryTable], sine[kRotaryTable];
    griddep_launch_dependents();
    griddep_wait();
    const int token0 = blockIdx.x * p.tokens, tokens = min(p.tokens, p.b - token0), tasks = tokens * p.per_token;
    constexpr int kBatch = !PAIRS && N == 8 && TYPE == kTypeF32 ? 1 : 2;
    constexpr int kPairs = PAIRS ? N / 2 : N;                  // of a task
    float x[kBatch][N], z[kBatch][N];
    void* row[kBatch];                                         // of the output, at the task's head
    int angle[kBatch], column[kBatch];                         // angle: the first one's place, -1 in a task that copies
    const auto fetch = [&](int first) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            // (past the end: the last task once more, which is not stored)
            const AttnQuotient token = attn_divide(min(first + j * kRotaryThreads, tasks - 1), p.per_token, p.per_per_token);
            const AttnQuotient head = attn_divide(token.rest, p.per_head, p.per_per_head);
            const bool which = head.quotient >= p.heads[0];
            const int h = which ? head.quotient - p.heads[0] : head.quotient, u = head.rest;
            const size_t at = static_cast<size_t>(token0 + token.quotient);
            constexpr int kBytes = TYPE == kTypeF32 ? 4 : 2;
            const size_t from = at * (which ? p.src_ld[1] : p.src_ld[0]) + h * p.head_dim, to = at * (which ? p.dst_ld[1] : p.dst_ld[0]) + h * p.head_dim;
            const void* src = which ? p.src[1] : p.src[0];
            row[j] = static_cast<uint8_t*>(which ? p.dst[1] : p.dst[0]) + to * kBytes;
            const bool turns = u < p.turned;
            angle[j] = turns ? token.quotient * p.n + u * kPairs : -1;
            column[j] = PAIRS || turns ? u * N : 2 * p.n + (u - p.turned) * N;
            load_n<TYPE, N>(src, from + column[j], x[j]);
            if (!PAIRS) load_n<TYPE, N>(src, from + column[j] + (turns ? p.n : 0), z[j]);
        }
    };
    fetch(threadIdx.x);
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
    for (int first = threadIdx.x; first < tasks; first += kBatch * kRotaryThreads) {
        if (first >= kRotaryThreads) fetch(first);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (first + j * kRotaryThreads >= tasks) break;
            if (angle[j] >= 0) {
                const float *c = cosine + angle[j], *s = sine + angle[j];
                if (PAIRS) {
                    // the last of the eight columns may be behind the rotated part
                    const int in = p.n - (column[j] >> 1);
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) {
                        if (i >= in) break;
                        const float u = x[j][2 * i], v = x[j][2 * i + 1];
                        x[j][2 * i] = u * c[i] - v * s[i];
                        x[j][2 * i + 1] = v * c[i] + u * s[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float u = x[j][i], v = z[j][i];
                        x[j][i] = u * c[i] - v * s[i];
                        z[j][i] = v * c[i] + u * s[i];
                    }
                    store_n<TYPE, N>(row[j], column[j] + p.n, z[j]);
                }
            }
            store_n<TYPE, N>(row[j], column[j], x[j]);
        }
    }
}

}  // namespace slope
