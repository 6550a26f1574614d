// Layer norm between the sparse layers, forward and backward, and the 8-bit checkpoints of activations that the backward
// pass reads in place of bf16 ones.
//
//   forward    h = X (+ residual),  m = mean(h),  s = 1 / sqrt(mean((h - m)^2) + eps),  y = (h - m) s gamma + beta
//   backward   x = (h - m) s,  g = dY gamma,  dX = s (g - mean(g) - x mean(g x)) (+ dH),
//              dgamma = sum over the tokens of dY x,  dbeta = sum over the tokens of dY
//
// Every matrix is read once from HBM and written once; a row stays in registers or shared memory between its statistics and its output.  All sums
// are fp32; the variance is that of the differences from the mean, not mean(h^2) - m^2, which cancels where a row's mean is large beside its
// spread.  Sums that leave fp32's range are taken again in larger units.
//
// Checkpoint of a matrix [rows x cols], cols a multiple of 32: each block of 32 consecutive values of a row is 32 signed bytes
// times one power of two, 2^k, k the smallest integer for which the block's largest magnitude is at most 127.5 * 2^k, within
// [-126, 121]; codes are rounded half to even and held in [-127, 127].  A value is off by at most half a unit of 2^k, i.e. 1/127
// of the block's largest magnitude at most, but for the ends of k's range: 2^-127 in any block at k = -126, and up to a whole unit for an fp32
// value beyond 127.5 * 2^121 (a power of two wastes at most half of the code's range; e4m3 codes, with the
// same 8 bits, are off by up to 1/16 of a value, for Gaussian activations 2.4 % (root mean square) against 0.8 %).  A code has seven
// significant bits, so a value that is read back is exact in bf16, and a product with it has exactly that operand.
// Memory: rows * cols codes, then rows * cols / 32 bytes k + 127 (the exponent field of 2^k as fp32); 255, with codes of 0, in a block
// that holds an infinity or a NaN, whose values are NaN, so that an overflow still shows in the gradients.
#pragma once
#include <cfloat>

#include "gemm_kernels.cuh"

namespace slope {

constexpr int kTypeBf16 = 0, kTypeF32 = 1, kTypeQ8 = 2;          // == slope_type_t
constexpr int kQBlock = 32;

// ---------------------------------------------------------------- eight values of a row, as fp32
// In four pairs, for the instructions that work on two fp32 values at once: what these kernels issue is what HBM has to wait for (see below).
using Pair = unsigned long long;
struct V8 {
    Pair p[4];
};
__device__ __forceinline__ Pair pair(uint32_t lo, uint32_t hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ Pair pair(float lo, float hi) { return pair(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ Pair both(float v) { return pair(v, v); }
__device__ __forceinline__ float low(Pair v) { return __uint_as_float(static_cast<uint32_t>(v)); }
__device__ __forceinline__ float high(Pair v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ V8 zeros() { return V8{{0, 0, 0, 0}}; }
__device__ __forceinline__ V8 from_bf16(const uint4& w) {
    return V8{{pair(w.x << 16, w.x & 0xFFFF0000u), pair(w.y << 16, w.y & 0xFFFF0000u), pair(w.z << 16, w.z & 0xFFFF0000u),
               pair(w.w << 16, w.w & 0xFFFF0000u)}};
}
__device__ __forceinline__ uint4 to_bf16(const V8& v) {
    return make_uint4(pack_bf16x2(low(v.p[0]), high(v.p[0])), pack_bf16x2(low(v.p[1]), high(v.p[1])),
                      pack_bf16x2(low(v.p[2]), high(v.p[2])), pack_bf16x2(low(v.p[3]), high(v.p[3])));
}
__device__ __forceinline__ V8 from_f32(const uint4& a, const uint4& b) {
    return V8{{pair(a.x, a.y), pair(a.z, a.w), pair(b.x, b.y), pair(b.z, b.w)}};
}
// The byte q of `w` is put into the mantissa of 2^23 as q + 128; taking 2^23 + 128 away leaves q.  (A multiplication by 2^k is exact.)
__device__ __forceinline__ V8 from_q8(const uint2& w, uint32_t e) {
    const uint32_t u[2] = {w.x ^ 0x80808080u, w.y ^ 0x80808080u};
    const Pair offset = both(-8388736.0f), unit = both(__uint_as_float(e << 23));
    V8 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t s = i >> 1, sel = 0x7650u | (2 * (i & 1));
        v.p[i] = mul2(add2(pair(prmt(u[s], 0x4B000000u, sel), prmt(u[s], 0x4B000000u, sel + 1)), offset), unit);
    }
    return v;
}
// from global memory (SLOPE_Q8: `count` values in all, the exponents stand behind them) ...
template <int TYPE>
__device__ __forceinline__ V8 load8(const void* base, size_t at, size_t count) {
    if (TYPE == kTypeBf16) return from_bf16(ld_v4(static_cast<const uint16_t*>(base) + at));
    if (TYPE == kTypeF32) {
        const float* p = static_cast<const float*>(base) + at;
        const uint4 a = ld_v4(p), b = ld_v4(p + 4);
        return from_f32(a, b);
    }
    const uint8_t* p = static_cast<const uint8_t*>(base);
    const uint2 w = ld_v2(p + at);
    return from_q8(w, ld_u8(p + count + at / kQBlock));
}
// ... and from a row in shared memory (SLOPE_Q8: `e`, the block's exponent byte, comes from elsewhere)
__device__ __forceinline__ uint4 lds_v4(uint32_t saddr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(saddr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds_v2(uint32_t saddr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(saddr) : "memory");
    return v;
}
template <int TYPE>
__device__ __forceinline__ V8 shared8(uint32_t row, int col, uint32_t e = 0) {
    if (TYPE == kTypeBf16) return from_bf16(lds_v4(row + 2 * col));
    if (TYPE == kTypeF32) {
        const uint4 a = lds_v4(row + 4 * col), b = lds_v4(row + 4 * col + 16);
        return from_f32(a, b);
    }
    return from_q8(lds_v2(row + col), e);
}
template <int TYPE>
__device__ __forceinline__ void store8(void* base, size_t at, const V8& v) {
    if (TYPE == kTypeBf16) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) = to_bf16(v);
    } else {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
        p[0] = make_float4(low(v.p[0]), high(v.p[0]), low(v.p[1]), high(v.p[1]));
        p[1] = make_float4(low(v.p[2]), high(v.p[2]), low(v.p[3]), high(v.p[3]));
    }
}

// The larger magnitude of three values; NaN if there is one.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
// Eight values to codes; four neighbouring lanes hold a block.  All lanes of the warp take part.  The exponent: that of the
// largest magnitude less 6, one more where its mantissa is above 127.5 / 64 (0x7F0000: then 0xFFFF carries into the exponent).
// Rounding: 1.5 * 2^23 added (fused with the exact multiplication by 2^-k) leaves the code in the low byte.  Only a block whose largest
// magnitude is 127.5 units (one in 128 of bf16 values), or that is held at k = 121, has a code to hold at 127.
__device__ __forceinline__ uint2 encode8(const V8& v, uint32_t& e) {
    float largest = max_abs(low(v.p[0]), high(v.p[0]), low(v.p[1]));
    largest = max_abs(largest, high(v.p[1]), low(v.p[2]));
    largest = max_abs(largest, high(v.p[2]), low(v.p[3]));
    largest = max_abs(largest, high(v.p[3]), 0.0f);
    uint32_t m = __float_as_uint(largest);
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    if (m >= 0x7F800000u) {
        e = 255u;
        return make_uint2(0u, 0u);
    }
    e = static_cast<uint32_t>(min(max(static_cast<int>((m + 0xFFFFu) >> 23) - 6, 1), 248));
    const float per_unit = __uint_as_float((254u - e) << 23);
    V8 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t.p[i] = fma2(v.p[i], both(per_unit), both(12582912.0f));
    if (__uint_as_float(m) * per_unit >= 127.5f) {
        auto held = [](float x) { return fminf(fmaxf(x, 12582912.0f - 127.0f), 12582912.0f + 127.0f); };
#pragma unroll
        for (int i = 0; i < 4; ++i) t.p[i] = pair(held(low(t.p[i])), held(high(t.p[i])));
    }
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = prmt(static_cast<uint32_t>(t.p[i]), static_cast<uint32_t>(t.p[i] >> 32), 0x0040u);
    return make_uint2(prmt(c[0], c[1], 0x5410u), prmt(c[2], c[3], 0x5410u));
}
// `at`: the place of the eight values in the matrix of `count`; `live`: whether the lane has any
__device__ __forceinline__ void store_q8(void* ckpt, size_t at, size_t count, bool live, const V8& v) {
    uint32_t e;
    const uint2 codes = encode8(v, e);
    if (!live) return;
    uint8_t* p = static_cast<uint8_t*>(ckpt);
    *reinterpret_cast<uint2*>(p + at) = codes;
    if ((threadIdx.x & 3) == 0) p[count + at / kQBlock] = static_cast<uint8_t>(e);
}

// ---------------------------------------------------------------- matrices to checkpoints and back
// A thread takes eight values at a time, two times in one go so that twice the bytes are in flight; `n8` eights in all, a multiple of 4, so that a
// block's four lanes live or rest together.  HBM-bound: 16384 x 11008 to 8 bits and back 1093 MB in 182 us, 6.0 TB/s (one at a time: 197 us).
template <int TYPE>
__global__ void __launch_bounds__(256) checkpoint_store_kernel(const void* X, size_t n8, void* ckpt) {
    griddep_stream(8);
    const size_t stride = static_cast<size_t>(gridDim.x) * 512;
    for (size_t first = static_cast<size_t>(blockIdx.x) * 512; first < n8; first += stride) {
        V8 v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const size_t i = first + 256 * k + threadIdx.x;
            v[k] = i < n8 ? load8<TYPE>(X, 8 * i, 0) : zeros();
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const size_t i = first + 256 * k + threadIdx.x;
            store_q8(ckpt, 8 * i, 8 * n8, i < n8, v[k]);
        }
    }
}
template <int TYPE>
__global__ void __launch_bounds__(256) checkpoint_load_kernel(const void* ckpt, size_t n8, void* X) {
    griddep_stream(8);
    const size_t stride = static_cast<size_t>(gridDim.x) * 512;
    for (size_t first = static_cast<size_t>(blockIdx.x) * 512; first < n8; first += stride) {
        const size_t i = first + threadIdx.x;
        const bool two = i + 256 < n8;
        if (i >= n8) continue;
        const V8 a = load8<kTypeQ8>(ckpt, 8 * i, 8 * n8);
        if (two) {
            const V8 b = load8<kTypeQ8>(ckpt, 8 * (i + 256), 8 * n8);
            store8<TYPE>(X, 8 * (i + 256), b);
        }
        store8<TYPE>(X, 8 * i, a);
    }
}

// ---------------------------------------------------------------- layer norm
// Blocks fill the SMs and stay.  A row belongs to a group of `row_warps` warps; a lane holds CHUNKS times eight of its columns, chunk i of lane l at
// column 8 (l + 32 row_warps i), the same ones in all rows, so that the sums of gamma's and beta's gradients can stay in registers.
// Rows come in by bulk copies, ahead of their use, into the group's ring in shared memory: the bytes in flight that HBM needs (some 35 KB
// per SM) cost no registers.  A stage holds `batch` adjacent rows (several where they are short), one copy per matrix; the group's first lane
// asks for the next ones when the group has read it.  Groups have nothing to do with one another.
//
// What bounds them: HBM for long rows (16384 x 4096: forward 6.0, backward 5.6 of 6.45 TB/s), else what is issued and waited for per row:
// at HBM's rate an SM has 890 clocks for a row of 5120 values.  us of the forward of 8192 x 5120 with fp32 parameters, 168 MB (floor 26),
// as it went: rows loaded by the warps, one fp32 value per instruction 62; the same from the ring, instances without branches on what a
// call leaves out, two values per instruction (23.6 -> 11.6 instructions per value) 43; 24 warps instead of 16 37; loads that leave L2
// first 35.
constexpr int kNormMaxWidth = 16384;
constexpr int kNormFwdWarps = 24, kNormBwdWarps = 16;             // of a block at most: so many as leave a row its registers
constexpr int kNormWarps = kNormFwdWarps;
constexpr int kNormMaxStages = 2, kNormMaxSources = 3;
constexpr int kNormSharedBytes = 224 * 1024;                   // of a block; beside it stands what NormShared takes

struct NormRing {
    const uint8_t* src[kNormMaxSources];      // row-major matrices; nullptr: none
    int row_bytes[kNormMaxSources];           // multiples of 16
    int batch, stages, groups, row_warps, b, d;
    int leave_first;                          // rows that have been read leave L2 before others
    const void* param[2];                     // gamma, beta (nullptr: ones, zeros)
    int p_f32;
    int params;                               // how many of them are kept in shared memory
    __host__ __device__ int param_bytes() const { return 4 * d * params; }
    __host__ __device__ int stage_bytes() const { return batch * (row_bytes[0] + row_bytes[1] + row_bytes[2]); }
    __host__ __device__ int bytes() const { return groups * stages * stage_bytes(); }
};

__device__ __forceinline__ uint64_t l2_policy_evict_normal() {
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
__device__ __forceinline__ void bulk_load(uint32_t smem_dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(smem_dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

struct NormShared {
    uint64_t full[kNormWarps][kNormMaxStages];
    alignas(16) float part[4][2 * kNormWarps];                    // partial sums of a row's warps in multiples of four places, zeros in the rest
    int abort_flag;
};

// One thread's place in its block, and its way through the rows.  A wait that runs out (see mbar_wait) does not take the thread out of its group's
// barriers: it goes on with what the stage holds, without further waits or copies, and the status word tells.
struct NormRows {
    const NormRing& r;
    NormShared& sh;
    uint32_t data, place, params;             // the group's ring in shared memory, its present stage; gamma and beta
    int lane, group, threads;                 // lane: 0 ... threads - 1 within the group
    int stage = 0, at = 0;                    // at: row within the stage
    uint32_t phase = 0;
    uint32_t row, step;                       // step: rows from a stage's first row to that of the group's next stage
    bool ok = true;

    __device__ __forceinline__ NormRows(const NormRing& ring, NormShared& shared, const uint8_t* smem) : r(ring), sh(shared) {
        threads = 32 * r.row_warps;
        group = threadIdx.x / threads;
        lane = threadIdx.x - group * threads;
        data = place = smem_u32(smem) + group * r.stages * r.stage_bytes();
        row = (blockIdx.x * r.groups + group) * r.batch;
        step = gridDim.x * r.groups * r.batch;
        for (int i = threadIdx.x; i < 8 * kNormWarps; i += blockDim.x) (&sh.part[0][0])[i] = 0.0f;
        if (lane == 0) {
            for (int s = 0; s < r.stages; ++s) mbar_init(&sh.full[group][s], 1);
            if (group == 0) sh.abort_flag = 0;
            fence_mbar_init();
        }
        __syncthreads();
        // (the set-up above may overlap the preceding kernel's tail; nothing touches global memory before it is done)
        griddep_launch_dependents();
        griddep_wait();
        params = smem_u32(smem) + r.bytes();
        if (lane == 0)
            for (int s = 0; s < r.stages; ++s) fill(s, row + s * step);
    }
    // gamma and beta into shared memory, as fp32, each as [low, high half of every eight][d / 8] x 16 bytes, so that a warp's reads touch
    // every bank once; four loads of a thread are under way at a time
    __device__ __forceinline__ void keep_params() const {
        const int units = r.d / 8, last = units * r.params;
        for (int first = threadIdx.x; first < last; first += 4 * blockDim.x) {
            V8 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = first + k * blockDim.x;
                if (i >= last) continue;
                const void* from = r.param[i >= units];
                const int at = 8 * (i < units ? i : i - units);
                const Pair none = i < units ? both(1.0f) : both(0.0f);
                v[k] = V8{{none, none, none, none}};
                if (from) v[k] = r.p_f32 ? load8<kTypeF32>(from, at, 0) : load8<kTypeBf16>(from, at, 0);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = first + k * blockDim.x;
                if (i >= last) continue;
                const uint32_t to = params + (i < units ? 16 * i : 4 * r.d + 16 * (i - units));
                store_pairs(to, v[k].p[0], v[k].p[1]);
                store_pairs(to + 2 * r.d, v[k].p[2], v[k].p[3]);
            }
        }
        __syncthreads();
    }
    static __device__ __forceinline__ void store_pairs(uint32_t to, Pair a, Pair b) {
        asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(to), "l"(a), "l"(b) : "memory");
    }
    // gamma (0) or beta (1) of eight columns
    __device__ __forceinline__ V8 param(int which, int col) const {
        const uint32_t at = params + which * 4 * r.d + 2 * col;
        const uint4 a = lds_v4(at), b = lds_v4(at + 2 * r.d);
        return from_f32(a, b);
    }
    __device__ __forceinline__ bool live() const { return row < static_cast<uint32_t>(r.b); }
    __device__ __forceinline__ void fill(int s, uint32_t first) const {
        if (first >= static_cast<uint32_t>(r.b)) return;
        const uint32_t rows = min(static_cast<uint32_t>(r.batch), r.b - first);
        uint64_t* bar = &sh.full[group][s];
        const uint64_t policy = r.leave_first ? l2_policy_evict_first() : l2_policy_evict_normal();
        mbar_expect_tx(bar, rows * (r.row_bytes[0] + r.row_bytes[1] + r.row_bytes[2]));
        uint32_t to = data + s * r.stage_bytes();
#pragma unroll
        for (int k = 0; k < kNormMaxSources; ++k) {
            if (r.src[k]) bulk_load(to, r.src[k] + static_cast<size_t>(first) * r.row_bytes[k], rows * r.row_bytes[k], bar, policy);
            to += r.batch * r.row_bytes[k];
        }
    }
    // waits for the row; the address of source k's row is then source(k)
    __device__ __forceinline__ void wait() {
        if (at == 0) ok = ok && mbar_wait(&sh.full[group][stage], phase, &sh.abort_flag);
    }
    __device__ __forceinline__ uint32_t source(int k) const {
        uint32_t a = place + at * r.row_bytes[k];
        for (int j = 0; j < k; ++j) a += r.batch * r.row_bytes[j];
        return a;
    }
    __device__ __forceinline__ bool ends_stage() const { return at + 1 == r.batch || row + 1 == static_cast<uint32_t>(r.b); }
    // the group's row after this one
    __device__ __forceinline__ uint32_t next() const { return ends_stage() ? row - at + step : row + 1; }
    // (barrier 0 is __syncthreads; a group of one warp needs none)
    __device__ __forceinline__ void sync() const {
        if (r.row_warps == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
    }
    // to the next row, once all threads of the group have read this one (a sync() lies behind their reads)
    __device__ __forceinline__ void advance() {
        if (!ends_stage()) {
            ++at;
            ++row;
            return;
        }
        const uint32_t first = row - at;
        if (lane == 0 && ok) fill(stage, first + r.stages * step);
        place += r.stage_bytes();
        if (++stage == r.stages) {
            stage = 0;
            place = data;
            phase ^= 1u;
        }
        at = 0;
        row = first + step;
    }
    // copies that are still under way after a wait ran out land before the block's memory goes
    __device__ __forceinline__ void leave() const {
        __syncthreads();
        if (*const_cast<volatile int*>(&sh.abort_flag)) drain_after_abort();
    }
    // the sum over the group's lanes; of several sums in flight each has a `slot` of its own
    __device__ __forceinline__ void begin_sum(float& v, int slot) const {
        v = warp_sum(v);
        if (r.row_warps > 1 && (lane & 31) == 0) sh.part[slot][group * padded(r.row_warps) + (lane >> 5)] = v;
    }
    static __device__ __forceinline__ int padded(int row_warps) { return (row_warps + 3) & ~3; }
    // (a sync() lies between the two)
    __device__ __forceinline__ float end_sum(float v, int slot) const {
        if (r.row_warps == 1) return v;
        const float4* part = reinterpret_cast<const float4*>(sh.part[slot] + group * padded(r.row_warps));
        float4 t = part[0];
        for (int w = 4; w < r.row_warps; w += 4) {
            const float4 u = part[w >> 2];
            t = make_float4(t.x + u.x, t.y + u.y, t.z + u.z, t.w + u.w);
        }
        return (t.x + t.y) + (t.z + t.w);
    }
};

__device__ __forceinline__ float min_nan(float a, float b) {
    float m;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}

struct NormFwdParams {
    NormRing ring;                // X, residual
    void *H, *Y, *H_ckpt, *Y_ckpt;
    float *mean, *rstd;
    float eps;
};

// The rows of a group among which some left fp32: their sum, or the sum of their squared differences.  They stand there with an rstd of 0
// or NaN and are done once more from the beginning: the mean in units of 2^16 (d / 2^16 of the largest number at most), the variance
// in units of 2^144, of which d differences of at most 2^128 have d 2^112.  A difference that is itself none of fp32's, or an infinity
// or a NaN in the row, leaves rstd and Y NaN.  Which rows: those that the loop left so, found by its own sums once more, so that a
// row's bits do not depend on its neighbours.  h comes from H or, where none is kept, from the inputs (H may be one of them); every
// thread writes what it has written before.
// Behind the loop over the rows, out of line and without arguments that the loop would have to keep, so that other rows pay one minimum.
// us, without / so / called within the loop / inlined behind it: 8192 x 5120 34.9 / 34.8 / 36.2 / 38.4, 8192 x 2304
// 16.7 / 16.6 / 17.6 / 17.7, 4096 x 8448 31.4 / 31.4 / 33.1 / 32.8, 4096 x 16384 with residual 105 / 98 / 99 / 99, 16384 x 4096 in
// fp32 with residual 128 / 130 / 126 / 135.
template <int TYPE, bool RESIDUAL, bool CKPT>
__device__ __noinline__ void layer_norm_wide_rows(const NormFwdParams& p, NormShared& sh, const uint8_t* smem) {
    const int d = p.ring.d, warps = p.ring.row_warps, threads = 32 * warps, group = threadIdx.x / threads, lane = threadIdx.x - group * threads;
    const uint32_t params = smem_u32(smem) + p.ring.bytes();
    const float per = 1.0f / d;
    const size_t count = static_cast<size_t>(p.ring.b) * d;
    size_t base = 0;
    const auto stream = [&](int col) {
        if (!RESIDUAL) return load8<TYPE>(p.ring.src[0], base + col, 0);
        if (p.H) return load8<TYPE>(p.H, base + col, 0);
        V8 h = load8<TYPE>(p.ring.src[0], base + col, 0);
        const V8 r = load8<kTypeBf16>(p.ring.src[1], base + col, 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) h.p[k] = add2(h.p[k], r.p[k]);
        return TYPE == kTypeBf16 ? from_bf16(to_bf16(h)) : h;
    };
    const auto group_sum = [&](const Pair (&part)[2], int slot) {
        const Pair both_parts = add2(part[0], part[1]);
        const float v = warp_sum(low(both_parts) + high(both_parts));
        if (warps == 1) return v;
        float* place = sh.part[slot] + group * NormRows::padded(warps);
        if ((lane & 31) == 0) place[lane >> 5] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
        const float4* sums = reinterpret_cast<const float4*>(place);              // (as NormRows::end_sum adds them)
        float4 t = sums[0];
        for (int w = 4; w < warps; w += 4) {
            const float4 u = sums[w >> 2];
            t = make_float4(t.x + u.x, t.y + u.y, t.z + u.z, t.w + u.w);
        }
        return (t.x + t.y) + (t.z + t.w);
    };
    // The row's sum and that of its squared differences, in units and with the loop's order of additions
    const auto sum_of = [&](float unit, int slot) {
        Pair part[2] = {0, 0};
        for (int col = 8 * lane; col < d; col += 8 * threads) {
            const V8 h = stream(col);
#pragma unroll
            for (int k = 0; k < 4; ++k) part[k & 1] = fma2(h.p[k], both(unit), part[k & 1]);
        }
        return group_sum(part, slot);
    };
    const auto squares_of = [&](float mean, float unit, int slot) {
        Pair part[2] = {0, 0};
        for (int col = 8 * lane; col < d; col += 8 * threads) {
            const V8 h = stream(col);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const Pair v = mul2(add2(h.p[k], both(-mean)), both(unit));
                part[k & 1] = fma2(v, v, part[k & 1]);
            }
        }
        return group_sum(part, slot);
    };
    // (batches of adjacent rows, as NormRows goes through them)
    const uint32_t b = p.ring.b, batch = p.ring.batch, step = gridDim.x * p.ring.groups * batch;
    for (uint32_t first = (blockIdx.x * p.ring.groups + group) * batch; first < b; first += step) {
        for (uint32_t row = first; row < min(first + batch, b); ++row) {
            base = static_cast<size_t>(row) * d;
            if (squares_of(sum_of(1.0f, 0) * per, 1.0f, 1) * per + p.eps <= FLT_MAX) continue;
            const float mean = sum_of(0x1p-16f, 2) * per * 0x1p16f;
            const float var = squares_of(mean, 0x1p-72f, 3) * per + p.eps * 0x1p-72f * 0x1p-72f;
            const Pair less = both(-mean);
            const float rstd = var <= FLT_MAX ? rsqrtf(var) * 0x1p-72f : __uint_as_float(0x7FC00000u);
            if (p.mean && lane == 0) {
                p.mean[row] = mean;
                p.rstd[row] = rstd;
            }
            for (int at = 0; at < d; at += 8 * threads) {
                const int col = at + 8 * lane;
                V8 y = zeros();
                if (col < d) {
                    y = stream(col);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint4 g = lds_v4(params + 2 * col + 2 * d * half), c = lds_v4(params + 4 * d + 2 * col + 2 * d * half);
                        Pair* v = y.p + 2 * half;
                        v[0] = fma2(mul2(add2(v[0], less), both(rstd)), pair(g.x, g.y), pair(c.x, c.y));
                        v[1] = fma2(mul2(add2(v[1], less), both(rstd)), pair(g.z, g.w), pair(c.z, c.w));
                    }
                    const uint4 w = to_bf16(y);
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.Y) + base + col) = w;
                    if (CKPT && p.Y_ckpt) y = from_bf16(w);
                }
                if (CKPT && p.Y_ckpt) store_q8(p.Y_ckpt, base + col, count, col < d, y);
            }
        }
    }
}

// FULL: every lane has all its columns.  CKPT: with checkpoints.
template <int TYPE, int CHUNKS, bool FULL, bool RESIDUAL, bool CKPT>
__global__ void __launch_bounds__(32 * kNormFwdWarps, 1) layer_norm_fwd_kernel(const __grid_constant__ NormFwdParams p) {
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ NormShared sh;
    NormRows rows(p.ring, sh, smem);
    rows.keep_params();
    const int d = p.ring.d;
    const float per = 1.0f / d;
    const size_t count = static_cast<size_t>(p.ring.b) * d;
    const int col0 = 8 * rows.lane, col_step = 8 * rows.threads;
    float least = 1.0f;                       // of the rows' rstd: 0 or NaN where a sum left fp32's range
    while (rows.live()) {
        const uint32_t row = rows.row;
        const size_t base = static_cast<size_t>(row) * d + col0;
        rows.wait();
        const uint32_t x_row = rows.source(0), r_row = rows.source(1);
        V8 h[CHUNKS];
        Pair part[2] = {0, 0};                 // (sums in turn: each addition takes four clocks)
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = col0 + col_step * i;
            if (!FULL) h[i] = zeros();
            if (FULL || col < d) {
                h[i] = shared8<TYPE>(x_row, col);
                if (RESIDUAL) {
                    const V8 r = shared8<kTypeBf16>(r_row, col);
#pragma unroll
                    for (int k = 0; k < 4; ++k) h[i].p[k] = add2(h[i].p[k], r.p[k]);
                    // the stream as it is stored is what is normalised, so that the backward pass sees the same one
                    if (TYPE == kTypeBf16) {
                        const uint4 w = to_bf16(h[i]);
                        if (p.H) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.H) + base + col_step * i) = w;
                        h[i] = from_bf16(w);
                    } else if (p.H) {
                        store8<TYPE>(p.H, base + col_step * i, h[i]);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) part[k & 1] = add2(part[k & 1], h[i].p[k]);
        }
        part[0] = add2(part[0], part[1]);
        float sum = low(part[0]) + high(part[0]);
        rows.begin_sum(sum, 0);
        rows.sync();
        const float mean = rows.end_sum(sum, 0) * per;
        rows.advance();
        const Pair less = both(-mean);
        part[0] = part[1] = 0;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const bool live = FULL || col0 + col_step * i < d;
            if (CKPT && p.H_ckpt) store_q8(p.H_ckpt, base + col_step * i, count, live, h[i]);
            if (live) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    h[i].p[k] = add2(h[i].p[k], less);
                    part[k & 1] = fma2(h[i].p[k], h[i].p[k], part[k & 1]);
                }
            }
        }
        part[0] = add2(part[0], part[1]);
        float sq = low(part[0]) + high(part[0]);
        rows.begin_sum(sq, 1);
        rows.sync();
        const float var = rows.end_sum(sq, 1) * per + p.eps;
        const float rstd = rsqrtf(var);
        least = min_nan(least, rstd);
        if (p.mean && rows.lane == 0) {
            p.mean[row] = mean;
            p.rstd[row] = rstd;
        }
        const Pair scale = both(rstd);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = col0 + col_step * i;
            const bool live = FULL || col < d;
            V8 y = h[i];
            if (live) {
#pragma unroll
                for (int k = 0; k < 4; ++k) y.p[k] = mul2(y.p[k], scale);
                const V8 g = rows.param(0, col), c = rows.param(1, col);
#pragma unroll
                for (int k = 0; k < 4; ++k) y.p[k] = fma2(y.p[k], g.p[k], c.p[k]);
                const uint4 w = to_bf16(y);
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.Y) + base + col_step * i) = w;
                if (CKPT && p.Y_ckpt) y = from_bf16(w);                   // the checkpoint is that of the Y which the linears read
            }
            if (CKPT && p.Y_ckpt) store_q8(p.Y_ckpt, base + col_step * i, count, live, y);
        }
    }
    if (!(least > 0.0f)) layer_norm_wide_rows<TYPE, RESIDUAL, CKPT>(p, sh, smem);      // (the same in all threads of the group)
    rows.leave();
}

struct NormBwdParams {
    NormRing ring;                // H (codes, if it is a checkpoint), dY, dH
    const uint8_t* exponents;     // of a checkpoint
    const float *mean, *rstd;
    void *dX, *dgamma, *dbeta;
    float* partial;               // [blocks][2][d]: sums of dY x and of dY over the block's rows
};

__device__ __forceinline__ void store_param(void* base, bool f32, int at, float v) {
    if (f32) static_cast<float*>(base)[at] = v;
    else static_cast<uint16_t*>(base)[at] = to_bf16(v);
}

// gamma's and beta's gradients grow in registers; at the end the groups' sums meet in shared memory (where the ring was) and are added in
// order, and the blocks' sums are added in order by layer_norm_params_kernel (a single block writes the gradients itself).  The order
// depends on the sizes alone.
// Registers are what it is short of: four chunks' sums take 64, so that from three chunks on a row's values are not kept between its two
// sums and its output but read from the ring and normalised again.  us, one / two (kept) / four (read again) chunks per lane: 16384 x 4096
// 140 / 94 / 94, 8192 x 5120 from 8 bits 76 / 98 / 76, 4096 x 8192 56 / 58 / 56, 8192 x 768 from 8 bits 18.9 / 21 / 18.9 (three chunks).
// At 128 registers ten of the 96 instances spill 4 to 48 bytes (the full one of four chunks in bf16 with dH 12, from 8 bits 44).
template <int TYPE, int DX_TYPE, int CHUNKS, bool FULL, bool SIDE>
__global__ void __launch_bounds__(32 * kNormBwdWarps, 1) layer_norm_bwd_kernel(const __grid_constant__ NormBwdParams p) {
    constexpr bool kReread = CHUNKS > 2;      // a row does not fit in registers beside its columns' sums: it is read from the ring twice
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ NormShared sh;
    NormRows rows(p.ring, sh, smem);
    const int d = p.ring.d;
    const int col0 = 8 * rows.lane, col_step = 8 * rows.threads;
    const float per = 1.0f / d;
    const bool gain = p.ring.param[0] != nullptr;
    V8 acc_g[CHUNKS], acc_b[CHUNKS], gamma[kReread ? 1 : CHUNKS];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) acc_g[i] = acc_b[i] = zeros();
    uint32_t e[CHUNKS] = {};
    float next_mean = 0.0f, next_rstd = 0.0f;
    // what is not in the ring, one row ahead
    auto ahead = [&](uint32_t row) {
        if (row >= static_cast<uint32_t>(p.ring.b)) return;
        next_mean = __uint_as_float(ld_u32(p.mean + row));
        next_rstd = __uint_as_float(ld_u32(p.rstd + row));
        if (TYPE == kTypeQ8) {
            const uint8_t* at = p.exponents + (static_cast<size_t>(row) * d + col0) / kQBlock;
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (FULL || col0 + col_step * i < d) e[i] = ld_u8(at + rows.threads / 4 * i);
        }
    };
    ahead(rows.row);
    if (kReread) {
        rows.keep_params();
    } else {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = col0 + col_step * i, at = kReread ? 0 : i;
            gamma[at] = V8{{both(1.0f), both(1.0f), both(1.0f), both(1.0f)}};
            if (gain && col < d) gamma[at] = p.ring.p_f32 ? load8<kTypeF32>(p.ring.param[0], col, 0) : load8<kTypeBf16>(p.ring.param[0], col, 0);
        }
    }
    for (int slot = 0; rows.live(); slot ^= 2) {
        const size_t base = static_cast<size_t>(rows.row) * d + col0;
        rows.wait();
        const uint32_t h_row = rows.source(0), g_row = rows.source(1), r_row = rows.source(2);
        const float rstd = next_rstd;
        const Pair less = both(-next_mean), scale = both(rstd);
        V8 g[kReread ? 1 : CHUNKS], x[kReread ? 1 : CHUNKS];
        Pair p1[2] = {0, 0}, p2[2] = {0, 0};  // (sums in turn: each addition takes four clocks)
        // normalised values of chunk i
        auto normalised = [&](int i) {
            V8 v = shared8<TYPE>(h_row, col0 + col_step * i, e[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) v.p[k] = mul2(add2(v.p[k], less), scale);
            return v;
        };
        // dY gamma of chunk i from dY
        auto gained = [&](int i, V8& v) {
            const V8 w = kReread ? rows.param(0, col0 + col_step * i) : gamma[kReread ? 0 : i];
#pragma unroll
            for (int k = 0; k < 4; ++k) v.p[k] = mul2(v.p[k], w.p[k]);
        };
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int at = kReread ? 0 : i, col = col0 + col_step * i;
            if (FULL || col < d) {
                x[at] = normalised(i);
                g[at] = shared8<kTypeBf16>(g_row, col);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    acc_g[i].p[k] = fma2(g[at].p[k], x[at].p[k], acc_g[i].p[k]);
                    acc_b[i].p[k] = add2(acc_b[i].p[k], g[at].p[k]);
                }
                gained(i, g[at]);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    p1[k & 1] = add2(p1[k & 1], g[at].p[k]);
                    p2[k & 1] = fma2(g[at].p[k], x[at].p[k], p2[k & 1]);
                }
            }
        }
        if (!kReread) ahead(rows.next());
        p1[0] = add2(p1[0], p1[1]);
        p2[0] = add2(p2[0], p2[1]);
        float s1 = low(p1[0]) + high(p1[0]), s2 = low(p2[0]) + high(p2[0]);
        rows.begin_sum(s1, slot);
        rows.begin_sum(s2, slot + 1);
        rows.sync();
        const Pair m1 = both(-rows.end_sum(s1, slot) * per), m2 = both(-rows.end_sum(s2, slot + 1) * per);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int at = kReread ? 0 : i, col = col0 + col_step * i;
            if (FULL || col < d) {
                if (kReread) {
                    x[0] = normalised(i);
                    g[0] = shared8<kTypeBf16>(g_row, col);
                    gained(i, g[0]);
                }
                const V8 r = SIDE ? shared8<DX_TYPE>(r_row, col) : zeros();
                V8 dx;
#pragma unroll
                for (int k = 0; k < 4; ++k) dx.p[k] = fma2(scale, fma2(x[at].p[k], m2, add2(g[at].p[k], m1)), r.p[k]);
                store8<DX_TYPE>(p.dX, base + col_step * i, dx);
            }
        }
        if (kReread) ahead(rows.next());
        if (kReread || SIDE) rows.sync();                         // the stage was read behind the sums' barrier
        rows.advance();
    }
    rows.leave();
    if (!p.dgamma && !p.dbeta) return;
    float* out = p.partial + static_cast<size_t>(blockIdx.x) * 2 * d;
    if (p.ring.groups == 1 && gridDim.x > 1) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = col0 + col_step * i;
            if (col >= d) continue;
            store8<kTypeF32>(out, col, acc_g[i]);
            store8<kTypeF32>(out + d, col, acc_b[i]);
        }
        return;
    }
    float* sums = reinterpret_cast<float*>(smem);                 // [groups][2][d]
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int col = col0 + col_step * i;
        if (col >= d) continue;
        store8<kTypeF32>(sums + rows.group * 2 * d, col, acc_g[i]);
        store8<kTypeF32>(sums + rows.group * 2 * d + d, col, acc_b[i]);
    }
    __syncthreads();
    for (int at = 4 * threadIdx.x; at < 2 * d; at += 4 * blockDim.x) {
        float4 t = *reinterpret_cast<const float4*>(sums + at);
        for (int k = 1; k < p.ring.groups; ++k) {
            const float4 u = *reinterpret_cast<const float4*>(sums + k * 2 * d + at);
            t = make_float4(t.x + u.x, t.y + u.y, t.z + u.z, t.w + u.w);
        }
        if (gridDim.x > 1) {
            *reinterpret_cast<float4*>(out + at) = t;
        } else {
            void* grad = at < d ? p.dgamma : p.dbeta;
            const int c = at < d ? at : at - d;
            if (!grad) continue;
            store_param(grad, p.ring.p_f32, c, t.x);
            store_param(grad, p.ring.p_f32, c + 1, t.y);
            store_param(grad, p.ring.p_f32, c + 2, t.z);
            store_param(grad, p.ring.p_f32, c + 3, t.w);
        }
    }
}

// dgamma and dbeta from the blocks' sums: a block takes 32 of the 2 d columns, its 32 slices of 8 threads every 32nd of the sums, which are
// then added in order.
__global__ void __launch_bounds__(256) layer_norm_params_kernel(const float* partial, int blocks, int d, void* dgamma, void* dbeta, int p_f32) {
    __shared__ float part[32][33];
    griddep_launch_dependents();
    griddep_wait();
    const int slice = threadIdx.x >> 3, c4 = 4 * (threadIdx.x & 7), col = 32 * blockIdx.x + c4;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (col < 2 * d) {
#pragma unroll 5
        for (int s = slice; s < blocks; s += 32) {
            const uint4 v = ld_v4(partial + static_cast<size_t>(s) * 2 * d + col);
            sum.x += __uint_as_float(v.x);
            sum.y += __uint_as_float(v.y);
            sum.z += __uint_as_float(v.z);
            sum.w += __uint_as_float(v.w);
        }
    }
    part[slice][c4] = sum.x;
    part[slice][c4 + 1] = sum.y;
    part[slice][c4 + 2] = sum.z;
    part[slice][c4 + 3] = sum.w;
    __syncthreads();
    const int at = 32 * blockIdx.x + threadIdx.x;
    if (threadIdx.x < 32 && at < 2 * d) {
        float total = part[0][threadIdx.x];
#pragma unroll
        for (int s = 1; s < 32; ++s) total += part[s][threadIdx.x];
        if (at < d) {
            if (dgamma) store_param(dgamma, p_f32, at, total);
        } else if (dbeta) {
            store_param(dbeta, p_f32, at - d, total);
        }
    }
}

}  // namespace slope
