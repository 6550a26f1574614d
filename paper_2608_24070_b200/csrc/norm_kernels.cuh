// Layer norm between the sparse layers, forward and backward, and the 8-bit checkpoints of activations that the backward
// pass reads in place of bf16 ones.
//
//   forward    h = X (+ residual),  m = mean(h),  s = 1 / sqrt(mean((h - m)^2) + eps),  y = (h - m) s gamma + beta
//   backward   x = (h - m) s,  g = dY gamma,  dX = s (g - mean(g) - x mean(g x)) (+ dH),
//              dgamma = sum over the tokens of dY x,  dbeta = sum over the tokens of dY
//
// Everything here is bound by HBM: every matrix is read once and written once, and a row stays in registers
// between its statistics and its output.  All sums are fp32; the variance is that of the differences from the mean, not
// mean(h^2) - m^2, which cancels where a row's mean is large beside its spread.
//
// Checkpoint of a matrix [rows x cols], cols a multiple of 32: each block of 32 consecutive values of a row is 32 signed bytes
// times one power of two, 2^k, k the smallest integer for which the block's largest magnitude is at most 127.5 * 2^k, within
// [-126, 121]; codes are rounded half to even and held in [-127, 127].  A value is off by at most half a unit of 2^k, i.e.
// 1/127 of the block's largest magnitude at most (a power of two wastes at most half of the code's range; e4m3 codes, with the
// same 8 bits, are off by up to 1/16 of a value, for Gaussian activations 2.6 % in the mean square against 0.7 %).  A code has seven
// significant bits, so a value that is read back is exact in bf16, and a product with it has exactly that operand.
// Memory: rows * cols codes, then rows * cols / 32 bytes k + 127 (the exponent field of 2^k as fp32); 255, with codes of 0, in a block
// that holds an infinity or a NaN, whose values are NaN, so that an overflow still shows in the gradients.
#pragma once
#include "ptx.cuh"

namespace slope {

constexpr int kTypeBf16 = 0, kTypeF32 = 1, kTypeQ8 = 2;          // == slope_type_t
constexpr int kQBlock = 32;

// ---------------------------------------------------------------- eight values of a row, as fp32
__device__ __forceinline__ void unpack_bf16(const uint4& w, float (&v)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack_bf16(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ void unpack_f32(const uint4& a, const uint4& b, float (&v)[8]) {
    const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
}
// The byte q of `w` is put into the mantissa of 2^23 as q + 128; taking 2^23 + 128 away leaves q.  (A multiplication by 2^k is exact.)
__device__ __forceinline__ void unpack_q8(const uint2& w, float unit, float (&v)[8]) {
    const uint32_t u[2] = {w.x ^ 0x80808080u, w.y ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = (__uint_as_float(prmt(u[i >> 2], 0x4B000000u, 0x7650u | (i & 3))) - 8388736.0f) * unit;
}
// Raw words of eight values, so that a row can be in flight before it is needed.
template <int TYPE>
struct Raw8;
template <>
struct Raw8<kTypeBf16> {
    uint4 w;
    __device__ __forceinline__ void load(const void* base, size_t at, size_t) { w = ld_v4(static_cast<const uint16_t*>(base) + at); }
    __device__ __forceinline__ void values(float (&v)[8]) const { unpack_bf16(w, v); }
};
template <>
struct Raw8<kTypeF32> {
    uint4 w0, w1;
    __device__ __forceinline__ void load(const void* base, size_t at, size_t) {
        w0 = ld_v4(static_cast<const float*>(base) + at);
        w1 = ld_v4(static_cast<const float*>(base) + at + 4);
    }
    __device__ __forceinline__ void values(float (&v)[8]) const { unpack_f32(w0, w1, v); }
};
template <>
struct Raw8<kTypeQ8> {
    uint2 w;
    uint32_t e;
    // `count`: values of the whole matrix; the exponents stand behind them
    __device__ __forceinline__ void load(const void* base, size_t at, size_t count) {
        const uint8_t* p = static_cast<const uint8_t*>(base);
        w = ld_v2(p + at);
        e = ld_u8(p + count + at / kQBlock);
    }
    __device__ __forceinline__ void values(float (&v)[8]) const { unpack_q8(w, __uint_as_float(e << 23), v); }
};
// parameters: of the type that `f32` says
__device__ __forceinline__ void load_params(const void* base, bool f32, int at, float (&v)[8]) {
    if (f32) {
        const float* p = static_cast<const float*>(base) + at;
        unpack_f32(ld_v4(p), ld_v4(p + 4), v);
    } else {
        unpack_bf16(ld_v4(static_cast<const uint16_t*>(base) + at), v);
    }
}
template <int TYPE>
__device__ __forceinline__ void store8(void* base, size_t at, const float (&v)[8]) {
    if (TYPE == kTypeBf16) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) = pack_bf16(v);
    } else {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
        p[0] = make_float4(v[0], v[1], v[2], v[3]);
        p[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// Eight values to codes; four neighbouring lanes hold a block.  All lanes of the warp take part.  The exponent: that of the
// largest magnitude less 6, one more where its mantissa is above 127.5 / 64 (0x7F0000: then 0xFFFF carries into the exponent).
// Rounding: 1.5 * 2^23 added (fused with the exact multiplication by 2^-k) leaves the code in the low byte.
__device__ __forceinline__ uint2 encode8(const float (&v)[8], uint32_t& e) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    if (m >= 0x7F800000u) {
        e = 255u;
        return make_uint2(0u, 0u);
    }
    e = static_cast<uint32_t>(min(max(static_cast<int>((m + 0xFFFFu) >> 23) - 6, 1), 248));
    const float per_unit = __uint_as_float((254u - e) << 23);
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = __fmaf_rn(v[i], per_unit, 12582912.0f);
        c[i] = __float_as_uint(fminf(fmaxf(t, 12582912.0f - 127.0f), 12582912.0f + 127.0f));
    }
    return make_uint2(prmt(prmt(c[0], c[1], 0x0040u), prmt(c[2], c[3], 0x0040u), 0x5410u),
                      prmt(prmt(c[4], c[5], 0x0040u), prmt(c[6], c[7], 0x0040u), 0x5410u));
}
// `at`: the place of the eight values in the matrix of `count`; `live`: whether the lane has any
__device__ __forceinline__ void store_q8(void* ckpt, size_t at, size_t count, bool live, const float (&v)[8]) {
    uint32_t e;
    const uint2 codes = encode8(v, e);
    if (!live) return;
    uint8_t* p = static_cast<uint8_t*>(ckpt);
    *reinterpret_cast<uint2*>(p + at) = codes;
    if ((threadIdx.x & 3) == 0) p[count + at / kQBlock] = static_cast<uint8_t>(e);
}

// ---------------------------------------------------------------- matrices to checkpoints and back
// A thread takes eight values at a time; `n8` of them in all, a multiple of 4, so that a block's four lanes live or rest together.
template <int TYPE>
__global__ void __launch_bounds__(256) checkpoint_store_kernel(const void* X, size_t n8, void* ckpt) {
    griddep_stream(8);
    const size_t stride = static_cast<size_t>(gridDim.x) * blockDim.x;
    for (size_t first = static_cast<size_t>(blockIdx.x) * blockDim.x; first < n8; first += stride) {
        const size_t i = first + threadIdx.x;
        const bool live = i < n8;
        float v[8] = {};
        if (live) {
            Raw8<TYPE> x;
            x.load(X, 8 * i, 0);
            x.values(v);
        }
        store_q8(ckpt, 8 * i, 8 * n8, live, v);
    }
}
template <int TYPE>
__global__ void __launch_bounds__(256) checkpoint_load_kernel(const void* ckpt, size_t n8, void* X) {
    griddep_stream(8);
    const size_t stride = static_cast<size_t>(gridDim.x) * blockDim.x;
    for (size_t i = static_cast<size_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < n8; i += stride) {
        Raw8<kTypeQ8> x;
        float v[8];
        x.load(ckpt, 8 * i, 8 * n8);
        x.values(v);
        store8<TYPE>(X, 8 * i, v);
    }
}

// ---------------------------------------------------------------- layer norm
// A row belongs to a group of `row_warps` warps; a lane holds CHUNKS times eight of its columns, chunk i of lane l at
// column 8 (l + 32 row_warps i).  A block has as many groups as fit, each walks over rows of its own.
struct RowGroup {
    int lane, group, groups, threads;      // lane: 0 ... threads - 1 within the group
    __device__ __forceinline__ explicit RowGroup(int row_warps) {
        threads = 32 * row_warps;
        groups = blockDim.x / threads;
        group = threadIdx.x / threads;
        lane = threadIdx.x - group * threads;
    }
    // (barrier 0 is __syncthreads)
    __device__ __forceinline__ void sync() const { asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory"); }
};
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
constexpr int kNormMaxWidth = 16384, kNormMaxGroups = 15;
constexpr int kNormThreads = 512;                                 // threads of a block at most, unless one row needs more

struct NormFwdParams {
    const void *X, *residual, *gamma, *beta;
    void *H, *Y, *H_ckpt, *Y_ckpt;
    float *mean, *rstd;
    int b, d, row_warps, p_f32;
    float eps;
};

template <int TYPE, int CHUNKS>
__global__ void __launch_bounds__(kNormThreads) layer_norm_fwd_kernel(const NormFwdParams p) {
    __shared__ float part[2][kNormThreads / 32];
    griddep_launch_dependents();
    griddep_wait();
    const RowGroup rg(p.row_warps);
    const int warp0 = rg.group * p.row_warps;
    const float per = 1.0f / p.d;
    const size_t count = static_cast<size_t>(p.b) * p.d;
    // the sum over the row of what the lanes hold; `slot` alternates, so that one barrier per sum is enough
    auto row_sum = [&](float v, int slot) {
        v = warp_sum(v);
        if (p.row_warps == 1) return v;
        if ((rg.lane & 31) == 0) part[slot][threadIdx.x >> 5] = v;
        rg.sync();
        float total = 0.0f;
        for (int w = 0; w < p.row_warps; ++w) total += part[slot][warp0 + w];
        return total;
    };
    for (size_t row = static_cast<size_t>(blockIdx.x) * rg.groups + rg.group; row < static_cast<size_t>(p.b);
         row += static_cast<size_t>(gridDim.x) * rg.groups) {
        const size_t base = row * p.d;
        float h[CHUNKS][8];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = 8 * (rg.lane + rg.threads * i);
#pragma unroll
            for (int k = 0; k < 8; ++k) h[i][k] = 0.0f;
            if (col < p.d) {
                Raw8<TYPE> x;
                x.load(p.X, base + col, 0);
                x.values(h[i]);
                if (p.residual) {
                    float r[8];
                    unpack_bf16(ld_v4(static_cast<const uint16_t*>(p.residual) + base + col), r);
#pragma unroll
                    for (int k = 0; k < 8; ++k) h[i][k] += r[k];
                    // the stream as it is stored is what is normalised, so that the backward pass sees the same one
                    if (TYPE == kTypeBf16) unpack_bf16(pack_bf16(h[i]), h[i]);
                    if (p.H) store8<TYPE>(p.H, base + col, h[i]);
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += h[i][k];
        }
        const float mean = row_sum(sum, 0) * per;
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = 8 * (rg.lane + rg.threads * i);
            if (p.H_ckpt) store_q8(p.H_ckpt, base + col, count, col < p.d, h[i]);
            if (col < p.d) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    h[i][k] -= mean;
                    sq = __fmaf_rn(h[i][k], h[i][k], sq);
                }
            }
        }
        const float rstd = rsqrtf(row_sum(sq, 1) * per + p.eps);
        if (p.mean && rg.lane == 0) {
            p.mean[row] = mean;
            p.rstd[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = 8 * (rg.lane + rg.threads * i);
            float y[8] = {};
            if (col < p.d) {
                float g[8], c[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    g[k] = 1.0f;
                    c[k] = 0.0f;
                }
                if (p.gamma) load_params(p.gamma, p.p_f32, col, g);
                if (p.beta) load_params(p.beta, p.p_f32, col, c);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = __fmaf_rn(h[i][k] * rstd, g[k], c[k]);
                const uint4 w = pack_bf16(y);
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.Y) + base + col) = w;
                unpack_bf16(w, y);                                // the checkpoint is that of the Y which the linears read
            }
            if (p.Y_ckpt) store_q8(p.Y_ckpt, base + col, count, col < p.d, y);
        }
    }
}

struct NormBwdParams {
    const void *dY, *H, *gamma, *dH;
    const float *mean, *rstd;
    void *dX, *dgamma, *dbeta;
    float* partial;               // [blocks][2][d]: sums of dY x and of dY over the block's rows
    int b, d, row_warps, p_f32;
};

__device__ __forceinline__ void store_param(void* base, bool f32, int at, float v) {
    if (f32) static_cast<float*>(base)[at] = v;
    else static_cast<uint16_t*>(base)[at] = to_bf16(v);
}

// The columns of a lane are the same in all rows, so gamma's and beta's gradients grow in registers; at the end the groups of a block
// add theirs in order through shared memory, and the blocks' sums are added in order by layer_norm_params_kernel (a single
// block writes the gradients itself).
template <int TYPE, int DX_TYPE, int CHUNKS, int THREADS>
__global__ void __launch_bounds__(THREADS) layer_norm_bwd_kernel(const NormBwdParams p) {
    __shared__ float2 part[2][32];
    extern __shared__ float4 sums4[];                             // [2][d], only with several groups
    float* sums = reinterpret_cast<float*>(sums4);
    griddep_launch_dependents();
    griddep_wait();
    const RowGroup rg(p.row_warps);
    const int warp0 = rg.group * p.row_warps;
    const float per = 1.0f / p.d;
    const size_t count = static_cast<size_t>(p.b) * p.d;
    const bool params = p.dgamma || p.dbeta;
    float acc_g[CHUNKS][8] = {}, acc_b[CHUNKS][8] = {};
    int slot = 0;
    for (size_t row = static_cast<size_t>(blockIdx.x) * rg.groups + rg.group; row < static_cast<size_t>(p.b);
         row += static_cast<size_t>(gridDim.x) * rg.groups, slot ^= 1) {
        const size_t base = row * p.d;
        const float mean = __uint_as_float(ld_u32(p.mean + row)), rstd = __uint_as_float(ld_u32(p.rstd + row));
        float g[CHUNKS][8], x[CHUNKS][8];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = 8 * (rg.lane + rg.threads * i);
            if (col < p.d) {
                Raw8<TYPE> raw;
                raw.load(p.H, base + col, count);
                unpack_bf16(ld_v4(static_cast<const uint16_t*>(p.dY) + base + col), g[i]);
                raw.values(x[i]);
                float w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = 1.0f;
                if (p.gamma) load_params(p.gamma, p.p_f32, col, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    x[i][k] = (x[i][k] - mean) * rstd;
                    acc_g[i][k] = __fmaf_rn(g[i][k], x[i][k], acc_g[i][k]);
                    acc_b[i][k] += g[i][k];
                    g[i][k] *= w[k];
                    s1 += g[i][k];
                    s2 = __fmaf_rn(g[i][k], x[i][k], s2);
                }
            }
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if (p.row_warps > 1) {
            if ((rg.lane & 31) == 0) part[slot][threadIdx.x >> 5] = make_float2(s1, s2);
            rg.sync();
            s1 = s2 = 0.0f;
            for (int w = 0; w < p.row_warps; ++w) {
                const float2 v = part[slot][warp0 + w];
                s1 += v.x;
                s2 += v.y;
            }
        }
        s1 *= per;
        s2 *= per;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int col = 8 * (rg.lane + rg.threads * i);
            if (col < p.d) {
                float dx[8], r[8] = {};
                if (p.dH) {
                    Raw8<DX_TYPE> raw;
                    raw.load(p.dH, base + col, 0);
                    raw.values(r);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) dx[k] = __fmaf_rn(rstd, g[i][k] - s1 - x[i][k] * s2, r[k]);
                store8<DX_TYPE>(p.dX, base + col, dx);
            }
        }
    }
    if (!params) return;
    // the groups' sums, one group after the other
    for (int turn = 0; turn < rg.groups; ++turn) {
        if (rg.group == turn) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int col = 8 * (rg.lane + rg.threads * i);
                if (col >= p.d) continue;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (turn) {
                        acc_g[i][k] += sums[col + k];
                        acc_b[i][k] += sums[p.d + col + k];
                    }
                    if (turn + 1 < rg.groups) {
                        sums[col + k] = acc_g[i][k];
                        sums[p.d + col + k] = acc_b[i][k];
                    }
                }
                if (turn + 1 < rg.groups) continue;
                if (gridDim.x > 1) {
                    float* out = p.partial + static_cast<size_t>(blockIdx.x) * 2 * p.d + col;
                    store8<kTypeF32>(out, 0, acc_g[i]);
                    store8<kTypeF32>(out + p.d, 0, acc_b[i]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (p.dgamma) store_param(p.dgamma, p.p_f32, col + k, acc_g[i][k]);
                        if (p.dbeta) store_param(p.dbeta, p.p_f32, col + k, acc_b[i][k]);
                    }
                }
            }
        }
        if (turn + 1 < rg.groups) __syncthreads();
    }
}

// dgamma and dbeta from the blocks' sums: a block takes 128 of the 2 d columns, its warps every eighth of the sums, which are
// then added in order.
__global__ void __launch_bounds__(256) layer_norm_params_kernel(const float* partial, int blocks, int d, void* dgamma, void* dbeta, int p_f32) {
    __shared__ float4 part[8][32];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int col = 4 * (blockIdx.x * 32 + lane);                 // d is a multiple of 8: four columns are all of dgamma or all of dbeta
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (col < 2 * d) {
        for (int s = warp; s < blocks; s += 8) {
            const uint4 v = ld_v4(partial + static_cast<size_t>(s) * 2 * d + col);
            sum.x += __uint_as_float(v.x);
            sum.y += __uint_as_float(v.y);
            sum.z += __uint_as_float(v.z);
            sum.w += __uint_as_float(v.w);
        }
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && col < 2 * d) {
        for (int w = 1; w < 8; ++w) {
            const float4 v = part[w][lane];
            sum.x += v.x;
            sum.y += v.y;
            sum.z += v.z;
            sum.w += v.w;
        }
        void* out = col < d ? dgamma : dbeta;
        const int at = col < d ? col : col - d;
        if (!out) return;
        store_param(out, p_f32, at, sum.x);
        store_param(out, p_f32, at + 1, sum.y);
        store_param(out, p_f32, at + 2, sum.z);
        store_param(out, p_f32, at + 3, sum.w);
    }
}

}  // namespace slope
