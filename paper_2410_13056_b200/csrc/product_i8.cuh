// Device side of the 8-bit linear layers and the gated block: a row's quantization, what a product does with its sums.
#pragma once

#include <cfloat>

#include "epilogue.cuh"
#include "linear_i8.cuh"

namespace cmpq {

constexpr int kQtThreads = 256;

// load8 without the read-only path, which is for memory that nobody writes as long as a kernel runs.  WRITTEN: of rows that a kernel
// may have written while this one was on its way, from L2.  Else of rows that this kernel writes too (a residual may be the
// output), entries that nobody but the reading thread writes, and it only later: ordinary loads, whose second half of a sector
// is in L1 (777 tokens 11008 -> 4096 45.1 us, 46.2 from L2).
template <bool WRITTEN>
__device__ __forceinline__ uint4 load8_ordinary(const uint16_t* p, int64_t left, bool wide) {
    const auto load = [](const auto* at) { return WRITTEN ? __ldcg(at) : __ldca(at); };
    if (wide && left >= 8) return load(reinterpret_cast<const uint4*>(p));
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = 2 * i < left ? load(p + 2 * i) : 0u, hi = 2 * i + 1 < left ? load(p + 2 * i + 1) : 0u;
        w[i] = lo | hi << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct RowParts {  // in shared memory
    uint32_t m[kQtThreads / 32];
    float s[kQtThreads / 32];
};

// Largest of the threads' `m` and total of their `s`, the same bits in each of them.
template <class Sync>
__device__ __forceinline__ void all_max_sum(uint32_t& m, float& s, int t, RowParts& parts, Sync sync) {
    m = __reduce_max_sync(0xffffffffu, m);
#pragma unroll
    for (int i = 16; i; i >>= 1) s += __shfl_xor_sync(0xffffffffu, s, i);
    if ((t & 31) == 0) parts.m[t >> 5] = m, parts.s[t >> 5] = s;
    sync();
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < kQtThreads / 32; ++i) m = max(m, parts.m[i]), s += parts.s[i];
}

// The squares of eight entries times f: a row of 16384 entries goes through at most 8 + 5 + 5 + 8 roundings one after the other.
__device__ __forceinline__ float sum_squares(const float (&x)[8], float f) {
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) a = __fmaf_rn(x[i] * f, x[i] * f, a), b = __fmaf_rn(x[i + 4] * f, x[i + 4] * f, b);
    return a + b;
}

// The larger of m and |v|, a NaN if one of them is.
__device__ __forceinline__ float larger(float m, float v) {
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(fabsf(v)));
    return m;
}

struct RowNorm {
    const uint16_t* weight;  // or null
    int wide;                // 16-byte aligned
    float eps;
};

// Codes of eight values: |v * inv| is at most 127 (1 + 2^-22), so adding 1.5 * 2^23 leaves the integer that rounding to even
// gives in the sum's low byte, in two's complement: one addition instead of a conversion, which has a quarter of its rate.
__device__ __forceinline__ uint2 round_codes(const float (&v)[8], float inv) {
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = v[2 * j] * inv + 12582912.0f, b = v[2 * j + 1] * inv + 12582912.0f;  // two roundings each: -fmad=false
        c[j] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040);
    }
    return make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
}

// Scale of a row whose largest magnitude is given, and what its values are multiplied with.
__device__ __forceinline__ float2 scale_of(float amax) {
    const float s = amax * (1.0f / 127.0f);
    return amax < 0x1p-120f ? make_float2(0.0f, 0.0f) : make_float2(s, 1.0f / s);
}

// Codes and scale of a row behind a root-mean-square norm, by 256 threads (t is a thread's number).  A row's codes do not depend
// on its norm: code = rint(v 127 / max|v|) with v = x g, whatever v is divided by; the norm enters the scale alone.  So nothing
// waits for the sum of squares, and the codes are as exact as without a norm.  v is one fp32 product, so magnitudes are
// compared in fp32.  A sum that passes fp32 (entries above 2^54 or so) is taken again of entries times 2^-80; entries that vanish
// there vanish beside it too.  A thread keeps v of KEEP groups of eight; what is longer is read again.
template <int DT, int KEEP>
__device__ __forceinline__ void norm_quantize_row(const uint16_t* row, int64_t d, bool wide, const RowNorm& norm, int8_t* out, float* scale,
                                                  int32_t* nonfinite, int t, RowParts& parts) {
    const int64_t groups = (d + 15) / 16 * 2;  // the codes' padding up to 16 is written too
    const auto sync = [] { __syncthreads(); };
    uint4 x[KEEP], w[KEEP];
    float v[KEEP][8], e[8];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t g = t + (int64_t)i * kQtThreads;
        x[i] = w[i] = make_uint4(0u, 0u, 0u, 0u);
        if (8 * g < d) x[i] = load8(row + 8 * g, d - 8 * g, wide), w[i] = load8(norm.weight + 8 * g, d - 8 * g, norm.wide);
    }
    auto weighted = [&](int64_t g, float (&p)[8]) {
        widen8<DT>(load8(row + 8 * g, d - 8 * g, wide), e);
        widen8<DT>(load8(norm.weight + 8 * g, d - 8 * g, norm.wide), p);
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = e[j] * p[j];
    };
    float most = 0.0f, sum = 0.0f;
    auto look = [&](const float (&p)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) most = larger(most, p[j]);
        sum += sum_squares(e, 1.0f);
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        widen8<DT>(x[i], e);
        widen8<DT>(w[i], v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = e[j] * v[i][j];
        look(v[i]);
    }
    for (int64_t g = t + (int64_t)KEEP * kQtThreads; g < groups; g += kQtThreads) {
        float p[8];
        weighted(g, p);
        look(p);
    }
    uint32_t m = __float_as_uint(most);  // compared as bit patterns from here on: NaN above infinity
    all_max_sum(m, sum, t, parts, sync);
    float2 s = scale_of(__uint_as_float(m));
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t g = t + (int64_t)i * kQtThreads;
        if (g < groups) *reinterpret_cast<uint2*>(out + 8 * g) = round_codes(v[i], s.y);
    }
    for (int64_t g = t + (int64_t)KEEP * kQtThreads; g < groups; g += kQtThreads) {
        float p[8];
        weighted(g, p);
        *reinterpret_cast<uint2*>(out + 8 * g) = round_codes(p, s.y);
    }
    float f = 1.0f;
    if (sum > FLT_MAX && m < 0x7f800000u) {  // the same in all threads; not a row with a NaN
        f = 0x1p-80f, sum = 0.0f;
        for (int64_t g = t; 8 * g < d; g += kQtThreads) {
            widen8<DT>(load8(row + 8 * g, d - 8 * g, wide), e);
            sum += sum_squares(e, f);
        }
        sync();  // the parts have been read
        all_max_sum(m, sum, t, parts, sync);
    }
    if (t == 0) {
        if (s.x > 0.0f) s.x *= f / sqrtf(sum / (float)d + norm.eps * f * f);
        *scale = s.x;
        if (m >= 0x7f800000u && nonfinite) atomicOr(nonfinite, 1);
    }
}

// ---- products ----

struct ProductArgs {
    const float *xs, *ws, *us;         // us, ubias: of the second projection of a gated product
    const uint16_t *bias, *ubias;
    uint16_t* y;
    int64_t ldy;
    const uint16_t* residual;          // or null
    int64_t ldr;
    int act, wide_residual;
    int n, d_out, kblocks;  // kblocks: 128-byte blocks of the sum
    int64_t cols;           // rows of weights: d_out, or twice that
    int wide;               // y takes 16-byte stores
    int n_tiles, m_tiles;   // tiles of channels, of tokens
    int stages, per_stage, bn, rows;  // tile kernel: stages, blocks of the sum in each, columns of a tile, token rows that a box brings
    int slices;  // of a tile's sum, over an instruction or over the CTAs of a cluster
    int32_t* failed;
};

// Columns [c0, c1) of a warp's 32 accumulator rows: fl16(fl(fl(sum * xs) * ws) + bias) into y + column, of which `left`
// exist.  c0 and c1 are multiples of 16; scale_bias holds (ws, bias) of the tile's columns.
template <int DT>
__device__ __forceinline__ void store_rows(uint32_t tmem, int c0, int c1, const float2* scale_bias, bool has_bias, float xs, bool real,
                                           uint16_t* y, int left, bool wide) {
    for (int c = c0; c < c1; c += 16) {
        uint32_t r[16], w[8];
        tc5::tmem_ld16(tmem + c, r);
        tc5::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            const float4 sb = *reinterpret_cast<const float4*>(scale_bias + c + j);
            float a = (float)(int)r[j] * xs * sb.x, b = (float)(int)r[j + 1] * xs * sb.z;
            if (has_bias) a += sb.y, b += sb.w;
            w[j / 2] = round16x2<DT>(a, b);
        }
        if (!real) continue;
        if (wide && c + 16 <= left) {
            *reinterpret_cast<uint4*>(y + c) = make_uint4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<uint4*>(y + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < left) y[c + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
        }
    }
}

// Sixteen 16-bit entries of a residual's row, of which `left` exist, as floats.
template <int DT>
__device__ __forceinline__ void load16(const uint16_t* p, int left, bool wide, float (&f)[16]) {
    float a[8], b[8];
    widen8<DT>(load8_ordinary<false>(p, left, wide), a);
    widen8<DT>(load8_ordinary<false>(p + 8, left - 8, wide), b);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = a[i], f[i + 8] = b[i];
}

// The same with fl16(act(...) + residual).  y may be the residual: a thread reads its sixteen entries before it writes them.
template <int DT>
__device__ __forceinline__ void store_finished(uint32_t tmem, int c0, int c1, const float2* scale_bias, const ProductArgs& A, float xs, bool real,
                                               uint16_t* y, const uint16_t* residual, int left) {
    with_act(A.act, [&](auto act) {
        for (int c = c0; c < c1; c += 16) {
            uint32_t r[16], w[8];
            float f[16];
            tc5::tmem_ld16(tmem + c, r);
            if (A.residual && real) load16<DT>(residual + c, left - c, A.wide_residual, f);
            tc5::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const float4 sb = *reinterpret_cast<const float4*>(scale_bias + c + j);
                float a = (float)(int)r[j] * xs * sb.x, b = (float)(int)r[j + 1] * xs * sb.z;
                if (A.bias) a += sb.y, b += sb.w;
                a = activate<decltype(act)::value>(a), b = activate<decltype(act)::value>(b);
                if (A.residual) a += f[j], b += f[j + 1];
                w[j / 2] = round16x2<DT>(a, b);
            }
            if (!real) continue;
            if (A.wide && c + 16 <= left) {
                *reinterpret_cast<uint4*>(y + c) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(y + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (c + j < left) y[c + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            }
        }
    });
}

// Columns [c0, c1), multiples of 8, of a gated product: the accumulator's and scale_bias's first `half` columns are the gate,
// the others the second projection; y = fl16(act(gate) * second), rows of y on 16 bytes.
template <int DT>
__device__ __forceinline__ void store_gated(uint32_t tmem, int c0, int c1, int half, const float2* scale_bias, const ProductArgs& A, float xs, bool real,
                                            uint16_t* y, int left) {
    with_act(A.act, [&](auto act) {
        for (int c = c0; c < c1; c += 8) {
            uint32_t g[8], u[8], w[4];
            tc5::tmem_ld8(tmem + c, g);
            tc5::tmem_ld8(tmem + half + c, u);
            tc5::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float4 gs = *reinterpret_cast<const float4*>(scale_bias + c + j), us = *reinterpret_cast<const float4*>(scale_bias + half + c + j);
                float g0 = (float)(int)g[j] * xs * gs.x, g1 = (float)(int)g[j + 1] * xs * gs.z;
                float u0 = (float)(int)u[j] * xs * us.x, u1 = (float)(int)u[j + 1] * xs * us.z;
                if (A.bias) g0 += gs.y, g1 += gs.w;
                if (A.ubias) u0 += us.y, u1 += us.w;
                w[j / 2] = round16x2<DT>(activate<decltype(act)::value>(g0) * u0, activate<decltype(act)::value>(g1) * u1);
            }
            if (!real) continue;
            if (c + 8 <= left) {
                *reinterpret_cast<uint4*>(y + c) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < left) y[c + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            }
        }
    });
}

// Eight columns of a token's row: z, or of a gated product both projections' (u), finished and written.
template <int DT, int KIND>
__device__ __forceinline__ void store_eight(const ProductArgs& A, const int (&z)[8], const int (&u)[8], const float2* scale_bias, const float2* up_scale_bias,
                                            float xs, uint16_t* y, const uint16_t* residual, int left) {
    float f[8];
    if (KIND == kFinish && A.residual) widen8<DT>(load8_ordinary<false>(residual, left, A.wide_residual), f);
    auto finish = [&](auto act) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float v[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float2 sb = scale_bias[j + k];
                v[k] = (float)z[j + k] * xs * sb.x;
                if (A.bias) v[k] += sb.y;
                v[k] = activate<decltype(act)::value>(v[k]);
                if (KIND == kGated) {
                    const float2 us = up_scale_bias[j + k];
                    float o = (float)u[j + k] * xs * us.x;
                    if (A.ubias) o += us.y;
                    v[k] *= o;
                }
                if (KIND == kFinish && A.residual) v[k] += f[j + k];
            }
            w[j / 2] = round16x2<DT>(v[0], v[1]);
        }
        if ((KIND == kGated || A.wide) && left >= 8) {
            *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) y[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
        }
    };
    if (KIND == kPlain)
        finish(ActIs<CMPQ_ACT_NONE>());
    else
        with_act(A.act, finish);
}

// Scale and bias of column i of a tile whose channels begin at o0: of a gated tile the first half's, then the second's.
template <int DT, int KIND>
__device__ __forceinline__ float2 column_scale(const ProductArgs& A, int o0, int i, int columns) {
    const bool second = KIND == kGated && i >= columns / 2;
    const int o = min(o0 + (second ? i - columns / 2 : i), A.d_out - 1);
    const uint16_t* bias = second ? A.ubias : A.bias;
    return make_float2(__ldg((second ? A.us : A.ws) + o), bias ? widen16<DT>(bias[o]) : 0.0f);
}

// A thread's columns [c0, c1) of the residual, on their way into L2 while the products run.
__device__ __forceinline__ void ask_for(const uint16_t* row, int c0, int c1) {
    const uintptr_t end = reinterpret_cast<uintptr_t>(row + c1);
    for (uintptr_t p = reinterpret_cast<uintptr_t>(row + c0) & ~(uintptr_t)127; c0 < c1 && p < end; p += 128)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}

}  // namespace cmpq
