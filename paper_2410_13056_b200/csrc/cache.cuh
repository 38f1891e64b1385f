// Shared by the kernels on the paged 8-bit cache: argument checks, where a token lies, 16-bit rounding.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace cmpq {

constexpr int kWordNonfinite = 1, kWordTable = 4, kWordInternal = 8;  // bits of the device word
constexpr float kScaleLo = 0x1p-60f, kScaleHi = 0x1p60f;

// Two floats rounded to 16 bits into one word, `lo` in the low half.
template <int DT>
__device__ __forceinline__ uint32_t round16x2(float lo, float hi) {
    if (DT == CMPQ_BF16) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&b);
    } else {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}

// Eight 16-bit elements from `p` on, of which `left` exist; `wide`: p is 16-byte aligned.
__device__ __forceinline__ uint4 load8(const uint16_t* p, int64_t left, bool wide) {
    if (wide && left >= 8) return __ldg(reinterpret_cast<const uint4*>(p));
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = 2 * i < left ? p[2 * i] : 0u, hi = 2 * i + 1 < left ? p[2 * i + 1] : 0u;
        w[i] = lo | hi << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int DT>
__device__ __forceinline__ void widen8(uint4 g, float (&f)[8]) {
    const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 p = widen16x2<DT>(w[i]);
        f[2 * i] = p.x;
        f[2 * i + 1] = p.y;
    }
}

// Codes of entries whose scale may have been cut off at its upper end: clamped, then rounded to even by adding
// 1.5 * 2^23, which leaves the integer in the sum's low byte (a conversion has a quarter of an addition's rate).  A NaN
// gives -127.
__device__ __forceinline__ uint32_t code_bits(float x, float inv) {
    return __float_as_uint(fminf(fmaxf(x * inv, -127.0f), 127.0f) + 12582912.0f);
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
    return __byte_perm(__byte_perm(code_bits(a, inv), code_bits(b, inv), 0x0040), __byte_perm(code_bits(c, inv), code_bits(d, inv), 0x0040), 0x5410);
}
__device__ __forceinline__ uint2 codes_of(const float (&f)[8], float inv) {
    return make_uint2(codes4(f[0], f[1], f[2], f[3], inv), codes4(f[4], f[5], f[6], f[7], inv));
}

// Four codes as floats: 0x4b000000 | u is 2^23 + u.
__device__ __forceinline__ void widen_codes(uint32_t c, float (&f)[4]) {
    const uint32_t u = c ^ 0x80808080u;
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 + e)) - 8388736.0f;
}

// The number of i in [1, last] with `below(i)`, for a predicate that holds up to some i and not after it; every
// thread of the block calls it with the same arguments.  One parallel look per blockDim.x candidates instead of a
// chain of dependent loads.
template <class Below>
__device__ __forceinline__ int block_count(int64_t last, Below below) {
    int found = 0;
    for (int64_t base = 1; base <= last; base += blockDim.x) {
        const int64_t i = base + threadIdx.x;
        const int c = __syncthreads_count(i <= last && below(i));
        found += c;
        if (c < (int)blockDim.x) break;
    }
    return found;
}

inline bool cache_ok(const cmpq_cache* c, cmpq_status* why) {
    *why = CMPQ_ERR_INVALID_ARG;
    if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || c->n_pages < 1 || c->n_pages > INT32_MAX ||
        c->n_kv_heads < 1 || c->n_kv_heads > 1024)
        return false;
    if (!aligned_to(c->k_codes, 16) || !aligned_to(c->v_codes, 16) || !aligned_to(c->k_scale, 4) || !aligned_to(c->v_scale, 4))
        return false;
    const int d = c->head_dim, p = c->page_tokens;
    if ((d != 64 && d != 128 && d != 256) || (p != 16 && p != 32 && p != 64 && p != 128)) {
        *why = CMPQ_ERR_UNSUPPORTED;
        return false;
    }
    return true;
}

inline bool batch_ok(const cmpq_batch* b) {
    return b && b->n_seq >= 0 && b->n_seq <= 65536 && b->n_tok >= 0 && b->n_tok < INT32_MAX && b->ld_table >= 0 && b->table_cols >= 0 &&
           (b->n_seq == 0 || b->n_tok == 0 ||
            (b->tok_off && b->lens && b->table && b->ld_table >= 1 && aligned_to(b->tok_off, 4) && aligned_to(b->lens, 4) &&
             aligned_to(b->table, 4)));
}

// The batch with the number of entries that a table row has.
inline cmpq_batch bounded(cmpq_batch b) {
    if (b.table_cols == 0) b.table_cols = b.ld_table;
    return b;
}

}  // namespace cmpq
