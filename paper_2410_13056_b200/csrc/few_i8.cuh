// Products for up to four tokens, shared by the linear layer and the gated block: every block quantizes all tokens into its
// shared memory while its first weights are on their way.
#pragma once

#include <algorithm>

#include "product_i8.cuh"

namespace cmpq {

constexpr int kFewThreads = 320;  // a warp for the weights, one for the products, eight that compute
constexpr int kFewMaxStages = 64;
constexpr int kFewSmem = 224 << 10;
constexpr int kFewRows = 8, kFewColumns = 16;  // of the tokens' operand and of an accumulator: the least there is

struct TokenRows {
    const uint16_t* x;
    int64_t ldx;
    int wide;  // rows on 16 bytes
    RowNorm norm;
    int64_t d;
    int n;
    int32_t* word;  // or null
};

// The computing warps' barrier.
__device__ __forceinline__ void meet() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// Where the codes of token `row` from byte k on stand in the tokens' operand: blocks of 128 bytes of the sum, in each eight rows
// in the 128-byte swizzle.
__device__ __forceinline__ uint8_t* code_at(uint8_t* base, int row, int k) {
    return base + (k >> 7) * kFewRows * 128 + row * 128 + (((k >> 4 & 7) ^ row) << 4) + (k & 15);
}

struct TokenParts {  // in shared memory
    uint32_t m[kFewTokens][8];
    float s[kFewTokens][8];
};

// Eight entries of every token, and of the norm's weight.
struct TokenGroup {
    uint4 w, x[kFewTokens];

    template <bool NORM>
    __device__ __forceinline__ void load(const TokenRows& A, int64_t g) {
        const uint4 none = make_uint4(0u, 0u, 0u, 0u);
        const bool there = 8 * g < A.d;
        w = NORM && there ? load8(A.norm.weight + 8 * g, A.d - 8 * g, A.norm.wide) : none;
#pragma unroll
        for (int r = 0; r < kFewTokens; ++r) x[r] = r < A.n && there ? load8_ordinary<true>(A.x + r * A.ldx + 8 * g, A.d - 8 * g, A.wide) : none;
    }
};
constexpr int kFewHeld = 2;  // groups that a thread keeps

// Codes of all tokens, of entry k of token r to place(r, k), their scales into `scale`, by 256 threads, all rows at once so that
// their loads are on their way together.  Each thread takes the groups that norm_quantize_row gives it, so a token gets the
// same bytes from either.
template <int DT, bool NORM, class Place>
__device__ __forceinline__ void quantize_tokens(const TokenRows& A, Place place, float* scale, TokenParts& parts, int t) {
    constexpr int R = kFewTokens;
    const int n = A.n;
    const int64_t d = A.d, groups = (d + 7) / 8;
    TokenGroup held[kFewHeld];
#pragma unroll
    for (int i = 0; i < kFewHeld; ++i) held[i].load<NORM>(A, t + i * 256);
    // f(row, group, entries, v) for this thread's groups
    auto every = [&](auto f) {
        auto one = [&](int64_t g, const TokenGroup& k) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r >= n || g >= groups) break;
                float e[8], v[8];
                widen8<DT>(k.x[r], e);
                if (NORM) widen8<DT>(k.w, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = NORM ? e[j] * v[j] : e[j];
                f(r, g, e, v);
            }
        };
#pragma unroll
        for (int i = 0; i < kFewHeld; ++i) one(t + i * 256, held[i]);
        for (int64_t g = t + kFewHeld * 256; g < groups; g += 256) {
            TokenGroup k;
            k.load<NORM>(A, g);
            one(g, k);
        }
    };
    uint32_t m[R] = {};
    float sum[R] = {}, f = 1.0f;
    auto add_up = [&] {  // over the block: the same bits in all threads
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = __reduce_max_sync(0xffffffffu, m[r]);
#pragma unroll
            for (int i = 16; i && NORM; i >>= 1) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], i);
            if ((t & 31) == 0) parts.m[r][t >> 5] = m[r], parts.s[r][t >> 5] = sum[r];
        }
        meet();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sum[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) m[r] = max(m[r], parts.m[r][i]), sum[r] += parts.s[r][i];
        }
    };
    every([&](int r, int64_t, const float(&e)[8], const float(&v)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) m[r] = __float_as_uint(larger(__uint_as_float(m[r]), v[j]));
        if (NORM) sum[r] += sum_squares(e, f);
    });
    add_up();
    float2 s[R];
    float factor[R], squares[R];
    bool passed = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        s[r] = scale_of(__uint_as_float(m[r])), squares[r] = sum[r], factor[r] = 1.0f;
        if (NORM && sum[r] > FLT_MAX && m[r] < 0x7f800000u) passed = true, factor[r] = 0x1p-80f;
    }
    if (passed) {  // see norm_quantize_row; the same in all threads
        f = 0x1p-80f;
#pragma unroll
        for (int r = 0; r < R; ++r) sum[r] = 0.0f;
        every([&](int r, int64_t, const float(&e)[8], const float(&)[8]) { sum[r] += sum_squares(e, f); });
        meet();  // the parts have been read
        add_up();
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (factor[r] != 1.0f) squares[r] = sum[r];
    }
    every([&](int r, int64_t g, const float(&)[8], const float(&v)[8]) { *reinterpret_cast<uint2*>(place(r, 8 * (int)g)) = round_codes(v, s[r].y); });
    if (t == 0)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r >= n) break;
            if (NORM && s[r].x > 0.0f) s[r].x *= factor[r] / sqrtf(squares[r] / (float)d + A.norm.eps * factor[r] * factor[r]);
            scale[r] = s[r].x;
            if (m[r] >= 0x7f800000u && A.word && blockIdx.x == 0) atomicOr(A.word, kWordNonfinite);
        }
}

// Equal tiles of channels for the blocks, in as few rounds as 128 channels allow.
inline void plan_tiles(ProductArgs& p) {
    const int64_t sms = sm_count(), rounds = ceil_div(p.d_out, 128 * sms);
    p.bn = (int)std::min<int64_t>(128, ceil_div(ceil_div(p.d_out, rounds * sms), 8) * 8);
    p.n_tiles = (int)ceil_div(p.d_out, p.bn);
}
// Bytes for stages of weights.  Behind them are the tokens' codes; products read 128 rows of weights and 16 of tokens, whatever
// there is.
inline int few_ring(int token_bytes) { return kFewSmem - 1024 - std::max(token_bytes + 1024, 128 * 128); }
// Stages of 16 to 32 KB: with less of a row at a time memory is slower (4096 x 11008 in boxes of 32 rows x 128 bytes: 23.5 us
// one by one, 10.1 by fours, 8.8 by eights).
inline void plan_stages(ProductArgs& p, int block_bytes, int ring) {
    p.per_stage = std::max(1, (32 << 10) / block_bytes);
    p.stages = std::min(ring / (p.per_stage * block_bytes), kFewMaxStages);
}

}  // namespace cmpq
