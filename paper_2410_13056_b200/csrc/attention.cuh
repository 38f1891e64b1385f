// Shared by the attention kernels on the paged 8-bit cache.
#pragma once

#include "cache.cuh"
#include "tc5.cuh"

namespace cmpq {

struct AttnArgs {
    cmpq_cache c;
    cmpq_batch b;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t ldq, ldo;
    int max_new, max_len, window;
    float scale;  // times log2(e): scores are kept in powers of two
    int n_heads, group, causal;
    int page_bits;  // log2 of a page's tokens
    int wide_q, wide_o;
    int32_t* word;
    int* counters;  // one per block, zero between calls; the last is set when a kernel gave up, so that later calls tell too
    float* parts;   // two parts per block, then one per worker
    int workers;
};

// Weights are kept relative to 2^kWeightBits: times their value scale the largest of a row are near the top of fp16, whose
// 30 octaves below that all count.
constexpr float kWeightBits = 15.0f;
constexpr int kGaveUp = CMPQ_ATTENTION_ZEROED / (int)sizeof(int) - 1;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A query row's way into fp16 and back: its entries times `down`, its scores times `up`, both powers of two with a product
// of 1.  The largest magnitude lands in [2^13, 2^14), so entries down to 2^-27 of it keep all their bits; the exponent is
// held to [-113, 126], where both powers are normal numbers: rows of bf16 subnormals stay smaller, of 2^127 end below 2^15.
struct RowScale {
    float down, up;
};
__device__ __forceinline__ RowScale row_scale(float largest) {
    const int e = min(max((int)(__float_as_uint(largest) >> 23) - 127, -113), 126);
    return {__uint_as_float((uint32_t)(127 + 13 - e) << 23), __uint_as_float((uint32_t)(127 - 13 + e) << 23)};
}

// log2 of a page's value scale; a page of zeros has scale 0 and counts as 2^-80.
__device__ __forceinline__ float scale_log2(float scale) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fmaxf(scale, 0x1p-80f)));
    return y;
}

// Four int8 codes (already offset by 128) as two pairs of fp16: 0x6400 | u is 1024 + u, and 1024 + 128 comes off.
__device__ __forceinline__ uint32_t half_pair(uint32_t u, uint32_t pick) {
    const uint32_t h = __byte_perm(u, 0x64646464u, pick);
    const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&h), __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&d);
}

// An earlier call on this work space gave up: its counters cannot be relied on.
__device__ __forceinline__ void report_stale(const AttnArgs& A) {
    if (A.word && A.counters[kGaveUp]) atomicOr(A.word, kWordInternal);
}
__device__ __forceinline__ void report_gave_up(const AttnArgs& A) {
    atomicOr(A.counters + kGaveUp, 1);
    if (A.word) atomicOr(A.word, kWordInternal);
}

constexpr int kPfSplits = 8;  // most blocks of the prompts' kernel that share out a unit's keys

// Whole prompts (cache_prefill.cu): head_dim 64 and 128.
cmpq_status launch_prefill(const AttnArgs& a, cmpq_dtype dt, cudaStream_t st);
size_t prefill_parts_bytes(int head_dim);  // behind the counters

}  // namespace cmpq
