// Shared by the 8-bit linear layers and the gated block: the checks of their arguments, and the launches of the tokens'
// quantization and of products, for callers that have made those checks.
#pragma once

#include <cfloat>

#include "cache.cuh"
#include "epilogue.cuh"
#include "plan_i8.h"
#include "tc5.cuh"

namespace cmpq {

// What a product does with its sums: scale and bias; activation and residual too; or two projections at once, of which the
// first, activated, multiplies the second.
enum { kPlain = 0, kFinish = 1, kGated = 2 };

using Weight8 = cmpq_weight_i8;
struct TokenCodes {
    const int8_t* codes;
    int64_t ld;
    const float* scale;
};
struct Finish {
    cmpq_act act;
    const void* residual;
    int64_t ldr;
};

// y = the product of the tokens with w, finished as f says; with `u`, fl16(act(product with w) * product with u), y's rows on
// 16 bytes.  word: where a kernel that gave up says so.  behind: it may start while the tokens are being quantized.
cmpq_status enqueue_product(const TokenCodes& x, cmpq_dtype dt, int64_t n, int64_t d_in, const Weight8& w, int64_t d_out, const Weight8* u,
                            const Finish& f, void* y, int64_t ldy, int32_t* word, bool behind, cudaStream_t st);
// `norm` may be null; `clear`, if given, is set to 0.
cmpq_status enqueue_quantize(const void* X, cmpq_dtype dt, int64_t n, int64_t d, int64_t ldx, const void* norm, float eps, int8_t* codes, int64_t ldc,
                             float* scale, int32_t* word, int32_t* clear, cudaStream_t st);

// Both in one launch, for up to kFewTokens tokens whose rows few_fits; word (may be null): where a NaN or an infinity is
// reported.  behind: it may start while the kernel in front of it, which was launched without this, writes X.
constexpr int kFewTokens = CMPQ_GATED_FEW_TOKENS, kFewBlocks = 100;  // blocks of 128 entries whose codes a block of the kernel holds
bool few_fits(int64_t d_in);
cmpq_status enqueue_few(const void* X, cmpq_dtype dt, int64_t n, int64_t d_in, int64_t ldx, const void* norm, float eps, const Weight8& w, int64_t d_out,
                        const Weight8* u, const Finish& f, void* y, int64_t ldy, int32_t* word, int32_t* gave_up, bool behind, cudaStream_t st);

size_t linear_i8_codes_bytes(int64_t n, int64_t d_in);

inline bool linear_sizes_ok(int64_t n, int64_t d_in, int64_t d_out) {
    return n >= 0 && n <= INT32_MAX - 256 /* tiles of tokens end past the last one */ && d_in >= 1 && d_in <= CMPQ_MAX_D_IN_I8 && d_out >= 1 && d_out <= CMPQ_MAX_D_IN;
}
inline bool weight_rows_ok(const Weight8& w, int64_t d_in) { return w.ld >= d_in && w.ld % 16 == 0; }
inline bool weight_ok(const Weight8& w) {
    return w.codes && w.scale && aligned_to(w.codes, 16) && aligned_to(w.scale, 4) && aligned_to(w.bias, 2);
}
inline bool norm_ok(const void* norm, float eps) { return !norm || (aligned_to(norm, 2) && eps >= FLT_MIN && eps <= FLT_MAX); }
inline bool finish_ok(cmpq_act act, const void* residual, int64_t ldr, int64_t d_out) {
    return act_ok(act) && (!residual || (aligned_to(residual, 2) && ldr >= d_out));
}

}  // namespace cmpq
