// Gated feed-forward block in 8 bits.
#include "linear_i8.cuh"

namespace cmpq {

// The work space: counters and the mark of a kernel that gave up; h; the codes of the tokens, later of h; both scales.
struct GatedSpace {
    int32_t* counters;
    uint16_t* h;
    int8_t* codes;
    float *x_scale, *h_scale;
    int64_t ldh, ldc_in, ldc_ff;
    size_t bytes;

    GatedSpace(void* ws, int64_t n, int64_t d_in, int64_t d_ff) {
        Workspace w(ws, SIZE_MAX);
        ldh = (int64_t)round_up(d_ff, 8), ldc_in = (int64_t)round_up(d_in, 16), ldc_ff = (int64_t)round_up(d_ff, 16);
        counters = w.take<int32_t>(CMPQ_GATED_ZEROED / 4);
        h = w.take<uint16_t>((size_t)n * ldh);
        codes = w.take<int8_t>((size_t)n * (ldc_in > ldc_ff ? ldc_in : ldc_ff));
        x_scale = w.take<float>(n);
        h_scale = w.take<float>(n);
        bytes = w.used;
    }
};

}  // namespace cmpq

using namespace cmpq;

static bool gated_sizes_ok(int64_t n, int64_t d_in, int64_t d_ff, int64_t d_out) {
    return linear_sizes_ok(n, d_in, d_ff) && linear_sizes_ok(n, d_ff, d_out);
}

extern "C" size_t cmpq_gated_i8_ws_bytes(int64_t n, int64_t d_in, int64_t d_ff, int64_t d_out) {
    return gated_sizes_ok(n, d_in, d_ff, d_out) ? GatedSpace(nullptr, n, d_in, d_ff).bytes : 0;
}

extern "C" cmpq_status cmpq_gated_i8(const void* X, cmpq_dtype dt, int64_t n, int64_t d_in, int64_t ldx, const void* norm, float eps,
                                     const cmpq_weight_i8* gate, const cmpq_weight_i8* up, const cmpq_weight_i8* down, int64_t d_ff, int64_t d_out,
                                     cmpq_act act, const void* residual, int64_t ldr, void* y, int64_t ldy, int32_t* word, void* ws, size_t ws_bytes,
                                     void* stream) {
    if (!gate || !up || !down || !gated_sizes_ok(n, d_in, d_ff, d_out) || ldx < d_in || ldy < d_out) return CMPQ_ERR_INVALID_ARG;
    if (!weight_rows_ok(*gate, d_in) || !weight_rows_ok(*up, d_in) || !weight_rows_ok(*down, d_ff)) return CMPQ_ERR_INVALID_ARG;
    if ((dt != CMPQ_F16 && dt != CMPQ_BF16) || !norm_ok(norm, eps) || !finish_ok(act, residual, ldr, d_out)) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!X || !y || !weight_ok(*gate) || !weight_ok(*up) || !weight_ok(*down) || !aligned_to(X, 2) || !aligned_to(y, 2)) return CMPQ_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < cmpq_gated_i8_ws_bytes(n, d_in, d_ff, d_out)) return CMPQ_ERR_WORKSPACE;
    const GatedSpace g(ws, n, d_in, d_ff);
    const auto st = static_cast<cudaStream_t>(stream);
    int32_t* mark = g.counters + CMPQ_GATED_ZEROED / 4 - 1;
    int32_t* gave_up = word ? word : mark;
    cmpq_status s = enqueue_quantize(X, dt, n, d_in, ldx, norm, eps, g.codes, g.ldc_in, g.x_scale, word, nullptr, st);
    if (s != CMPQ_OK) return s;
    s = enqueue_product({g.codes, g.ldc_in, g.x_scale}, dt, n, d_in, *gate, d_ff, up, {act, nullptr, 0}, g.h, g.ldh, gave_up, true, st);
    if (s != CMPQ_OK) return s;
    s = enqueue_quantize(g.h, dt, n, d_ff, g.ldh, nullptr, 0.0f, g.codes, g.ldc_ff, g.h_scale, word, nullptr, st);
    if (s != CMPQ_OK) return s;
    return enqueue_product({g.codes, g.ldc_ff, g.h_scale}, dt, n, d_ff, *down, d_out, nullptr, {CMPQ_ACT_NONE, residual, ldr}, y, ldy, gave_up, true, st);
}
