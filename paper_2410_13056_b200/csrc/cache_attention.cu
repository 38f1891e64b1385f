// Attention over the paged 8-bit cache.
#include "cache.cuh"

namespace cmpq {

struct AttnArgs {
    cmpq_cache c;
    cmpq_batch b;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t ldq, ldo, max_new, max_len, window;
    float scale;
    int n_heads, causal;
    int32_t* word;
};

// One warp per query row and head: the lanes share the head's entries, one key after the other.
template <int DT, int D>
__global__ void __launch_bounds__(128)
attention_row_kernel(const __grid_constant__ AttnArgs A) {
    const int lane = threadIdx.x & 31, P = A.c.page_tokens, H = A.c.n_kv_heads;
    const int32_t* off = A.b.tok_off;
    const int64_t t = blockIdx.x;
    const int s = block_count(A.b.n_seq, [&](int64_t i) { return off[i] <= t; });
    if (s >= A.b.n_seq) return;
    const int64_t len = A.b.lens[s], pos = len - off[s + 1] + t;
    if (len < 0 || len > A.max_len || off[s + 1] - off[s] > A.max_new) {
        if (threadIdx.x == 0 && A.word) atomicOr(A.word, kWordTable);
        return;
    }
    const int64_t hi = A.causal ? min(len, pos + 1) : len;
    const int64_t lo = A.window > 0 ? max((int64_t)0, pos - A.window + 1) : 0;
    constexpr int E = D / 32;
    for (int h = threadIdx.x >> 5; h < A.n_heads; h += 4) {
        const int kv = h / (A.n_heads / H);
        float q[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            q[e] = widen16<DT>(A.q[t * A.ldq + h * D + lane + 32 * e]);
            o[e] = 0.0f;
        }
        for (int64_t j = lo; j < hi; ++j) {
            const int64_t page = j / P;
            const int id = page < A.b.ld_table ? A.b.table[s * A.b.ld_table + page] : -1;
            if (id < 0 || id >= A.c.n_pages) {
                if (lane == 0 && A.word) atomicOr(A.word, kWordTable);
                continue;
            }
            const int64_t at = (int64_t)id * H + kv, row = (at * P + j % P) * D;
            float dot = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) dot = fmaf(q[e], (float)A.c.k_codes[row + lane + 32 * e], dot);
#pragma unroll
            for (int x = 16; x; x >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, x);
            dot *= A.c.k_scale[at] * A.scale;
            const float top = fmaxf(m, dot), keep = __expf(m - top), p = __expf(dot - top);
            l = fmaf(l, keep, p);
            const float pv = p * A.c.v_scale[at];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], keep, pv * (float)A.c.v_codes[row + lane + 32 * e]);
            m = top;
        }
        const float r = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) A.out[t * A.ldo + h * D + lane + 32 * e] = round16<DT>(o[e] * r);
        if (A.lse && lane == 0) A.lse[t * A.n_heads + h] = l > 0.0f ? m + logf(l) : -INFINITY;
    }
}

template <int DT>
static void launch_rows(const AttnArgs& a, cudaStream_t st) {
    const unsigned n = (unsigned)a.b.n_tok;
    if (a.c.head_dim == 64) attention_row_kernel<DT, 64><<<n, 128, 0, st>>>(a);
    else if (a.c.head_dim == 128) attention_row_kernel<DT, 128><<<n, 128, 0, st>>>(a);
    else attention_row_kernel<DT, 256><<<n, 128, 0, st>>>(a);
}

}  // namespace cmpq

using namespace cmpq;

extern "C" size_t cmpq_cache_attention_ws_bytes(int64_t n_seq, int64_t n_tok, int64_t max_new, int64_t max_len,
                                                int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
    if (n_seq < 0 || n_tok < 0 || max_new < 0 || max_len < 0 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads ||
        head_dim < 1)
        return 0;
    return 256;
}

extern "C" cmpq_status cmpq_cache_attention(const cmpq_cache* cache, const cmpq_batch* batch, const void* q, int64_t ldq,
                                            cmpq_dtype dt, int32_t n_heads, int64_t max_new, int64_t max_len, float scale,
                                            int32_t causal, int64_t window, void* out, int64_t ldo, float* lse,
                                            int32_t* word, void* ws, size_t ws_bytes, void* stream) {
    cmpq_status why;
    if (!cache_ok(cache, &why)) return why;
    if (!batch_ok(batch) || (dt != CMPQ_F16 && dt != CMPQ_BF16)) return CMPQ_ERR_INVALID_ARG;
    if (n_heads < 1 || n_heads > 4096 || n_heads % cache->n_kv_heads || max_new < 0 || max_len < 0 || max_len > INT32_MAX)
        return CMPQ_ERR_INVALID_ARG;
    if (window < 0 || (window > 0 && !causal) || !(scale > 0.0f) || isinf(scale)) return CMPQ_ERR_INVALID_ARG;
    const int64_t row = (int64_t)n_heads * cache->head_dim;
    if (ldq < row || ldo < row) return CMPQ_ERR_INVALID_ARG;
    if (batch->n_seq == 0 || batch->n_tok == 0) return CMPQ_OK;
    if (!q || !out || !aligned_to(q, 2) || !aligned_to(out, 2) || !aligned_to(lse, 4)) return CMPQ_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 256) ||
        ws_bytes < cmpq_cache_attention_ws_bytes(batch->n_seq, batch->n_tok, max_new, max_len, n_heads, cache->n_kv_heads, cache->head_dim))
        return CMPQ_ERR_WORKSPACE;
    AttnArgs a{*cache, *batch, static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out), lse, ldq, ldo, max_new, max_len,
               window, scale, n_heads, causal != 0, word};
    auto st = static_cast<cudaStream_t>(stream);
    if (dt == CMPQ_BF16)
        launch_rows<CMPQ_BF16>(a, st);
    else
        launch_rows<CMPQ_F16>(a, st);
    return launch_status();
}
