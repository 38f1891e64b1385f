// Paged 8-bit cache of keys and values: append with the rotation on the way, and the values read back.
#include "cache.cuh"

namespace cmpq {

struct AppendArgs {
    cmpq_cache c;
    cmpq_batch b;
    const uint16_t *k, *v, *q;
    uint16_t* q_out;
    int64_t ldk, ldv, ldq, ldqo;
    const float *cos, *sin;
    int64_t n_pos;
    int rot, interleaved, n_heads;
    int wide_k, wide_v, wide_q;
    int32_t* word;
    int groups;    // groups of eight entries rotate with groups of eight, cosines and sines can be read four at a time
    int few;       // few new tokens a sequence
    int q_tokens, q_heads;  // tokens and heads that a block of the queries takes
    unsigned kv_blocks;
};

__device__ __forceinline__ void report(int32_t* word, int bit) {
    if (word) atomicOr(word, bit);
}

__device__ __forceinline__ void load_floats(const float* p, float (&f)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}

// Eight rotated entries of a head from entry j on (j a multiple of eight).  `row` is the head's first entry,
// `at` the position's row in the cosine and sine arrays.
template <int DT>
__device__ __forceinline__ void rotated8(const AppendArgs& A, const uint16_t* row, int j, bool wide, int64_t at,
                                         float (&f)[8]) {
    widen8<DT>(load8(row + j, 8, wide), f);
    const int rot = A.rot, half = rot / 2;
    if (j >= rot) return;
    const float *cs = A.cos + at * half, *sn = A.sin + at * half;
    if (A.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            if (j + i < rot) {  // rot is even
                const float c = __ldg(cs + (j + i) / 2), s = __ldg(sn + (j + i) / 2), x = f[i], y = f[i + 1];
                f[i] = x * c - y * s;
                f[i + 1] = y * c + x * s;
            }
        }
        return;
    }
    if (A.groups) {  // the partners of eight entries are eight neighbouring entries
        float g[8], c[8], s[8];
        const bool low = j < half;
        const int jj = low ? j : j - half;
        widen8<DT>(load8(row + (low ? j + half : jj), 8, wide), g);
        load_floats(cs + jj, c);
        load_floats(sn + jj, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = low ? f[i] * c[i] - g[i] * s[i] : f[i] * c[i] + g[i] * s[i];
        return;
    }
    for (int i = 0; i < 8; ++i) {
        const int e = j + i;
        if (e >= rot) break;
        const int p = e < half ? e : e - half;
        const float c = __ldg(cs + p), s = __ldg(sn + p);
        const float o = widen16<DT>(row[e < half ? e + half : p]);
        f[i] = e < half ? f[i] * c - o * s : f[i] * c + o * s;
    }
}

template <int DT>
__device__ __forceinline__ uint4 round8(const float (&f)[8]) {
    return make_uint4(round16x2<DT>(f[0], f[1]), round16x2<DT>(f[2], f[3]), round16x2<DT>(f[4], f[5]), round16x2<DT>(f[6], f[7]));
}

// Heads [first, last) of the queries of one token.  Where groups of eight rotate with groups of eight, a thread takes such a pair of groups
// (or a group that has no partner) of every head that is `heads` further on: its cosines and sines are loaded once for
// all heads, what it reads it alone writes, and several heads' loads are under way together.
template <int DT>
__device__ __forceinline__ void rotate_queries(const AppendArgs& A, const uint16_t* src, uint16_t* dst, int64_t pos, int first, int last) {
    const int D = A.c.head_dim, G = D / 8, rot = A.rot, half = rot / 2, tid = threadIdx.x;
    if (A.groups && A.wide_q) {
        const int pairs = A.interleaved ? 0 : rot / 16, units = A.interleaved ? G : G - pairs, heads = (int)blockDim.x / units;
        const int u = tid % units, h0 = tid / units;
        if (h0 >= heads) return;
        if (u < pairs) {
            float c[8], s[8];
            load_floats(A.cos + pos * half + 8 * u, c);
            load_floats(A.sin + pos * half + 8 * u, s);
#pragma unroll 4
            for (int h = first + h0; h < last; h += heads) {
                float x[8], y[8], a[8], b[8];
                widen8<DT>(*reinterpret_cast<const uint4*>(src + h * D + 8 * u), x);
                widen8<DT>(*reinterpret_cast<const uint4*>(src + h * D + half + 8 * u), y);
#pragma unroll
                for (int i = 0; i < 8; ++i) a[i] = x[i] * c[i] - y[i] * s[i], b[i] = y[i] * c[i] + x[i] * s[i];
                *reinterpret_cast<uint4*>(dst + h * D + 8 * u) = round8<DT>(a);
                *reinterpret_cast<uint4*>(dst + h * D + half + 8 * u) = round8<DT>(b);
            }
        } else if (A.interleaved && 8 * u < rot) {
            const float4 c = __ldg(reinterpret_cast<const float4*>(A.cos + pos * half + 4 * u)), s = __ldg(reinterpret_cast<const float4*>(A.sin + pos * half + 4 * u));
            const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll 4
            for (int h = first + h0; h < last; h += heads) {
                float x[8], a[8];
                widen8<DT>(*reinterpret_cast<const uint4*>(src + h * D + 8 * u), x);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[2 * i] = x[2 * i] * cc[i] - x[2 * i + 1] * ss[i];
                    a[2 * i + 1] = x[2 * i + 1] * cc[i] + x[2 * i] * ss[i];
                }
                *reinterpret_cast<uint4*>(dst + h * D + 8 * u) = round8<DT>(a);
            }
        } else if (src != dst) {
            const int j = A.interleaved ? 8 * u : rot + 8 * (u - pairs);
#pragma unroll 4
            for (int h = first + h0; h < last; h += heads)
                *reinterpret_cast<uint4*>(dst + h * D + j) = *reinterpret_cast<const uint4*>(src + h * D + j);
        }
        return;
    }
    const int g = tid % G, r0 = tid / G, heads = (int)blockDim.x / G;
    for (int h0 = first; h0 < last; h0 += heads) {  // in place: a block of heads is read before it is written
        const int h = h0 + r0;
        float f[8];
        if (h < last) rotated8<DT>(A, src + h * D, 8 * g, A.wide_q, pos, f);
        __syncthreads();
        if (h < last) {
            const uint4 w = round8<DT>(f);
            const uint32_t e[4] = {w.x, w.y, w.z, w.w};
            uint16_t* o = dst + h * D + 8 * g;
            if (A.wide_q) {
                *reinterpret_cast<uint4*>(o) = w;
            } else {
                for (int i = 0; i < 8; ++i) o[i] = (uint16_t)(e[i >> 1] >> (16 * (i & 1)));
            }
        }
    }
}

// The first kv_blocks blocks take (page of a sequence, head, keys or values); the others rotate q_heads heads of
// the queries of q_tokens tokens.
//
// The pages of sequence s start at slot tok_off[s] / P + 2 s: n new tokens touch at most (n + 2P - 2) / P pages,
// and that many slots lie between two neighbouring starts.  So a block finds its sequence from its index alone
// and the grid needs no length from the device; a slot without a page ends at once.
//
// A block reads its new tokens, keeps the first NIT groups of a thread rotated in fp32 registers (all of them for
// prompts; blocks of one warp, which are for single tokens, read a later row again), agrees on the largest magnitude,
// and writes codes; earlier codes of the page are touched only when the scale grows.  Each row of a head is D/8 threads
// of eight entries, so global accesses are 16 bytes (inputs) and 8 bytes (codes), whole lines per row.
template <int DT, int NIT, int THREADS>
__global__ void __launch_bounds__(THREADS)
cache_append_kernel(const __grid_constant__ AppendArgs A) {
    const int D = A.c.head_dim, P = A.c.page_tokens, G = D / 8;
    const int32_t* off = A.b.tok_off;
    const int tid = threadIdx.x;
    if (blockIdx.x >= A.kv_blocks) {
        const int chunks = (A.n_heads + A.q_heads - 1) / A.q_heads, block = blockIdx.x - A.kv_blocks, first = block % chunks * A.q_heads;
        const int64_t t0 = (int64_t)(block / chunks) * A.q_tokens;
        int s = block_count(A.b.n_seq, [&](int64_t i) { return off[i] <= t0; });
        for (int64_t t = t0; t < min(t0 + A.q_tokens, A.b.n_tok); ++t) {
            while (s < A.b.n_seq && off[s + 1] <= t) ++s;
            if (s >= A.b.n_seq) return;  // a row past the last sequence
            const int64_t pos = (int64_t)A.b.lens[s] - off[s + 1] + t;
            if (pos < 0 || (A.rot && pos >= A.n_pos)) {
                if (tid == 0) report(A.word, kWordTable);
                continue;
            }
            rotate_queries<DT>(A, A.q + t * A.ldq, A.q_out + t * A.ldqo, pos, first, min(A.n_heads, first + A.q_heads));
        }
        return;
    }
    const int g = tid % G, r0 = tid / G, rows_at_once = THREADS / G;
    const int H = A.c.n_kv_heads;
    const bool is_v = blockIdx.x & 1;
    const int head = (blockIdx.x >> 1) % H;
    const int64_t slot = (blockIdx.x >> 1) / H;
    const int s = block_count(A.b.n_seq - 1, [&](int64_t i) { return off[i] / P + 2 * i <= slot; });
    const int64_t n = off[s + 1] - off[s], len = A.b.lens[s], start = len - n;
    if (n <= 0) return;
    if (start < 0 || off[s] < 0 || off[s + 1] > A.b.n_tok) {
        if (tid == 0) report(A.word, kWordTable);
        return;
    }
    const int64_t page = start / P + (slot - (off[s] / P + 2 * (int64_t)s));
    if (page * P >= len || page < start / P) return;
    const int64_t lo = max(start, page * P), hi = min(len, (page + 1) * P);
    const int id = page < A.b.ld_table ? A.b.table[s * A.b.ld_table + page] : -1;
    if (id < 0 || id >= A.c.n_pages || (!is_v && A.rot && hi > A.n_pos)) {
        if (tid == 0) report(A.word, kWordTable);
        return;
    }
    const int64_t at = (int64_t)id * H + head;
    float* scale = (is_v ? A.c.v_scale : A.c.k_scale) + at;
    int8_t* codes = (is_v ? A.c.v_codes : A.c.k_codes) + at * P * D;
    const int held = (int)(lo - page * P), fresh = (int)(hi - lo);
    const float before = held ? *scale : 0.0f;
    const int64_t t0 = off[s] + (lo - start), ld = is_v ? A.ldv : A.ldk;
    const uint16_t* src = (is_v ? A.v : A.k) + t0 * ld + head * D;

    auto entries = [&](int r, float (&f)[8]) {
        if (is_v)
            widen8<DT>(load8(src + r * ld + 8 * g, 8, A.wide_v), f);
        else
            rotated8<DT>(A, src + r * ld, 8 * g, A.wide_k, lo + r, f);
    };
    float f[NIT][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
        const int r = r0 + i * rows_at_once;
        if (r < fresh) {
            entries(r, f[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[i][e]) & 0x7fffffffu);
        }
    }
    for (int r = r0 + NIT * rows_at_once; r < fresh; r += rows_at_once) {
        float x[8];
        entries(r, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if (THREADS > 32) {
        __shared__ uint32_t part[THREADS / 32];
        if ((tid & 31) == 0) part[tid >> 5] = m;
        __syncthreads();  // every thread has read the scale too
#pragma unroll
        for (int i = 0; i < THREADS / 32; ++i) m = max(m, part[i]);
    }
    const float step = __uint_as_float(m) * (1.0f / 127.0f);
    const float after = fmaxf(before, fminf(fmaxf(step, kScaleLo), kScaleHi)), inv = 1.0f / after;
    __syncwarp();
    if (tid == 0) {
        if (m >= 0x7f800000u) report(A.word, kWordNonfinite);
        *scale = after;
    }
    if (after > before) {
        const float again = before * inv;
        for (int i = tid; i < held * G; i += THREADS) {
            uint2* p = reinterpret_cast<uint2*>(codes) + i;
            const uint2 c = *p;
            float x[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = (float)(int8_t)(c.x >> (8 * e));
                x[4 + e] = (float)(int8_t)(c.y >> (8 * e));
            }
            *p = codes_of(x, again);
        }
    }
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
        const int r = r0 + i * rows_at_once;
        if (r < fresh) *reinterpret_cast<uint2*>(codes + (int64_t)(held + r) * D + 8 * g) = codes_of(f[i], inv);
    }
    for (int r = r0 + NIT * rows_at_once; r < fresh; r += rows_at_once) {
        float x[8];
        entries(r, x);
        *reinterpret_cast<uint2*>(codes + (int64_t)(held + r) * D + 8 * g) = codes_of(x, inv);
    }
}

struct ReadArgs {
    cmpq_cache c;
    cmpq_batch b;
    uint16_t *k, *v;
    int64_t ldo;
    int wide;
    int32_t* word;
};

// A block takes TOKENS tokens, a thread 16 codes of each at a time (keys of all heads, then values): the tokens' loads
// are under way together.
template <int DT, int TOKENS>
__global__ void __launch_bounds__(256)
cache_read_kernel(const __grid_constant__ ReadArgs A) {
    const int D = A.c.head_dim, P = A.c.page_tokens, H = A.c.n_kv_heads, G = D / 16;
    const int32_t* off = A.b.tok_off;
    const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
    int s = block_count(A.b.n_seq, [&](int64_t i) { return off[i] <= t0; });
    int id[TOKENS], in_page[TOKENS];
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
        const int64_t t = t0 + j;
        id[j] = -1, in_page[j] = 0;
        if (t < A.b.n_tok) {
            while (s < A.b.n_seq && off[s + 1] <= t) ++s;
            if (s < A.b.n_seq) {
                const int64_t pos = (int64_t)A.b.lens[s] - off[s + 1] + t, page = pos >= 0 ? pos / P : 0;
                id[j] = pos >= 0 && page < A.b.ld_table ? A.b.table[s * A.b.ld_table + page] : -1;
                in_page[j] = (int)(pos - page * P);
                if (id[j] < 0 || id[j] >= A.c.n_pages) {
                    id[j] = -1;
                    if (threadIdx.x == 0) report(A.word, kWordTable);
                }
            }
        }
    }
    for (int i = threadIdx.x; i < 2 * H * G; i += blockDim.x) {
        const bool is_v = i >= H * G;
        const int k = is_v ? i - H * G : i, h = k / G, g = k % G;
        uint4 c[TOKENS];
        float sc[TOKENS];
#pragma unroll
        for (int j = 0; j < TOKENS; ++j) {
            if (id[j] < 0) continue;
            const int64_t at = (int64_t)id[j] * H + h;
            c[j] = __ldg(reinterpret_cast<const uint4*>((is_v ? A.c.v_codes : A.c.k_codes) + (at * P + in_page[j]) * D) + g);
            sc[j] = __ldg((is_v ? A.c.v_scale : A.c.k_scale) + at);
        }
#pragma unroll
        for (int j = 0; j < TOKENS; ++j) {
            if (id[j] < 0) continue;
            const uint32_t x[4] = {c[j].x, c[j].y, c[j].z, c[j].w};
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t two = x[e >> 1] >> (16 * (e & 1));
                w[e] = round16x2<DT>((float)(int8_t)two * sc[j], (float)(int8_t)(two >> 8) * sc[j]);
            }
            uint16_t* o = (is_v ? A.v : A.k) + (t0 + j) * A.ldo + h * D + 16 * g;
            if (A.wide) {
                *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(o + 8) = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
                for (int e = 0; e < 16; ++e) o[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
            }
        }
    }
}

template <int DT>
static void launch_append(const AppendArgs& a, unsigned blocks, cudaStream_t st) {
    if (a.few) {
        cache_append_kernel<DT, 2, 32><<<blocks, 32, 0, st>>>(a);
        return;
    }
    switch (a.c.head_dim * a.c.page_tokens / 2048) {  // groups of eight entries per thread of a 256-thread block
        case 0: case 1: cache_append_kernel<DT, 1, 256><<<blocks, 256, 0, st>>>(a); break;
        case 2: cache_append_kernel<DT, 2, 256><<<blocks, 256, 0, st>>>(a); break;
        case 4: cache_append_kernel<DT, 4, 256><<<blocks, 256, 0, st>>>(a); break;
        case 8: cache_append_kernel<DT, 8, 256><<<blocks, 256, 0, st>>>(a); break;
        default: cache_append_kernel<DT, 8, 512><<<blocks, 512, 0, st>>>(a); break;
    }
}

template <int DT>
static void launch_read(const ReadArgs& a, cudaStream_t st) {
    // four tokens to a block once that leaves blocks enough
    if (a.b.n_tok >= 4096)
        cache_read_kernel<DT, 4><<<(unsigned)((a.b.n_tok + 3) / 4), 256, 0, st>>>(a);
    else
        cache_read_kernel<DT, 1><<<(unsigned)a.b.n_tok, 256, 0, st>>>(a);
}

}  // namespace cmpq

using namespace cmpq;

extern "C" cmpq_status cmpq_check_cache(const int32_t* word, void* stream) {
    if (!word) return CMPQ_ERR_INVALID_ARG;
    int32_t host = 0;
    auto st = static_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(&host, word, sizeof(host), cudaMemcpyDeviceToHost, st) != cudaSuccess) return CMPQ_ERR_CUDA;
    if (cudaStreamSynchronize(st) != cudaSuccess) return CMPQ_ERR_CUDA;
    return host & kWordInternal ? CMPQ_ERR_INTERNAL : host & kWordTable ? CMPQ_ERR_INVALID_ARG : host ? CMPQ_ERR_NONFINITE : CMPQ_OK;
}

extern "C" cmpq_status cmpq_cache_append(const cmpq_cache* cache, const cmpq_batch* batch, const void* k, int64_t ldk,
                                         const void* v, int64_t ldv, cmpq_dtype dt, const float* cos, const float* sin,
                                         int64_t n_pos, int32_t rot_dim, int32_t interleaved, const void* q, int64_t ldq,
                                         int32_t n_heads, void* q_out, int64_t ldqo, int32_t* word, void* stream) {
    cmpq_status why;
    if (!cache_ok(cache, &why)) return why;
    if (!batch_ok(batch) || (dt != CMPQ_F16 && dt != CMPQ_BF16)) return CMPQ_ERR_INVALID_ARG;
    const int64_t row = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (ldk < row || ldv < row || rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 2 || n_pos < 0) return CMPQ_ERR_INVALID_ARG;
    if (rot_dim && (!cos || !sin || !aligned_to(cos, 4) || !aligned_to(sin, 4))) return CMPQ_ERR_INVALID_ARG;
    if (q && (!q_out || n_heads < 1 || n_heads > 4096 || ldq < (int64_t)n_heads * cache->head_dim || ldqo < (int64_t)n_heads * cache->head_dim))
        return CMPQ_ERR_INVALID_ARG;
    if (batch->n_seq == 0 || batch->n_tok == 0) return CMPQ_OK;
    if (!k || !v || !aligned_to(k, 2) || !aligned_to(v, 2) || !aligned_to(q, 2) || !aligned_to(q_out, 2)) return CMPQ_ERR_INVALID_ARG;
    AppendArgs a;
    a.c = *cache;
    a.b = *batch;
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.q = static_cast<const uint16_t*>(q);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.ldk = ldk, a.ldv = ldv, a.ldq = ldq, a.ldqo = ldqo;
    a.cos = cos, a.sin = sin, a.n_pos = n_pos;
    a.rot = rot_dim, a.interleaved = interleaved, a.n_heads = n_heads;
    a.wide_k = aligned_to(k, 16) && ldk % 8 == 0;
    a.wide_v = aligned_to(v, 16) && ldv % 8 == 0;
    a.wide_q = aligned_to(q, 16) && aligned_to(q_out, 16) && ldq % 8 == 0 && ldqo % 8 == 0;
    a.word = word;
    const int64_t kv = (batch->n_tok / cache->page_tokens + 2 * batch->n_seq) * cache->n_kv_heads * 2;
    a.groups = rot_dim % (interleaved ? 8 : 16) == 0 && aligned_to(cos, 16) && aligned_to(sin, 16);
    // Four new tokens a sequence or fewer: blocks of one warp, without barriers, for a page and head or 16 heads of a
    // query; otherwise all threads that a full page occupies, and the queries of four tokens once that leaves enough blocks.
    a.few = batch->n_tok <= 4 * batch->n_seq;
    a.q_tokens = !a.few && batch->n_tok >= 4096 ? 4 : 1;
    a.q_heads = a.few ? 16 : n_heads;
    const int64_t blocks = kv + (q ? (batch->n_tok + a.q_tokens - 1) / a.q_tokens * ((n_heads + a.q_heads - 1) / a.q_heads) : 0);
    if (blocks > INT32_MAX) return CMPQ_ERR_UNSUPPORTED;
    a.kv_blocks = (unsigned)kv;
    auto st = static_cast<cudaStream_t>(stream);
    if (dt == CMPQ_BF16)
        launch_append<CMPQ_BF16>(a, (unsigned)blocks, st);
    else
        launch_append<CMPQ_F16>(a, (unsigned)blocks, st);
    return launch_status();
}

extern "C" cmpq_status cmpq_cache_read(const cmpq_cache* cache, const cmpq_batch* batch, cmpq_dtype dt, void* k_out,
                                       void* v_out, int64_t ldo, int32_t* word, void* stream) {
    cmpq_status why;
    if (!cache_ok(cache, &why)) return why;
    if (!batch_ok(batch) || (dt != CMPQ_F16 && dt != CMPQ_BF16)) return CMPQ_ERR_INVALID_ARG;
    if (ldo < (int64_t)cache->n_kv_heads * cache->head_dim) return CMPQ_ERR_INVALID_ARG;
    if (batch->n_seq == 0 || batch->n_tok == 0) return CMPQ_OK;
    if (!k_out || !v_out || !aligned_to(k_out, 2) || !aligned_to(v_out, 2)) return CMPQ_ERR_INVALID_ARG;
    ReadArgs a{*cache, *batch, static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out), ldo,
               aligned_to(k_out, 16) && aligned_to(v_out, 16) && ldo % 8 == 0, word};
    auto st = static_cast<cudaStream_t>(stream);
    if (dt == CMPQ_BF16)
        launch_read<CMPQ_BF16>(a, st);
    else
        launch_read<CMPQ_F16>(a, st);
    return launch_status();
}
