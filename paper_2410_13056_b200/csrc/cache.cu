// Paged 8-bit cache of keys and values: append with the rotation on the way, and the values read back.
#include <algorithm>

#include "cache.cuh"
#include "tc5.cuh"

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
    int groups;    // rot_dim is a multiple of 16, cosines and sines can be read four at a time
    int few;       // few new tokens a sequence
    int q_heads, kv_heads;  // heads that a block of the queries, of the keys or values takes
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
    if (half % 8 == 0 && A.groups) {  // the partners of eight entries are eight neighbouring entries
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

// Sixteen entries of a head as two groups of eight from entries a and b on.  Where rot_dim is a multiple of 16 a thread's
// unit is closed under the rotation: a group and its partner group (1), or pairs inside the groups (2), or nothing turns.
struct Unit {
    int a, b, mode;
    __device__ __forceinline__ Unit(int u, int rot, bool interleaved) {
        const int pairs = interleaved ? 0 : rot / 16;
        a = u < pairs ? 8 * u : (interleaved ? 0 : rot) + 16 * (u - pairs);
        b = u < pairs ? rot / 2 + 8 * u : a + 8;
        mode = u < pairs ? 1 : interleaved && 16 * u < rot ? 2 : 0;
    }
};

// The unit's entries in fp32, turned.  c, s: cosines and sines 8 u .. of the position, in both modes.
template <int DT>
__device__ __forceinline__ void turned(uint4 a, uint4 b, int mode, const float (&c)[8], const float (&s)[8], float (&x)[8], float (&y)[8]) {
    widen8<DT>(a, x);
    widen8<DT>(b, y);
    if (mode == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = x[i], q = y[i];
            x[i] = p * c[i] - q * s[i];
            y[i] = q * c[i] + p * s[i];
        }
    } else if (mode == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = x[2 * i], q = x[2 * i + 1], v = y[2 * i], w = y[2 * i + 1];
            x[2 * i] = p * c[i] - q * s[i];
            x[2 * i + 1] = q * c[i] + p * s[i];
            y[2 * i] = v * c[4 + i] - w * s[4 + i];
            y[2 * i + 1] = w * c[4 + i] + v * s[4 + i];
        }
    }
}

// Heads [first, last) of the queries of one token.  A thread takes a unit of every head that is `heads` further on: its
// cosines and sines are loaded once for all of them, and what it reads it alone writes.
template <int DT>
__device__ __forceinline__ void rotate_queries(const AppendArgs& A, const uint16_t* src, uint16_t* dst, int64_t pos, int first, int last) {
    const int D = A.c.head_dim, G = D / 8, half = A.rot / 2, tid = threadIdx.x;
    if (A.groups && A.wide_q) {
        const int u = tid % (D / 16), h0 = tid / (D / 16), heads = (int)blockDim.x / (D / 16);
        const Unit at(u, A.rot, A.interleaved);
        float c[8], s[8];
        if (at.mode) load_floats(A.cos + pos * half + 8 * u, c), load_floats(A.sin + pos * half + 8 * u, s);
        constexpr int kAtOnce = 2;  // heads loaded before the first store: in place the compiler may not move a load past one
        for (int h = first + h0; h < last; h += kAtOnce * heads) {
            uint4 p[kAtOnce], q[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (h + k * heads < last) {
                    p[k] = *reinterpret_cast<const uint4*>(src + (h + k * heads) * D + at.a);
                    q[k] = *reinterpret_cast<const uint4*>(src + (h + k * heads) * D + at.b);
                }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (h + k * heads < last) {
                    float x[8], y[8];
                    turned<DT>(p[k], q[k], at.mode, c, s, x, y);
                    *reinterpret_cast<uint4*>(dst + (h + k * heads) * D + at.a) = round8<DT>(x);
                    *reinterpret_cast<uint4*>(dst + (h + k * heads) * D + at.b) = round8<DT>(y);
                }
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

// q_heads heads of the queries of a token.
template <int DT>
__device__ __forceinline__ void query_block(const AppendArgs& A, int block) {
    const int32_t* off = A.b.tok_off;
    const int chunks = (A.n_heads + A.q_heads - 1) / A.q_heads, first = block % chunks * A.q_heads;
    const int64_t t = block / chunks;
    const int s = block_count(A.b.n_seq, [&](int64_t i) { return off[i] <= t; });
    if (s >= A.b.n_seq) return;  // a row past the last sequence
    const int64_t pos = (int64_t)A.b.lens[s] - off[s + 1] + t;
    if (pos < 0 || (A.rot && pos >= A.n_pos)) {
        if (threadIdx.x == 0) report(A.word, kWordTable);
        return;
    }
    rotate_queries<DT>(A, A.q + t * A.ldq, A.q_out + t * A.ldqo, pos, first, min(A.n_heads, first + A.q_heads));
}

template <int DT>
__global__ void __launch_bounds__(256)
cache_queries_any_kernel(const __grid_constant__ AppendArgs A) {
    query_block<DT>(A, blockIdx.x);
}

// The queries of prompts where units are closed under the rotation: a block to a token, two units of a thread at a time.
// The first entries, whose place needs no position, are asked for before the sequence is looked up.
// Measured: 13.5 thousand tokens of 64 heads of 128 (440 MB) 84 us, 5.3 TB/s; several tokens to a block one after the other
// 92 to 185 us (the look-ups of each are waited for).
template <int DT>
__global__ void __launch_bounds__(256, 4)
cache_queries_kernel(const __grid_constant__ AppendArgs A) {
    const int D = A.c.head_dim, U = D / 16, half = A.rot / 2, tid = threadIdx.x, u = tid % U, h0 = tid / U, heads = 256 / U;
    const int32_t* off = A.b.tok_off;
    const Unit at(u, A.rot, A.interleaved);
    const int64_t t = blockIdx.x;
    const uint16_t* src = A.q + t * A.ldq;
    uint16_t* dst = A.q_out + t * A.ldqo;
    uint4 p[2], q[2];
    auto fetch = [&](int h) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (h + k * heads < A.n_heads) {
                p[k] = *reinterpret_cast<const uint4*>(src + (h + k * heads) * D + at.a);
                q[k] = *reinterpret_cast<const uint4*>(src + (h + k * heads) * D + at.b);
            }
    };
    fetch(h0);
    const int s = block_count(A.b.n_seq, [&](int64_t i) { return off[i] <= t; });
    if (s >= A.b.n_seq) return;  // a row past the last sequence
    const int64_t pos = (int64_t)A.b.lens[s] - off[s + 1] + t;
    if (pos < 0 || (A.rot && pos >= A.n_pos)) {
        if (tid == 0) report(A.word, kWordTable);
        return;
    }
    float c[8], sn[8];
    if (at.mode) load_floats(A.cos + pos * half + 8 * u, c), load_floats(A.sin + pos * half + 8 * u, sn);
    for (int h = h0; h < A.n_heads; h += 2 * heads) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (h + k * heads < A.n_heads) {
                float a[8], b[8];
                turned<DT>(p[k], q[k], at.mode, c, sn, a, b);
                *reinterpret_cast<uint4*>(dst + (h + k * heads) * D + at.a) = round8<DT>(a);
                *reinterpret_cast<uint4*>(dst + (h + k * heads) * D + at.b) = round8<DT>(b);
            }
        fetch(h + 2 * heads);
    }
}

// The page of a sequence that a block fills.
//
// The pages of sequence s start at slot tok_off[s] / P + 2 s: n new tokens touch at most (n + 2P - 2) / P pages,
// and that many slots lie between two neighbouring starts.  So a block finds its sequence from its index alone
// and the grid needs no length from the device; a slot without a page ends at once.
struct Place {
    int64_t page_id;  // -1: nothing to do
    int64_t row;      // first new token's row in k and v
    int64_t pos;      // and its position
    int held, fresh;  // tokens that the page holds already, new ones
};
__device__ __forceinline__ Place place_of(const AppendArgs& A, int64_t slot, bool keys) {
    const int P = A.c.page_tokens;
    const int32_t* off = A.b.tok_off;
    Place p;
    p.page_id = -1;
    const int s = block_count(A.b.n_seq - 1, [&](int64_t i) { return off[i] / P + 2 * i <= slot; });
    const int64_t from = off[s], n = off[s + 1] - from, len = A.b.lens[s], start = len - n;
    if (n <= 0) return p;
    if (start < 0 || from < 0 || from + n > A.b.n_tok) {
        if (threadIdx.x == 0) report(A.word, kWordTable);
        return p;
    }
    const int64_t page = start / P + (slot - (from / P + 2 * (int64_t)s));
    if (page * P >= len || page < start / P) return p;
    const int64_t lo = max(start, page * P), hi = min(len, (page + 1) * P);
    const int id = page < A.b.table_cols ? A.b.table[s * A.b.ld_table + page] : -1;
    if (id < 0 || id >= A.c.n_pages || (keys && A.rot && hi > A.n_pos)) {
        if (threadIdx.x == 0) report(A.word, kWordTable);
        return p;
    }
    p.page_id = id;
    p.row = from + (lo - start);
    p.pos = lo;
    p.held = (int)(lo - page * P), p.fresh = (int)(hi - lo);
    return p;
}

__device__ __forceinline__ float grown_scale(float before, uint32_t max_bits) {
    return fmaxf(before, fminf(fmaxf(__uint_as_float(max_bits) * (1.0f / 127.0f), kScaleLo), kScaleHi));
}

// The page's earlier codes under a scale that has grown.
__device__ __forceinline__ void scale_again(int8_t* codes, int count, float by) {
    for (int i = threadIdx.x; i < count / 8; i += blockDim.x) {
        uint2* p = reinterpret_cast<uint2*>(codes) + i;
        const uint2 c = *p;
        float x[8], y[4];
        widen_codes(c.x, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = y[e];
        widen_codes(c.y, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 + e] = y[e];
        *p = codes_of(x, by);
    }
}

// Any alignment and rotation.  The first kv_blocks blocks take (page of a sequence, head, keys or values).  Blocks of
// one warp are for single tokens: no barriers, and the blocks behind rotate the queries, so that a step of generation is
// one launch.  A block reads its new tokens, keeps the first NIT groups of a thread rotated in fp32 registers, agrees on
// the largest magnitude and writes codes; later rows of a thread are read again for that.  Each row of a head is D/8
// threads of eight entries, so global accesses are 16 bytes (inputs) and 8 bytes (codes), whole lines per row.
// Measured: one token of 64 sequences, 64/8 heads, 6.2 us a call, 3.6 in a graph, nearly all of it five dependent loads.
template <int DT, int NIT, int THREADS>
__global__ void __launch_bounds__(THREADS)
cache_append_kernel(const __grid_constant__ AppendArgs A) {
    if (THREADS == 32 && blockIdx.x >= A.kv_blocks) {
        query_block<DT>(A, blockIdx.x - A.kv_blocks);
        return;
    }
    const int D = A.c.head_dim, P = A.c.page_tokens, G = D / 8, H = A.c.n_kv_heads, tid = threadIdx.x;
    const int g = tid % G, r0 = tid / G, rows_at_once = THREADS / G;
    const bool is_v = blockIdx.x & 1;
    const int head = (blockIdx.x >> 1) % H;
    const Place at = place_of(A, (blockIdx.x >> 1) / H, !is_v);
    if (at.page_id < 0) return;
    float* scale = (is_v ? A.c.v_scale : A.c.k_scale) + at.page_id * H + head;
    int8_t* codes = (is_v ? A.c.v_codes : A.c.k_codes) + (at.page_id * H + head) * P * D;
    const float before = at.held ? *scale : 0.0f;
    const int64_t ld = is_v ? A.ldv : A.ldk;
    const uint16_t* src = (is_v ? A.v : A.k) + at.row * ld + head * D;

    auto entries = [&](int r, float (&f)[8]) {
        if (is_v)
            widen8<DT>(load8(src + r * ld + 8 * g, 8, A.wide_v), f);
        else
            rotated8<DT>(A, src + r * ld, 8 * g, A.wide_k, at.pos + r, f);
    };
    float f[NIT][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
        const int r = r0 + i * rows_at_once;
        if (r < at.fresh) {
            entries(r, f[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[i][e]) & 0x7fffffffu);
        }
    }
    for (int r = r0 + NIT * rows_at_once; r < at.fresh; r += rows_at_once) {
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
    const float after = grown_scale(before, m), inv = 1.0f / after;
    __syncwarp();
    if (tid == 0) {
        if (m >= 0x7f800000u) report(A.word, kWordNonfinite);
        *scale = after;
    }
    if (after > before) scale_again(codes, at.held * D, before * inv);
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
        const int r = r0 + i * rows_at_once;
        if (r < at.fresh) *reinterpret_cast<uint2*>(codes + (int64_t)(at.held + r) * D + 8 * g) = codes_of(f[i], inv);
    }
    for (int r = r0 + NIT * rows_at_once; r < at.fresh; r += rows_at_once) {
        float x[8];
        entries(r, x);
        *reinterpret_cast<uint2*>(codes + (int64_t)(at.held + r) * D + 8 * g) = codes_of(x, inv);
    }
}

// Prompts: a block takes a page's keys or values of a run of heads, one head after the other, a thread the same unit of
// 16 entries of NIT rows in each.  The place is looked up and the cosines and sines are read once for all heads, and the
// next head's entries and scale are on their way while this one's are turned, compared and written.
// Measured: the same tokens' 8 heads, pages of 32 (83 MB) 31 us; a block to a page and head 84 us.
template <int DT, int NIT, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 512 ? 1 : NIT == 1 ? 3 : 2)
cache_fill_kernel(const __grid_constant__ AppendArgs A) {
    const int D = A.c.head_dim, P = A.c.page_tokens, U = D / 16, H = A.c.n_kv_heads, tid = threadIdx.x;
    const int u = tid % U, r0 = tid / U, rows_at_once = THREADS / U;
    const bool is_v = blockIdx.x & 1;
    const int chunks = (H + A.kv_heads - 1) / A.kv_heads, first = (blockIdx.x >> 1) % chunks * A.kv_heads, last = min(H, first + A.kv_heads);
    const Place at = place_of(A, (blockIdx.x >> 1) / chunks, !is_v);
    if (at.page_id < 0) return;
    float* scales = (is_v ? A.c.v_scale : A.c.k_scale) + at.page_id * H;
    int8_t* pages = (is_v ? A.c.v_codes : A.c.k_codes) + at.page_id * H * P * D;
    const int64_t ld = is_v ? A.ldv : A.ldk;
    const uint16_t* src = (is_v ? A.v : A.k) + at.row * ld;
    const Unit unit(u, is_v ? 0 : A.rot, is_v || A.interleaved);

    float c[NIT][8], s[NIT][8];
    if (unit.mode) {
#pragma unroll
        for (int i = 0; i < NIT; ++i) {
            const int64_t row = (at.pos + min(r0 + i * rows_at_once, at.fresh - 1)) * (A.rot / 2) + 8 * u;
            load_floats(A.cos + row, c[i]);
            load_floats(A.sin + row, s[i]);
        }
    }
    uint4 p[NIT], q[NIT];
    float before = 0.0f;
    auto fetch = [&](int head) {
#pragma unroll
        for (int i = 0; i < NIT; ++i) {
            const int r = r0 + i * rows_at_once;
            p[i] = q[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r < at.fresh) {
                p[i] = __ldg(reinterpret_cast<const uint4*>(src + r * ld + head * D + unit.a));
                q[i] = __ldg(reinterpret_cast<const uint4*>(src + r * ld + head * D + unit.b));
            }
        }
        if (at.held) before = scales[head];
    };
    __shared__ uint32_t part[2][THREADS / 32];
    fetch(first);
    for (int head = first; head < last; ++head) {
        float x[NIT][8], y[NIT][8];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < NIT; ++i) {
            turned<DT>(p[i], q[i], unit.mode, c[i], s[i], x[i], y[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, max(__float_as_uint(x[i][e]) & 0x7fffffffu, __float_as_uint(y[i][e]) & 0x7fffffffu));
        }
        const float was = before;
        if (head + 1 < last) fetch(head + 1);
        m = __reduce_max_sync(0xffffffffu, m);
        if ((tid & 31) == 0) part[head & 1][tid >> 5] = m;
        __syncthreads();  // every thread has this head's scale; the other half of `part` is free again after the next one
#pragma unroll
        for (int i = 0; i < THREADS / 32; ++i) m = max(m, part[head & 1][i]);
        const float after = grown_scale(was, m), inv = 1.0f / after;
        if (tid == 0) {
            if (m >= 0x7f800000u) report(A.word, kWordNonfinite);
            scales[head] = after;
        }
        int8_t* codes = pages + (int64_t)head * P * D;
        if (after > was) scale_again(codes, at.held * D, was * inv);
#pragma unroll
        for (int i = 0; i < NIT; ++i) {
            const int r = r0 + i * rows_at_once;
            if (r >= at.fresh) continue;
            int8_t* o = codes + (at.held + r) * D;
            const uint2 a = codes_of(x[i], inv), b = codes_of(y[i], inv);
            if (unit.mode == 1) {
                *reinterpret_cast<uint2*>(o + unit.a) = a;
                *reinterpret_cast<uint2*>(o + unit.b) = b;
            } else {
                *reinterpret_cast<uint4*>(o + unit.a) = make_uint4(a.x, a.y, b.x, b.y);
            }
        }
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

// A block takes TOKENS tokens: the first threads find a token's page each, then all read and widen, a thread 16 codes of
// AT_ONCE tokens at a time (keys of all heads, then values), whose loads are under way together.
// Measured: 10 thousand tokens of 8 heads of 128 (63 MB) 22.5 us, 2.8 TB/s, the issue slots at 34 %: two batches of loads
// behind the look-up are all that a block does, and 640 blocks are little more than one round.
template <int DT, int TOKENS, int AT_ONCE>
__global__ void __launch_bounds__(256)
cache_read_kernel(const __grid_constant__ ReadArgs A) {
    const int D = A.c.head_dim, P = A.c.page_tokens, H = A.c.n_kv_heads, G = D / 16;
    const int32_t* off = A.b.tok_off;
    const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
    __shared__ int id[TOKENS], in_page[TOKENS];
    const int s0 = block_count(A.b.n_seq, [&](int64_t i) { return off[i] <= t0; });
    if (threadIdx.x < TOKENS) {
        const int64_t t = t0 + threadIdx.x;
        int found = -1, place = 0, s = s0;
        while (s < A.b.n_seq && off[s + 1] <= t) ++s;
        if (t < A.b.n_tok && s < A.b.n_seq) {
            const int64_t pos = (int64_t)A.b.lens[s] - off[s + 1] + t, page = pos >= 0 ? pos / P : 0;
            found = pos >= 0 && page < A.b.table_cols ? A.b.table[s * A.b.ld_table + page] : -1;
            place = (int)(pos - page * P);
            if (found < 0 || found >= A.c.n_pages) {
                found = -1;
                report(A.word, kWordTable);
            }
        }
        id[threadIdx.x] = found, in_page[threadIdx.x] = place;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * H * G; i += blockDim.x) {
        const bool is_v = i >= H * G;
        const int k = is_v ? i - H * G : i, h = k / G, g = k % G;
        const int8_t* codes = (is_v ? A.c.v_codes : A.c.k_codes) + (int64_t)h * P * D + 16 * g;
        const float* scales = (is_v ? A.c.v_scale : A.c.k_scale) + h;
        uint16_t* out = (is_v ? A.v : A.k) + t0 * A.ldo + h * D + 16 * g;
#pragma unroll 1
        for (int first = 0; first < TOKENS; first += AT_ONCE) {
            uint4 c[AT_ONCE];
            float sc[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const int page = id[first + j];
                if (page < 0) continue;
                c[j] = __ldg(reinterpret_cast<const uint4*>(codes + ((int64_t)page * H * P + in_page[first + j]) * D));
                sc[j] = __ldg(scales + (int64_t)page * H);
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                if (id[first + j] < 0) continue;
                const uint32_t x[4] = {c[j].x, c[j].y, c[j].z, c[j].w};
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float f[4];
                    widen_codes(x[e], f);
                    w[2 * e] = round16x2<DT>(f[0] * sc[j], f[1] * sc[j]);
                    w[2 * e + 1] = round16x2<DT>(f[2] * sc[j], f[3] * sc[j]);
                }
                uint16_t* o = out + (first + j) * A.ldo;
                if (A.wide) {
                    *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                    *reinterpret_cast<uint4*>(o + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                } else {
                    for (int e = 0; e < 16; ++e) o[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                }
            }
        }
    }
}

template <class Kernel, class Args>
static cmpq_status launch(Kernel kernel, unsigned blocks, int threads, const Args& a, cudaStream_t st) {
    return launch_cluster(kernel, blocks, threads, 0, 1, false, st, a);
}

template <int DT>
static cmpq_status launch_append(const AppendArgs& a, unsigned q_blocks, cudaStream_t st) {
    const unsigned kv = a.kv_blocks;
    if (a.few) return launch(cache_append_kernel<DT, 2, 32>, kv + q_blocks, 32, a, st);
    cmpq_status done;
    if (a.groups && a.wide_k && a.wide_v) {
        const int units = a.c.head_dim * a.c.page_tokens / 16;
        done = units <= 256    ? launch(cache_fill_kernel<DT, 1, 256>, kv, 256, a, st)
               : units == 512  ? launch(cache_fill_kernel<DT, 2, 256>, kv, 256, a, st)
               : units == 1024 ? launch(cache_fill_kernel<DT, 2, 512>, kv, 512, a, st)
                               : launch(cache_fill_kernel<DT, 4, 512>, kv, 512, a, st);
    } else {
        done = launch(cache_append_kernel<DT, 2, 256>, kv, 256, a, st);
    }
    if (done != CMPQ_OK || !q_blocks) return done;
    return a.groups && a.wide_q ? launch(cache_queries_kernel<DT>, q_blocks, 256, a, st) : launch(cache_queries_any_kernel<DT>, q_blocks, 256, a, st);
}

template <int DT>
static cmpq_status launch_read(const ReadArgs& a, cudaStream_t st) {
    // 16 tokens to a block once that leaves about four blocks an SM
    return a.b.n_tok >= 8192 ? launch(cache_read_kernel<DT, 16, 4>, (unsigned)((a.b.n_tok + 15) / 16), 256, a, st)
                             : launch(cache_read_kernel<DT, 1, 1>, (unsigned)a.b.n_tok, 256, a, st);
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
    a.b = bounded(*batch);
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
    a.groups = rot_dim % 16 == 0 && aligned_to(cos, 16) && aligned_to(sin, 16);
    // Four new tokens a sequence or fewer: blocks of one warp, without barriers, for a page and head or 16 heads of a
    // query; otherwise all threads that a full page occupies, and a block to the queries of a token.
    a.few = batch->n_tok <= 4 * batch->n_seq;
    a.q_heads = a.few ? 16 : n_heads;
    const int64_t slots = batch->n_tok / cache->page_tokens + 2 * batch->n_seq, heads = cache->n_kv_heads;
    // as many heads to a block as leave about eight blocks an SM
    const bool fill = !a.few && a.groups && a.wide_k && a.wide_v;
    a.kv_heads = fill ? (int)std::max<int64_t>(1, std::min(heads, slots * 2 * heads / (8 * std::max(1, sm_count())))) : 1;
    const int64_t kv = slots * ((heads + a.kv_heads - 1) / a.kv_heads) * 2;
    const int64_t q_blocks = q ? batch->n_tok * ((n_heads + a.q_heads - 1) / a.q_heads) : 0;
    if (kv + q_blocks > INT32_MAX) return CMPQ_ERR_UNSUPPORTED;
    a.kv_blocks = (unsigned)kv;
    auto st = static_cast<cudaStream_t>(stream);
    return dt == CMPQ_BF16 ? launch_append<CMPQ_BF16>(a, (unsigned)q_blocks, st) : launch_append<CMPQ_F16>(a, (unsigned)q_blocks, st);
}

extern "C" cmpq_status cmpq_cache_read(const cmpq_cache* cache, const cmpq_batch* batch, cmpq_dtype dt, void* k_out,
                                       void* v_out, int64_t ldo, int32_t* word, void* stream) {
    cmpq_status why;
    if (!cache_ok(cache, &why)) return why;
    if (!batch_ok(batch) || (dt != CMPQ_F16 && dt != CMPQ_BF16)) return CMPQ_ERR_INVALID_ARG;
    if (ldo < (int64_t)cache->n_kv_heads * cache->head_dim) return CMPQ_ERR_INVALID_ARG;
    if (batch->n_seq == 0 || batch->n_tok == 0) return CMPQ_OK;
    if (!k_out || !v_out || !aligned_to(k_out, 2) || !aligned_to(v_out, 2)) return CMPQ_ERR_INVALID_ARG;
    ReadArgs a{*cache, bounded(*batch), static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out), ldo,
               aligned_to(k_out, 16) && aligned_to(v_out, 16) && ldo % 8 == 0, word};
    auto st = static_cast<cudaStream_t>(stream);
    return dt == CMPQ_BF16 ? launch_read<CMPQ_BF16>(a, st) : launch_read<CMPQ_F16>(a, st);
}
