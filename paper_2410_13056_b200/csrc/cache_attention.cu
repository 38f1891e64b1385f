// Attention over the paged 8-bit cache.
//
// out = softmax(scale q K^T) V with K = S_k[page] c, V = S_v[page] c, c int8.  The codes are exact in fp16, so both
// products run on the tensor cores in fp16 with fp32 accumulation, a page's scale being one factor of its scores (keys)
// or of its weights (values); a query row is scaled by a power of two into fp16's range first, and a row's weights, times
// their value scales, by one that puts the largest near fp16's top.
#include <algorithm>
#include <cmath>

#include "attention.cuh"

namespace cmpq {

// ---- few query rows: warps share out the cache -------------------------------------------------------------------
//
// The time is that of reading the cache once, so the keys are split over all warps of the GPU.  The rows of a sequence
// and key-value head (its new tokens times the query heads of the group) are taken R = 8 NT at a time; such a unit is a
// run of tiles of 64 or 32 tokens.  All units' tiles, one behind the other, are dealt to the workers (warps) in equal
// contiguous runs: sequences of any lengths balance, and a worker meets few unit borders.  A unit inside one worker's run
// is finished there.  The parts of one that is cut are joined by the block that holds them and, where several do, by the
// last block to arrive, always in the order of the workers: the same bytes every time.
//
// Measured, D = 128: 64 sequences of up to 8191 tokens, 64/8 heads (608 MB): 126 to 131 us, 4.7 TB/s, 0.72 of the copy rate;
// two of up to 131072 (515 MB): 107 us; one of 2049, 32 heads: 16.2 us in a stream of calls.  What is left: the SMs get
// unequal shares of the memory (the blocks' loops of the second case end between 62 and 90 us), and some 10 us of look-ups,
// first loads and joins.
// Dealing the last 10 to 30 % in short runs to whichever block is free costs more in look-ups and joins than it evens out
// (136 to 139 and 138 to 157 us); asking for later tiles in L2 makes it slower (129 / 154 / 180 us for 1 / 2 / 4 tiles
// ahead).
constexpr int kMaxBlocks = 512;  // counters: one per block here, behind them those of the prompts' kernel, the last for kGaveUp

template <int D, int NT>
struct Rows {
    static constexpr int kR = 8 * NT;
    static constexpr int kWarps = 4;
    static constexpr int kTile = NT == 1 && D <= 128 ? 64 : 32;             // tokens; what the registers allow
    static constexpr int kTileBytes = kTile * D;                            // keys; as many for the values
    static constexpr int kBuffers = kTile == 64 ? 1 : 2;
    static constexpr int kPerSm = NT == 1 && D <= 128 ? 3 : D == 256 ? 1 : 2;
    static constexpr int kRing = kBuffers * 2 * kTileBytes > kR * (D + 2) * 4 ? kBuffers * 2 * kTileBytes : (kR * (D + 2) * 4 + 1023) / 1024 * 1024;
    static constexpr int kSmem = kWarps * kRing + 1024;
    static constexpr int kPart = kR * (D + 2);                              // floats of a partial result
};

struct SeqPlan {
    int first, n, len;  // row of the first query, queries, cached tokens
    int tile0, tiles, blocks;
    bool bad;
};

// What a sequence needs: its tiles per unit (one at least, so that rows without a key are written too) and its row
// blocks.  `count` of its tiles is tiles * blocks * heads, 0 for a sequence without queries or with bad lengths.
__device__ __forceinline__ SeqPlan seq_plan(const AttnArgs& A, int64_t s, int rows, int tile) {
    SeqPlan p;
    p.first = A.b.tok_off[s];
    p.n = A.b.tok_off[s + 1] - p.first;
    p.len = A.b.lens[s];
    p.bad = p.len < 0 || p.len > A.max_len || p.n < 0 || p.n > A.max_new || p.first < 0 || (int64_t)p.first + p.n > A.b.n_tok;
    const int lo = A.window > 0 ? max(0, max(0, p.len - p.n) - A.window + 1) : 0;  // a position may be far below 0
    p.tile0 = lo / tile;
    p.tiles = p.bad ? 1 : max(1, (p.len + tile - 1) / tile - p.tile0);
    p.blocks = p.bad ? 0 : (p.n * A.group + rows - 1) / rows;
    return p;
}
__device__ __forceinline__ int64_t seq_tiles(const AttnArgs& A, const SeqPlan& p) {
    return (int64_t)p.tiles * p.blocks * A.c.n_kv_heads;
}

// Inclusive sums over the warp's lanes.
__device__ __forceinline__ int64_t warp_scan(int64_t v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += o;
    }
    return v;
}
// Quotient and remainder of a dividend that nearly always has 32 bits.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b, int* rest) {
    if ((uint64_t)a >> 32 == 0 && (uint64_t)b >> 32 == 0) {
        const uint32_t q = (uint32_t)a / (uint32_t)b;
        *rest = (int)((uint32_t)a - q * (uint32_t)b);
        return q;
    }
    *rest = (int)(a % b);
    return a / b;
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Bytes of token t's entries from d on in a tile: rows of 128 bytes (two tokens of 64 entries, or half a token of 256 in
// a plane of its own), 16-byte groups swizzled by the row as the tensor map leaves them.
template <int D, int TILE>
__device__ __forceinline__ uint32_t tile_at(int t, int d) {
    if (D == 64) {
        const int row = t >> 1;
        return row * 128 + ((((t & 1) * 4 + (d >> 4)) ^ (row & 7)) << 4) + (d & 15);
    }
    const int plane = D == 256 ? d >> 7 : 0, e = D == 256 ? d & 127 : d;
    return plane * (TILE * 128) + t * 128 + (((e >> 4) ^ (t & 7)) << 4) + (e & 15);
}

// A worker's part of a unit: tiles [from, to) are the unit's, rows at output rows first.. of the head, block rb.
struct Piece {
    int64_t from, to;
    const float* at;
    int first, head, rb, rows;
};

// Joins n parts (rows of D entries, then maximum and sum of each row) in their order: into `into`, or, where that is
// null, into the output.  Every thread of the block; a thread takes four entries of a row at a time and sixteen parts'
// values are under way together (eight: 111 instead of 109 us for two streams of up to 131072 tokens, which join 28
// parts).
template <int DT, int D, int R, class Part>
__device__ __forceinline__ void join_parts(const AttnArgs& A, const Piece& u, int n, Part part, float* into) {
    constexpr int kAtOnce = 16;
    for (int i = threadIdx.x; i < u.rows * (D / 4); i += blockDim.x) {
        const int row = i / (D / 4), d = i % (D / 4) * 4;
        float top = -INFINITY, sum = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int k = 0; k < n; k += kAtOnce) {
            float2 ml[kAtOnce];
            float4 v[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                ml[j] = make_float2(-INFINITY, 0.0f);
                v[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (k + j < n) {
                    const float* p = part(k + j);
                    ml[j] = *reinterpret_cast<const float2*>(p + R * D + 2 * row);
                    v[j] = *reinterpret_cast<const float4*>(p + row * D + d);
                }
            }
            float most = top;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) most = fmaxf(most, ml[j].x);
            const float at = most == -INFINITY ? 0.0f : most, keep = ex2(top - at);
            top = most;
            sum *= keep, o.x *= keep, o.y *= keep, o.z *= keep, o.w *= keep;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const float f = ex2(ml[j].x - at);
                sum = fmaf(f, ml[j].y, sum);
                o.x = fmaf(f, v[j].x, o.x), o.y = fmaf(f, v[j].y, o.y), o.z = fmaf(f, v[j].z, o.z), o.w = fmaf(f, v[j].w, o.w);
            }
        }
        if (into) {
            *reinterpret_cast<float4*>(into + row * D + d) = o;
            if (d == 0) *reinterpret_cast<float2*>(into + R * D + 2 * row) = make_float2(top, sum);
            continue;
        }
        const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
        const int q = u.rb * R + row, h = u.head * A.group + q % A.group;
        const int64_t t = u.first + q / A.group;
        uint16_t* dst = A.out + t * A.ldo + (int64_t)h * D + d;
        const uint2 w = make_uint2(round16x2<DT>(o.x * f, o.y * f), round16x2<DT>(o.z * f, o.w * f));
        if (A.wide_o) {
            *reinterpret_cast<uint2*>(dst) = w;
        } else {
            dst[0] = (uint16_t)w.x, dst[1] = (uint16_t)(w.x >> 16), dst[2] = (uint16_t)w.y, dst[3] = (uint16_t)(w.y >> 16);
        }
        if (A.lse && d == 0) A.lse[t * A.n_heads + h] = sum > 0.0f ? (top - kWeightBits + log2f(sum)) * kLn2 : -INFINITY;
    }
}

// A lane's place in the m16n8k16 fragments: r = lane / 4, c = lane % 4.
//   scores   S^T[token][row] = K Q^T: a lane reads 16 bytes of keys of tokens r and r + 8 at a time, which are the A
//            entries of four instructions when the sum runs over the entries in the order 16 (2c + j) + 4 w + {0..3}
//            (w the instruction, any order serves as long as Q has the same); for D = 64 the 16 bytes are group c.
//   weights  the score fragment, rounded to fp16 and transposed eight by eight, is the B operand of
//   output   O^T[entry][row] = V^T P^T: a lane reads D/8 neighbouring entries of tokens 2c, 2c+1, 2c+8, 2c+9 and pairs
//            the tokens' bytes; entry i of its run is row r (i even) or r + 8 (i odd) of instruction i / 2.
// So keys and values are read from shared memory once, 16 bytes a time and without bank conflicts for D >= 128, and a
// lane ends up with D/8 neighbouring entries of two output rows.  Widening a code takes about 1.4 of a lane's
// instructions; all in all a tile of 64 tokens is some 1300 warp instructions, 40 % of the issue slots.
template <int DT, int D, int NT>
__global__ void __launch_bounds__(128, Rows<D, NT>::kPerSm)
attention_rows_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                      const __grid_constant__ AttnArgs A) {
    using C = Rows<D, NT>;
    constexpr int kR = C::kR, kTile = C::kTile, kBuffers = C::kBuffers, MT = kTile / 16;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[C::kWarps][2][kBuffers];
    __shared__ float2 page_scale[C::kWarps][64];  // key and value scales of the last 64 pages asked for
    __shared__ int failed[C::kWarps], is_last;
    __shared__ Piece pieces[C::kWarps][2], list[2 * C::kWarps];
    __shared__ int listed;
    uint8_t* smem = raw + ((1024u - (tc5::smem_addr(raw) & 1023u)) & 1023u);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, c = lane & 3;
    const int H = A.c.n_kv_heads, g = A.group, P = A.c.page_tokens, page_bits = A.page_bits;
    if (lane == 0) {
        for (int i = 0; i < kBuffers; ++i) tc5::mbar_init(&bars[warp][0][i], 1), tc5::mbar_init(&bars[warp][1][i], 1);
        failed[warp] = 0;
        pieces[warp][0].at = pieces[warp][1].at = nullptr;
        tc5::mbar_init_fence();
    }

    if (blockIdx.x == gridDim.x - 1 && tid == 127) report_stale(A);
    if (A.zero_behind) zero_behind(A, blockIdx.x, gridDim.x, tid, 32 * C::kWarps);

    // The total, this warp's run, and the sequence it starts in: every warp for itself, 32 sequences at a time.
    int64_t total = 0, mine = 0, upto = 0;
    for (int64_t at = 0; at < A.b.n_seq; at += 32) {
        mine = 0;
        if (at + lane < A.b.n_seq) {
            const SeqPlan p = seq_plan(A, at + lane, kR, kTile);
            mine = seq_tiles(A, p);
            if (p.bad && blockIdx.x == 0 && warp == 0 && A.word) atomicOr(A.word, kWordTable);
        }
        upto = total + warp_scan(mine);
        total = __shfl_sync(0xffffffffu, upto, 31);
    }
    const int64_t per = max((int64_t)1, (total + A.workers - 1) / A.workers);
    const int worker = blockIdx.x * C::kWarps + warp;
    const int64_t begin = worker * per, end = min(total, begin + per);
    int64_t s = 0, base = 0;
    if (begin < end) {
        for (int64_t at = 0, before = 0;; at += 32) {
            if (A.b.n_seq > 32) {  // the sums again; of 32 sequences or fewer they are still there
                mine = at + lane < A.b.n_seq ? seq_tiles(A, seq_plan(A, at + lane, kR, kTile)) : 0;
                upto = before + warp_scan(mine);
                before = __shfl_sync(0xffffffffu, upto, 31);
            }
            const unsigned here = __ballot_sync(0xffffffffu, upto - mine <= begin && begin < upto);
            if (here) {
                const int l = __ffs(here) - 1;
                s = at + l, base = __shfl_sync(0xffffffffu, upto - mine, l);
                break;
            }
        }
    }

    uint8_t* ring = smem + warp * C::kRing;  // keys, then values
    volatile int* gave_up = &failed[warp];
    int slot[2] = {0, 0}, phase[2] = {0, 0}, next[2] = {0, 0};  // of the keys and of the values: next to read, to fill

    for (int64_t x = begin; x < end;) {
        const SeqPlan p = seq_plan(A, s, kR, C::kTile);
        const int64_t all = seq_tiles(A, p);
        if (x >= base + all) {  // also a sequence without tiles
            base += all;
            ++s;
            continue;
        }
        int t_from, rb;
        const int64_t unit = divide(x - base, p.tiles, &t_from);
        const int head = (int)divide(unit, p.blocks, &rb);
        const int t_to = (int)min((int64_t)p.tiles, t_from + (end - x));  // tiles of this unit that are this worker's
        const int rows = min(kR, p.n * g - rb * kR);
        // positions of the block's first and last query; keys that any of them sees
        const int p0 = p.len - p.n + (rb * kR) / g, p1 = p.len - p.n + (rb * kR + rows - 1) / g;
        const int key_hi = A.causal ? max(0, p1 + 1) : p.len;
        const int key_lo = A.window > 0 ? max(0, max(0, p0) - A.window + 1) : 0;
        const int live_from = max(t_from, key_lo / kTile - p.tile0);
        const int live_to = min(t_to, (key_hi + kTile - 1) / kTile - p.tile0);
        // from this token on some row does not see a tile whole, and up to this one
        const int whole_hi = A.causal ? min(p.len, p0 + 1) : p.len, whole_lo = A.window > 0 ? max(0, p1) - A.window + 1 : 0;
        int row_pos[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) row_pos[nt][e] = p.len - p.n + (rb * kR + nt * 8 + 2 * c + e) / g;

        // Pages are looked up 32 at a time, one per lane.  The first tiles are asked for as soon as their pages are known;
        // the queries and the pages' scales are fetched under way.
        const int page0 = ((p.tile0 + live_from) * kTile) >> page_bits;
        const int page_end = (p.len + P - 1) >> page_bits;
        int my_page = -1, have = 0;  // pages page0 .. page0 + have are known
        auto fetch_pages = [&]() {
            const int page = page0 + have + lane;
            my_page = -1;
            if (page < page_end) {
                my_page = page < A.b.table_cols ? __ldg(A.b.table + s * A.b.ld_table + page) : -1;
                if (my_page < 0 || my_page >= A.c.n_pages) {
                    my_page = -1;
                    if (A.word) atomicOr(A.word, kWordTable);
                }
            }
            have += 32;
        };
        auto fetch_scales = [&]() {  // of the pages looked up last
            float2 sc = make_float2(0.0f, 0.0f);
            if (my_page >= 0) {
                const int64_t at = (int64_t)my_page * H + head;
                sc = make_float2(__ldg(A.c.k_scale + at), __ldg(A.c.v_scale + at));
            }
            page_scale[warp][(have - 32 + lane) & 63] = sc;
            __syncwarp();
        };
        auto ask = [&](int t, int which) {  // keys (0) or values (1) of tile t of the unit
            const int token = (p.tile0 + t) * kTile;
            const int page = (token >> page_bits) - page0;
            if (page >= have) fetch_pages(), fetch_scales();  // 32 pages hold whole tiles
            constexpr int kLine = D < 128 ? 128 / D : 1;  // tokens per row of the tensor map
            const int pieces = P < kTile ? kTile >> page_bits : 1, tokens = P < kTile ? P : kTile;
            const int first_id = __shfl_sync(0xffffffffu, my_page, page & 31);
            if (pieces == 1) {
                if (lane == 0) {
                    uint64_t* bar = &bars[warp][which][next[which]];
                    uint8_t* to = ring + (which * kBuffers + next[which]) * C::kTileBytes;
                    tc5::mbar_expect_tx(bar, first_id >= 0 ? C::kTileBytes : 0);
                    if (first_id >= 0) {
                        const int row = (int)(((((int64_t)first_id * H + head) << page_bits) + (token & (P - 1))) / kLine);
#pragma unroll
                        for (int plane = 0; plane < (D + 127) / 128; ++plane)
                            tc5::tma_load_2d(to + plane * kTile * 128, which ? &vmap : &kmap, bar, plane * 128, row);
                    }
                }
            } else {
                // a lane per page: the first lanes look at the pages that follow
                const int id = __shfl_sync(0xffffffffu, my_page, (page + lane) & 31);
                const bool mine_too = lane < pieces && id >= 0;
                const int n = __popc(__ballot_sync(0xffffffffu, mine_too));
                uint64_t* bar = &bars[warp][which][next[which]];
                if (lane == 0) tc5::mbar_expect_tx(bar, n * tokens * D);
                __syncwarp();
                if (mine_too) {
                    uint8_t* to = ring + (which * kBuffers + next[which]) * C::kTileBytes + lane * tokens * (D < 128 ? D : 128);
                    const int row = (int)((((int64_t)id * H + head) << page_bits) / kLine);
#pragma unroll
                    for (int plane = 0; plane < (D + 127) / 128; ++plane)
                        tc5::tma_load_2d(to + plane * kTile * 128, which ? &vmap : &kmap, bar, plane * 128, row);
                }
            }
            if (++next[which] == kBuffers) next[which] = 0;
        };
        fetch_pages();
        for (int t = live_from; t < live_to && t < live_from + kBuffers; ++t) ask(t, 0), ask(t, 1);

        // the queries, scaled into fp16
        uint32_t qf[NT][D / 16][2];
        float qs[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = nt * 8 + r, i = (rb * kR + row) / g, h = head * g + (rb * kR + row) % g;
            float f[D / 4];
            float m = 0.0f;
#pragma unroll
            for (int e = 0; e < D / 4; e += 8) {  // e / 16 the group of 16 entries, 16 (2c + e/16) (D = 64: 16 c)
                const int d = (D == 64 ? 16 * c : 16 * (2 * c + ((e >> 4) & 1)) + (e >> 5) * 128) + (e & 15);
                float v[8];
                if (row < rows) {
                    const uint16_t* src = A.q + (int64_t)(p.first + i) * A.ldq + (int64_t)h * D + d;
                    widen8<DT>(load8(src, 8, A.wide_q), v);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) f[e + j] = v[j], m = fmaxf(m, fabsf(v[j]));
            }
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const RowScale by = row_scale(m);
#pragma unroll
            for (int e = 0; e < D / 4; e += 2) {
                const __half2 hh = __floats2half2_rn(f[e] * by.down, f[e + 1] * by.down);
                qf[nt][e >> 2][(e >> 1) & 1] = *reinterpret_cast<const uint32_t*>(&hh);
            }
            const float mine = A.scale * by.up;  // of row r; the score fragment has rows 2c, 2c + 1
            qs[nt][0] = __shfl_sync(0xffffffffu, mine, (2 * c) * 4);
            qs[nt][1] = __shfl_sync(0xffffffffu, mine, (2 * c + 1) * 4);
        }

        float o[NT][D / 16][4], m2[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.0f;
            m2[nt][0] = m2[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.0f;
        }

        fetch_scales();

        for (int t = live_from; t < live_to; ++t) {
            const int token = (p.tile0 + t) * kTile;
            const int page = (token >> page_bits) - page0;
            float2 sc[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sc[mt] = page_scale[warp][(page + ((mt * 16) >> page_bits)) & 63];

            if (!tc5::mbar_wait_warp(&bars[warp][0][slot[0]], phase[0], gave_up)) break;
            const uint8_t* kt = ring + slot[0] * C::kTileBytes;
            float st[NT][MT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st[nt][mt][e] = 0.0f;
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const int d = D == 64 ? 16 * c : 16 * (2 * c + (j & 1)) + (j >> 1) * 128;
                    const uint4 lo = *reinterpret_cast<const uint4*>(kt + tile_at<D, kTile>(mt * 16 + r, d));
                    const uint4 hi = *reinterpret_cast<const uint4*>(kt + tile_at<D, kTile>(mt * 16 + r + 8, d));
                    const uint32_t a[4] = {lo.x, lo.y, lo.z, lo.w}, b[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t ua = a[w] ^ 0x80808080u, ub = b[w] ^ 0x80808080u;
                        const uint32_t a0 = half_pair(ua, 0x4140), a1 = half_pair(ub, 0x4140), a2 = half_pair(ua, 0x4342), a3 = half_pair(ub, 0x4342);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma_f16(st[nt][mt], a0, a1, a2, a3, qf[nt][4 * j + w][0], qf[nt][4 * j + w][1]);
                    }
                }
            }
            __syncwarp();  // every lane has read the keys
            if (++slot[0] == kBuffers) slot[0] = 0, phase[0] ^= 1;
            if (t + kBuffers < live_to) ask(t + kBuffers, 0);

            // scores in powers of two, what is not seen at -infinity
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st[nt][mt][e] *= qs[nt][e & 1] * sc[mt].x;
            if (token + kTile > whole_hi || token < whole_lo) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int pos = row_pos[nt][e & 1];
                        const int hi = A.causal ? min(p.len, pos + 1) : p.len, lo = A.window > 0 ? max(0, pos) - A.window : -1;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            const int key = token + mt * 16 + r + (e >> 1) * 8;
                            if (key >= hi || key <= lo) st[nt][mt][e] = -INFINITY;
                        }
                    }
            }
            // m2 is the row's largest score plus log2 of its page's value scale so far: what goes to fp16 is weight times value
            // scale, and the largest of those that the row sees is 2^15, which fp16 has: a row with one key that counts loses
            // nothing
            float above[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) above[mt] = scale_log2(sc[mt].y);
            uint32_t pf[NT][MT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float keep[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = fmaxf(st[nt][0][e], st[nt][0][e + 2]) + above[0];
#pragma unroll
                    for (int mt = 1; mt < MT; ++mt) top = fmaxf(top, fmaxf(st[nt][mt][e], st[nt][mt][e + 2]) + above[mt]);
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                    top = fmaxf(top, m2[nt][e]);
                    const float ref = top == -INFINITY ? 0.0f : top, at = ref - kWeightBits;
                    keep[e] = ex2(m2[nt][e] - ref);
                    m2[nt][e] = top;
                    float sum = 0.0f;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float w = ex2(st[nt][mt][e + 2 * k] - at);
                            sum += w;
                            st[nt][mt][e + 2 * k] = w * sc[mt].y;
                        }
                    l[nt][e] = fmaf(l[nt][e], keep[e], sum);  // this lane's tokens only; joined at the end
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const __half2 hh = __floats2half2_rn(st[nt][mt][2 * k], st[nt][mt][2 * k + 1]);
                        pf[nt][mt][k] = transpose8x8(*reinterpret_cast<const uint32_t*>(&hh));
                    }
                if (__any_sync(0xffffffffu, keep[0] != 1.0f || keep[1] != 1.0f)) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nt][i][e] *= keep[e & 1];
                }
            }
            if (!tc5::mbar_wait_warp(&bars[warp][1][slot[1]], phase[1], gave_up)) break;
            const uint8_t* vt = ring + (kBuffers + slot[1]) * C::kTileBytes;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int half = 0; half < (D + 127) / 128; ++half) {
                    constexpr int kW = D == 64 ? 2 : 4;  // words of a lane's run
                    uint32_t v[4][kW];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint8_t* at = vt + tile_at<D, kTile>(mt * 16 + 2 * c + (k & 1) + (k >> 1) * 8, D == 64 ? 8 * r : half * 128 + 16 * r);
                        if (D == 64) {
                            const uint2 x = *reinterpret_cast<const uint2*>(at);
                            v[k][0] = x.x ^ 0x80808080u, v[k][1] = x.y ^ 0x80808080u;
                        } else {
                            const uint4 x = *reinterpret_cast<const uint4*>(at);
                            v[k][0] = x.x ^ 0x80808080u, v[k][1] = x.y ^ 0x80808080u;
                            v[k][2 % kW] = x.z ^ 0x80808080u, v[k][3 % kW] = x.w ^ 0x80808080u;
                        }
                    }
#pragma unroll
                    for (int w = 0; w < kW; ++w) {
                        const uint32_t a01 = __byte_perm(v[0][w], v[1][w], 0x5140), a23 = __byte_perm(v[0][w], v[1][w], 0x7362);
                        const uint32_t b01 = __byte_perm(v[2][w], v[3][w], 0x5140), b23 = __byte_perm(v[2][w], v[3][w], 0x7362);
                        const uint32_t f0 = half_pair(a01, 0x4140), f1 = half_pair(a01, 0x4342), f2 = half_pair(b01, 0x4140), f3 = half_pair(b01, 0x4342);
                        const uint32_t h0 = half_pair(a23, 0x4140), h1 = half_pair(a23, 0x4342), h2 = half_pair(b23, 0x4140), h3 = half_pair(b23, 0x4342);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma_f16(o[nt][half * 8 + 2 * w], f0, f1, f2, f3, pf[nt][mt][0], pf[nt][mt][1]);
                            mma_f16(o[nt][half * 8 + 2 * w + 1], h0, h1, h2, h3, pf[nt][mt][0], pf[nt][mt][1]);
                        }
                    }
                }
            __syncwarp();  // every lane has read the values
            if (++slot[1] == kBuffers) slot[1] = 0, phase[1] ^= 1;
            if (t + kBuffers < live_to) ask(t + kBuffers, 1);
        }
        if (*gave_up) break;

        // The unit's rows: whole, or this worker's part of them.  A part after which the worker goes on to another unit
        // is put into the work space, since the copies for that unit take the shared memory; the last stays there.
        const bool whole = t_from == 0 && t_to == p.tiles;
        x += t_to - t_from;
        float* part = x < end ? A.parts + (int64_t)(A.workers / C::kWarps * 2 + worker) * C::kPart : reinterpret_cast<float*>(ring);
        if (!whole && lane == 0) {
            Piece& e = pieces[warp][x < end ? 0 : 1];
            e.from = base + unit * p.tiles, e.to = e.from + p.tiles;
            e.at = part;
            e.first = p.first, e.head = head, e.rb = rb, e.rows = rows;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[nt][e];
                sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                const int row = nt * 8 + 2 * c + e;
                if (row >= rows) continue;
                const float f = whole && sum > 0.0f ? 1.0f / sum : 0.0f;
                // entries 16 r (8 r for D = 64) and following of the row, in order
                if (whole) {
                    const int i = (rb * kR + row) / g, h = head * g + (rb * kR + row) % g;
                    uint16_t* dst = A.out + (int64_t)(p.first + i) * A.ldo + (int64_t)h * D;
#pragma unroll
                    for (int j = 0; j < D / 16; j += 4) {
                        const int d = D == 64 ? 8 * r : (j >> 3) * 128 + 16 * r + (j & 7) * 2;
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[k] = round16x2<DT>(o[nt][j + k][e] * f, o[nt][j + k][e + 2] * f);
                        if (A.wide_o) {
                            *reinterpret_cast<uint4*>(dst + d) = make_uint4(w[0], w[1], w[2], w[3]);
                        } else {
#pragma unroll
                            for (int k = 0; k < 8; ++k) dst[d + k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
                        }
                    }
                    if (A.lse && r == 0) A.lse[(int64_t)(p.first + i) * A.n_heads + h] = sum > 0.0f ? (m2[nt][e] - kWeightBits + log2f(sum)) * kLn2 : -INFINITY;
                } else {
#pragma unroll
                    for (int j = 0; j < D / 16; j += 2) {
                        const int d = D == 64 ? 8 * r + 2 * j : (j >> 3) * 128 + 16 * r + (j & 7) * 2;
                        *reinterpret_cast<float4*>(part + row * D + d) =
                            make_float4(o[nt][j][e], o[nt][j][e + 2], o[nt][j + 1][e], o[nt][j + 1][e + 2]);
                    }
                    if (r == 0) part[kR * D + 2 * row] = m2[nt][e], part[kR * D + 2 * row + 1] = sum;
                }
            }
    }
    if (*gave_up) {  // copies that were asked for have to land before the shared memory is given back
        const long long start = clock64();
        while (clock64() - start < (1ll << 21)) __nanosleep(1000);
        if (lane == 0) report_gave_up(A);
    }
    __syncthreads();

    // Parts of one unit that this block's warps hold, one behind the other, are joined here: into the result if the
    // unit lies in the block's run, otherwise into the block's part.  The block that adds the last of a unit's parts
    // (a counter at the block that began the unit tells) joins those, in the blocks' order, and clears the counter.
    if (warp == 0) {  // the parts there are, without gaps
        const Piece* mine_at = &pieces[0][0] + lane;
        const bool there = lane < 2 * C::kWarps && mine_at->at != nullptr;
        const unsigned all = __ballot_sync(0xffffffffu, there);
        if (there) list[__popc(all & ((1u << lane) - 1))] = *mine_at;
        if (lane == 0) listed = __popc(all);
    }
    __syncthreads();
    const int64_t block_run = per * C::kWarps, block_from = blockIdx.x * block_run, block_to = block_from + block_run;
    for (int first = 0; first < listed;) {
        const Piece& e = list[first];
        int n = 1;
        while (first + n < listed && list[first + n].from == e.from) ++n;
        auto local = [&](int k) { return list[first + k].at; };
        const bool complete = e.from >= block_from && e.to <= block_to;
        float* mine_out = A.parts + ((int64_t)blockIdx.x * 2 + (e.from >= block_from)) * C::kPart;
        join_parts<DT, D, kR>(A, e, n, local, complete ? nullptr : mine_out);
        if (!complete) {
            const int64_t b0 = e.from / block_run, b1 = (e.to - 1) / block_run;
            __threadfence();
            __syncthreads();
            if (tid == 0) is_last = atomicAdd(A.counters + b0, 1) == (int)(b1 - b0);
            __syncthreads();
            if (is_last) {
                __threadfence();
                auto far = [&](int k) { return (const float*)(A.parts + ((b0 + k) * 2 + (k == 0)) * (int64_t)C::kPart); };
                join_parts<DT, D, kR>(A, e, (int)(b1 - b0) + 1, far, nullptr);
                if (tid == 0) A.counters[b0] = 0;
            }
        }
        first += n;
    }
}

template <int DT, int D, int NT>
static cmpq_status launch_rows(AttnArgs a, cudaStream_t st) {
    using C = Rows<D, NT>;
    const cmpq_cache& c = a.c;
    CUtensorMap kmap, vmap;
    const int64_t tokens = c.n_pages * c.n_kv_heads * c.page_tokens;
    const int box_tokens = std::min(c.page_tokens, C::kTile);
    const int64_t rows = D == 64 ? tokens / 2 : tokens, width = D == 256 ? 256 : 128;
    if (rows > INT32_MAX) return CMPQ_ERR_UNSUPPORTED;
    const int box = D == 64 ? box_tokens / 2 : box_tokens;
    if (!make_byte_map(&kmap, c.k_codes, rows, width, width, box) || !make_byte_map(&vmap, c.v_codes, rows, width, width, box)) return CMPQ_ERR_CUDA;
    static bool raised[64];
    if (!raise_smem_limit_once(attention_rows_kernel<DT, D, NT>, C::kSmem, raised)) return CMPQ_ERR_CUDA;
    const int blocks = std::min(sm_count() * C::kPerSm, kMaxBlocks);
    a.workers = blocks * C::kWarps;
    return launch_cluster(attention_rows_kernel<DT, D, NT>, blocks, 32 * C::kWarps, C::kSmem, 1, false, st, kmap, vmap, a);
}

template <int DT, int D>
static cmpq_status launch_attention(const AttnArgs& a, cudaStream_t st) {
    // row blocks of 8 while one holds all rows of a sequence, of 16 otherwise
    const int64_t rows = (int64_t)a.max_new * a.group;
    return rows <= 8 ? launch_rows<DT, D, 1>(a, st) : launch_rows<DT, D, 2>(a, st);
}

// Which kernel takes a batch.  Up to 32 rows of a sequence and key-value head the warps that share out the cache, above
// 128 the one for prompts.  Between, the one for prompts too, unless its blocks, at the most splits of the keys, leave more
// than half of the SMs idle.  Measured over 771 batches (40 to 128 rows, 1 to 64 sequences of one length or of several, 512 to
// 32768 tokens, 1 to 32 heads of 64 and 128, with and without a window): 1 % above the better kernel on average, always
// the warps 56 %, always the other 4 %.  Microseconds, warps / other, D = 128, one sequence to 2048 and 16 to 8192 tokens: 4 heads,
// 64 rows 22 / 30 and 134 / 84; 8 heads, 40 rows 22 / 29 and 185 / 134.
static bool prefill_pays(const AttnArgs& a) {
    const int64_t rows = (int64_t)a.max_new * a.group, units = a.b.n_seq * a.c.n_kv_heads;
    if (a.c.head_dim > 128 || rows <= 32) return false;
    return rows > 128 || units * kPfSplits * 2 > sm_count();
}

// The counters, then two parts per block and one per worker, of the kernel that has most, or the parts of the prompts'.
static size_t attention_ws_bytes(int d) {
    const size_t narrow = (size_t)Rows<64, 1>::kPerSm * 6 * 8, wide = (size_t)Rows<64, 2>::kPerSm * 6 * 16;
    const size_t blocks = std::min(std::max(1, sm_count()), kMaxBlocks / Rows<64, 1>::kPerSm);
    return CMPQ_ATTENTION_ZEROED + std::max(blocks * std::max(narrow, wide) * (d + 2) * sizeof(float), prefill_parts_bytes(d));
}

}  // namespace cmpq

using namespace cmpq;

extern "C" size_t cmpq_cache_attention_ws_bytes(int64_t n_seq, int64_t n_tok, int64_t max_new, int64_t max_len,
                                                int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
    if (n_seq < 0 || n_tok < 0 || max_new < 0 || max_len < 0 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads ||
        head_dim < 1 || head_dim > 256)
        return 0;
    return round_up(attention_ws_bytes(head_dim), 256);
}

extern "C" cmpq_status cmpq_cache_attention(const cmpq_cache* cache, const cmpq_batch* batch, const void* q, int64_t ldq,
                                            cmpq_dtype dt, int32_t n_heads, int64_t max_new, int64_t max_len, float scale,
                                            int32_t causal, int64_t window, void* out, int64_t ldo, float* lse,
                                            int32_t* word, void* ws, size_t ws_bytes, void* stream) {
    cmpq_status why;
    if (!cache_ok(cache, &why)) return why;
    if (!batch_ok(batch) || (dt != CMPQ_F16 && dt != CMPQ_BF16)) return CMPQ_ERR_INVALID_ARG;
    if (n_heads < 1 || n_heads > 4096 || n_heads % cache->n_kv_heads || max_new < 0 || max_new > INT32_MAX || max_len < 0 || max_len > INT32_MAX - 256)
        return CMPQ_ERR_INVALID_ARG;
    const int zero = causal & CMPQ_ZERO_BEHIND;
    causal &= ~CMPQ_ZERO_BEHIND;
    if (window < 0 || (window > 0 && !causal) || !(scale > 0.0f) || isinf(scale)) return CMPQ_ERR_INVALID_ARG;
    const int64_t row = (int64_t)n_heads * cache->head_dim;
    if (ldq < row || ldo < row) return CMPQ_ERR_INVALID_ARG;
    if (batch->n_tok == 0 || (batch->n_seq == 0 && !zero)) return CMPQ_OK;
    if (!q || !out || !aligned_to(q, 2) || !aligned_to(out, 2) || !aligned_to(lse, 4)) return CMPQ_ERR_INVALID_ARG;
    if (batch->n_seq == 0)
        return cudaMemset2DAsync(out, ldo * 2, 0, row * 2, batch->n_tok, static_cast<cudaStream_t>(stream)) == cudaSuccess ? CMPQ_OK : CMPQ_ERR_CUDA;
    if (batch->n_tok * std::max(n_heads, cache->n_kv_heads) > INT32_MAX - 64) return CMPQ_ERR_UNSUPPORTED;
    if (!ws || !aligned_to(ws, 256) ||
        ws_bytes < cmpq_cache_attention_ws_bytes(batch->n_seq, batch->n_tok, max_new, max_len, n_heads, cache->n_kv_heads, cache->head_dim))
        return CMPQ_ERR_WORKSPACE;
    AttnArgs a{*cache, bounded(*batch), static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out), lse, ldq, ldo, (int)max_new, (int)max_len,
               (int)std::min<int64_t>(window, INT32_MAX), scale * kLog2e, n_heads, n_heads / cache->n_kv_heads, causal != 0, zero,
               31 - __builtin_clz(cache->page_tokens), aligned_to(q, 16) && ldq % 8 == 0, aligned_to(out, 16) && ldo % 8 == 0,
               word, static_cast<int*>(ws), reinterpret_cast<float*>(static_cast<char*>(ws) + CMPQ_ATTENTION_ZEROED), 0};
    auto st = static_cast<cudaStream_t>(stream);
    a.max_new = (int)std::min<int64_t>(max_new, batch->n_tok);  // a sequence has no more: a loose bound costs nothing
    if (window >= max_len) a.window = 0;  // it reaches every key: a position is below max_len
    const bool bf = dt == CMPQ_BF16;
    if (prefill_pays(a)) return launch_prefill(a, dt, st);
    switch (cache->head_dim) {
        case 64: return bf ? launch_attention<CMPQ_BF16, 64>(a, st) : launch_attention<CMPQ_F16, 64>(a, st);
        case 128: return bf ? launch_attention<CMPQ_BF16, 128>(a, st) : launch_attention<CMPQ_F16, 128>(a, st);
        default: return bf ? launch_attention<CMPQ_BF16, 256>(a, st) : launch_attention<CMPQ_F16, 256>(a, st);
    }
}
