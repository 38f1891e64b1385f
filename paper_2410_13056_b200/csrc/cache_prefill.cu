// Attention of many query rows over the paged 8-bit cache: both products on tcgen05, accumulators in TMEM.
#include <algorithm>
#include <type_traits>

#include "attention.cuh"

namespace cmpq {

// A block takes 256 query rows of a sequence and key-value head (its new tokens times the query heads of the group,
// next to each other, so that grouped heads share the keys) as two tiles of 128 and walks over the keys 128 at a time:
//   4 warps   widen the tile's keys and values from int8 to fp16 into shared memory, a buffer ahead
//   1 thread  (of four warps, the others idle) issues S_w = Q_w K^T and O_w += P_w V for the two row tiles in turn
//   2 x 4 warps, a thread per row: weights P_w = exp2(S_w - m) in fp16 over S_w's own TMEM columns
// While one row tile's weights are made the other's products run.  TMEM holds S (2 x 128 columns) and O (2 x D).
// The weights carry the value scale of their page as part of the exponent, and the row's sum takes it out again page by
// page.  The reference m is the row's own largest of score plus log2 of the value scale, over keys that it sees, so pages
// that it does not see, or hardly weighs, cost the others no bits of fp16.  It follows the true maximum only when that
// has grown by more than 2^8, so what goes to fp16 ends in [2^7, 2^15]: then, rarely after the first tiles, O is multiplied
// in TMEM.  Rows of keys and of queries keep the order of their entries 16 c + 8 p + e as plane p, group c, entry e, so
// that the 16 codes a lane widens go to the same group of two planes and a row's lanes to different banks.
// With 128 rows or fewer the two accumulators take every other tile of keys of the one row tile and are joined at the end;
// fewer units than SMs are split over the keys, the last block to arrive joining the parts in their order.
//
// Measured: 2 x up to 2048 queries over up to 6145 tokens, 32 heads, D = 128: 292 us, 762 TFLOP/s of visible pairs, 0.47 of
// the library's bf16 product; the tensor pipe is at 43 %.  Per 256 rows x 128 keys the weights' warps work 3000 cycles and
// wait 1050 for scores, the warps that widen wait 1220, the products' thread 1490 of 4100; the floor of the exponential unit
// is 2048, of the products about the same.  Tried when the whole took 292 us: steps of 32 keys 307, of 128 (registers spill)
// 309; scores of 64 keys in two buffers, so that the weights never wait, 301 (twice the barriers, and M = 128, N = 64 products
// read shared memory 1.5 times as long).
constexpr int kPfKeys = 128, kPfThreads = 16 * 32;
constexpr float kPfSlack = 8.0f;
// Registers a thread: launched with 128, four warps of each of the four groups; 2 x 168 + 112 + 64 = 4 x 128.
constexpr int kPfRegsRows = 168, kPfRegsWiden = 112, kPfRegsOther = 64;
static_assert(2 * kPfRegsRows + kPfRegsWiden + kPfRegsOther <= 4 * (65536 / kPfThreads), "shares of what the block is launched with");

template <int D>
struct Prefill {
    static constexpr int kPlanes = D / 64;
    static constexpr int kTileBytes = 128 * D * 2;                      // 128 rows or keys in fp16
    static constexpr int kSmem = 2 * kTileBytes + 4 * kTileBytes + 1024;  // queries; keys and values, two buffers each
};

// Where group (of eight entries) j of row t lies in a tile of 128 rows: see above for the order of the groups.
template <int D>
__device__ __forceinline__ uint32_t pf_at(int t, int j) {
    const int c = j >> 1, p = j & 1;
    if (D == 128) return p * (128 * 128) + t * 128 + ((c ^ (t & 7)) << 4);
    return t * 128 + (((p * 4 + c) ^ (t & 7)) << 4);
}

// Two floats in one register pair, and the instructions on such pairs.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ float low(uint64_t p) { return __uint_as_float((uint32_t)p); }
__device__ __forceinline__ float high(uint64_t p) { return __uint_as_float((uint32_t)(p >> 32)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// How the units (row block, sequence, key-value head) are dealt to blocks: `splits` blocks share out a unit's keys.
struct PrefillPlan {
    int row_blocks, per_row_block, splits;
};
constexpr int kPfCounters = 512;  // where its counters begin

// A row's entries, times f, as 16 bits into `dst` or as they are into `part`.  columns(c, x, y) gives the accumulator's
// columns c.. and D/2 + c.. and is called by all lanes; `real`: the row exists.
template <int DT, int D, class Columns>
__device__ __forceinline__ void store_row(Columns columns, float f, bool real, float* part, uint16_t* dst, bool wide) {
#pragma unroll
    for (int c = 0; c < D / 2; c += 32) {
        uint32_t x[32], y[32];
        __syncwarp();
        columns(c, x, y);
        if (!real) continue;
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) * f), y[j] = __float_as_uint(__uint_as_float(y[j]) * f);
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
            if (part) {
                uint4* o = reinterpret_cast<uint4*>(part + 2 * (c + j));
                o[0] = make_uint4(x[j], x[j + 1], x[j + 2], x[j + 3]);
                o[1] = make_uint4(x[j + 4], x[j + 5], x[j + 6], x[j + 7]);
                o[2] = make_uint4(y[j], y[j + 1], y[j + 2], y[j + 3]);
                o[3] = make_uint4(y[j + 4], y[j + 5], y[j + 6], y[j + 7]);
                continue;
            }
            uint32_t a[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                a[k] = round16x2<DT>(__uint_as_float(x[j + 2 * k]), __uint_as_float(x[j + 2 * k + 1]));
                a[4 + k] = round16x2<DT>(__uint_as_float(y[j + 2 * k]), __uint_as_float(y[j + 2 * k + 1]));
            }
            uint16_t* o = dst + 2 * (c + j);
            if (wide) {
                *reinterpret_cast<uint4*>(o) = make_uint4(a[0], a[1], a[2], a[3]);
                *reinterpret_cast<uint4*>(o + 8) = make_uint4(a[4], a[5], a[6], a[7]);
            } else {
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = (uint16_t)(a[k >> 1] >> (16 * (k & 1)));
            }
        }
    }
}

// PAGES: pages that 64 neighbouring keys lie on at most.
template <int DT, int D, int PAGES>
__global__ void __launch_bounds__(kPfThreads, 1)
attention_prefill_kernel(const __grid_constant__ AttnArgs A, const __grid_constant__ PrefillPlan plan) {
    using C = Prefill<D>;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024u - (tc5::smem_addr(raw) & 1023u)) & 1023u);
    uint8_t* const sq = smem;
    uint8_t* const sk = smem + 2 * C::kTileBytes;
    uint8_t* const sv = smem + 4 * C::kTileBytes;
    __shared__ uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_full[2];
    __shared__ uint32_t tmem_at;
    __shared__ int failed, is_last;
    __shared__ float2 half_ml[128];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int H = A.c.n_kv_heads, g = A.group, page_bits = A.page_bits;
    if (blockIdx.x == 0 && tid == kPfThreads - 1) report_stale(A);
    // the last row blocks see most keys and come first
    const int splits = plan.splits, unit = blockIdx.x / splits, z = blockIdx.x % splits;
    const int rb = plan.row_blocks - 1 - unit / plan.per_row_block, s = unit % plan.per_row_block / H, head = unit % H;

    if (A.zero_behind && z == 0 && s == A.b.n_seq - 1) zero_behind(A, rb * H + head, (int64_t)plan.row_blocks * H, tid, kPfThreads);
    const int first = A.b.tok_off[s], n = A.b.tok_off[s + 1] - first, len = A.b.lens[s];
    if (len < 0 || len > A.max_len || n < 0 || n > A.max_new || first < 0 || (int64_t)first + n > A.b.n_tok) {
        if (tid == 0 && A.word) atomicOr(A.word, kWordTable);
        return;
    }
    const int rows = min(256, n * g - rb * 256);
    if (rows <= 0) return;
    const bool two = rows > 128;
    // positions of the first and last query, keys that any of them sees, tiles of keys
    const int p0 = len - n + (rb * 256) / g, p1 = len - n + (rb * 256 + rows - 1) / g;
    const int key_hi = A.causal ? max(0, p1 + 1) : len, key_lo = A.window > 0 ? max(0, max(0, p0) - A.window + 1) : 0;  // p0 may be far below 0
    const int tile0 = key_lo / kPfKeys, all_tiles = key_hi > key_lo ? (key_hi + kPfKeys - 1) / kPfKeys - tile0 : 0;
    const int t0 = tile0 + all_tiles * z / splits, tiles = tile0 + all_tiles * (z + 1) / splits - t0;  // this block's
    const int32_t* table = A.b.table + (int64_t)s * A.b.ld_table;
    const int pages = (len + (1 << page_bits) - 1) >> page_bits;
    auto page_of = [&](int page) {  // -1 where there is none
        const int id = page < pages && page < A.b.table_cols ? __ldg(table + page) : -1;
        if (id >= 0 && id < A.c.n_pages) return id;
        if (page < pages && A.word) atomicOr(A.word, kWordTable);
        return -1;
    };

    if (tid == 0) {
        tc5::mbar_init(&q_full, 8);
        for (int i = 0; i < 2; ++i) {
            tc5::mbar_init(k_full + i, 4), tc5::mbar_init(v_full + i, 4);
            tc5::mbar_init(k_empty + i, 1), tc5::mbar_init(v_empty + i, 1);
            tc5::mbar_init(s_full + i, 1), tc5::mbar_init(p_full + i, 4), tc5::mbar_init(o_full + i, 1);
        }
        failed = 0;
        tc5::mbar_init_fence();
    }
    if (warp == 12) tc5::tmem_alloc<1>(&tmem_at, 512);
    tc5::fence_before_sync();
    __syncthreads();
    tc5::fence_after_sync();
    const uint32_t tmem = tmem_at, tmem_o = tmem + 256;

    if (warp >= 12) {
        tc5::give_registers<kPfRegsOther>();
        if (warp == 12 && tiles > 0 && tc5::elect_one()) {
            constexpr uint32_t kScores = tc5::idesc_f16(128, 128), kOut = tc5::idesc_f16(128, D) | tc5::kTransposedB;
            const uint32_t aq = tc5::smem_addr(sq), ak = tc5::smem_addr(sk), av = tc5::smem_addr(sv);
            auto scores = [&](int w, int t) {
                const uint64_t a = tc5::desc_k_sw128(aq + (two ? w : 0) * C::kTileBytes), b = tc5::desc_k_sw128(ak + (t & 1) * C::kTileBytes);
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    const uint32_t at = (j >> 2) * (128 * 128 >> 4) + (j & 3) * 2;
                    tc5::mma_f16_ss(tmem + w * 128, a + at, b + at, kScores, j != 0);
                }
                tc5::mma_commit(s_full + w);
            };
            auto outputs = [&](int w, int t) {
                const uint64_t b = tc5::desc_mn_sw128(av + (t & 1) * C::kTileBytes, 128 * 128);
#pragma unroll
                for (int j = 0; j < kPfKeys / 16; ++j)
                    tc5::mma_f16_ts(tmem_o + w * 128, tmem + w * 128 + j * 8, b + j * (2048 >> 4), kOut, (two ? t : t >> 1) != 0 || j != 0);
            };
            bool ok = tc5::mbar_wait(&q_full, 0, &failed) && tc5::mbar_wait(k_full, 0, &failed);
            tc5::fence_after_sync();
            if (ok && two) {
                scores(0, 0);
                scores(1, 0);
                tc5::mma_commit(k_empty);
                for (int t = 0; ok && t < tiles; ++t) {
                    const int slot = t & 1, next = (t + 1) & 1;
                    ok = tc5::mbar_wait(v_full + slot, (t >> 1) & 1, &failed);
                    if (ok && t + 1 < tiles) ok = tc5::mbar_wait(k_full + next, ((t + 1) >> 1) & 1, &failed);
#pragma unroll 1
                    for (int w = 0; ok && w < 2; ++w) {
                        if (!(ok = tc5::mbar_wait(p_full + w, t & 1, &failed))) break;
                        tc5::fence_after_sync();
                        outputs(w, t);
                        if (t + 1 < tiles) {
                            scores(w, t + 1);
                        } else {
                            tc5::mma_commit(o_full + w);
                        }
                    }
                    tc5::mma_commit(v_empty + slot);
                    if (t + 1 < tiles) tc5::mma_commit(k_empty + next);
                }
            } else if (ok) {  // one row tile: the two accumulators take every other tile of keys
                scores(0, 0);
                tc5::mma_commit(k_empty);
                if (tiles > 1) {
                    ok = tc5::mbar_wait(k_full + 1, 0, &failed);
                    tc5::fence_after_sync();
                    scores(1, 1);
                    tc5::mma_commit(k_empty + 1);
                }
                for (int t = 0; ok && t < tiles; ++t) {
                    const int w = t & 1, phase = (t >> 1) & 1;
                    ok = tc5::mbar_wait(v_full + w, phase, &failed) && tc5::mbar_wait(p_full + w, phase, &failed);
                    if (ok && t + 2 < tiles) ok = tc5::mbar_wait(k_full + w, phase ^ 1, &failed);
                    if (!ok) break;
                    tc5::fence_after_sync();
                    outputs(w, t);
                    tc5::mma_commit(v_empty + w);
                    if (t + 2 < tiles) {
                        scores(w, t + 2);
                        tc5::mma_commit(k_empty + w);
                    } else {
                        tc5::mma_commit(o_full + w);
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp >= 8) {
        tc5::give_registers<kPfRegsWiden>();
        // a row's lanes: D/16 of them, 16 codes each
        constexpr int kLanes = D / 16, kRows = 32 / kLanes, kSteps = 32 / kRows;  // rows of a warp at a time, times per tile
        const int w = warp - 8, c = lane % kLanes, q = lane / kLanes;
        const int r0 = D == 64 ? (q & 1) * 4 + (q >> 1) : q;  // eight neighbouring lanes write to different banks
        uint4 kc[kSteps], vc[kSteps];
        // the warp's 32 keys lie on one page or, of 16 tokens, on two
        int64_t at[2];
        auto pages_of = [&](int t) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int key = (t0 + t) * kPfKeys + w * 32 + k * 16, id = page_of(key >> page_bits);
                at[k] = id < 0 ? -1 : ((((int64_t)id * H + head) << page_bits) + (key & ((1 << page_bits) - 1)) + r0) * D + 16 * c;
            }
        };
        auto fetch = [&](const int8_t* codes, uint4 (&x)[kSteps]) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int k = i * kRows / 16;
                x[i] = make_uint4(0u, 0u, 0u, 0u);
                if (at[k] >= 0) x[i] = __ldg(reinterpret_cast<const uint4*>(codes + at[k] + (i * kRows - 16 * k) * D));
            }
        };
        auto put = [&](uint8_t* tile, const uint4 (&x)[kSteps]) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int row = w * 32 + i * kRows + r0;
                const uint32_t a = x[i].x ^ 0x80808080u, b = x[i].y ^ 0x80808080u, d = x[i].z ^ 0x80808080u, e = x[i].w ^ 0x80808080u;
                *reinterpret_cast<uint4*>(tile + pf_at<D>(row, 2 * c)) =
                    make_uint4(half_pair(a, 0x4140), half_pair(a, 0x4342), half_pair(b, 0x4140), half_pair(b, 0x4342));
                *reinterpret_cast<uint4*>(tile + pf_at<D>(row, 2 * c + 1)) =
                    make_uint4(half_pair(d, 0x4140), half_pair(d, 0x4342), half_pair(e, 0x4140), half_pair(e, 0x4342));
            }
        };
        if (tiles > 0) pages_of(0), fetch(A.c.k_codes, kc), fetch(A.c.v_codes, vc);
        for (int t = 0; t < tiles; ++t) {
            const int slot = t & 1, phase = ((t >> 1) & 1) ^ 1;
            if (!tc5::mbar_wait_warp(k_empty + slot, phase, &failed)) break;
            put(sk + slot * C::kTileBytes, kc);
            tc5::fence_async_smem();
            __syncwarp();
            if (lane == 0) tc5::mbar_arrive(k_full + slot);
            if (t + 1 < tiles) pages_of(t + 1), fetch(A.c.k_codes, kc);
            if (!tc5::mbar_wait_warp(v_empty + slot, phase, &failed)) break;
            put(sv + slot * C::kTileBytes, vc);
            tc5::fence_async_smem();
            __syncwarp();
            if (lane == 0) tc5::mbar_arrive(v_full + slot);
            if (t + 1 < tiles) fetch(A.c.v_codes, vc);
        }
    } else {
        tc5::take_registers<kPfRegsRows>();
        const int w = warp >> 2, local = tid & 127, in_block = (two ? w : 0) * 128 + local, row = rb * 256 + in_block;
        const bool real = in_block < rows;
        const int i = row / g, h = head * g + row % g, pos = len - n + i;
        // this row's query into shared memory, scaled by a power of two into fp16's range
        float qs = 0.0f;
        {
            const uint16_t* src = A.q + (int64_t)(first + i) * A.ldq + (int64_t)h * D;
            uint4 x[D / 8];
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < D / 8; ++j) {
                x[j] = real ? load8(src + 8 * j, 8, A.wide_q) : make_uint4(0u, 0u, 0u, 0u);
                const uint32_t e[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) m = max(m, max(e[k] & 0x7fffu, e[k] >> 16 & 0x7fffu));
            }
            const RowScale by = row_scale(widen16<DT>((uint16_t)m));
#pragma unroll
            for (int j = 0; j < D / 8; ++j) {
                float f[8];
                uint32_t y[4];
                widen8<DT>(x[j], f);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = round16x2<CMPQ_F16>(f[2 * k] * by.down, f[2 * k + 1] * by.down);
                if (two || w == 0) *reinterpret_cast<uint4*>(sq + w * C::kTileBytes + pf_at<D>(local, j)) = make_uint4(y[0], y[1], y[2], y[3]);
            }
            qs = A.scale * by.up;
            tc5::fence_async_smem();
            __syncwarp();
            if (lane == 0) tc5::mbar_arrive(&q_full);
        }
        const uint32_t lanes = (uint32_t)(warp & 3) << 21, ts = tmem + w * 128 + lanes, to = tmem_o + w * 128 + lanes;
        const int span_bits = min(7, page_bits), per_tile = kPfKeys >> span_bits;
        // Lane k holds the scales of the tile's k-th page.  Those of the next tile are under way, and so is the look-up of the
        // page in the tile behind that: neither is waited for (one look-up at a time stalled each tile for a memory latency).
        float2 sc, sc_next = make_float2(0.0f, 0.0f);
        int id_next = -1;
        auto look_up = [&](int t) {  // not looked at here; the warps that widen the codes report what is no page
            const int page = ((t0 + t) * kPfKeys >> page_bits) + lane;
            return lane < per_tile && t < tiles && page < min(pages, (int)min((int64_t)INT32_MAX, A.b.table_cols)) ? __ldg(table + page) : -1;
        };
        auto scales = [&](int id) {
            return id < 0 || id >= A.c.n_pages ? make_float2(0.0f, 0.0f)
                                               : make_float2(__ldg(A.c.k_scale + (int64_t)id * H + head), __ldg(A.c.v_scale + (int64_t)id * H + head));
        };
        // with one row tile the second four warps take every other tile of keys
        const int t_first = two ? 0 : w, t_step = two ? 1 : 2;
        const bool work = t_first < tiles;
        if (work) sc_next = scales(look_up(t_first)), id_next = look_up(t_first + t_step);
        float m = -INFINITY, l = 0.0f;
        // keys [lo, hi) are seen by this row; a tile inside [all_lo, all_hi) is seen whole by the warp's rows
        const int hi = real ? (A.causal ? min(len, pos + 1) : len) : INT32_MAX, lo = real && A.window > 0 ? max(0, pos) - A.window + 1 : 0;
        const int all_hi = __reduce_min_sync(0xffffffffu, hi), all_lo = __reduce_max_sync(0xffffffffu, lo);
        // The reference maximum has moved before keys 32 step.. of tile t: what was weighted with the old one.
        auto rescale = [&](int t, int step, float keep) {
            if (t > t_first) {  // the products into O that came before have ended: S was committed after them
#pragma unroll 1
                for (int c = 0; c < D; c += 16) {
                    uint32_t x[16];
                    tc5::tmem_ld16(to + c, x);
                    tc5::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) * keep);
                    tc5::tmem_st16(to + c, x);
                }
            }
#pragma unroll 1
            for (int k = 0; k < step; ++k) {  // weights of this tile
                uint32_t x[16];
                tc5::tmem_st_wait();
                tc5::tmem_ld16(ts + k * 16, x);
                tc5::tmem_ld_wait();
                const __half2 by = __float2half2_rn(keep);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&x[j]), by);
                    x[j] = *reinterpret_cast<const uint32_t*>(&y);
                }
                tc5::tmem_st16(ts + k * 16, x);
            }
        };
        bool ok = true;
        for (int t = t_first; t < tiles; t += t_step) {
            sc = sc_next;
            const float bias = scale_log2(sc.y), inv_vs = ex2(-bias);
            sc_next = scales(id_next);
            id_next = look_up(t + 2 * t_step);
            if (!(ok = tc5::mbar_wait_warp(s_full + w, (two ? t : t >> 1) & 1, &failed))) break;
            tc5::fence_after_sync();
            const int key0 = (t0 + t) * kPfKeys;
            const int from = lo - key0, upto = hi - key0;
            auto tile = [&](auto masked) {
                #pragma unroll
                for (int step = 0; step < 2; ++step) {  // 64 keys, on PAGES pages at most
                    constexpr int kCols = 64 / PAGES;
                    uint32_t v[64];
                    tc5::tmem_ld32(ts + step * 64, v);
                    tc5::tmem_ld32(ts + step * 64 + 32, v + 32);
                    tc5::tmem_ld_wait();
                    if (decltype(masked)::value) {
#pragma unroll
                        for (int j = 0; j < 64; ++j)
                            if (step * 64 + j < from || step * 64 + j >= upto) v[j] = 0xff800000u;  // -infinity
                    }
                    float f[PAGES], b[PAGES], top = -INFINITY;
#pragma unroll
                    for (int k = 0; k < PAGES; ++k) {
                        f[k] = fmaxf(qs * __shfl_sync(0xffffffffu, sc.x, (step * 64 + k * kCols) >> span_bits), 0x1p-126f);
                        b[k] = __shfl_sync(0xffffffffu, bias, (step * 64 + k * kCols) >> span_bits);
                        float most[4];  // side by side
#pragma unroll
                        for (int j = 0; j < 4; ++j) most[j] = __uint_as_float(v[k * kCols + j]);
#pragma unroll
                        for (int j = 4; j < kCols; j += 2) most[j >> 1 & 3] = fmaxf(fmaxf(most[j >> 1 & 3], __uint_as_float(v[k * kCols + j])), __uint_as_float(v[k * kCols + j + 1]));
                        top = fmaxf(top, fmaf(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])), f[k], b[k]));
                    }
                    const bool grown = top > m + kPfSlack;
                    if (__any_sync(0xffffffffu, grown)) {
                        const float now = grown ? top : m, keep = grown ? ex2(m - now) : 1.0f;
                        m = now;
                        l *= keep;
                        rescale(t, 2 * step, keep);
                    }
                    const float at = (m == -INFINITY ? 0.0f : m) - (kWeightBits - kPfSlack);
                    uint32_t y[32];
#pragma unroll
                    for (int k = 0; k < PAGES; ++k) {
                        const int page = (step * 64 + k * kCols) >> span_bits;
                        const float add = b[k] - at;
                        const uint64_t ff = pair(f[k], f[k]), aa = pair(add, add);
                        uint64_t sum[2] = {0, 0};
#pragma unroll
                        for (int j = 0; j < kCols; j += 2) {
                            const uint64_t z = fma2(pair(__uint_as_float(v[k * kCols + j]), __uint_as_float(v[k * kCols + j + 1])), ff, aa);
                            const float a = ex2(low(z)), b = ex2(high(z));
                            sum[j >> 1 & 1] = add2(sum[j >> 1 & 1], pair(a, b));
                            y[(k * kCols + j) / 2] = round16x2<CMPQ_F16>(a, b);
                        }
                        const uint64_t both = add2(sum[0], sum[1]);
                        l = fmaf(low(both) + high(both), __shfl_sync(0xffffffffu, inv_vs, page), l);
                    }
                    tc5::tmem_st32(ts + step * 32, y);
                }
            };
            if (key0 + kPfKeys > all_hi || key0 < all_lo)
                tile(std::true_type());
            else
                tile(std::false_type());
            tc5::tmem_st_wait();
            tc5::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc5::mbar_arrive(p_full + w);
        }
        if (work && ok) ok = tc5::mbar_wait_warp(o_full + w, 0, &failed);
        if (!two && w == 1 && tiles > 0 && ok) ok = tc5::mbar_wait_warp(o_full, 0, &failed);  // all products have ended
        tc5::fence_after_sync();
        // entries 2 c .. 2 c + 63 of the row: columns c.. and D/2 + c.., whose groups 2 j and 2 j + 1 alternate
        auto columns = [&](int c, uint32_t (&x)[32], uint32_t (&y)[32]) {
            if (work) {
                tc5::tmem_ld32(to + c, x);
                tc5::tmem_ld32(to + D / 2 + c, y);
                tc5::tmem_ld_wait();
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) x[j] = y[j] = 0u;
            }
        };
        float mine = 1.0f, others = 0.0f;
        if (!two) {  // the second half's sums, by way of the keys' shared memory: no product reads it any more
            float* held = reinterpret_cast<float*>(sk) + local;
            if (w == 1) {
                half_ml[local] = make_float2(m, l);
#pragma unroll
                for (int c = 0; c < D / 2; c += 32) {
                    uint32_t x[32], y[32];
                    columns(c, x, y);
#pragma unroll
                    for (int j = 0; j < 32; ++j) held[(c + j) * 128] = __uint_as_float(x[j]), held[(D / 2 + c + j) * 128] = __uint_as_float(y[j]);
                }
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            const float2 o = half_ml[local];
            const float top = fmaxf(m, o.x), at = top == -INFINITY ? 0.0f : top;
            mine = ex2(m - at), others = ex2(o.x - at);
            l = l * mine + o.y * others;
            m = top;
        }
        if (ok && (two || w == 0)) {  // all lanes: the warp reads TMEM together
            // whole: the normalised row; a part: as it is, with maximum and sum behind the rows
            float* part = splits > 1 ? A.parts + (int64_t)blockIdx.x * (256 * (D + 2)) : nullptr;
            const float f = part ? 1.0f : l > 0.0f ? 1.0f / l : 0.0f;
            uint16_t* dst = A.out + (int64_t)(first + i) * A.ldo + (int64_t)h * D;
            const float* held = reinterpret_cast<const float*>(sk) + local;
            store_row<DT, D>(
                [&](int c, uint32_t (&x)[32], uint32_t (&y)[32]) {
                    columns(c, x, y);
                    if (!two) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            x[j] = __float_as_uint(fmaf(__uint_as_float(x[j]), mine, held[(c + j) * 128] * others));
                            y[j] = __float_as_uint(fmaf(__uint_as_float(y[j]), mine, held[(D / 2 + c + j) * 128] * others));
                        }
                    }
                },
                f, real, part ? part + in_block * D : nullptr, dst, A.wide_o);
            if (part && real) {
                reinterpret_cast<float2*>(part + 256 * D)[in_block] = make_float2(m, l);
                __threadfence();
            } else if (real && A.lse) {
                A.lse[(int64_t)(first + i) * A.n_heads + h] = l > 0.0f ? (m - (kWeightBits - kPfSlack) + log2f(l)) * kLn2 : -INFINITY;
            }
        }
        tc5::fence_before_sync();
        if (splits > 1) {  // the block that adds a unit's last part joins them, in order, a thread per row
            const int first_part = blockIdx.x - z;
            asm volatile("bar.sync 1, 256;" ::: "memory");  // all rows' parts are written
            if (tid == 0) {
                __threadfence();
                is_last = atomicAdd(A.counters + kPfCounters + unit, 1) == splits - 1;
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (is_last && tid < rows) {
                __threadfence();
                const float* parts = A.parts + (int64_t)first_part * (256 * (D + 2));
                constexpr int kStep = 256 * (D + 2);
                float m = -INFINITY, l = 0.0f, by[kPfSplits];
#pragma unroll
                for (int k = 0; k < kPfSplits; ++k) {
                    by[k] = -INFINITY;
                    if (k < splits) by[k] = reinterpret_cast<const float2*>(parts + k * kStep + 256 * D)[tid].x;
                    m = fmaxf(m, by[k]);
                }
                const float at = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int k = 0; k < kPfSplits; ++k) {
                    by[k] = ex2(by[k] - at);
                    if (k < splits) l = fmaf(by[k], reinterpret_cast<const float2*>(parts + k * kStep + 256 * D)[tid].y, l);
                }
                const int row = rb * 256 + tid, i = row / g, h = head * g + row % g;
                const float f = l > 0.0f ? 1.0f / l : 0.0f;
                uint16_t* dst = A.out + (int64_t)(first + i) * A.ldo + (int64_t)h * D;
                for (int c = 0; c < D; c += 8) {
                    float o[8] = {};
#pragma unroll
                    for (int k = 0; k < kPfSplits; ++k)
                        if (k < splits) {
                            const float4* p = reinterpret_cast<const float4*>(parts + k * kStep + tid * D + c);
                            const float4 a = p[0], b = p[1];
                            o[0] = fmaf(by[k], a.x, o[0]), o[1] = fmaf(by[k], a.y, o[1]), o[2] = fmaf(by[k], a.z, o[2]), o[3] = fmaf(by[k], a.w, o[3]);
                            o[4] = fmaf(by[k], b.x, o[4]), o[5] = fmaf(by[k], b.y, o[5]), o[6] = fmaf(by[k], b.z, o[6]), o[7] = fmaf(by[k], b.w, o[7]);
                        }
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = round16x2<DT>(o[2 * k] * f, o[2 * k + 1] * f);
                    if (A.wide_o) {
                        *reinterpret_cast<uint4*>(dst + c) = make_uint4(w[0], w[1], w[2], w[3]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) dst[c + k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
                    }
                }
                if (A.lse) A.lse[(int64_t)(first + i) * A.n_heads + h] = l > 0.0f ? (m - (kWeightBits - kPfSlack) + log2f(l)) * kLn2 : -INFINITY;
            }
            if (is_last && tid == 0) A.counters[kPfCounters + unit] = 0;
        }
    }
    __syncwarp();
    __syncthreads();
    if (failed) {  // products and arrivals that were asked for have to end before the memory is given back
        if (tid == 0) {
            const long long start = clock64();
            while (clock64() - start < (1ll << 21)) __nanosleep(1000);
            report_gave_up(A);
        }
        __syncthreads();
    }
    if (warp == 12) tc5::tmem_free<1>(tmem, 512);
}

template <int DT, int D, int PAGES>
static cmpq_status launch_prefill_of(const AttnArgs& a, cudaStream_t st) {
    static bool raised[64];
    if (!raise_smem_limit_once(attention_prefill_kernel<DT, D, PAGES>, Prefill<D>::kSmem, raised)) return CMPQ_ERR_CUDA;
    const int64_t row_blocks = ((int64_t)a.max_new * a.group + 255) / 256, per = a.b.n_seq * a.c.n_kv_heads, units = row_blocks * per, sms = sm_count();
    // Fewer units than SMs: each is split over the keys, three tiles of them to a block at least.  Splitting the last round
    // of many does not pay: 2 x 2048 queries, 32 heads (512 units, 3.5 rounds) took 334 us so, and 314 whole, since the
    // blocks of the earlier rounds do not end together.
    const int splits = units < sms ? (int)std::max<int64_t>(1, std::min({sms / units, (int64_t)kPfSplits, ((int64_t)a.max_len + kPfKeys - 1) / kPfKeys / 3})) : 1;
    const int64_t blocks = units * splits;
    if (blocks > INT32_MAX) return CMPQ_ERR_UNSUPPORTED;
    const PrefillPlan plan{(int)row_blocks, (int)per, splits};
    return launch_cluster(attention_prefill_kernel<DT, D, PAGES>, (unsigned)blocks, kPfThreads, Prefill<D>::kSmem, 1, false, st, a, plan);
}

size_t prefill_parts_bytes(int d) { return d > 128 ? 0 : (size_t)std::max(1, sm_count()) * 256 * (d + 2) * sizeof(float); }

cmpq_status launch_prefill(const AttnArgs& a, cmpq_dtype dt, cudaStream_t st) {
    const bool bf = dt == CMPQ_BF16, small = a.c.page_tokens < 64;
    if (a.c.head_dim == 64) {
        if (small) return bf ? launch_prefill_of<CMPQ_BF16, 64, 4>(a, st) : launch_prefill_of<CMPQ_F16, 64, 4>(a, st);
        return bf ? launch_prefill_of<CMPQ_BF16, 64, 1>(a, st) : launch_prefill_of<CMPQ_F16, 64, 1>(a, st);
    }
    if (small) return bf ? launch_prefill_of<CMPQ_BF16, 128, 4>(a, st) : launch_prefill_of<CMPQ_F16, 128, 4>(a, st);
    return bf ? launch_prefill_of<CMPQ_BF16, 128, 1>(a, st) : launch_prefill_of<CMPQ_F16, 128, 1>(a, st);
}

}  // namespace cmpq
