// Gated feed-forward block in 8 bits.
#include <algorithm>

#include "few_i8.cuh"

namespace cmpq {

// The work space: h; the codes of the tokens, later of h; their scales.  For few tokens h, the down projection's sums and how
// many parts of each tile's are there.
struct GatedSpace {
    int32_t* sums;
    uint16_t* h;
    int8_t* codes;
    float *x_scale, *h_scale;
    int64_t ldh, ldc_in, ldc_ff;
    size_t bytes;

    GatedSpace(void* ws, int64_t n, int64_t d_in, int64_t d_ff, int64_t d_out) {
        Workspace w(ws, SIZE_MAX);
        ldh = (int64_t)round_up(d_ff, 8), ldc_in = (int64_t)round_up(d_in, 16), ldc_ff = (int64_t)round_up(d_ff, 16);
        h = w.take<uint16_t>((size_t)n * ldh);
        codes = w.take<int8_t>((size_t)n * (ldc_in > ldc_ff ? ldc_in : ldc_ff));
        x_scale = w.take<float>(n);
        h_scale = w.take<float>(n);
        sums = n <= kFewTokens ? w.take<int32_t>((size_t)n * (d_out + 128) + d_out / 8 + 8) : nullptr;
        bytes = w.used;
    }
};

// ---- few tokens: the whole block in one kernel ----------------------------------------------------------------
//
// While tokens are few the weights are the time, and between two kernels their stream stops: four launches take 35 us for a
// token through 4096 -> 11008 -> 4096 whose weights come in 20.6.  Here one block to an SM walks through all of it (a
// cooperative launch: its blocks wait for one another, once):
//   every block quantizes all tokens into its shared memory
//   tiles of channels of both projections; h and its rows' maxima go to memory            state 0: blocks done
//   units of the down projection, some channels by a part of the sum: a block quantizes the part of h that it needs; 32-bit
//   integers are added in memory, where their order does not matter, and whoever adds a tile's last part finishes it
// Channels are the accumulator's rows, tokens its columns: an instruction reads 128 rows of its first operand whatever they
// hold (40 cycles for up to 32 columns), so it should hold the weights, which are what there is much of.
//
// The weights depend on nothing.  The warp that brings them runs ahead through all of this as far as shared memory reaches, 4.4
// us of the memory's time, so that the memory goes on while the blocks quantize.  Each product has stages of its own size over
// the same bytes.
//
// What blocks hand to one another goes through L2: stores, a fence, an atomic on the counter; an acquiring load of it, then
// loads past L1.
//
// Measured in graphs, weights from memory: one token 4096 -> 11008 -> 4096 29.9 us (4.5 TB/s), 4 tokens 30.9, one token 8192 ->
// 28672 -> 8192 121 (5.8 TB/s).  A block's time for the first: its tokens quantized at 3.4 us, the products of both projections
// over at 16.4, h seen by all at 19.2, its part of h quantized at 20.6, the last products at 25.3, sums joined at 26.5.  Between
// 16 and 20 the memory fills shared memory and rests a little; asking for more into L2 meanwhile gained nothing, since from
// there to the SMs no more than 1.4 times the memory's rate was had.

constexpr int kRowMax = 2, kMark = CMPQ_GATED_STATE_BYTES / 4 - 1;  // in the state: rows' maxima, the mark of a kernel that gave up

struct FewArgs {
    TokenRows x;
    ProductArgs up, down;  // bn: channels of a tile; stages, per_stage; of up: y is h
    int d_in, d_ff;
    int ring;                             // bytes that the stages share
    int parts, part_blocks, block_units;  // of the down projection: of its sum, of units to a block
    int32_t* sums;                        // [n][ld_sums], then a count for every tile
    int64_t ld_sums;
    int32_t *state, *word;  // word: the caller's, or null
};

// Waits until *count has reached `target`; gives up after about a second, or when another wait of this call has.
__device__ __forceinline__ bool wait_count(const int32_t* count, int target, volatile int* failed, const int32_t* mark) {
    const long long start = clock64();
    for (;;) {
        int32_t v;
        asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(count) : "memory");
        if (v >= target) return true;
        if (*failed) return false;
        if (clock64() - start > (1ll << 31) || *reinterpret_cast<const volatile int32_t*>(mark)) {
            *failed = 1;
            return false;
        }
    }
}
// The count before this block's addition, for thread 0 of them; what all of them wrote before is seen by whoever sees it.
__device__ __forceinline__ int add_count(int32_t* count, int t) {
    meet();
    if (t != 0) return 0;
    __threadfence();
    return atomicAdd(count, 1);
}

template <int DT, bool NORM>
__global__ void __launch_bounds__(kFewThreads, 1)
gated_few_kernel(const __grid_constant__ CUtensorMap gate_map, const __grid_constant__ CUtensorMap up_map, const __grid_constant__ CUtensorMap down_map,
                 const __grid_constant__ FewArgs A) {
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024u - (tc5::smem_addr(raw) & 1023u)) & 1023u);
    uint8_t* tokens = smem + A.ring;  // codes of the tokens, later of a part of h
    __shared__ uint64_t full[2][kFewMaxStages], empty[2][kFewMaxStages], acc_full[2], acc_empty[2], tokens_there;  // [1]: of the down projection
    __shared__ TokenParts parts;
    __shared__ float scale[kFewTokens], inverse[kFewTokens];  // of the tokens, later of the rows of h
    __shared__ uint32_t tmem_at;
    __shared__ int failed, go;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = A.up.n, t = (int)threadIdx.x - 64;  // t: of the computing threads
    const int tile_bytes = A.up.bn * 128, unit_bytes = A.down.bn * 128;  // of a block of the sum
    if (threadIdx.x < 2 * kFewMaxStages) tc5::mbar_init(&full[0][0] + threadIdx.x, 1), tc5::mbar_init(&empty[0][0] + threadIdx.x, 1);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) tc5::mbar_init(acc_full + i, 1), tc5::mbar_init(acc_empty + i, 8);
        tc5::mbar_init(&tokens_there, 8);
        failed = 0;
        if (blockIdx.x == 0 && A.state[kMark] && A.word) atomicOr(A.word, kWordInternal);
    }
    tc5::mbar_init_fence();
    if (warp == 1) tc5::tmem_alloc<1>(&tmem_at, 64);
    tc5::fence_before_sync();
    __syncthreads();
    tc5::fence_after_sync();
    const uint32_t tmem = tmem_at;
    const int units = A.down.n_tiles * A.parts, first_unit = blockIdx.x * A.block_units, end_unit = min(first_unit + A.block_units, units);
    // Stages of either product lie over the same bytes.  Stage j of the up projection was filled fills(j) times; the down
    // projection begins with the stage behind the last one that the up projection filled, where bytes are free first.
    const int up_bytes = A.up.per_stage * 2 * tile_bytes, down_bytes = A.down.per_stage * unit_bytes;
    const int up_fills = (blockIdx.x < A.up.n_tiles ? (A.up.n_tiles - 1 - blockIdx.x) / gridDim.x + 1 : 0) * ((A.up.kblocks + A.up.per_stage - 1) / A.up.per_stage);
    const int down_first = (up_fills % A.up.stages * up_bytes + down_bytes - 1) / down_bytes % A.down.stages;
    if (warp == 0) {
        if (tc5::elect_one()) {
            int slot = 0, phase = 1;  // a new barrier counts as empty
            bool ok = true;
            for (int tile = blockIdx.x; ok && tile < A.up.n_tiles; tile += gridDim.x)
                for (int k = 0; k < A.up.kblocks; k += A.up.per_stage) {
                    if (!(ok = tc5::mbar_wait(empty[0] + slot, phase, &failed))) break;
                    const int count = min(A.up.per_stage, A.up.kblocks - k);
                    uint8_t* at = smem + slot * up_bytes;
                    tc5::mbar_expect_tx(full[0] + slot, count * 2 * tile_bytes);
                    for (int i = k; i < k + count; ++i, at += 2 * tile_bytes) {
                        tc5::tma_load_2d(at, &gate_map, full[0] + slot, i * 128, tile * A.up.bn);
                        tc5::tma_load_2d(at + tile_bytes, &up_map, full[0] + slot, i * 128, tile * A.up.bn);
                    }
                    if (++slot == A.up.stages) slot = 0, phase ^= 1;
                }
            slot = down_first, phase = 1;
            bool fresh = true;  // not filled by this product yet
            for (int unit = first_unit; ok && unit < end_unit; ++unit) {
                const int row = unit % A.down.n_tiles * A.down.bn, begin = unit / A.down.n_tiles * A.part_blocks, end = min(begin + A.part_blocks, A.down.kblocks);
                for (int k = begin; ok && k < end; k += A.down.per_stage) {
                    if (fresh) {
                        for (int j = slot * down_bytes / up_bytes; ok && j <= min(((slot + 1) * down_bytes - 1) / up_bytes, A.up.stages - 1); ++j) {
                            const int fills = up_fills > j ? (up_fills - j + A.up.stages - 1) / A.up.stages : 0;
                            if (fills) ok = tc5::mbar_wait(empty[0] + j, (fills - 1) & 1, &failed);
                        }
                    } else {
                        ok = tc5::mbar_wait(empty[1] + slot, phase, &failed);
                    }
                    if (!ok) break;
                    const int count = min(A.down.per_stage, end - k);
                    uint8_t* at = smem + slot * down_bytes;
                    tc5::mbar_expect_tx(full[1] + slot, count * unit_bytes);
                    for (int i = k; i < k + count; ++i, at += unit_bytes) tc5::tma_load_2d(at, &down_map, full[1] + slot, i * 128, row);
                    if (++slot == A.down.stages) slot = 0;
                    if (slot == down_first) fresh = false, phase ^= 1;
                }
            }
        }
    } else if (warp == 1) {
        if (tc5::elect_one()) {
            const uint32_t idesc = tc5::idesc_i8(128, kFewColumns);
            const uint64_t x0 = tc5::desc_k_sw128(tc5::smem_addr(tokens));
            constexpr uint64_t kRowStep = kFewRows * 8;  // descriptors count 16 bytes
            int slot = 0, phase = 0, acc = 0, acc_phase = 1, there = 1;
            bool ok = tc5::mbar_wait(&tokens_there, 0, &failed);  // also where a block has no tile for them
            auto accumulator = [&] {
                ok = tc5::mbar_wait(acc_empty + acc, acc_phase, &failed);
                tc5::fence_after_sync();
                return tmem + acc * 2 * kFewColumns;
            };
            auto done = [&] {
                tc5::mma_commit(acc_full + acc);
                acc ^= 1;
                if (acc == 0) acc_phase ^= 1;
            };
            for (int tile = blockIdx.x; ok && tile < A.up.n_tiles; tile += gridDim.x) {
                const uint32_t into = accumulator();
                uint64_t x = x0;
                for (int k = 0; ok && k < A.up.kblocks; k += A.up.per_stage) {
                    if (!(ok = tc5::mbar_wait(full[0] + slot, phase, &failed))) break;
                    tc5::fence_after_sync();
                    uint64_t w = tc5::desc_k_sw128(tc5::smem_addr(smem + slot * up_bytes));
                    for (int i = k; i < min(k + A.up.per_stage, A.up.kblocks); ++i, x += kRowStep, w += 2 * tile_bytes / 16)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            tc5::mma_i8<1>(into, w + 2 * j, x + 2 * j, idesc, (i | j) != 0);
                            tc5::mma_i8<1>(into + kFewColumns, w + tile_bytes / 16 + 2 * j, x + 2 * j, idesc, (i | j) != 0);
                        }
                    tc5::mma_commit(empty[0] + slot);
                    if (++slot == A.up.stages) slot = 0, phase ^= 1;
                }
                done();
            }
            slot = down_first, phase = 0;
            for (int unit = first_unit, held = -1; ok && unit < end_unit; ++unit) {
                const int part = unit / A.down.n_tiles, blocks = min(A.part_blocks, A.down.kblocks - part * A.part_blocks);
                const uint32_t into = accumulator();
                if (ok && part != held) ok = tc5::mbar_wait(&tokens_there, there, &failed), there ^= 1, held = part;
                uint64_t x = x0;
                for (int k = 0; ok && k < blocks; k += A.down.per_stage) {
                    if (!(ok = tc5::mbar_wait(full[1] + slot, phase, &failed))) break;
                    tc5::fence_after_sync();
                    uint64_t w = tc5::desc_k_sw128(tc5::smem_addr(smem + slot * down_bytes));
                    for (int i = k; i < min(k + A.down.per_stage, blocks); ++i, x += kRowStep, w += unit_bytes / 16)
#pragma unroll
                        for (int j = 0; j < 4; ++j) tc5::mma_i8<1>(into, w + 2 * j, x + 2 * j, idesc, (i | j) != 0);
                    tc5::mma_commit(empty[1] + slot);
                    if (++slot == A.down.stages) slot = 0;
                    if (slot == down_first) phase ^= 1;
                }
                done();
            }
        }
    } else {
        const int quad = warp & 3;
        const bool reads = warp < 6;  // the accumulators, whose 128 rows are four warps' and which have kFewTokens columns that count
        const uint32_t lanes = tmem + ((uint32_t)quad << 21);
        // the operand that this warp wrote is seen by the products
        auto tokens_written = [&] {
            tc5::fence_async_smem();
            __syncwarp();
            if (lane == 0) tc5::mbar_arrive(&tokens_there);
        };
        quantize_tokens<DT, NORM>(A.x, [&](int r, int k) { return code_at(tokens, r, k); }, scale, parts, t);
        tokens_written();
        int32_t* tile_parts = A.sums + n * A.ld_sums;
        for (int64_t i = (int64_t)blockIdx.x * 256 + t; i < (n * A.ld_sums + A.down.n_tiles + 3) / 4; i += (int64_t)gridDim.x * 256)
            reinterpret_cast<int4*>(A.sums)[i] = make_int4(0, 0, 0, 0);
        int acc = 0, parity = 0;
        bool ok = true;
        auto accumulator = [&] {
            ok = ok && tc5::mbar_wait_warp(acc_full + acc, parity, &failed);
            tc5::fence_after_sync();
            return ok;
        };
        auto give_back = [&] {
            tc5::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc5::mbar_arrive(acc_empty + acc);
            acc ^= 1;
            if (acc == 0) parity ^= 1;
        };
        uint32_t* row_max = reinterpret_cast<uint32_t*>(A.state) + kRowMax;
        meet();  // the scales are there
        for (int tile = blockIdx.x; tile < A.up.n_tiles; tile += gridDim.x) {
            const int c = quad * 32 + lane, o = tile * A.up.bn + c;
            const bool real = c < A.up.bn && o < A.d_ff;
            const float2 gs = column_scale<DT, kPlain>(A.up, o, 0, 1);
            const float us = __ldg(A.up.us + min(o, A.d_ff - 1)), ub = A.up.ubias ? widen16<DT>(A.up.ubias[min(o, A.d_ff - 1)]) : 0.0f;
            if (accumulator() && reads && quad * 32 < A.up.bn)
                with_act(A.up.act, [&](auto act) {
                    uint32_t g[kFewTokens], u[kFewTokens], most = 0;
                    tc5::tmem_ld4(lanes + acc * 2 * kFewColumns, g);
                    tc5::tmem_ld4(lanes + acc * 2 * kFewColumns + kFewColumns, u);
                    tc5::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < kFewTokens; ++j) {
                        const float xs = scale[min(j, n - 1)];
                        float a = (float)(int)g[j] * xs * gs.x, b = (float)(int)u[j] * xs * us;
                        if (A.up.bias) a += gs.y;
                        if (A.up.ubias) b += ub;
                        g[j] = round16x2<DT>(activate<decltype(act)::value>(a) * b, 0.0f);
                        if (real && j < n) A.up.y[j * A.up.ldy + o] = (uint16_t)g[j];
                    }
#pragma unroll
                    for (int j = 0; j < kFewTokens; ++j) {
                        const uint32_t m = __reduce_max_sync(0xffffffffu, real ? g[j] & 0x7fffu : 0u);  // bit patterns: NaN above infinity
                        if (lane == j) most = m;
                    }
                    if (lane < n && most) atomicMax(row_max + lane, most);
                });
            give_back();
        }
        add_count(A.state, t);
        if (t == 0) go = wait_count(A.state, gridDim.x, &failed, A.state + kMark);
        meet();
        const bool on = go != 0;  // one answer for all threads
        const ProductArgs& D = A.down;
        for (int unit = first_unit, held = -1; on && unit < end_unit; ++unit) {
            const int tile = unit % D.n_tiles, part = unit / D.n_tiles, c = quad * 32 + lane;
            const int at = tile * D.bn + lane * 4, left = lane * 4 < D.bn ? D.d_out - at : 0;  // this thread's channels, should it finish the tile
            float ws[4], bias[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int channel = min(at + j, D.d_out - 1);
                ws[j] = __ldg(D.ws + channel), bias[j] = D.bias ? widen16<DT>(D.bias[channel]) : 0.0f;
            }
            if (D.residual && warp - 2 < n && left > 0) ask_for(D.residual + (warp - 2) * D.ldr + at, 0, min(4, left));
            if (part != held) {  // what was held has been used: its accumulator has been waited for
                const int begin = part * A.part_blocks * 128, groups = (min(begin + A.part_blocks * 128, A.d_ff) - begin + 7) / 8;
                uint4 h[kFewTokens];
                auto ask = [&](int g) {
#pragma unroll
                    for (int r = 0; r < kFewTokens; ++r)
                        if (r < n && g < groups) h[r] = __ldcg(reinterpret_cast<const uint4*>(A.up.y + r * A.up.ldy + begin + 8 * g));
                };
                ask(t);  // while the scales are on their way
                if (held < 0) {
                    if (t < n) {
                        const uint32_t most = __ldcg(row_max + t);
                        const float2 s = scale_of(widen16<DT>((uint16_t)most));
                        scale[t] = s.x, inverse[t] = s.y;
                        if (blockIdx.x == 0 && A.word && most >= (DT == CMPQ_BF16 ? 0x7f80u : 0x7c00u)) atomicOr(A.word, kWordNonfinite);
                    }
                    meet();
                }
                held = part;
                for (int g = t; g < groups; ) {
#pragma unroll
                    for (int r = 0; r < kFewTokens; ++r) {
                        if (r >= n) break;
                        float v[8];
                        widen8<DT>(h[r], v);
                        *reinterpret_cast<uint2*>(code_at(tokens, r, 8 * g)) = round_codes(v, inverse[r]);
                    }
                    ask(g += 256);
                }
                tokens_written();
            }
            if (accumulator() && reads) {
                uint32_t r[kFewTokens];
                tc5::tmem_ld4(lanes + acc * 2 * kFewColumns, r);
                tc5::tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < kFewTokens; ++j)
                    if (j < n && c < D.bn) atomicAdd(A.sums + j * A.ld_sums + tile * D.bn + c, (int)r[j]);
            }
            give_back();
            const int before = add_count(tile_parts + tile, t);
            if (t == 0) go = before == A.parts - 1;
            meet();
            if (!go || !ok) continue;
            __threadfence();
            const int row = warp - 2;
            if (row < n && left > 0) {
                const int4 sum = __ldcg(reinterpret_cast<const int4*>(A.sums + row * A.ld_sums + at));
                const uint16_t* res = D.residual + row * D.ldr + at;
                uint16_t* y = D.y + row * D.ldy + at;
                float f[4] = {(float)sum.x, (float)sum.y, (float)sum.z, (float)sum.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    f[j] = f[j] * scale[row] * ws[j];
                    if (D.bias) f[j] += bias[j];
                    if (D.residual && j < left) f[j] += widen16<DT>(res[j]);
                }
                const uint32_t lo = round16x2<DT>(f[0], f[1]), hi = round16x2<DT>(f[2], f[3]);
                if (D.wide && left >= 4) {
                    *reinterpret_cast<uint2*>(y) = make_uint2(lo, hi);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < left) y[j] = (uint16_t)((j < 2 ? lo : hi) >> (16 * (j & 1)));
                }
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (failed) {  // the loads that were asked for have to land before the shared memory is given back
        if (threadIdx.x == 0) {
            const long long start = clock64();
            while (clock64() - start < (1ll << 21)) __nanosleep(1000);
            atomicOr(A.state + kMark, kWordInternal);
            if (A.word) atomicOr(A.word, kWordInternal);
        }
        __syncthreads();
    } else if (warp == 0) {
        int last = 0;
        if (lane == 0) last = atomicAdd(A.state + 1, 1) == (int)gridDim.x - 1;
        if (__shfl_sync(0xffffffffu, last, 0) && lane < kRowMax + kFewTokens) A.state[lane] = 0;  // the last block: nobody waits or reads any more
    }
    if (warp == 1) tc5::tmem_free<1>(tmem, 64);
}

// Tiles, parts and stages; false where separate kernels are as fast, or the tokens' codes would take too much of the shared
// memory.  In graphs, 1 token 4096 -> 11008 -> 4096 takes 29.7 us here and 32.4 in four kernels, 2048 -> 5632 -> 2048 16.5 and
// 18.5, 1024 -> 2816 -> 1024 14.2 and 13.9.  Where the kernel that quantizes its own tokens does for both products, two of it
// are faster (4096 -> 4096 -> 4096 20.2 here, 17.4 in two; 4 tokens 21.6 and 19.7).
static bool plan_few(FewArgs& a) {
    ProductArgs &u = a.up, &d = a.down;
    const int sms = sm_count();
    if ((few_fits(a.d_in) && few_fits(a.d_ff)) || (2 * (int64_t)a.d_in + d.d_out) * a.d_ff < (16 << 20)) return false;
    u.kblocks = (int)ceil_div(a.d_in, 128), d.kblocks = (int)ceil_div(a.d_ff, 128);
    if (u.kblocks > kFewBlocks) return false;
    plan_tiles(u);
    // channels and part of the sum of a unit, so that the block with the most of them is soonest done, in cycles: 23 bytes come
    // in one, a block of the sum takes 150 and a unit 1500 besides
    int64_t least = INT64_MAX;
    for (int bn = 128; bn >= 8; bn -= 8)
        for (int full = 1; full <= 2; ++full) {  // units that fill the blocks once or twice
            const int64_t tiles = ceil_div(d.d_out, bn), parts = std::min({std::max(full * sms / tiles, ceil_div(d.kblocks, kFewBlocks)), (int64_t)d.kblocks, (int64_t)32});
            const int64_t blocks = ceil_div(d.kblocks, parts), each = ceil_div(tiles * ceil_div(d.kblocks, blocks), sms);
            const int64_t cost = each * (blocks * (bn * 128 / 23 + 150) + 1500);
            if (blocks <= kFewBlocks && cost < least) {
                least = cost, d.bn = bn, d.n_tiles = (int)tiles;
                a.part_blocks = (int)blocks, a.parts = (int)ceil_div(d.kblocks, blocks), a.block_units = (int)each;
            }
        }
    if (least == INT64_MAX) return false;
    a.ld_sums = (int64_t)d.n_tiles * d.bn;
    d.wide = aligned_to(d.y, 8) && d.ldy % 4 == 0;
    a.ring = few_ring(kFewRows * 128 * std::max(u.kblocks, a.part_blocks));
    plan_stages(u, 2 * u.bn * 128, a.ring);
    plan_stages(d, d.bn * 128, a.ring);
    return true;
}

template <int DT>
static cmpq_status launch_few(const FewArgs& a, const Weight8& gate, const Weight8& up, const Weight8& down, cudaStream_t st) {
    CUtensorMap gate_map, up_map, down_map;
    if (!make_byte_map(&gate_map, gate.codes, a.d_ff, a.d_in, gate.ld, a.up.bn) || !make_byte_map(&up_map, up.codes, a.d_ff, a.d_in, up.ld, a.up.bn) ||
        !make_byte_map(&down_map, down.codes, a.down.d_out, a.d_ff, down.ld, a.down.bn))
        return CMPQ_ERR_CUDA;
    const auto launch = [&](auto kernel, bool (&raised)[64]) {
        if (!raise_smem_limit_once(kernel, kFewSmem, raised)) return CMPQ_ERR_CUDA;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)std::min<int64_t>(std::max<int64_t>(a.up.n_tiles, ceil_div((int64_t)a.down.n_tiles * a.parts, a.block_units)), sm_count()));
        cfg.blockDim = dim3(kFewThreads);
        cfg.dynamicSmemBytes = kFewSmem;  // one block to an SM
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeCooperative;
        attr.val.cooperative = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, kernel, gate_map, up_map, down_map, a) == cudaSuccess ? launch_status() : CMPQ_ERR_CUDA;
    };
    static bool raised[2][64];
    return a.x.norm.weight ? launch(gated_few_kernel<DT, true>, raised[0]) : launch(gated_few_kernel<DT, false>, raised[1]);
}

}  // namespace cmpq

using namespace cmpq;

static bool gated_sizes_ok(int64_t n, int64_t d_in, int64_t d_ff, int64_t d_out) {
    return linear_sizes_ok(n, d_in, d_ff) && linear_sizes_ok(n, d_ff, d_out);
}

extern "C" size_t cmpq_gated_i8_ws_bytes(int64_t n, int64_t d_in, int64_t d_ff, int64_t d_out) {
    return gated_sizes_ok(n, d_in, d_ff, d_out) ? GatedSpace(nullptr, n, d_in, d_ff, d_out).bytes : 0;
}

extern "C" cmpq_status cmpq_gated_i8(const void* X, cmpq_dtype dt, int64_t n, int64_t d_in, int64_t ldx, const void* norm, float eps,
                                     const cmpq_weight_i8* gate, const cmpq_weight_i8* up, const cmpq_weight_i8* down, int64_t d_ff, int64_t d_out,
                                     cmpq_act act, const void* residual, int64_t ldr, void* y, int64_t ldy, int32_t* word, void* state, void* ws,
                                     size_t ws_bytes, void* stream) {
    if (!gate || !up || !down || !gated_sizes_ok(n, d_in, d_ff, d_out) || ldx < d_in || ldy < d_out) return CMPQ_ERR_INVALID_ARG;
    if (!weight_rows_ok(*gate, d_in) || !weight_rows_ok(*up, d_in) || !weight_rows_ok(*down, d_ff)) return CMPQ_ERR_INVALID_ARG;
    if ((dt != CMPQ_F16 && dt != CMPQ_BF16) || !norm_ok(norm, eps) || !finish_ok(act, residual, ldr, d_out)) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!X || !y || !weight_ok(*gate) || !weight_ok(*up) || !weight_ok(*down) || !aligned_to(X, 2) || !aligned_to(y, 2)) return CMPQ_ERR_INVALID_ARG;
    if (!state || !aligned_to(state, 16)) return CMPQ_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < cmpq_gated_i8_ws_bytes(n, d_in, d_ff, d_out)) return CMPQ_ERR_WORKSPACE;
    const GatedSpace g(ws, n, d_in, d_ff, d_out);
    const auto st = static_cast<cudaStream_t>(stream);
    auto* kept = static_cast<int32_t*>(state);
    if (sm_count() <= 0) return CMPQ_ERR_CUDA;  // no device to plan for
    if (n <= kFewTokens) {
        FewArgs a = {};
        a.x = {static_cast<const uint16_t*>(X), ldx, aligned_to(X, 16) && ldx % 8 == 0, {static_cast<const uint16_t*>(norm), aligned_to(norm, 16), eps},
               d_in, (int)n, word};
        a.sums = g.sums;
        a.up.ws = gate->scale, a.up.us = up->scale;
        a.up.bias = static_cast<const uint16_t*>(gate->bias), a.up.ubias = static_cast<const uint16_t*>(up->bias);
        a.up.y = g.h, a.up.ldy = g.ldh, a.up.act = act, a.up.d_out = (int)d_ff;
        a.down.ws = down->scale, a.down.bias = static_cast<const uint16_t*>(down->bias);
        a.down.y = static_cast<uint16_t*>(y), a.down.ldy = ldy, a.down.d_out = (int)d_out;
        a.down.residual = static_cast<const uint16_t*>(residual), a.down.ldr = ldr;
        a.up.n = a.down.n = (int)n, a.d_in = (int)d_in, a.d_ff = (int)d_ff;
        a.state = kept, a.word = word;
        if (plan_few(a)) return dt == CMPQ_BF16 ? launch_few<CMPQ_BF16>(a, *gate, *up, *down, st) : launch_few<CMPQ_F16>(a, *gate, *up, *down, st);
    }
    int32_t* gave_up = word ? word : kept + kMark;
    if (n <= kFewTokens && few_fits(d_in) && few_fits(d_ff)) {
        const cmpq_status s = enqueue_few(X, dt, n, d_in, ldx, norm, eps, *gate, d_ff, up, {act, nullptr, 0}, g.h, g.ldh, word, gave_up, false, st);
        return s != CMPQ_OK ? s
                            : enqueue_few(g.h, dt, n, d_ff, g.ldh, nullptr, 0.0f, *down, d_out, nullptr, {CMPQ_ACT_NONE, residual, ldr}, y, ldy, word, gave_up,
                                          true, st);
    }
    cmpq_status s = enqueue_quantize(X, dt, n, d_in, ldx, norm, eps, g.codes, g.ldc_in, g.x_scale, word, nullptr, st);
    if (s != CMPQ_OK) return s;
    s = enqueue_product({g.codes, g.ldc_in, g.x_scale}, dt, n, d_in, *gate, d_ff, up, {act, nullptr, 0}, g.h, g.ldh, gave_up, true, st);
    if (s != CMPQ_OK) return s;
    s = enqueue_quantize(g.h, dt, n, d_ff, g.ldh, nullptr, 0.0f, g.codes, g.ldc_ff, g.h_scale, word, nullptr, st);
    if (s != CMPQ_OK) return s;
    return enqueue_product({g.codes, g.ldc_ff, g.h_scale}, dt, n, d_ff, *down, d_out, nullptr, {CMPQ_ACT_NONE, residual, ldr}, y, ldy, gave_up, true, st);
}
