// Products of up to four tokens with 8-bit weights, from 16-bit tokens: one launch.
#include "few_i8.cuh"

namespace cmpq {

struct FewProduct {
    TokenRows x;
    ProductArgs p;      // bn: channels of a tile; kblocks: of a slice; stages, per_stage
    int slices, rows;   // of the sum; of the tokens' operand
    int ring, reduce;   // where the tokens' codes and the slices' sums begin in shared memory
};

// A block takes tiles of up to 128 channels (of both projections where KIND is kGated), the accumulator's rows; the tokens are
// its columns: an instruction reads 128 rows of its first operand whatever they hold (40 cycles for up to 32 columns), so it
// should hold the weights.  Where the channels are spread over all SMs and a tile has 64 or 32 of them, its sum is cut into two
// or four slices, every second or fourth block of it, each with rows and columns of its own: an instruction then takes as many blocks of the sum, what a slice's
// rows make of another one's columns is left, and the slices are added up at the end (a token 4096 -> 4096 takes 32
// instructions instead of 128, 2 us less).  Launched behind a kernel that writes its tokens, a block asks for its first
// weights before that has ended.
// Measured in graphs, weights from memory, against the quantization and the tile kernel, one token: 4096 -> 4096 6.6 us and 9.2,
// 4096 -> 11008 11.0 and 12.2, 512 -> 512 4.4 and 4.4; in eager calls, where a launch more counts, 8.2 and 10.4, 12.3 and 14.4,
// 6.2 and 9.1.  Of the 6.6 the weights' way takes 2.6; launch, the tokens' loads and sums and the products take turns.
template <int DT, bool NORM, int KIND>
__global__ void __launch_bounds__(kFewThreads, 1)
few_product_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap umap, const __grid_constant__ FewProduct A) {
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024u - (tc5::smem_addr(raw) & 1023u)) & 1023u);
    uint8_t* tokens = smem + A.ring;
    int32_t* reduce = reinterpret_cast<int32_t*>(smem + A.reduce);
    __shared__ uint64_t full[kFewMaxStages], empty[kFewMaxStages], acc_full[2], acc_empty[2], tokens_there;
    __shared__ TokenParts parts;
    __shared__ float scale[kFewTokens];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    const ProductArgs& P = A.p;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = A.x.n, t = (int)threadIdx.x - 64;  // t: of the computing threads
    const int S = A.slices, high = 128 / S, box_bytes = P.bn * 128, slice_bytes = S == 1 ? box_bytes : high * 128;
    const int half_bytes = S * slice_bytes, block_bytes = KIND == kGated ? 2 * half_bytes : half_bytes;  // of a projection, of a block of all slices
    const int all = (P.n_tiles - 1 - blockIdx.x) / gridDim.x + 1;  // tiles
    if (threadIdx.x < P.stages) tc5::mbar_init(full + threadIdx.x, 1), tc5::mbar_init(empty + threadIdx.x, 1);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) tc5::mbar_init(acc_full + i, 1), tc5::mbar_init(acc_empty + i, 4);
        tc5::mbar_init(&tokens_there, 8);
        failed = 0;
    }
    tc5::mbar_init_fence();
    if (warp == 1) tc5::tmem_alloc<1>(&tmem_at, 64);
    tc5::dependents_may_start();
    tc5::fence_before_sync();
    __syncthreads();
    tc5::fence_after_sync();
    const uint32_t tmem = tmem_at;
    if (warp == 0) {
        if (tc5::elect_one()) {
            int slot = 0, phase = 1;  // a new barrier counts as empty
            bool ok = true;
            for (int i = 0, tile = blockIdx.x; ok && i < all; ++i, tile += gridDim.x)
                for (int k = 0; k < P.kblocks; k += P.per_stage) {
                    if (!(ok = tc5::mbar_wait(empty + slot, phase, &failed))) break;
                    const int count = min(P.per_stage, P.kblocks - k);
                    uint8_t* at = smem + slot * P.per_stage * block_bytes;
                    tc5::mbar_expect_tx(full + slot, count * S * (KIND == kGated ? 2 : 1) * box_bytes);
                    for (int b = k; b < k + count; ++b, at += block_bytes)
                        for (int q = 0; q < S; ++q) {
                            tc5::tma_load_2d(at + q * slice_bytes, &wmap, full + slot, (b * S + q) * 128, tile * P.bn);
                            if (KIND == kGated) tc5::tma_load_2d(at + half_bytes + q * slice_bytes, &umap, full + slot, (b * S + q) * 128, tile * P.bn);
                        }
                    if (++slot == P.stages) slot = 0, phase ^= 1;
                }
        }
    } else if (warp == 1) {
        if (tc5::elect_one()) {
            const uint32_t idesc = tc5::idesc_i8(128, kFewColumns);
            int slot = 0, phase = 0, acc = 0, acc_phase = 1;
            bool ok = tc5::mbar_wait(&tokens_there, 0, &failed);
            for (int i = 0; ok && i < all; ++i) {
                if (!(ok = tc5::mbar_wait(acc_empty + acc, acc_phase, &failed))) break;
                tc5::fence_after_sync();
                const uint32_t into = tmem + acc * 2 * kFewColumns;
                uint64_t x = tc5::desc_k_sw128(tc5::smem_addr(tokens));
                for (int k = 0; k < P.kblocks; k += P.per_stage) {
                    if (!(ok = tc5::mbar_wait(full + slot, phase, &failed))) break;
                    tc5::fence_after_sync();
                    uint64_t w = tc5::desc_k_sw128(tc5::smem_addr(smem + slot * P.per_stage * block_bytes));  // counts 16 bytes
                    for (int b = k; b < min(k + P.per_stage, P.kblocks); ++b, x += A.rows * 8, w += block_bytes / 16)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            tc5::mma_i8<1>(into, w + 2 * j, x + 2 * j, idesc, (b | j) != 0);
                            if (KIND == kGated) tc5::mma_i8<1>(into + kFewColumns, w + half_bytes / 16 + 2 * j, x + 2 * j, idesc, (b | j) != 0);
                        }
                    tc5::mma_commit(empty + slot);
                    if (++slot == P.stages) slot = 0, phase ^= 1;
                }
                tc5::mma_commit(acc_full + acc);
                acc ^= 1;
                if (acc == 0) acc_phase ^= 1;
            }
        }
    } else {
        tc5::wait_for_previous();
        // token r's codes of slice q are row 4 q + r of the operand
        auto place = [&](int r, int k) {
            const int block = k >> 7, row = 4 * (block & (S - 1)) + r;
            return tokens + (block >> (S >> 1)) * A.rows * 128 + row * 128 + (((k >> 4 & 7) ^ (row & 7)) << 4) + (k & 15);  // S is 1, 2 or 4
        };
        quantize_tokens<DT, NORM>(A.x, place, scale, parts, t);
        tc5::fence_async_smem();
        __syncwarp();
        if (lane == 0) tc5::mbar_arrive(&tokens_there);
        meet();  // the scales are there
        // The accumulators' 128 rows are four warps'.  Row `row` holds slice q's sum of channel row - q high, tokens in columns 4 q
        // .. 4 q + 3.  A thread finishes channel c of tokens first, first + S ..
        const int row = (warp & 3) * 32 + lane, q = row / high, c = S == 1 ? row : t % high, first = S == 1 ? 0 : t / high;
        int acc = 0, parity = 0;
        bool ok = true;
        for (int i = 0, tile = blockIdx.x; warp < 6 && i < all; ++i, tile += gridDim.x) {
            const int o = tile * P.bn + c, at = min(o, P.d_out - 1);
            const bool real = c < P.bn && o < P.d_out;
            const float2 ws = column_scale<DT, kPlain>(P, at, 0, 1);
            const float us = KIND == kGated ? __ldg(P.us + at) : 0.0f, ub = KIND == kGated && P.ubias ? widen16<DT>(P.ubias[at]) : 0.0f;
            float res[kFewTokens];
#pragma unroll
            for (int j = 0; j < kFewTokens; ++j) res[j] = KIND == kFinish && P.residual && real && j < n ? widen16<DT>(P.residual[j * P.ldr + o]) : 0.0f;
            ok = ok && tc5::mbar_wait_warp(acc_full + acc, parity, &failed);
            tc5::fence_after_sync();
            uint32_t a[kFewTokens], b[kFewTokens];
            if (ok) {
                const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + acc * 2 * kFewColumns + 4 * q;
                tc5::tmem_ld4(from, a);
                if (KIND == kGated) tc5::tmem_ld4(from + kFewColumns, b);
                tc5::tmem_ld_wait();
            }
            tc5::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc5::mbar_arrive(acc_empty + acc);
            acc ^= 1;
            if (acc == 0) parity ^= 1;
            if (S > 1) {  // [projection][slice][token][channel]
                const auto four = [] { asm volatile("bar.sync 2, 128;" ::: "memory"); };
#pragma unroll
                for (int j = 0; j < kFewTokens; ++j) {
                    reduce[q * 4 * high + j * high + row % high] = (int)a[j];
                    if (KIND == kGated) reduce[512 + q * 4 * high + j * high + row % high] = (int)b[j];
                }
                four();
#pragma unroll
                for (int j = 0; j < kFewTokens; ++j) {
                    int sum = 0, other = 0;
                    for (int k = 0; k < S; ++k) {
                        sum += reduce[k * 4 * high + j * high + c];
                        if (KIND == kGated) other += reduce[512 + k * 4 * high + j * high + c];
                    }
                    a[j] = (uint32_t)sum, b[j] = (uint32_t)other;
                }
                four();  // they have been read
            }
            if (!ok) continue;
            auto store = [&](auto act) {
#pragma unroll
                for (int j = 0; j < kFewTokens; ++j) {
                    if (j >= n) break;
                    if (S > 1 && j % S != first) continue;
                    float z = (float)(int)a[j] * scale[j] * ws.x;
                    if (P.bias) z += ws.y;
                    z = activate<decltype(act)::value>(z);
                    if (KIND == kGated) {
                        float u = (float)(int)b[j] * scale[j] * us;
                        if (P.ubias) u += ub;
                        z *= u;
                    }
                    if (KIND == kFinish && P.residual) z += res[j];
                    if (real) P.y[j * P.ldy + o] = (uint16_t)round16x2<DT>(z, 0.0f);
                }
            };
            if (KIND == kPlain)
                store(ActIs<CMPQ_ACT_NONE>());
            else
                with_act(P.act, store);
        }
    }
    __syncwarp();
    __syncthreads();
    if (failed) {  // the loads that were asked for have to land before the shared memory is given back
        if (threadIdx.x == 0) {
            const long long start = clock64();
            while (clock64() - start < (1ll << 21)) __nanosleep(1000);
            atomicOr(P.failed, kWordInternal);
        }
        __syncthreads();
    }
    if (warp == 1) tc5::tmem_free<1>(tmem, 64);
}

template <int DT, int KIND>
static cmpq_status launch_few(FewProduct& a, const Weight8& w, const Weight8* u, bool behind, cudaStream_t st) {
    CUtensorMap wmap, umap;
    if (!make_byte_map(&wmap, w.codes, a.p.d_out, a.x.d, w.ld, a.p.bn)) return CMPQ_ERR_CUDA;
    umap = wmap;
    if (u && !make_byte_map(&umap, u->codes, a.p.d_out, a.x.d, u->ld, a.p.bn)) return CMPQ_ERR_CUDA;
    const unsigned grid = (unsigned)std::min(a.p.n_tiles, sm_count());
    static bool raised[2][64];
    const auto launch = [&](auto kernel, bool (&done)[64]) {
        if (!raise_smem_limit_once(kernel, kFewSmem, done)) return CMPQ_ERR_CUDA;
        return launch_cluster(kernel, grid, kFewThreads, kFewSmem, 1, behind, st, wmap, umap, a);
    };
    return a.x.norm.weight ? launch(few_product_kernel<DT, true, KIND>, raised[0]) : launch(few_product_kernel<DT, false, KIND>, raised[1]);
}

// Rows of which a thread keeps its share: longer ones are read three times by every block (4 tokens 11008 -> 4096: 15.9 us here,
// 12.8 in two kernels; 8192 -> 8192 19.7 and 18.0; one token 13.9 and 12.7, 16.6 and 18.2; one token 4096 -> 4096 6.6 and 8.3).
bool few_fits(int64_t d_in) { return d_in <= 4096; }

cmpq_status enqueue_few(const void* X, cmpq_dtype dt, int64_t n, int64_t d_in, int64_t ldx, const void* norm, float eps, const Weight8& w, int64_t d_out,
                        const Weight8* u, const Finish& f, void* y, int64_t ldy, int32_t* word, int32_t* gave_up, bool behind, cudaStream_t st) {
    if (sm_count() <= 0) return CMPQ_ERR_CUDA;  // no device to plan for
    FewProduct a = {};
    a.x = {static_cast<const uint16_t*>(X), ldx, aligned_to(X, 16) && ldx % 8 == 0, {static_cast<const uint16_t*>(norm), aligned_to(norm, 16), eps},
           d_in, (int)n, word};
    ProductArgs& p = a.p;
    p.ws = w.scale, p.bias = static_cast<const uint16_t*>(w.bias);
    if (u) p.us = u->scale, p.ubias = static_cast<const uint16_t*>(u->bias);
    p.y = static_cast<uint16_t*>(y), p.ldy = ldy;
    p.residual = static_cast<const uint16_t*>(f.residual), p.ldr = f.ldr, p.act = f.act;
    p.n = (int)n, p.d_out = (int)d_out, p.kblocks = (int)ceil_div(d_in, 128);
    p.failed = gave_up;
    plan_tiles(p);
    a.slices = p.kblocks <= 8 || p.bn > 64 ? 1 : p.bn > 32 ? 2 : 4;  // short sums are not worth the adding up
    a.rows = a.slices == 4 ? 16 : 8;
    p.kblocks = (int)ceil_div(p.kblocks, a.slices);
    const int token_bytes = p.kblocks * a.rows * 128, block = (u ? 2 : 1) * (a.slices == 1 ? p.bn * 128 : 128 * 128);
    a.ring = few_ring(token_bytes + 4096);
    a.reduce = a.ring + token_bytes + 1024;
    plan_stages(p, block, a.ring);
    auto launch = [&](auto type) {
        constexpr int DT = decltype(type)::value;
        return u ? launch_few<DT, kGated>(a, w, u, behind, st)
               : f.act == CMPQ_ACT_NONE && !f.residual ? launch_few<DT, kPlain>(a, w, u, behind, st) : launch_few<DT, kFinish>(a, w, u, behind, st);
    };
    return dt == CMPQ_BF16 ? launch(ActIs<CMPQ_BF16>()) : launch(ActIs<CMPQ_F16>());
}

}  // namespace cmpq
