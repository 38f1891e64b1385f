// 8-bit linear layers: quantization of tokens and the integer product with scales per token and channel.
#include <algorithm>

#include "cache.cuh"
#include "tc5.cuh"
#include "walk.cuh"

namespace cmpq {

constexpr int kQtThreads = 256;

// The larger magnitudes of two packed pairs, entry by entry; a NaN stays.
template <int DT>
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) {
    if (DT == CMPQ_BF16) {
        const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
        return *reinterpret_cast<const uint32_t*>(&m);
    } else {
        const __half2 m = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), __habs2(*reinterpret_cast<const __half2*>(&b)));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
}
template <int DT>
__device__ __forceinline__ uint32_t group_max(uint32_t m, uint4 g) {
    return larger2<DT>(larger2<DT>(larger2<DT>(larger2<DT>(m, g.x), g.y), g.z), g.w);
}

// Codes of eight entries.  |x * inv| is at most 127 (1 + 2^-22) here, so adding 1.5 * 2^23 leaves the integer that
// rounding to even gives in the sum's low byte, in two's complement: one addition instead of a conversion, which has a
// quarter of its rate.
template <int DT>
__device__ __forceinline__ uint2 group_codes(uint4 g, float inv) {
    const uint32_t w[4] = {g.x, g.y, g.z, g.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = widen16x2<DT>(w[i]);
        const float a = f.x * inv + 12582912.0f, b = f.y * inv + 12582912.0f;  // two roundings each: -fmad=false
        c[i] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040);
    }
    return make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
}

// One block per token.  Magnitudes are compared two at a time in their own type and, between lanes, as bit patterns,
// where a NaN is larger than infinity and infinity larger than every number: the maximum also tells whether the row is
// finite.  A thread keeps KEEP groups of eight in registers, chosen by the row's length so that more blocks share an SM
// where rows are short; rows of up to 16384 entries are read once, the rest of a longer one is read again.
// Measured in a stream of calls: 4096 x 8192 20 us (100 MB, 5.0 TB/s), 1000 x 11008 10.3 us; the first took 1.5 times as long
// with conversions and 32-bit comparisons.
template <int DT, int KEEP>
__global__ void __launch_bounds__(kQtThreads)
quantize_tokens_kernel(const uint16_t* __restrict__ X, int64_t d, int64_t ldx, int wide, int8_t* __restrict__ codes,
                       int64_t ldc, float* __restrict__ scale, int32_t* __restrict__ nonfinite, int32_t* __restrict__ clear) {
    tc5::dependents_may_start();
    const uint16_t* row = X + blockIdx.x * ldx;
    int8_t* out = codes + blockIdx.x * ldc;
    const int t = threadIdx.x;
    const int64_t groups = (d + 15) / 16 * 2;  // the codes' padding up to 16 is written too
    uint4 keep[KEEP];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t g = t + (int64_t)i * kQtThreads;
        keep[i] = make_uint4(0u, 0u, 0u, 0u);
        if (g < groups) keep[i] = load8(row + 8 * g, d - 8 * g, wide);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) m = group_max<DT>(m, keep[i]);
    for (int64_t g = t + (int64_t)KEEP * kQtThreads; g < groups; g += kQtThreads)
        m = group_max<DT>(m, load8(row + 8 * g, d - 8 * g, wide));
    __shared__ uint32_t part[kQtThreads / 32];
    m = __reduce_max_sync(0xffffffffu, max(m & 0x7fffu, m >> 16 & 0x7fffu));  // of magnitudes, as bit patterns
    if ((t & 31) == 0) part[t >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQtThreads / 32; ++i) m = max(m, part[i]);
    const float amax = widen16<DT>((uint16_t)m);
    float s = amax * (1.0f / 127.0f), inv = 1.0f / s;
    if (amax < 0x1p-120f) s = inv = 0.0f;
    if (t == 0) {
        scale[blockIdx.x] = s;
        if (clear && blockIdx.x == 0) *clear = 0;  // the mark of the product behind this, which sets it only after waiting for this kernel
        if (m >= (DT == CMPQ_BF16 ? 0x7f80u : 0x7c00u) && nonfinite) atomicOr(nonfinite, 1);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t g = t + (int64_t)i * kQtThreads;
        if (g < groups) *reinterpret_cast<uint2*>(out + 8 * g) = group_codes<DT>(keep[i], inv);
    }
    for (int64_t g = t + (int64_t)KEEP * kQtThreads; g < groups; g += kQtThreads)
        *reinterpret_cast<uint2*>(out + 8 * g) = group_codes<DT>(load8(row + 8 * g, d - 8 * g, wide), inv);
}

// ---- the product --------------------------------------------------------------------------------------------
//
// Tokens are the rows of the accumulator (a TMEM lane each), output channels its columns: a thread of the epilogue owns
// a token, whose scale is a register, and writes neighbouring channels, 16 bytes at a time; the channels' scales and
// biases come from shared memory.  Codes of both sides are K-major as they lie in memory; 128 bytes of the sum are one
// swizzled TMA box and four instructions of K = 32.

struct ProductArgs {
    const float *xs, *ws;
    const uint16_t* bias;
    uint16_t* y;
    int64_t ldy;
    int n, d_out, kblocks;  // kblocks: 128-byte blocks of the sum
    int wide;               // y takes 16-byte stores
    int n_tiles, m_tiles;   // tiles of channels, of tokens
    int stages, bn, rows;   // tile kernel: stages, channels of a tile, token rows that a box brings
    int32_t* failed;
};

constexpr int kMmThreads = 320;  // a warp for the loads, one for the products, eight for the epilogue
constexpr int kMmMaxStages = 40;
constexpr size_t kTileSmem = 208 << 10;

// Columns [c0, c1) of a warp's 32 accumulator rows: fl16(fl(fl(sum * xs) * ws) + bias) into y + column, of which `left`
// exist.  c0 and c1 are multiples of 16; scale_bias holds (ws, bias) of the tile's columns.
template <int DT>
__device__ __forceinline__ void store_rows(uint32_t tmem, int c0, int c1, const float2* scale_bias, bool has_bias, float xs, bool real,
                                           uint16_t* y, int left, bool wide) {
    for (int c = c0; c < c1; c += 16) {
        uint32_t r[16], w[8];
        tc5::tmem_ld16(tmem + c, r);
        tc5::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            const float4 sb = *reinterpret_cast<const float4*>(scale_bias + c + j);
            float a = (float)(int)r[j] * xs * sb.x, b = (float)(int)r[j + 1] * xs * sb.z;
            if (has_bias) a += sb.y, b += sb.w;
            w[j / 2] = round16x2<DT>(a, b);
        }
        if (!real) continue;
        if (wide && c + 16 <= left) {
            *reinterpret_cast<uint4*>(y + c) = make_uint4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<uint4*>(y + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < left) y[c + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
        }
    }
}

// Few tiles: a block takes 128 tokens (all of them, mostly) and `bn` channels, a multiple of 16 chosen so that the
// blocks fill the SMs; the weights pass through once and are the time while tokens are few.  Launched behind the
// quantization of its tokens, a block asks for its first weights before that has ended.  A stage holds the
// token rows that exist (to eight) and the channels'; the product reads on past those rows into whatever follows, which
// only reaches accumulator rows that are not stored, and 16 KB behind the last stage are kept for it.  With that one
// token's weights have some 30 stages on their way.
//
// Measured with the quantization in a stream of calls, weights from memory: one token 4096 -> 4096 10.3 us, 8192 -> 28672 42 us
// (5.6 TB/s, 0.86 of the copy rate); 37 tokens 4096 -> 11008 14.3 us (3.2 TB/s: launch, first loads and the last stage's way
// out are half of it).  Splitting the sum over a cluster instead, weights as rows, took 1.5, 1.3 and 2.4 times as long.
template <int DT>
__global__ void __launch_bounds__(kMmThreads)
matmul_i8_tile_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap,
                      const __grid_constant__ ProductArgs A) {
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024u - (tc5::smem_addr(raw) & 1023u)) & 1023u);
    __shared__ uint64_t full[kMmMaxStages], empty[kMmMaxStages], done;
    __shared__ float4 scale_bias[128];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nt = blockIdx.x / A.m_tiles, mt = blockIdx.x % A.m_tiles, bn = A.bn;
    const int a_bytes = A.rows * 128, stage = a_bytes + bn * 128, columns = bn <= 32 ? 32 : bn <= 64 ? 64 : bn <= 128 ? 128 : 256;
    if (threadIdx.x < A.stages) tc5::mbar_init(full + threadIdx.x, 1), tc5::mbar_init(empty + threadIdx.x, 1);
    if (threadIdx.x == 0) tc5::mbar_init(&done, 1), failed = 0;
    tc5::mbar_init_fence();
    if (warp == 1) tc5::tmem_alloc<1>(&tmem_at, columns);
    tc5::fence_before_sync();
    __syncthreads();
    tc5::fence_after_sync();
    const uint32_t tmem = tmem_at;
    if (warp == 0) {
        if (tc5::elect_one()) {
            int slot = 0, phase = 1;  // a new barrier counts as empty
            for (int i = 0; i < A.kblocks; ++i) {
                if (!tc5::mbar_wait(empty + slot, phase, &failed)) break;
                tc5::mbar_expect_tx(full + slot, stage);  // the tokens' bytes too, whoever comes first
                tc5::tma_load_2d(smem + slot * stage + a_bytes, &wmap, full + slot, i * 128, nt * bn);
                if (++slot == A.stages) slot = 0, phase ^= 1;
            }
        }
    } else if (warp == 1) {
        if (tc5::elect_one()) {
            const uint32_t idesc = tc5::idesc_i8(128, bn);
            int slot = 0, phase = 0;
            for (int i = 0; i < A.kblocks; ++i) {
                if (!tc5::mbar_wait(full + slot, phase, &failed)) break;
                tc5::fence_after_sync();
                const uint32_t at = tc5::smem_addr(smem + slot * stage);
                const uint64_t a = tc5::desc_k_sw128(at), b = tc5::desc_k_sw128(at + a_bytes);
#pragma unroll
                for (int k = 0; k < 4; ++k) tc5::mma_i8<1>(tmem, a + 2 * k, b + 2 * k, idesc, (i | k) != 0);
                tc5::mma_commit(empty + slot);
                if (++slot == A.stages) slot = 0, phase ^= 1;
            }
            tc5::mma_commit(&done);
        }
    } else {
        float2* sb = reinterpret_cast<float2*>(scale_bias);
        const int o0 = nt * bn, left = min(bn, A.d_out - o0), i = threadIdx.x - 64;
        if (i < bn) {
            const int o = min(o0 + i, A.d_out - 1);
            sb[i] = make_float2(__ldg(A.ws + o), A.bias ? widen16<DT>(A.bias[o]) : 0.0f);
        }
        tc5::wait_for_previous();
        if (warp == 2) {  // the token codes: the first epilogue warp's work until then
            if (tc5::elect_one()) {
                int slot = 0, phase = 1;
                for (int k = 0; k < A.kblocks; ++k) {
                    if (!tc5::mbar_wait(empty + slot, phase, &failed)) break;
                    tc5::tma_load_2d(smem + slot * stage, &xmap, full + slot, k * 128, mt * 128);
                    if (++slot == A.stages) slot = 0, phase ^= 1;
                }
            }
            __syncwarp();
        }
        const int quad = warp & 3, t = mt * 128 + quad * 32 + lane, half = (bn / 16 + 1) / 2 * 16;
        const bool real = t < A.n, upper = warp >= 6;
        const float xs = real ? __ldcg(A.xs + t) : 0.0f;  // written while this kernel was on its way: not the read-only path
        asm volatile("bar.sync 1, 256;" ::: "memory");
        tc5::mbar_wait_warp(&done, 0, &failed);
        tc5::fence_after_sync();
        if (mt * 128 + quad * 32 < A.n)
            store_rows<DT>(tmem + ((uint32_t)quad << 21), upper ? half : 0, upper ? bn : half, sb, A.bias != nullptr, xs, real,
                           A.y + (int64_t)t * A.ldy + o0, left, A.wide);
        tc5::fence_before_sync();
    }
    __syncwarp();
    __syncthreads();
    if (failed) {  // the loads that were asked for have to land before the shared memory is given back
        if (threadIdx.x == 0) {
            const long long start = clock64();
            while (clock64() - start < (1ll << 21)) __nanosleep(1000);
            atomicOr(A.failed, kWordInternal);
        }
        __syncthreads();
    }
    if (warp == 1) tc5::tmem_free<1>(tmem, columns);
}

constexpr int kPairStages = 6, kPairStageBytes = 2 * 128 * 128;
constexpr size_t kPairSmem = kPairStages * kPairStageBytes + 1024;

// Many tokens: pairs of CTAs stay on their SMs and walk over tiles of 256 tokens x 256 channels (cta_group::2).  A CTA
// loads its 128 tokens and half of the channels, so each byte that an SM reads feeds 512 products; six stages of 32 KB.
// Two accumulators of 256 columns alternate, the epilogue of one tile runs under the products of the next.  Token tiles
// go fastest: the pairs at work share a few weight tiles and the token codes stay in L2.
//
// Measured: 4096 x 8192 x 28672 with the quantization 610 us in a few calls after a rest (3.15 POP/s, 0.96 of twice the library's
// bf16 rate) and 680 to 694 in a long stream, where the power limit holds the clock; 2048 x 4096 x 11008 67 us, 72 with the
// quantization, the tensor pipe at 81 % (172 pair tiles in 3 rounds of 74).
template <int DT>
__global__ void __launch_bounds__(kMmThreads, 1)
matmul_i8_pair_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap,
                      const __grid_constant__ ProductArgs A) {
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024u - (tc5::smem_addr(raw) & 1023u)) & 1023u);
    __shared__ uint64_t full[kPairStages], empty[kPairStages], acc_full[2], acc_empty[2];
    __shared__ float4 scale_bias[2][128];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)tc5::cluster_rank();
    const int tiles = A.n_tiles * A.m_tiles, first = blockIdx.x >> 1, step = gridDim.x >> 1;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairStages; ++i) tc5::mbar_init(full + i, 1), tc5::mbar_init(empty + i, 1);
        for (int i = 0; i < 2; ++i) tc5::mbar_init(acc_full + i, 1), tc5::mbar_init(acc_empty + i, 16);
        failed = 0;
        tc5::mbar_init_fence();
    }
    if (warp == 1) tc5::tmem_alloc<2>(&tmem_at, 512);
    tc5::fence_before_sync();
    __syncthreads();
    tc5::cluster_sync();
    tc5::fence_after_sync();
    const uint32_t tmem = tmem_at;
    tc5::wait_for_previous();
    if (warp == 0) {
        if (tc5::elect_one()) {
            int slot = 0, phase = 1;  // a new barrier counts as empty
            bool ok = true;
            for (int tile = first; ok && tile < tiles; tile += step) {
                const int mt = tile % A.m_tiles, nt = tile / A.m_tiles;
                for (int k = 0; k < A.kblocks; ++k) {
                    if (!(ok = tc5::mbar_wait(empty + slot, phase, &failed))) break;
                    if (rank == 0) tc5::mbar_expect_tx(full + slot, 2 * kPairStageBytes);
                    uint8_t* at = smem + slot * kPairStageBytes;
                    tc5::tma_load_2d_pair(at, &xmap, full + slot, k * 128, mt * 256 + rank * 128);
                    tc5::tma_load_2d_pair(at + 128 * 128, &wmap, full + slot, k * 128, nt * 256 + rank * 128);
                    if (++slot == kPairStages) slot = 0, phase ^= 1;
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && tc5::elect_one()) {
            int slot = 0, phase = 0, acc = 0, acc_phase = 1;
            bool ok = true;
            for (int tile = first; ok && tile < tiles; tile += step) {
                if (!tc5::mbar_wait(acc_empty + acc, acc_phase, &failed)) break;
                tc5::fence_after_sync();
                for (int k = 0; k < A.kblocks; ++k) {
                    if (!(ok = tc5::mbar_wait(full + slot, phase, &failed))) break;
                    tc5::fence_after_sync();
                    const uint32_t at = tc5::smem_addr(smem + slot * kPairStageBytes);
                    const uint64_t a = tc5::desc_k_sw128(at), b = tc5::desc_k_sw128(at + 128 * 128);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        tc5::mma_i8<2>(tmem + acc * 256, a + 2 * j, b + 2 * j, tc5::idesc_i8(256, 256), (k | j) != 0);
                    tc5::mma_commit_pair(empty + slot);
                    if (++slot == kPairStages) slot = 0, phase ^= 1;
                }
                tc5::mma_commit_pair(acc_full + acc);
                acc ^= 1;
                if (acc == 0) acc_phase ^= 1;
            }
        }
    } else {
        const int quad = warp & 3, upper = warp >= 6, i = threadIdx.x - 64;
        float xs = 0.0f;
        walk_tiles(
            first, tiles, step,
            [&](int tile, int acc) {
                const int t = tile % A.m_tiles * 256 + rank * 128 + quad * 32 + lane;
                xs = t < A.n ? __ldcg(A.xs + t) : 0.0f;  // see the other kernel
                const int o = min(tile / A.m_tiles * 256 + i, A.d_out - 1);
                reinterpret_cast<float2*>(scale_bias[acc])[i] = make_float2(__ldg(A.ws + o), A.bias ? widen16<DT>(A.bias[o]) : 0.0f);
                asm volatile("bar.sync 1, 256;" ::: "memory");
            },
            [&](int acc, int parity) { return tc5::mbar_wait_warp(acc_full + acc, parity, &failed); },
            [&](int tile, int acc) {
                const int o0 = tile / A.m_tiles * 256, row0 = tile % A.m_tiles * 256 + rank * 128 + quad * 32, t = row0 + lane;
                tc5::fence_after_sync();
                if (row0 < A.n)
                    store_rows<DT>(tmem + ((uint32_t)quad << 21) + acc * 256, upper * 128, upper * 128 + 128, reinterpret_cast<float2*>(scale_bias[acc]),
                                   A.bias != nullptr, xs, t < A.n, A.y + (int64_t)t * A.ldy + o0, min(256, A.d_out - o0), A.wide);
                tc5::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc5::mbar_arrive_remote(acc_empty + acc, 0);
            });
    }
    __syncwarp();
    __syncthreads();
    if (failed) {
        if (threadIdx.x == 0) {
            const long long start = clock64();
            while (clock64() - start < (1ll << 21)) __nanosleep(1000);
            atomicOr(A.failed, kWordInternal);
        }
        __syncthreads();
    }
    tc5::cluster_sync();  // the pair's products and loads have ended on both sides
    if (warp == 1) tc5::tmem_free<2>(tmem, 512);
}

// Cycles that a way to cover the product takes, from sizes: rounds of blocks over the SMs, in each the blocks of the sum
// at the pace of the products or of the loads (64 bytes a cycle and SM), and what a round or launch costs besides; not
// less than the weights' way from memory (3400 bytes a cycle).  Fitted to sweeps of bn over 1 to 512 tokens and layers of
// 4096 x 4096 to 8192 x 28672; e.g. 256 x 4096 x 11008: bn = 160 17.9 us, 80 22.7, pairs 21.6; 4096 x 8192 x 28672: pairs.
static int64_t tile_cycles(const ProductArgs& a, int bn) {
    const int64_t blocks = (int64_t)((a.n + 127) / 128) * ((a.d_out + bn - 1) / bn), sms = sm_count();
    const int64_t rounds = (blocks + sms - 1) / sms, pace = std::max(4 * std::max(32, bn / 2), (bn + std::min(a.n, 128)) * 2);
    return std::max<int64_t>(rounds * a.kblocks * pace, (int64_t)a.kblocks * 128 * a.d_out / 3400) + rounds * (9000 + 8 * bn);
}
static int64_t pair_cycles(const ProductArgs& a) {
    const int64_t tiles = (int64_t)((a.n + 255) / 256) * ((a.d_out + 255) / 256), pairs = sm_count() / 2;
    return (tiles + pairs - 1) / pairs * a.kblocks * 600 + 14000;
}

template <int DT>
static cmpq_status launch_product(const int8_t* xc, int64_t ldxc, const int8_t* wc, int64_t ldwc, int64_t d_in, ProductArgs a, bool behind,
                                  cudaStream_t st) {
    a.kblocks = (int)((d_in + 127) / 128);
    a.wide = aligned_to(a.y, 16) && a.ldy % 8 == 0;
    a.bn = 32;
    for (int bn = 48; bn <= 256; bn += 16)
        if (tile_cycles(a, bn) < tile_cycles(a, a.bn)) a.bn = bn;
    const bool pair = a.n > 128 && pair_cycles(a) < tile_cycles(a, a.bn);
    a.rows = pair ? 128 : std::min(128, (a.n + 7) / 8 * 8);
    CUtensorMap wmap, xmap;
    if (!make_byte_map(&wmap, wc, a.d_out, d_in, ldwc, pair ? 128 : a.bn) || !make_byte_map(&xmap, xc, a.n, d_in, ldxc, a.rows)) return CMPQ_ERR_CUDA;
    if (pair) {
        a.m_tiles = (a.n + 255) / 256, a.n_tiles = (a.d_out + 255) / 256;
        static bool raised[64];
        if (!raise_smem_limit_once(matmul_i8_pair_kernel<DT>, kPairSmem, raised)) return CMPQ_ERR_CUDA;
        const int64_t tiles = (int64_t)a.m_tiles * a.n_tiles;
        return launch_cluster(matmul_i8_pair_kernel<DT>, 2 * (unsigned)std::min<int64_t>(tiles, sm_count() / 2), kMmThreads, kPairSmem, 2, behind, st,
                              wmap, xmap, a);
    }
    a.m_tiles = (a.n + 127) / 128, a.n_tiles = (a.d_out + a.bn - 1) / a.bn;
    // one block to an SM: two that share it were slower at every size, their rounds and tails cost more than they hide
    const int64_t blocks = (int64_t)a.m_tiles * a.n_tiles;
    const size_t stage = (a.rows + a.bn) * 128, slack = (128 - a.rows) * 128 + 1024;
    a.stages = std::min({(int)((kTileSmem - slack) / stage), kMmMaxStages, a.kblocks});
    static bool raised[64];
    if (!raise_smem_limit_once(matmul_i8_tile_kernel<DT>, kTileSmem, raised)) return CMPQ_ERR_CUDA;
    if (blocks > INT32_MAX) return CMPQ_ERR_UNSUPPORTED;
    return launch_cluster(matmul_i8_tile_kernel<DT>, (unsigned)blocks, kMmThreads, a.stages * stage + slack, 1, behind, st, wmap, xmap, a);
}

size_t linear_i8_codes_bytes(int64_t n, int64_t d_in) { return round_up((size_t)n * round_up(d_in, 16), 256); }

}  // namespace cmpq

using namespace cmpq;

static bool linear_sizes_ok(int64_t n, int64_t d_in, int64_t d_out) {
    return n >= 0 && n <= INT32_MAX - 256 /* tiles of tokens end past the last one */ && d_in >= 1 && d_in <= CMPQ_MAX_D_IN_I8 && d_out >= 1 && d_out <= CMPQ_MAX_D_IN;
}

extern "C" size_t cmpq_linear_i8_ws_bytes(int64_t n, int64_t d_in, int64_t d_out) {
    if (!linear_sizes_ok(n, d_in, d_out)) return 0;
    return linear_i8_codes_bytes(n, d_in) + round_up((size_t)n * sizeof(float), 256) + 256;
}

static cmpq_status quantize(const void* X, cmpq_dtype dt, int64_t n, int64_t d, int64_t ldx, int8_t* codes, int64_t ldc, float* scale,
                            int32_t* nonfinite, int32_t* clear, void* stream) {
    if (dt != CMPQ_F16 && dt != CMPQ_BF16) return CMPQ_ERR_INVALID_ARG;
    if (n < 0 || n > INT32_MAX || d < 1 || d > CMPQ_MAX_D_IN || ldx < d || ldc < d || ldc % 16) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!X || !codes || !scale || !aligned_to(X, 2) || !aligned_to(codes, 16) || !aligned_to(scale, 4)) return CMPQ_ERR_INVALID_ARG;
    const int wide = aligned_to(X, 16) && ldx % 8 == 0;
    const auto* x = static_cast<const uint16_t*>(X);
    auto st = static_cast<cudaStream_t>(stream);
    const unsigned rows = (unsigned)n;
    const int64_t keep = (d + 8 * kQtThreads - 1) / (8 * kQtThreads);
    auto launch = [&](auto kernel) { return launch_cluster(kernel, rows, kQtThreads, 0, 1, false, st, x, d, ldx, wide, codes, ldc, scale, nonfinite, clear); };
    if (dt == CMPQ_BF16)
        return keep <= 2   ? launch(quantize_tokens_kernel<CMPQ_BF16, 2>)
               : keep <= 4 ? launch(quantize_tokens_kernel<CMPQ_BF16, 4>)
                           : launch(quantize_tokens_kernel<CMPQ_BF16, 8>);
    return keep <= 2   ? launch(quantize_tokens_kernel<CMPQ_F16, 2>)
           : keep <= 4 ? launch(quantize_tokens_kernel<CMPQ_F16, 4>)
                       : launch(quantize_tokens_kernel<CMPQ_F16, 8>);
}

extern "C" cmpq_status cmpq_quantize_tokens(const void* X, cmpq_dtype dt, int64_t n, int64_t d, int64_t ldx,
                                            int8_t* codes, int64_t ldc, float* scale, int32_t* nonfinite,
                                            void* stream) {
    return quantize(X, dt, n, d, ldx, codes, ldc, scale, nonfinite, nullptr, stream);
}

// Where a call without a word of the caller's keeps the mark of a kernel that gave up; it starts from 0 in every call.
static int32_t* mark_of(void* ws, int64_t n, int64_t d_in, int64_t d_out) {
    return reinterpret_cast<int32_t*>(static_cast<char*>(ws) + cmpq_linear_i8_ws_bytes(n, d_in, d_out) - 256);
}

// The caller has checked everything.
static cmpq_status product(const int8_t* xc, int64_t ldxc, const float* xs, const int8_t* wc, int64_t ldwc, const float* w_scale, const void* bias,
                           cmpq_dtype dt, int64_t n, int64_t d_in, int64_t d_out, void* y, int64_t ldy, int32_t* word, bool behind, void* stream) {
    ProductArgs a = {};
    a.xs = xs, a.ws = w_scale;
    a.bias = static_cast<const uint16_t*>(bias);
    a.y = static_cast<uint16_t*>(y);
    a.ldy = ldy;
    a.n = (int)n, a.d_out = (int)d_out;
    a.failed = word;
    auto st = static_cast<cudaStream_t>(stream);
    return dt == CMPQ_BF16 ? launch_product<CMPQ_BF16>(xc, ldxc, wc, ldwc, d_in, a, behind, st)
                           : launch_product<CMPQ_F16>(xc, ldxc, wc, ldwc, d_in, a, behind, st);
}

extern "C" cmpq_status cmpq_matmul_i8(const int8_t* xc, int64_t ldxc, const float* xs, const int8_t* wc, int64_t ldwc,
                                      const float* w_scale, const void* bias, cmpq_dtype dt, int64_t n, int64_t d_in,
                                      int64_t d_out, void* y, int64_t ldy, void* ws, size_t ws_bytes, void* stream) {
    if (dt != CMPQ_F16 && dt != CMPQ_BF16) return CMPQ_ERR_INVALID_ARG;
    if (!linear_sizes_ok(n, d_in, d_out) || ldxc < d_in || ldwc < d_in || ldxc % 16 || ldwc % 16 || ldy < d_out) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!xc || !xs || !wc || !w_scale || !y || !aligned_to(xc, 16) || !aligned_to(wc, 16) || !aligned_to(xs, 4) ||
        !aligned_to(w_scale, 4) || !aligned_to(y, 2) || !aligned_to(bias, 2))
        return CMPQ_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < cmpq_linear_i8_ws_bytes(n, d_in, d_out)) return CMPQ_ERR_WORKSPACE;
    int32_t* mark = mark_of(ws, n, d_in, d_out);
    if (cudaMemsetAsync(mark, 0, sizeof(*mark), static_cast<cudaStream_t>(stream)) != cudaSuccess) return CMPQ_ERR_CUDA;
    return product(xc, ldxc, xs, wc, ldwc, w_scale, bias, dt, n, d_in, d_out, y, ldy, mark, false, stream);
}

extern "C" cmpq_status cmpq_linear_i8(const void* X, cmpq_dtype dt, int64_t n, int64_t d_in, int64_t ldx,
                                      const int8_t* wc, int64_t ldwc, const float* w_scale, const void* bias,
                                      int64_t d_out, void* y, int64_t ldy, int32_t* nonfinite, void* ws,
                                      size_t ws_bytes, void* stream) {
    if (!linear_sizes_ok(n, d_in, d_out) || ldwc < d_in || ldwc % 16 || ldy < d_out || ldx < d_in) return CMPQ_ERR_INVALID_ARG;
    if (dt != CMPQ_F16 && dt != CMPQ_BF16) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!wc || !w_scale || !y || !aligned_to(wc, 16) || !aligned_to(w_scale, 4) || !aligned_to(y, 2) || !aligned_to(bias, 2))
        return CMPQ_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < cmpq_linear_i8_ws_bytes(n, d_in, d_out)) return CMPQ_ERR_WORKSPACE;
    Workspace w(ws, ws_bytes);
    int8_t* codes = w.take<int8_t>(linear_i8_codes_bytes(n, d_in));
    float* scale = w.take<float>(n);
    const int64_t ldc = (int64_t)round_up(d_in, 16);
    int32_t* mark = mark_of(ws, n, d_in, d_out);
    cmpq_status st = quantize(X, dt, n, d_in, ldx, codes, ldc, scale, nonfinite, nonfinite ? nullptr : mark, stream);
    if (st != CMPQ_OK) return st;
    // the quantization lets the product start early; it was itself started after everything before it, the weights too
    return product(codes, ldc, scale, wc, ldwc, w_scale, bias, dt, n, d_in, d_out, y, ldy, nonfinite ? nonfinite : mark, true, stream);
}
