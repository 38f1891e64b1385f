// 8-bit linear layers: quantization of tokens and the integer product with scales per token and channel.
#include <algorithm>

#include "asked.h"
#include "product_i8.cuh"
#include "walk.cuh"

namespace cmpq {

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
// where rows are short, and twice as many threads where they are long; rows of up to 32768 entries are read once, the rest of a
// longer one is read again.
// Measured in graphs: 4096 x 8192 17.8 us (100 MB, 5.6 TB/s), 4096 x 28672 58 (6.1 TB/s; 88 with 256 threads, which read the end
// of the row twice); the first took 1.5 times as long with conversions and 32-bit comparisons.
template <int DT, int KEEP, int THREADS = kQtThreads>
__global__ void __launch_bounds__(THREADS)
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
        const int64_t g = t + (int64_t)i * THREADS;
        keep[i] = make_uint4(0u, 0u, 0u, 0u);
        if (g < groups) keep[i] = load8(row + 8 * g, d - 8 * g, wide);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) m = group_max<DT>(m, keep[i]);
    for (int64_t g = t + (int64_t)KEEP * THREADS; g < groups; g += THREADS)
        m = group_max<DT>(m, load8(row + 8 * g, d - 8 * g, wide));
    __shared__ uint32_t part[THREADS / 32];
    m = __reduce_max_sync(0xffffffffu, max(m & 0x7fffu, m >> 16 & 0x7fffu));  // of magnitudes, as bit patterns
    if ((t & 31) == 0) part[t >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) m = max(m, part[i]);
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
        const int64_t g = t + (int64_t)i * THREADS;
        if (g < groups) *reinterpret_cast<uint2*>(out + 8 * g) = group_codes<DT>(keep[i], inv);
    }
    for (int64_t g = t + (int64_t)KEEP * THREADS; g < groups; g += THREADS)
        *reinterpret_cast<uint2*>(out + 8 * g) = group_codes<DT>(load8(row + 8 * g, d - 8 * g, wide), inv);
}

// The same behind a norm.  Measured in graphs: 4096 x 8192 23 us (100 MB, 4.4 TB/s), 4096 x 4096 14 (3.6): the issue slots are two
// thirds full, of which a third goes to what a row costs besides its entries.
template <int DT, int KEEP>
__global__ void __launch_bounds__(kQtThreads)
norm_quantize_kernel(const uint16_t* __restrict__ X, int64_t d, int64_t ldx, int wide, RowNorm norm, int8_t* __restrict__ codes, int64_t ldc,
                     float* __restrict__ scale, int32_t* __restrict__ nonfinite, int32_t* __restrict__ clear) {
    tc5::dependents_may_start();
    __shared__ RowParts parts;
    if (threadIdx.x == 0 && clear && blockIdx.x == 0) *clear = 0;  // see the other kernel
    norm_quantize_row<DT, KEEP>(X + blockIdx.x * ldx, d, wide, norm, codes + blockIdx.x * ldc, scale + blockIdx.x, nonfinite, threadIdx.x, parts);
}

// ---- the product --------------------------------------------------------------------------------------------
//
// Tokens are the rows of the accumulator (a TMEM lane each), output channels its columns: a thread of the epilogue owns
// a token, whose scale is a register, and writes neighbouring channels, 16 bytes at a time; the channels' scales and
// biases come from shared memory.  Codes of both sides are K-major as they lie in memory; 128 bytes of the sum are one
// swizzled TMA box and four instructions of K = 32.

constexpr int kMmThreads = 320;  // a warp for the loads, one for the products, eight for the epilogue
constexpr int kMmMaxStages = 40;
constexpr size_t kTileSmem = 208 << 10;

// Few tiles: a block takes 128 tokens (all of them, mostly) and `bn` channels, a multiple of 16 chosen so that the
// blocks fill the SMs; the weights pass through once and are the time while tokens are few.  Launched behind the
// quantization of its tokens, a block asks for its first weights before that has ended.  A stage holds the
// token rows that exist (to eight) and the channels'; the product reads on past those rows into whatever follows, which
// only reaches accumulator rows that are not stored, and 16 KB behind the last stage are kept for it.  A stage holds one
// 128-byte block of the sum, or 48 to 64 KB of them where weights come from memory in narrow tiles (stage_of_one: why, and figures).
//
// Measured with the quantization in graphs, weights from memory: 8 tokens 4096 -> 4096 8.4 us, 8192 -> 28672 42.3 us (5.6 TB/s,
// 0.85 of the copy rate); 53 tokens 4096 -> 11008 11.9 us (3.8 TB/s: launch, first loads and the last stage's way out are
// half of it).  For these, weights as rows and the sum over a cluster took 1.5, 1.3 and 2.4 times as long.
//
// A gated tile's columns are bn / 2 channels of the gate and the same ones of the second projection, from maps of their own.
//
// kSliced: narrow tiles of few tokens leave most of an instruction's rows empty, and it takes 40 cycles all the same.  Every
// second or fourth block of the sum gets rows and columns of its own then, an instruction takes as many blocks, and the slices
// are added up at the end (see few_i8.cu): 8 tokens 11008 -> 4096 15.4 -> 12.9 us.  A kernel of its own, as its longer program
// cost small layers 0.2 us.
//
// kSplit: the sum of a tile is cut over two or four CTAs of a cluster, which lets a few wide tiles with long sums use all SMs and
// reads the tokens fewer times than as many narrow tiles.  Each CTA then takes a part of the tile's channels and adds up what the
// others send it of those.  128 tokens 28672 -> 1024: 40 us whole, 18 over four; 11008 -> 4096 19.4 and 16.7 over
// four; 256 tokens 11008 -> 2048 19.0 and 15.4.
//
// ONE: a stage is one block of the sum.  The loops over the blocks are the time of an issuing thread, so they are written out without
// those of a stage (4096 -> 4096, 320 tokens 12.6 us with both, 11.4 so).
enum { kWhole, kSliced, kSplit };
template <int DT, int KIND, int SUM, bool ONE>
__global__ void __launch_bounds__(kMmThreads, 1)
matmul_i8_tile_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap umap, const __grid_constant__ CUtensorMap xmap,
                      const __grid_constant__ ProductArgs A) {
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024u - (tc5::smem_addr(raw) & 1023u)) & 1023u);
    __shared__ uint64_t full[kMmMaxStages], empty[kMmMaxStages], done;
    __shared__ float4 scale_bias[128];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int parts = SUM == kSplit ? A.slices : 1, part = SUM == kSplit ? (int)tc5::cluster_rank() : 0, k0 = part * A.kblocks;
    const int nt = blockIdx.x / parts / A.m_tiles, mt = blockIdx.x / parts % A.m_tiles, bn = A.bn;
    const int S = SUM == kSliced ? A.slices : 1, N = S * bn, columns = N <= 32 ? 32 : N <= 64 ? 64 : N <= 128 ? 128 : 256;
    const int row_box = A.rows * 128, box = bn * 128, a_bytes = S * row_box, b_bytes = S * box, stage = (ONE ? 1 : A.per_stage) * (a_bytes + b_bytes);  // of a slice, of all
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
            for (int i = 0; ONE && i < A.kblocks; ++i) {
                if (!tc5::mbar_wait(empty + slot, phase, &failed)) break;
                tc5::mbar_expect_tx(full + slot, stage);  // the tokens' bytes too, whoever comes first
                uint8_t* at = smem + slot * stage + a_bytes;
                if (KIND == kGated) {
                    tc5::tma_load_2d(at, &wmap, full + slot, (k0 + i) * 128, nt * (bn / 2));
                    tc5::tma_load_2d(at + box / 2, &umap, full + slot, (k0 + i) * 128, nt * (bn / 2));
                } else {
                    tc5::tma_load_2d(at, &wmap, full + slot, (k0 + i) * 128, nt * bn);
                }
                if (++slot == A.stages) slot = 0, phase ^= 1;
            }
            for (int k = 0; !ONE && k < A.kblocks; k += A.per_stage) {
                if (!tc5::mbar_wait(empty + slot, phase, &failed)) break;
                const int count = min(A.per_stage, A.kblocks - k);
                tc5::mbar_expect_tx(full + slot, count * (a_bytes + b_bytes));  // the tokens' bytes too, whoever comes first
                uint8_t* at = smem + slot * stage + A.per_stage * a_bytes;
                for (int i = k0 + k * S; i < k0 + (k + count) * S; ++i, at += box) {
                    if (KIND == kGated) {
                        tc5::tma_load_2d(at, &wmap, full + slot, i * 128, nt * (bn / 2));
                        tc5::tma_load_2d(at + box / 2, &umap, full + slot, i * 128, nt * (bn / 2));
                    } else {
                        tc5::tma_load_2d(at, &wmap, full + slot, i * 128, nt * bn);
                    }
                }
                if (++slot == A.stages) slot = 0, phase ^= 1;
            }
        }
    } else if (warp == 1) {
        if (tc5::elect_one()) {
            const uint32_t idesc = tc5::idesc_i8(128, N);
            int slot = 0, phase = 0;
            for (int i = 0; ONE && i < A.kblocks; ++i) {
                if (!tc5::mbar_wait(full + slot, phase, &failed)) break;
                tc5::fence_after_sync();
                const uint32_t at = tc5::smem_addr(smem + slot * stage);
                const uint64_t a = tc5::desc_k_sw128(at), b = tc5::desc_k_sw128(at + a_bytes);
#pragma unroll
                for (int j = 0; j < 4; ++j) tc5::mma_i8<1>(tmem, a + 2 * j, b + 2 * j, idesc, (i | j) != 0);
                tc5::mma_commit(empty + slot);
                if (++slot == A.stages) slot = 0, phase ^= 1;
            }
            for (int k = 0; !ONE && k < A.kblocks; k += A.per_stage) {
                if (!tc5::mbar_wait(full + slot, phase, &failed)) break;
                tc5::fence_after_sync();
                const uint32_t at = tc5::smem_addr(smem + slot * stage);
                uint64_t a = tc5::desc_k_sw128(at), b = tc5::desc_k_sw128(at + A.per_stage * a_bytes);  // in units of 16 bytes
                for (int i = k; i < min(k + A.per_stage, A.kblocks); ++i, a += a_bytes / 16, b += b_bytes / 16)
#pragma unroll
                    for (int j = 0; j < 4; ++j) tc5::mma_i8<1>(tmem, a + 2 * j, b + 2 * j, idesc, (i | j) != 0);
                tc5::mma_commit(empty + slot);
                if (++slot == A.stages) slot = 0, phase ^= 1;
            }
            tc5::mma_commit(&done);
        }
        __syncwarp();
    } else {
        float2* sb = reinterpret_cast<float2*>(scale_bias);
        const int wide = KIND == kGated ? bn / 2 : bn;  // channels of the tile
        const int o0 = nt * wide, left = min(wide, A.d_out - o0), i = threadIdx.x - 64;
        if (i < bn) sb[i] = column_scale<DT, KIND>(A, o0, i, bn);
        tc5::wait_for_previous();
        if (warp == 2) {  // the token codes: the first epilogue warp's work until then
            if (tc5::elect_one()) {
                int slot = 0, phase = 1;
                for (int i = 0; ONE && i < A.kblocks; ++i) {
                    if (!tc5::mbar_wait(empty + slot, phase, &failed)) break;
                    tc5::tma_load_2d(smem + slot * stage, &xmap, full + slot, (k0 + i) * 128, mt * 128);
                    if (++slot == A.stages) slot = 0, phase ^= 1;
                }
                for (int k = 0; !ONE && k < A.kblocks; k += A.per_stage) {
                    if (!tc5::mbar_wait(empty + slot, phase, &failed)) break;
                    for (int i = 0; i < min(A.per_stage, A.kblocks - k) * S; ++i)
                        tc5::tma_load_2d(smem + slot * stage + i * row_box, &xmap, full + slot, (k0 + k * S + i) * 128, mt * 128);
                    if (++slot == A.stages) slot = 0, phase ^= 1;
                }
            }
            __syncwarp();
        }
        const int step = KIND == kGated ? 8 : 16, quad = warp & 3, t = mt * 128 + quad * 32 + lane, mine = wide / parts;
        const int half = SUM == kSplit ? (mine / 8 + 1) / 2 * 8 : (mine / step + 1) / 2 * step;
        const bool real = t < A.n, upper = warp >= 6;
        const int c0 = part * mine + (upper ? half : 0), c1 = part * mine + (upper ? mine : half);
        if (KIND == kFinish && A.residual && real) ask_for(A.residual + (int64_t)t * A.ldr + o0, c0, min(c1, left));
        const float xs = real ? __ldcg(A.xs + t) : 0.0f;  // written while this kernel was on its way: not the read-only path
        asm volatile("bar.sync 1, 256;" ::: "memory");
        tc5::mbar_wait_warp(&done, 0, &failed);
        tc5::fence_after_sync();
        if (SUM == kSplit) {
            // The CTA finishes `mine` of the tile's channels: the others' sums of those come through shared memory, which no copy
            // or product uses any more, [CTA][token][column]; rows 16 bytes more apart, for the banks.
            const int both = KIND == kGated ? 2 : 1, pitch = both * mine + 4, first = part * mine;
            const uint32_t rows = tmem + ((uint32_t)quad << 21);
            int32_t* sums = reinterpret_cast<int32_t*>(smem) + (quad * 32 + lane) * pitch;
            const bool warp_real = mt * 128 + quad * 32 < A.n;
            tc5::cluster_sync();  // everybody's products have ended
            if (warp_real)
                for (int p = 1; p < parts; ++p) {
                    const int to = (part + p) & (parts - 1);
                    for (int b = 0; b < both; ++b)
                        for (int c = c0 - first; c < c1 - first; c += 8) {
                            uint32_t r[8];
                            tc5::tmem_ld8(rows + b * wide + to * mine + c, r);
                            tc5::tmem_ld_wait();
                            if (real) {
                                int32_t* at = sums + (p - 1) * 128 * pitch + b * mine + c;
                                tc5::store_remote(at, to, r[0], r[1], r[2], r[3]);
                                tc5::store_remote(at + 4, to, r[4], r[5], r[6], r[7]);
                            }
                        }
                }
            __syncwarp();
            tc5::cluster_sync();
            if (warp_real)
                for (int o = c0; o < c1; o += 8) {
                    uint32_t r[8], s[8] = {};
                    tc5::tmem_ld8(rows + o, r);
                    if (KIND == kGated) tc5::tmem_ld8(rows + wide + o, s);
                    tc5::tmem_ld_wait();
                    int z[8], u[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = (int)r[j], u[j] = (int)s[j];
                    for (int p = 0; p < parts - 1; ++p)
#pragma unroll
                        for (int j = 0; j < 8; j += 4) {
                            const int32_t* at = sums + p * 128 * pitch + o - first + j;
                            const int4 a = *reinterpret_cast<const int4*>(at);
                            z[j] += a.x, z[j + 1] += a.y, z[j + 2] += a.z, z[j + 3] += a.w;
                            if (KIND == kGated) {
                                const int4 b = *reinterpret_cast<const int4*>(at + mine);
                                u[j] += b.x, u[j + 1] += b.y, u[j + 2] += b.z, u[j + 3] += b.w;
                            }
                        }
                    if (real && o < left)
                        store_eight<DT, KIND>(A, z, u, sb + o, sb + wide + o, xs, A.y + (int64_t)t * A.ldy + o0 + o, A.residual + (int64_t)t * A.ldr + o0 + o,
                                              left - o);
                }
        } else if (SUM == kSliced) {
            // Row q rows + t holds slice q's sums of token t, in columns q bn and on.  They are added up through shared memory, which
            // no copy or product uses any more: [slice][token][column].
            int32_t* sums = reinterpret_cast<int32_t*>(smem);
            const int row = quad * 32 + lane, mine = row / A.rows;
            for (int q = quad * 32 / A.rows; q < min(S, (quad * 32 + 31) / A.rows + 1); ++q)
                for (int c = upper ? 16 : 0; c < bn; c += 32) {
                    uint32_t r[16];
                    tc5::tmem_ld16(tmem + ((uint32_t)quad << 21) + q * bn + c, r);
                    tc5::tmem_ld_wait();
                    if (mine == q)
#pragma unroll
                        for (int j = 0; j < 16; j += 4) *reinterpret_cast<int4*>(sums + row * bn + c + j) = make_int4(r[j], r[j + 1], r[j + 2], r[j + 3]);
                }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            for (int i = threadIdx.x - 64; i < A.n * (wide / 8); i += 256) {
                const int token = i / (wide / 8), c = i % (wide / 8) * 8;
                int z[8] = {}, u[8] = {};
                for (int q = 0; q < S; ++q)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int32_t* from = sums + (q * A.rows + token) * bn + c + j;
                        z[j] += from[0];
                        if (KIND == kGated) u[j] += from[bn / 2];
                    }
                if (c < left)
                    store_eight<DT, KIND>(A, z, u, sb + c, sb + bn / 2 + c, __ldcg(A.xs + token), A.y + (int64_t)token * A.ldy + o0 + c,
                                          A.residual + (int64_t)token * A.ldr + o0 + c, left - c);
            }
        } else if (mt * 128 + quad * 32 < A.n) {
            const uint32_t rows = tmem + ((uint32_t)quad << 21);
            uint16_t* y = A.y + (int64_t)t * A.ldy + o0;
            if (KIND == kPlain) store_rows<DT>(rows, c0, c1, sb, A.bias != nullptr, xs, real, y, left, A.wide);
            if (KIND == kFinish) store_finished<DT>(rows, c0, c1, sb, A, xs, real, y, A.residual + (int64_t)t * A.ldr + o0, left);
            if (KIND == kGated) store_gated<DT>(rows, c0, c1, wide, sb, A, xs, real, y, left);
        }
        tc5::fence_before_sync();
    }
    __syncwarp();
    if (SUM == kSplit && warp < 2) tc5::cluster_sync(), tc5::cluster_sync();  // the epilogue's
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

constexpr int kPairStages = 6, kPairStageBytes = 2 * 128 * 128;  // room for the widest tile
constexpr size_t kPairSmem = kPairStages * kPairStageBytes + 1024;

// Many tokens: pairs of CTAs stay on their SMs and walk over tiles of 256 tokens x bn channels (cta_group::2), 256 of them or
// fewer, in steps of 32, where that fills the last round better.  A CTA loads its 128 tokens and half of the channels, so each
// byte that an SM reads feeds 512 products; six stages of 32 KB, whose weights are asked for while the tokens are quantized.
// Two accumulators of 256 columns alternate, the epilogue of one tile runs under the products of the next.  Token tiles
// go fastest: the pairs at work share a few weight tiles and the token codes stay in L2.
//
// Measured: 4096 x 8192 x 28672 with the quantization 610 us in a few calls after a rest (3.15 POP/s, 0.96 of twice the library's
// bf16 rate) and 670 in a long stream, where the power limit holds the clock; 2048 x 4096 x 11008 64 us, 71 with the
// quantization, the tensor pipe at 71 %: the SMs ask L2 for some 12 TB/s then, which is what holds the pace.
//
// A gated tile is 256 tokens x bn / 2 channels of both projections: the even CTA's half of the columns is the gate, the odd
// one's the second projection, so a thread of the epilogue finds both of a channel in its accumulator row; activations stay
// under the next tile's products.  2048 tokens 4096 -> 11008 take 114 us, the tensor pipe at 82 %.
template <int DT, int KIND>
__global__ void __launch_bounds__(kMmThreads, 1)
matmul_i8_pair_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap umap, const __grid_constant__ CUtensorMap xmap,
                      const __grid_constant__ ProductArgs A) {
    const int half = A.bn / 2, wide_tile = KIND == kGated ? half : A.bn;  // columns that a CTA loads; channels of a tile
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
    if (warp == 0) {
        if (tc5::elect_one()) {
            int slot = 0, phase = 1;  // a new barrier counts as empty
            bool ok = true;
            auto weights = [&](int nt, int k) {  // and both operands' bytes of both CTAs, whoever comes first
                if (rank == 0) tc5::mbar_expect_tx(full + slot, 2 * (128 + half) * 128);
                uint8_t* at = smem + slot * kPairStageBytes + 128 * 128;
                if (KIND == kGated)
                    tc5::tma_load_2d_pair(at, rank ? &umap : &wmap, full + slot, k * 128, nt * half);
                else
                    tc5::tma_load_2d_pair(at, &wmap, full + slot, k * 128, nt * A.bn + rank * half);
            };
            const int early = first < tiles ? min(kPairStages, A.kblocks) : 0;  // stages of weights that do not wait for the tokens
            for (slot = 0; slot < early; ++slot) weights(first / A.m_tiles, slot);
            slot = 0;
            tc5::wait_for_previous();
            for (int tile = first; ok && tile < tiles; tile += step) {
                const int mt = tile % A.m_tiles, nt = tile / A.m_tiles;
                for (int k = 0; k < A.kblocks; ++k) {
                    if (tile != first || k >= early) {
                        if (!(ok = tc5::mbar_wait(empty + slot, phase, &failed))) break;
                        weights(nt, k);
                    }
                    tc5::tma_load_2d_pair(smem + slot * kPairStageBytes, &xmap, full + slot, k * 128, mt * 256 + rank * 128);
                    if (++slot == kPairStages) slot = 0, phase ^= 1;
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && tc5::elect_one()) {
            const uint32_t idesc = tc5::idesc_i8(256, A.bn);
            int slot = 0, phase = 0, acc = 0, acc_phase = 1;
            bool ok = true;
            for (int tile = first; ok && tile < tiles; tile += step) {
                if (!tc5::mbar_wait<true>(acc_empty + acc, acc_phase, &failed)) break;
                tc5::fence_after_sync();
                for (int k = 0; k < A.kblocks; ++k) {
                    if (!(ok = tc5::mbar_wait(full + slot, phase, &failed))) break;
                    tc5::fence_after_sync();
                    const uint32_t at = tc5::smem_addr(smem + slot * kPairStageBytes);
                    const uint64_t a = tc5::desc_k_sw128(at), b = tc5::desc_k_sw128(at + 128 * 128);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        tc5::mma_i8<2>(tmem + acc * 256, a + 2 * j, b + 2 * j, idesc, (k | j) != 0);
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
        tc5::wait_for_previous();
        walk_tiles(
            first, tiles, step,
            [&](int tile, int acc) {
                const int t = tile % A.m_tiles * 256 + rank * 128 + quad * 32 + lane;
                xs = t < A.n ? __ldcg(A.xs + t) : 0.0f;  // see the other kernel
                const int o0 = tile / A.m_tiles * wide_tile;
                if (i < A.bn) reinterpret_cast<float2*>(scale_bias[acc])[i] = column_scale<DT, KIND>(A, o0, i, A.bn);
                if (KIND == kFinish && A.residual && t < A.n)
                    ask_for(A.residual + (int64_t)t * A.ldr + o0, min(upper * half, A.d_out - o0), min(upper * half + half, A.d_out - o0));
                asm volatile("bar.sync 1, 256;" ::: "memory");
            },
            [&](int acc, int parity) { return tc5::mbar_wait_warp(acc_full + acc, parity, &failed); },
            [&](int tile, int acc) {
                const int o0 = tile / A.m_tiles * wide_tile, row0 = tile % A.m_tiles * 256 + rank * 128 + quad * 32, t = row0 + lane;
                const int left = min(wide_tile, A.d_out - o0), c0 = upper * (wide_tile / 2), c1 = c0 + wide_tile / 2;
                tc5::fence_after_sync();
                if (row0 < A.n) {
                    const float2* sb = reinterpret_cast<float2*>(scale_bias[acc]);
                    const uint32_t rows = tmem + ((uint32_t)quad << 21) + acc * 256;
                    uint16_t* y = A.y + (int64_t)t * A.ldy + o0;
                    if (KIND == kPlain) store_rows<DT>(rows, c0, c1, sb, A.bias != nullptr, xs, t < A.n, y, left, A.wide);
                    if (KIND == kFinish) store_finished<DT>(rows, c0, c1, sb, A, xs, t < A.n, y, A.residual + (int64_t)t * A.ldr + o0, left);
                    if (KIND == kGated) store_gated<DT>(rows, c0, c1, half, sb, A, xs, t < A.n, y, left);
                }
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

// Clusters of `parts` CTAs, each on an SM of its own, that run at once: fewer than the SMs would allow (33 of four on 148 SMs), as
// a cluster keeps to one group of SMs.  Asked once per device; 0, and no error left behind, where that fails.
static int cluster_slots(int parts) {
    static AskedOnce asked[2];
    static bool raised[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return cudaGetLastError(), 0;
    return asked[parts == 4].get(dev, [parts] {
        const auto kernel = matmul_i8_tile_kernel<CMPQ_BF16, kPlain, kSplit, false>;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = parts, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(parts * sm_count()), cfg.blockDim = dim3(kMmThreads), cfg.dynamicSmemBytes = kTileSmem;
        cfg.attrs = &attr, cfg.numAttrs = 1;
        int n = 0;
        if (raise_smem_limit_once(kernel, kTileSmem, raised) && cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess) return n;
        cudaGetLastError();  // not the launch's that comes next, which does without clusters
        return 0;
    });
}

template <int DT, int KIND>
static cmpq_status launch_kind(const TokenCodes& x, int64_t d_in, const Weight8& w, const Weight8* u, ProductArgs a, bool behind, cudaStream_t st) {
    const int sms = sm_count();
    if (sms <= 0) return CMPQ_ERR_CUDA;  // no device to plan for
    a.kblocks = (int)((d_in + 127) / 128);
    a.wide = aligned_to(a.y, 16) && a.ldy % 8 == 0;
    a.wide_residual = aligned_to(a.residual, 16) && a.ldr % 8 == 0;
    a.cols = (KIND == kGated ? 2 : 1) * (int64_t)a.d_out;
    const ProductPlan plan = plan_product({a.n, a.cols, a.kblocks, sms}, cluster_slots);
    const bool pair = plan.pair;
    const int parts = plan.parts;
    a.bn = plan.bn, a.rows = plan.rows;
    CUtensorMap wmap, umap, xmap;
    const int box = pair || KIND == kGated ? a.bn / 2 : a.bn, channels = KIND == kGated ? a.bn / 2 : a.bn;
    if (!make_byte_map(&wmap, w.codes, a.d_out, d_in, w.ld, box) || !make_byte_map(&xmap, x.codes, a.n, d_in, x.ld, a.rows)) return CMPQ_ERR_CUDA;
    umap = wmap;
    if (u && !make_byte_map(&umap, u->codes, a.d_out, d_in, u->ld, box)) return CMPQ_ERR_CUDA;
    a.n_tiles = (a.d_out + channels - 1) / channels;
    static bool raised[6][64];
    if (pair) {
        a.m_tiles = (a.n + 255) / 256;
        if (!raise_smem_limit_once(matmul_i8_pair_kernel<DT, KIND>, kPairSmem, raised[0])) return CMPQ_ERR_CUDA;
        const int64_t tiles = (int64_t)a.m_tiles * a.n_tiles;
        return launch_cluster(matmul_i8_pair_kernel<DT, KIND>, 2 * (unsigned)std::min<int64_t>(tiles, sms / 2), kMmThreads, kPairSmem, 2, behind,
                              st, wmap, umap, xmap, a);
    }
    a.m_tiles = (a.n + 127) / 128;
    // one block to an SM: two that share it were slower at every size, their rounds and tails cost more than they hide
    const int64_t blocks = (int64_t)a.m_tiles * a.n_tiles;
    a.slices = parts > 1 ? parts : plan.slices;
    a.kblocks = (a.kblocks + a.slices - 1) / a.slices;
    a.per_stage = plan.per_stage;
    const int slices = plan.slices, block = slices * (a.rows + a.bn) * 128;
    const size_t stage = a.per_stage * block, slack = (128 - slices * a.rows) * 128 + 1024;
    a.stages = std::min({(int)((kTileSmem - slack) / stage), kMmMaxStages, (a.kblocks + a.per_stage - 1) / a.per_stage});
    if (blocks * parts > INT32_MAX) return CMPQ_ERR_UNSUPPORTED;
    const size_t exchange = (parts - 1) * 128 * (a.bn / parts + 4) * 4 + 1024;
    const auto launch = [&](auto kernel, bool (&done)[64]) {
        if (!raise_smem_limit_once(kernel, kTileSmem, done)) return CMPQ_ERR_CUDA;
        return launch_cluster(kernel, (unsigned)blocks * parts, kMmThreads, std::max(a.stages * stage + slack, exchange), parts, behind, st, wmap, umap, xmap, a);
    };
    const bool one = a.per_stage == 1;
    if (parts > 1) return one ? launch(matmul_i8_tile_kernel<DT, KIND, kSplit, true>, raised[5]) : launch(matmul_i8_tile_kernel<DT, KIND, kSplit, false>, raised[3]);
    if (a.slices > 1) return launch(matmul_i8_tile_kernel<DT, KIND, kSliced, false>, raised[1]);
    return one ? launch(matmul_i8_tile_kernel<DT, KIND, kWhole, true>, raised[4]) : launch(matmul_i8_tile_kernel<DT, KIND, kWhole, false>, raised[2]);
}

template <int DT>
static cmpq_status launch_product(const TokenCodes& x, int64_t n, int64_t d_in, const Weight8& w, int64_t d_out, const Weight8* u, const Finish& f,
                                  void* y, int64_t ldy, int32_t* word, bool behind, cudaStream_t st) {
    ProductArgs a = {};
    a.xs = x.scale, a.ws = w.scale;
    a.bias = static_cast<const uint16_t*>(w.bias);
    a.y = static_cast<uint16_t*>(y);
    a.ldy = ldy;
    a.residual = static_cast<const uint16_t*>(f.residual);
    a.ldr = f.ldr, a.act = f.act;
    a.n = (int)n, a.d_out = (int)d_out;
    a.failed = word;
    if (u) {
        a.us = u->scale;
        a.ubias = static_cast<const uint16_t*>(u->bias);
        return launch_kind<DT, kGated>(x, d_in, w, u, a, behind, st);
    }
    return f.act == CMPQ_ACT_NONE && !f.residual ? launch_kind<DT, kPlain>(x, d_in, w, nullptr, a, behind, st)
                                                 : launch_kind<DT, kFinish>(x, d_in, w, nullptr, a, behind, st);
}

cmpq_status enqueue_product(const TokenCodes& x, cmpq_dtype dt, int64_t n, int64_t d_in, const Weight8& w, int64_t d_out, const Weight8* u,
                            const Finish& f, void* y, int64_t ldy, int32_t* word, bool behind, cudaStream_t st) {
    return dt == CMPQ_BF16 ? launch_product<CMPQ_BF16>(x, n, d_in, w, d_out, u, f, y, ldy, word, behind, st)
                           : launch_product<CMPQ_F16>(x, n, d_in, w, d_out, u, f, y, ldy, word, behind, st);
}

template <int DT>
static cmpq_status launch_quantize(const uint16_t* x, int64_t n, int64_t d, int64_t ldx, const uint16_t* norm, float eps, int8_t* codes, int64_t ldc,
                                   float* scale, int32_t* word, int32_t* clear, cudaStream_t st) {
    const int wide = aligned_to(x, 16) && ldx % 8 == 0;
    const int64_t keep = (d + 8 * kQtThreads - 1) / (8 * kQtThreads);
    const unsigned rows = (unsigned)n;
    auto plain = [&](auto kernel, int threads) { return launch_cluster(kernel, rows, threads, 0, 1, false, st, x, d, ldx, wide, codes, ldc, scale, word, clear); };
    auto normed = [&](auto kernel) {
        return launch_cluster(kernel, rows, kQtThreads, 0, 1, false, st, x, d, ldx, wide, RowNorm{norm, aligned_to(norm, 16), eps}, codes, ldc, scale, word, clear);
    };
    if (norm)
        return keep <= 2   ? normed(norm_quantize_kernel<DT, 2>)
               : keep <= 4 ? normed(norm_quantize_kernel<DT, 4>)
                           : normed(norm_quantize_kernel<DT, 8>);
    return keep <= 2   ? plain(quantize_tokens_kernel<DT, 2>, kQtThreads)
           : keep <= 4 ? plain(quantize_tokens_kernel<DT, 4>, kQtThreads)
           : keep <= 8 ? plain(quantize_tokens_kernel<DT, 8>, kQtThreads)
                       : plain(quantize_tokens_kernel<DT, 8, 2 * kQtThreads>, 2 * kQtThreads);
}

cmpq_status enqueue_quantize(const void* X, cmpq_dtype dt, int64_t n, int64_t d, int64_t ldx, const void* norm, float eps, int8_t* codes, int64_t ldc,
                             float* scale, int32_t* word, int32_t* clear, cudaStream_t st) {
    const auto *x = static_cast<const uint16_t*>(X), *g = static_cast<const uint16_t*>(norm);
    return dt == CMPQ_BF16 ? launch_quantize<CMPQ_BF16>(x, n, d, ldx, g, eps, codes, ldc, scale, word, clear, st)
                           : launch_quantize<CMPQ_F16>(x, n, d, ldx, g, eps, codes, ldc, scale, word, clear, st);
}

size_t linear_i8_codes_bytes(int64_t n, int64_t d_in) { return round_up((size_t)n * round_up(d_in, 16), 256); }

}  // namespace cmpq

using namespace cmpq;

extern "C" size_t cmpq_linear_i8_ws_bytes(int64_t n, int64_t d_in, int64_t d_out) {
    if (!linear_sizes_ok(n, d_in, d_out)) return 0;
    return linear_i8_codes_bytes(n, d_in) + round_up((size_t)n * sizeof(float), 256) + 256;
}

extern "C" cmpq_status cmpq_norm_quantize_tokens(const void* X, cmpq_dtype dt, int64_t n, int64_t d, int64_t ldx, const void* norm, float eps,
                                                 int8_t* codes, int64_t ldc, float* scale, int32_t* nonfinite, void* stream) {
    if (dt != CMPQ_F16 && dt != CMPQ_BF16) return CMPQ_ERR_INVALID_ARG;
    if (n < 0 || n > INT32_MAX || d < 1 || d > CMPQ_MAX_D_IN || ldx < d || ldc < d || ldc % 16 || !norm_ok(norm, eps)) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!X || !codes || !scale || !aligned_to(X, 2) || !aligned_to(codes, 16) || !aligned_to(scale, 4)) return CMPQ_ERR_INVALID_ARG;
    return enqueue_quantize(X, dt, n, d, ldx, norm, eps, codes, ldc, scale, nonfinite, nullptr, static_cast<cudaStream_t>(stream));
}

extern "C" cmpq_status cmpq_quantize_tokens(const void* X, cmpq_dtype dt, int64_t n, int64_t d, int64_t ldx,
                                            int8_t* codes, int64_t ldc, float* scale, int32_t* nonfinite,
                                            void* stream) {
    return cmpq_norm_quantize_tokens(X, dt, n, d, ldx, nullptr, 0.0f, codes, ldc, scale, nonfinite, stream);
}

// Where a call without a word of the caller's keeps the mark of a kernel that gave up; it starts from 0 in every call.
static int32_t* mark_of(void* ws, int64_t n, int64_t d_in, int64_t d_out) {
    return reinterpret_cast<int32_t*>(static_cast<char*>(ws) + cmpq_linear_i8_ws_bytes(n, d_in, d_out) - 256);
}

extern "C" cmpq_status cmpq_matmul_i8(const int8_t* xc, int64_t ldxc, const float* xs, const int8_t* wc, int64_t ldwc,
                                      const float* w_scale, const void* bias, cmpq_dtype dt, int64_t n, int64_t d_in,
                                      int64_t d_out, void* y, int64_t ldy, void* ws, size_t ws_bytes, void* stream) {
    const cmpq_weight_i8 w = {wc, ldwc, w_scale, bias};
    if (dt != CMPQ_F16 && dt != CMPQ_BF16) return CMPQ_ERR_INVALID_ARG;
    if (!linear_sizes_ok(n, d_in, d_out) || ldxc < d_in || ldxc % 16 || ldy < d_out || !weight_rows_ok(w, d_in)) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!xc || !xs || !y || !weight_ok(w) || !aligned_to(xc, 16) || !aligned_to(xs, 4) || !aligned_to(y, 2)) return CMPQ_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < cmpq_linear_i8_ws_bytes(n, d_in, d_out)) return CMPQ_ERR_WORKSPACE;
    int32_t* mark = mark_of(ws, n, d_in, d_out);
    if (cudaMemsetAsync(mark, 0, sizeof(*mark), static_cast<cudaStream_t>(stream)) != cudaSuccess) return CMPQ_ERR_CUDA;
    return enqueue_product({xc, ldxc, xs}, dt, n, d_in, w, d_out, nullptr, {}, y, ldy, mark, false, static_cast<cudaStream_t>(stream));
}

extern "C" cmpq_status cmpq_linear_i8_fused(const void* X, cmpq_dtype dt, int64_t n, int64_t d_in, int64_t ldx, const void* norm, float eps,
                                            const cmpq_weight_i8* weight, int64_t d_out, cmpq_act act, const void* residual, int64_t ldr, void* y,
                                            int64_t ldy, int32_t* nonfinite, void* ws, size_t ws_bytes, void* stream) {
    if (!weight || !linear_sizes_ok(n, d_in, d_out) || !weight_rows_ok(*weight, d_in) || ldy < d_out || ldx < d_in) return CMPQ_ERR_INVALID_ARG;
    if ((dt != CMPQ_F16 && dt != CMPQ_BF16) || !norm_ok(norm, eps) || !finish_ok(act, residual, ldr, d_out)) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!X || !y || !weight_ok(*weight) || !aligned_to(X, 2) || !aligned_to(y, 2)) return CMPQ_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < cmpq_linear_i8_ws_bytes(n, d_in, d_out)) return CMPQ_ERR_WORKSPACE;
    Workspace w(ws, ws_bytes);
    int8_t* codes = w.take<int8_t>(linear_i8_codes_bytes(n, d_in));
    float* scale = w.take<float>(n);
    const int64_t ldc = (int64_t)round_up(d_in, 16);
    int32_t* mark = mark_of(ws, n, d_in, d_out);
    const auto st = static_cast<cudaStream_t>(stream);
    // One launch for few tokens, whose blocks read all of X and write y without waiting for one another: apart, then.
    const auto *x0 = static_cast<const uint16_t*>(X), *y0 = static_cast<const uint16_t*>(y);
    if (n <= kFewTokens && few_fits(d_in) && (x0 + (n - 1) * ldx + d_in <= y0 || y0 + (n - 1) * ldy + d_out <= x0)) {
        if (!nonfinite && cudaMemsetAsync(mark, 0, sizeof(*mark), st) != cudaSuccess) return CMPQ_ERR_CUDA;
        return enqueue_few(X, dt, n, d_in, ldx, norm, eps, *weight, d_out, nullptr, {act, residual, ldr}, y, ldy, nonfinite, nonfinite ? nonfinite : mark,
                           false, st);
    }
    const cmpq_status s = enqueue_quantize(X, dt, n, d_in, ldx, norm, eps, codes, ldc, scale, nonfinite, nonfinite ? nullptr : mark, st);
    if (s != CMPQ_OK) return s;
    // the quantization lets the product start early; it was itself started after everything before it, the weights too
    return enqueue_product({codes, ldc, scale}, dt, n, d_in, *weight, d_out, nullptr, {act, residual, ldr}, y, ldy, nonfinite ? nonfinite : mark, true, st);
}

extern "C" cmpq_status cmpq_linear_i8(const void* X, cmpq_dtype dt, int64_t n, int64_t d_in, int64_t ldx, const int8_t* wc,
                                      int64_t ldwc, const float* w_scale, const void* bias, int64_t d_out, void* y, int64_t ldy,
                                      int32_t* nonfinite, void* ws, size_t ws_bytes, void* stream) {
    const cmpq_weight_i8 w = {wc, ldwc, w_scale, bias};
    return cmpq_linear_i8_fused(X, dt, n, d_in, ldx, nullptr, 0.0f, &w, d_out, CMPQ_ACT_NONE, nullptr, 0, y, ldy, nonfinite, ws, ws_bytes, stream);
}
