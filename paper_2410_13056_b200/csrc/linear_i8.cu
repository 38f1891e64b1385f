// 8-bit linear layers: quantization of tokens and the integer product with scales per token and channel.
#include "cache.cuh"

namespace cmpq {

constexpr int kQtThreads = 256;
constexpr int kQtKeep = 8;  // groups of eight elements a thread keeps in registers between the two passes

template <int DT>
__device__ __forceinline__ uint32_t group_max(uint4 g) {
    uint32_t m = 0;
    const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = widen16x2<DT>(w[i]);
        m = max(m, max(__float_as_uint(f.x) & 0x7fffffffu, __float_as_uint(f.y) & 0x7fffffffu));
    }
    return m;
}

template <int DT>
__device__ __forceinline__ uint2 group_codes(uint4 g, float inv) {
    const uint32_t w[4] = {g.x, g.y, g.z, g.w};
    uint32_t c[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = widen16x2<DT>(w[i]);
        c[i >> 1] |= (code_of(f.x, inv) | code_of(f.y, inv) << 8) << (16 * (i & 1));
    }
    return make_uint2(c[0], c[1]);
}

// One block per token.  The magnitudes are compared as bit patterns, where a NaN is larger than infinity and
// infinity larger than every number, so the maximum also tells whether the row is finite.  A thread keeps its
// first kQtKeep groups in registers (rows of up to 16384 entries are read once); longer rows are read again.
template <int DT>
__global__ void __launch_bounds__(kQtThreads)
quantize_tokens_kernel(const uint16_t* __restrict__ X, int64_t d, int64_t ldx, int wide, int8_t* __restrict__ codes,
                       int64_t ldc, float* __restrict__ scale, int32_t* __restrict__ nonfinite) {
    const uint16_t* row = X + blockIdx.x * ldx;
    int8_t* out = codes + blockIdx.x * ldc;
    const int t = threadIdx.x;
    const int64_t groups = (d + 15) / 16 * 2;  // the codes' padding up to 16 is written too
    uint4 keep[kQtKeep];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kQtKeep; ++i) {
        const int64_t g = t + (int64_t)i * kQtThreads;
        keep[i] = make_uint4(0u, 0u, 0u, 0u);
        if (g < groups) keep[i] = load8(row + 8 * g, d - 8 * g, wide);
    }
#pragma unroll
    for (int i = 0; i < kQtKeep; ++i) m = max(m, group_max<DT>(keep[i]));
    for (int64_t g = t + (int64_t)kQtKeep * kQtThreads; g < groups; g += kQtThreads)
        m = max(m, group_max<DT>(load8(row + 8 * g, d - 8 * g, wide)));
    __shared__ uint32_t part[kQtThreads / 32];
    m = __reduce_max_sync(0xffffffffu, m);
    if ((t & 31) == 0) part[t >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQtThreads / 32; ++i) m = max(m, part[i]);
    const float amax = __uint_as_float(m);
    float s = amax * (1.0f / 127.0f), inv = 1.0f / s;
    if (amax < 0x1p-120f) s = inv = 0.0f;
    if (t == 0) {
        scale[blockIdx.x] = s;
        if (m >= 0x7f800000u && nonfinite) atomicOr(nonfinite, 1);
    }
#pragma unroll
    for (int i = 0; i < kQtKeep; ++i) {
        const int64_t g = t + (int64_t)i * kQtThreads;
        if (g < groups) *reinterpret_cast<uint2*>(out + 8 * g) = group_codes<DT>(keep[i], inv);
    }
    for (int64_t g = t + (int64_t)kQtKeep * kQtThreads; g < groups; g += kQtThreads)
        *reinterpret_cast<uint2*>(out + 8 * g) = group_codes<DT>(load8(row + 8 * g, d - 8 * g, wide), inv);
}

// Plain tiled product on the integer dot-product instruction: 64 x 64 outputs a block, 64 bytes of the sum at a
// time.
template <int DT>
__global__ void __launch_bounds__(256)
matmul_i8_kernel(const int8_t* __restrict__ xc, int64_t ldxc, const float* __restrict__ xs,
                 const int8_t* __restrict__ wc, int64_t ldwc, const float* __restrict__ ws,
                 const uint16_t* __restrict__ bias, int64_t n, int64_t d_in, int64_t d_out, uint16_t* __restrict__ y,
                 int64_t ldy) {
    __shared__ int a[64][17], b[64][17];
    const int64_t t0 = (int64_t)blockIdx.y * 64, o0 = (int64_t)blockIdx.x * 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int acc[4][4] = {};
    for (int64_t k = 0; k < d_in; k += 64) {
        for (int i = threadIdx.x; i < 64 * 16; i += 256) {
            const int r = i >> 4, w = i & 15;
            const int64_t j = k + 4 * w;
            int va = 0, vb = 0;
            if (j < d_in) {
                const int keep = d_in - j >= 4 ? -1 : (1 << (8 * (int)(d_in - j))) - 1;
                if (t0 + r < n) va = *reinterpret_cast<const int*>(xc + (t0 + r) * ldxc + j) & keep;
                if (o0 + r < d_out) vb = *reinterpret_cast<const int*>(wc + (o0 + r) * ldwc + j) & keep;
            }
            a[r][w] = va;
            b[r][w] = vb;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 16; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(a[ty + 16 * i][w], b[tx + 16 * j][w], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t t = t0 + ty + 16 * i, o = o0 + tx + 16 * j;
            if (t >= n || o >= d_out) continue;
            float v = (float)acc[i][j] * xs[t] * ws[o];
            if (bias) v += widen16<DT>(bias[o]);
            y[t * ldy + o] = round16<DT>(v);
        }
}

size_t linear_i8_codes_bytes(int64_t n, int64_t d_in) { return round_up((size_t)n * round_up(d_in, 16), 256); }

}  // namespace cmpq

using namespace cmpq;

static bool linear_sizes_ok(int64_t n, int64_t d_in, int64_t d_out) {
    return n >= 0 && n <= INT32_MAX && d_in >= 1 && d_in <= CMPQ_MAX_D_IN_I8 && d_out >= 1 && d_out <= CMPQ_MAX_D_IN;
}

extern "C" size_t cmpq_linear_i8_ws_bytes(int64_t n, int64_t d_in, int64_t d_out) {
    if (!linear_sizes_ok(n, d_in, d_out)) return 0;
    return linear_i8_codes_bytes(n, d_in) + round_up((size_t)n * sizeof(float), 256) + 256;
}

extern "C" cmpq_status cmpq_quantize_tokens(const void* X, cmpq_dtype dt, int64_t n, int64_t d, int64_t ldx,
                                            int8_t* codes, int64_t ldc, float* scale, int32_t* nonfinite,
                                            void* stream) {
    if (dt != CMPQ_F16 && dt != CMPQ_BF16) return CMPQ_ERR_INVALID_ARG;
    if (n < 0 || n > INT32_MAX || d < 1 || d > CMPQ_MAX_D_IN || ldx < d || ldc < d || ldc % 16) return CMPQ_ERR_INVALID_ARG;
    if (n == 0) return CMPQ_OK;
    if (!X || !codes || !scale || !aligned_to(X, 2) || !aligned_to(codes, 16) || !aligned_to(scale, 4)) return CMPQ_ERR_INVALID_ARG;
    const int wide = aligned_to(X, 16) && ldx % 8 == 0;
    const auto* x = static_cast<const uint16_t*>(X);
    auto st = static_cast<cudaStream_t>(stream);
    if (dt == CMPQ_BF16)
        quantize_tokens_kernel<CMPQ_BF16><<<(unsigned)n, kQtThreads, 0, st>>>(x, d, ldx, wide, codes, ldc, scale, nonfinite);
    else
        quantize_tokens_kernel<CMPQ_F16><<<(unsigned)n, kQtThreads, 0, st>>>(x, d, ldx, wide, codes, ldc, scale, nonfinite);
    return launch_status();
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
    const dim3 grid((unsigned)((d_out + 63) / 64), (unsigned)((n + 63) / 64));
    auto st = static_cast<cudaStream_t>(stream);
    const auto* b = static_cast<const uint16_t*>(bias);
    auto* out = static_cast<uint16_t*>(y);
    if (dt == CMPQ_BF16)
        matmul_i8_kernel<CMPQ_BF16><<<grid, 256, 0, st>>>(xc, ldxc, xs, wc, ldwc, w_scale, b, n, d_in, d_out, out, ldy);
    else
        matmul_i8_kernel<CMPQ_F16><<<grid, 256, 0, st>>>(xc, ldxc, xs, wc, ldwc, w_scale, b, n, d_in, d_out, out, ldy);
    return launch_status();
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
    cmpq_status st = cmpq_quantize_tokens(X, dt, n, d_in, ldx, codes, ldc, scale, nonfinite, stream);
    if (st != CMPQ_OK) return st;
    return cmpq_matmul_i8(codes, ldc, scale, wc, ldwc, w_scale, bias, dt, n, d_in, d_out, y, ldy, ws, ws_bytes, stream);
}
