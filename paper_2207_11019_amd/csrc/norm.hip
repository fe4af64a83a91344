// Layer normalisation over the channels of a row (a position of a sample), with trainable weight and bias:
//   mu = sum_c x / C,  r = 1 / sqrt(sum_c (x - mu)^2 / C + eps),  h = (x - mu) r,  y = gamma h + beta                     (forward)
//   g = dy gamma,  dx = r (g - mean_c g - h mean_c(g h)),  dgamma = sum over rows of dy h,  dbeta = sum over rows of dy    (backward)
// Both passes are bound by HBM: a row is read once into registers -- by 4 to 64 lanes of a wavefront or by a whole block, by its length -- and
// everything that the formulas ask of it is taken from there, the variance as the mean of squared differences.  All sums are float.  The input
// is there again in the backward pass, or its checkpoint in 8 bits is, which the forward pass stores on its way: the same bytes as lpm_ckpt8_pack.
// dgamma and dbeta: a thread adds up its channels over the rows it meets, a block its threads, a second kernel the blocks, each in an order
// that only the sizes decide (no atomics).  The next row's loads are under way while a row is summed up.  Measured, forward and backward with its columns: 65536 x 2048
// bf16 with checkpoints 126 us (5.4 TB/s) and 225 + 5 (3.6), 8192 x 1024 bf16 10.3 and 13 + 4, 10007 x 515 float 18 and 21 + 4 (without the loads ahead: 211 and
// 270 + 18, 13 and 16 + 20, 16 and 19 + 20).
#include "chunk.h"
#include "lpm_internal.h"
#include <initializer_list>

using namespace lpm;

namespace lpm {

constexpr int norm_threads(int g) { return g < 256 ? 256 : g; }      // of a block, with G threads a row
constexpr int NORM_MAX_C = 16384;          // what a block of 512 threads keeps in registers, 32 channels a thread

// Sums of N values over the G threads of a row; `red` holds N values per wavefront where the row is the block's.
template <int G, int N>
__device__ __forceinline__ void norm_sum(float (&a)[N], float* red) {
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = group_sum<(G < 64 ? G : 64)>(a[i]);
    if (G > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();                   // (the values of the sum before have been read)
#pragma unroll
        for (int i = 0; i < N; ++i) if ((threadIdx.x & 63) == 0) red[N * wave + i] = a[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a[i] = red[i];
#pragma unroll
            for (int w = 1; w < G / 64; ++w) a[i] += red[N * w + i];
        }
    }
}

// CH chunks of eight channels a thread: chunk k of thread t of the row's G is channel 8 (t + G k)
template <typename T, int G, int CH>
__global__ void __launch_bounds__(norm_threads(G)) norm_fwd_kernel(int64_t rows, int C, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                float eps, T* y, float* __restrict__ stats, uint8_t* __restrict__ q, uint8_t* __restrict__ ex) {
    constexpr int RB = norm_threads(G) / G;
    __shared__ float red[16];
    const int t = threadIdx.x % G, sub = threadIdx.x / G;
    float w[CH][8], b[CH][8];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = 8 * (t + G * k);
        if (gamma) chunk_values(ld_raw(gamma, c, C), c, C, true, w[k]);
        if (beta) chunk_values(ld_raw(beta, c, C), c, C, true, b[k]);
    }
    RawChunk<T> raw[CH];                   // the next row's
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        const T* xr = x + (row < rows ? row : 0) * C;
#pragma unroll
        for (int k = 0; k < CH; ++k) raw[k] = ld_raw(xr, 8 * (t + G * k), C);
    };
    load((int64_t)blockIdx.x * RB + sub);
    for (int64_t r0 = (int64_t)blockIdx.x * RB; r0 < rows; r0 += (int64_t)gridDim.x * RB) {
        const int64_t row = r0 + sub;
        const bool there = row < rows;
        float v[CH][8];
        float s[1] = {0.f};
#pragma unroll
        for (int k = 0; k < CH; ++k) chunk_values(raw[k], 8 * (t + G * k), C, there, v[k]);
        if (r0 + (int64_t)gridDim.x * RB < rows) load(row + (int64_t)gridDim.x * RB);
        if (q) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int c = 8 * (t + G * k), n = there ? C - c : 0;
                uint32_t top = chunk_top(v[k]);
                for (int o = 1; o < 4; o <<= 1) { const uint32_t a = (uint32_t)__shfl_xor((int)top, o, 64); top = a > top ? a : top; }
                const uint32_t byte = ckpt_byte(top);
                if (n > 0) st_bytes8(q + row * C + c, n, ckpt_quantise(v[k], byte));
                if (n > 0 && c % CKPT_BLOCK == 0) ex[row * ckpt_blocks(C) + c / CKPT_BLOCK] = (uint8_t)byte;
            }
        }
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += v[k][e];
        norm_sum<G>(s, red);
        const float mu0 = s[0] / (float)C;
        // what is left of the mean after the rounding of its sum comes with the squares: a row of equal elements has no variance
        float d2[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int n = C - 8 * (t + G * k);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = e < n ? v[k][e] - mu0 : 0.f;
                d2[0] += d;
                d2[1] = fmaf(d, d, d2[1]);
            }
        }
        norm_sum<G>(d2, red);
        const float rest = d2[0] / (float)C, mu = mu0 + rest;
        const float rs = rsqrtf(fmaxf(d2[1] / (float)C - rest * rest, 0.f) + eps);
        if (stats && t == 0 && there) { stats[2 * row] = mu; stats[2 * row + 1] = rs; }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (t + G * k), n = there ? C - c : 0;
            if (n <= 0) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float h = (v[k][e] - mu) * rs;
                if (gamma) h *= w[k][e];
                v[k][e] = beta ? h + b[k][e] : h;
            }
            st_chunk(y + row * C + c, n, v[k]);
        }
    }
}

// part (NULL: no weight gradients): [gridDim.x][2][C], the block's sums of dy h and of dy
template <typename T, int G, int CH, bool KEPT>
__global__ void __launch_bounds__(norm_threads(G)) norm_bwd_kernel(int64_t rows, int C, const T* x, const uint8_t* __restrict__ q, const uint8_t* __restrict__ ex,
                                                                const float* __restrict__ stats, const T* dy, const float* gamma, T* dx,
                                                                int accumulate, float* __restrict__ part) {
    constexpr int RB = norm_threads(G) / G;
    __shared__ float red[16];
    const int t = threadIdx.x % G, sub = threadIdx.x / G;
    const float inv = 1.f / (float)C;
    constexpr bool AHEAD = G < 512;        // (of the longest rows there is no room for two, nor for the weights)
    float dg[CH][8], db[CH][8], w[CH][8];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = 8 * (t + G * k);
        if (AHEAD && gamma) chunk_values(ld_raw(gamma, c, C), c, C, true, w[k]);
#pragma unroll
        for (int e = 0; e < 8; ++e) dg[k][e] = db[k][e] = 0.f;
    }
    // the next row's
    RawChunk<T> raw_g[CH], raw_x[KEPT ? 1 : CH];
    uint2 raw_q[KEPT ? CH : 1];
    uint32_t raw_e[KEPT ? CH : 1];
    float raw_mu, raw_rs;
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        const int64_t from = row < rows ? row : 0;
        raw_mu = stats[2 * from];
        raw_rs = stats[2 * from + 1];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (t + G * k);
            raw_g[k] = ld_raw(dy + from * C, c, C);
            if constexpr (KEPT) {
                raw_q[k] = ld_bytes8(q + from * C + (c < C ? c : 0), c < C ? C - c : 0);
                raw_e[k] = ex[from * ckpt_blocks(C) + (c < C ? c / CKPT_BLOCK : 0)];
            } else {
                raw_x[k] = ld_raw(x + from * C, c, C);
            }
        }
    };
    if (AHEAD) load((int64_t)blockIdx.x * RB + sub);
    for (int64_t r0 = (int64_t)blockIdx.x * RB; r0 < rows; r0 += (int64_t)gridDim.x * RB) {
        const int64_t row = r0 + sub;
        const bool there = row < rows;
        const int64_t base = (there ? row : 0) * C;
        if (!AHEAD) load(row);
        const float mu = raw_mu, rs = raw_rs;
        float h[CH][8], g[CH][8];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (t + G * k);
            chunk_values(raw_g[k], c, C, there, g[k]);
            if constexpr (KEPT) ckpt_values(raw_q[k], raw_e[k], h[k]);
            else chunk_values(raw_x[k], c, C, there, h[k]);
        }
        if (AHEAD && r0 + (int64_t)gridDim.x * RB < rows) load(row + (int64_t)gridDim.x * RB);
        float sums[2] = {0.f, 0.f};             // of g and of g h
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (t + G * k), n = there ? C - c : 0;
            if (!AHEAD && gamma) chunk_values(ld_raw(gamma, c, C), c, C, true, w[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[k][e] = e < n ? (h[k][e] - mu) * rs : 0.f;
                if (part) { dg[k][e] = fmaf(g[k][e], h[k][e], dg[k][e]); db[k][e] += g[k][e]; }
                if (gamma) g[k][e] *= w[k][e];
                sums[0] += g[k][e];
                sums[1] = fmaf(g[k][e], h[k][e], sums[1]);
            }
        }
        norm_sum<G>(sums, red);
        const float mg = sums[0] * inv, mgh = sums[1] * inv;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = 8 * (t + G * k), n = there ? C - c : 0;
            if (n <= 0) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = rs * (g[k][e] - mg - h[k][e] * mgh);
            if (accumulate) {
                float old[8];
                chunk_values(ld_raw(dx + base, c, C), c, C, true, old);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += old[e];
            }
            st_chunk(dx + base + c, n, v);
        }
    }
    if (!part) return;
    float* out = part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = which ? db[k][e] : dg[k][e];
            const int c = 8 * (t + G * k);
            if (G <= 64) {                 // rows of other lanes, then of the other wavefronts
                const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
                for (int o = G; o < 64; o <<= 1)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += __shfl_xor(v[e], o, 64);
                __shared__ float over[4 * 64 * 8];
                __syncthreads();
#pragma unroll
                for (int e = 0; e < 8; ++e) over[(wave * 8 + e) * 64 + lane] = v[e];
                __syncthreads();
                if (threadIdx.x < G && c < C) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = (over[e * 64 + lane] + over[(8 + e) * 64 + lane]) + (over[(16 + e) * 64 + lane] + over[(24 + e) * 64 + lane]);
                    st_chunk(out + which * C + c, C - c, v);
                }
            } else if (c < C) {
                st_chunk(out + which * C + c, C - c, v);
            }
        }
    }
}

// dst[c] (+)= the sum over blocks of part[block][c], for the 2 C columns (dgamma, then dbeta): a block has 16 columns, sixteen threads share one, each its
// sixteenth of the blocks, eight loads at a time
__global__ void __launch_bounds__(256) norm_columns_kernel(const float* __restrict__ part, int blocks, int C, float* __restrict__ dgamma, float* __restrict__ dbeta,
                                                           int accumulate) {
    __shared__ float sums[16][17];
    const int lane = threadIdx.x & 15, share = threadIdx.x >> 4, col = blockIdx.x * 16 + lane, from = min(col, 2 * C - 1);
    float s = 0.f;
    for (int b = share; b < blocks; b += 128) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = part[(int64_t)min(b + 16 * k, blocks - 1) * 2 * C + from];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += b + 16 * k < blocks ? v[k] : 0.f;
    }
    sums[share][lane] = s;
    __syncthreads();
    if (share || col >= 2 * C) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) s += sums[k][lane];
    float* dst = col < C ? dgamma : dbeta;
    if (!dst) return;
    const int c = col < C ? col : col - C;
    dst[c] = accumulate ? dst[c] + s : s;
}

// Threads of a row and chunks a thread, for C channels: a lane has a chunk where the row fits a wavefront, then up to four (no barrier), then the block shares it
struct NormShape { int g, ch; };
static NormShape norm_shape(int C) {
    for (int g = 4; g <= 64; g *= 2) if (C <= 8 * g) return {g, 1};
    for (int ch = 2; ch <= 4; ch *= 2) if (C <= 512 * ch) return {64, ch};
    for (int ch = 2; ch <= 4; ch *= 2) if (C <= 2048 * ch) return {256, ch};
    return {512, 4};
}
// Blocks of the backward pass: each adds a line of 2 C floats to what the second kernel reads.  (At most 512, 768, 1024: 228, 242, 251 us for 65536 x 2048 kept in 8
// bits, 22, 27, 25 for 10007 x 515 float.)
static int norm_bwd_blocks(int64_t rows, int C) {
    const int per = norm_threads(norm_shape(C).g) / norm_shape(C).g;
    const int64_t b = (rows + per - 1) / per;
    return (int)(b < 512 ? b : 512);
}
#define LPM_NORM_SHAPE(C_, ...)                                                                  \
    do {                                                                                         \
        const NormShape sh__ = norm_shape(C_);                                                   \
        if (sh__.g == 4) { constexpr int G = 4, CH = 1; __VA_ARGS__; }                           \
        else if (sh__.g == 8) { constexpr int G = 8, CH = 1; __VA_ARGS__; }                      \
        else if (sh__.g == 16) { constexpr int G = 16, CH = 1; __VA_ARGS__; }                    \
        else if (sh__.g == 32) { constexpr int G = 32, CH = 1; __VA_ARGS__; }                    \
        else if (sh__.g == 64 && sh__.ch == 1) { constexpr int G = 64, CH = 1; __VA_ARGS__; }    \
        else if (sh__.g == 64 && sh__.ch == 2) { constexpr int G = 64, CH = 2; __VA_ARGS__; }    \
        else if (sh__.g == 64) { constexpr int G = 64, CH = 4; __VA_ARGS__; }                    \
        else if (sh__.ch == 2) { constexpr int G = 256, CH = 2; __VA_ARGS__; }                   \
        else if (sh__.g == 256) { constexpr int G = 256, CH = 4; __VA_ARGS__; }                   \
        else { constexpr int G = 512, CH = 4; __VA_ARGS__; }                                     \
    } while (0)

template <typename T>
static hipError_t norm_fwd(int64_t rows, int C, const T* x, const float* gamma, const float* beta, float eps, T* y, float* stats, uint8_t* q, uint8_t* ex,
                           hipStream_t st) {
    const int per = norm_threads(norm_shape(C).g) / norm_shape(C).g;
    const int64_t b = (rows + per - 1) / per;
    const dim3 grid((unsigned)(b < 2048 ? b : 2048));
    LPM_NORM_SHAPE(C, hipLaunchKernelGGL((norm_fwd_kernel<T, G, CH>), grid, dim3(norm_threads(G)), 0, st, rows, C, x, gamma, beta, eps, y, stats, q, ex));
    return hipGetLastError();
}
template <typename T>
static hipError_t norm_bwd(int64_t rows, int C, const T* x, const uint8_t* q, const uint8_t* ex, const float* stats, const T* dy, const float* gamma, T* dx,
                           int dx_acc, float* dgamma, float* dbeta, int accumulate, float* ws, hipStream_t st) {
    const bool sums = dgamma || dbeta;
    const int blocks = norm_bwd_blocks(rows, C);
    if (rows > 0)
        LPM_NORM_SHAPE(C, if (q) hipLaunchKernelGGL((norm_bwd_kernel<T, G, CH, true>), dim3((unsigned)blocks), dim3(norm_threads(G)), 0, st, rows, C, x, q, ex, stats,
                                                    dy, gamma, dx, dx_acc, sums ? ws : nullptr);
                          else hipLaunchKernelGGL((norm_bwd_kernel<T, G, CH, false>), dim3((unsigned)blocks), dim3(norm_threads(G)), 0, st, rows, C, x, q, ex, stats,
                                                  dy, gamma, dx, dx_acc, sums ? ws : nullptr));
    if (sums) hipLaunchKernelGGL(norm_columns_kernel, dim3((unsigned)((2 * C + 15) / 16)), dim3(256), 0, st, (const float*)ws, blocks, C, dgamma, dbeta, accumulate);
    return hipGetLastError();
}

}  // namespace lpm

static int32_t norm_shape_check(int64_t rows, int32_t channels, int32_t dtype) {
    if (dtype != LPM_F32 && dtype != LPM_BF16) return fail(LPM_EINVAL, "dtype must be LPM_F32 or LPM_BF16");
    if (rows < 0 || channels <= 0 || channels > NORM_MAX_C || rows > ((int64_t)1 << 40) / channels)
        return fail(LPM_ESHAPE, "layer norm over %lld rows of %d channels (1 to %d)", (long long)rows, channels, NORM_MAX_C);
    return LPM_OK;
}
static bool norm_misaligned(std::initializer_list<const void*> ps) {
    for (const void* p : ps) if ((uintptr_t)p & 255u) return true;
    return false;
}

extern "C" int32_t lpm_norm_ws_bytes(int64_t rows, int32_t channels, int32_t dtype, size_t* bytes) {
    if (!bytes) return fail(LPM_EINVAL, "bytes is NULL");
    const int32_t rc = norm_shape_check(rows, channels, dtype);
    if (rc) return rc;
    *bytes = (size_t)norm_bwd_blocks(rows, channels) * 2 * channels * sizeof(float);
    return LPM_OK;
}

extern "C" int32_t lpm_norm_forward(int64_t rows, int32_t channels, int32_t dtype, const void* x, const float* gamma, const float* beta, float eps,
                                    void* y, float* stats, void* ckpt, void* stream) {
    const int32_t rc = norm_shape_check(rows, channels, dtype);
    if (rc) return rc;
    if (!(eps >= 0.f)) return fail(LPM_EINVAL, "eps must not be negative");
    if (rows == 0) return LPM_OK;
    if (!x || !y) return fail(LPM_EINVAL, "NULL argument");
    if (norm_misaligned({x, gamma, beta, y, stats, ckpt})) return fail(LPM_EALIGN, "device buffers must be 256-byte aligned");
    uint8_t* q = (uint8_t*)ckpt;
    uint8_t* ex = q ? q + ckpt_exponents_at(rows, channels) : nullptr;
    if (dtype == LPM_BF16)
        LPM_HIP(norm_fwd<bf16_t>(rows, channels, (const bf16_t*)x, gamma, beta, eps, (bf16_t*)y, stats, q, ex, (hipStream_t)stream));
    else
        LPM_HIP(norm_fwd<float>(rows, channels, (const float*)x, gamma, beta, eps, (float*)y, stats, q, ex, (hipStream_t)stream));
    return LPM_OK;
}

extern "C" int32_t lpm_norm_backward(int64_t rows, int32_t channels, int32_t dtype, const void* x, const void* ckpt, const float* stats, const void* dy,
                                     const float* gamma, void* dx, int32_t dx_accumulate, float* dgamma, float* dbeta, int32_t accumulate, void* ws,
                                     void* stream) {
    const int32_t rc = norm_shape_check(rows, channels, dtype);
    if (rc) return rc;
    if (rows > 0 && (!stats || !dy || !dx)) return fail(LPM_EINVAL, "NULL argument");
    if (rows > 0 && !x == !ckpt) return fail(LPM_EINVAL, "the input or its checkpoint, one of the two");
    if (rows > 0 && (dgamma || dbeta) && !ws) return fail(LPM_EINVAL, "scratch required");
    if (norm_misaligned({x, ckpt, stats, dy, gamma, dx, dgamma, dbeta, ws})) return fail(LPM_EALIGN, "device buffers must be 256-byte aligned");
    const uint8_t* q = (const uint8_t*)ckpt;
    const uint8_t* ex = q ? q + ckpt_exponents_at(rows, channels) : nullptr;
    if (dtype == LPM_BF16)
        LPM_HIP(norm_bwd<bf16_t>(rows, channels, (const bf16_t*)x, q, ex, stats, (const bf16_t*)dy, gamma, (bf16_t*)dx, dx_accumulate, dgamma, dbeta, accumulate,
                                 (float*)ws, (hipStream_t)stream));
    else
        LPM_HIP(norm_bwd<float>(rows, channels, (const float*)x, q, ex, stats, (const float*)dy, gamma, (float*)dx, dx_accumulate, dgamma, dbeta, accumulate,
                                (float*)ws, (hipStream_t)stream));
    return LPM_OK;
}
