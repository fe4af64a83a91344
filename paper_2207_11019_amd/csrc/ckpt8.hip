// Activation checkpoints in 8 bits: what a stash keeps of a tensor between F and B at half (a quarter) of its size, and the weight gradient
// that reads its layer's input from one.  The format is in chunk.h; a tensor is rows x channels, channels innermost.
#include "chunk.h"
#include "lpm_internal.h"

using namespace lpm;

namespace lpm {

// A thread has eight channels, four neighbours a block of 32, and every thread ITEMS such pieces, whose loads are all in flight before the first is
// used.  Bound: HBM; 100352 x 1000 bf16: pack 64 us (4.7 TB/s; 49 from the cache), unpack 51 (6.0).
constexpr int CKPT_ITEMS = 4, CKPT_THREADS = 256;

// The piece of item `at` of the block's items: row and first channel.  The block's first item is divided once, by all lanes alike; the rest are small.
struct CkptPlace { int64_t row0; int part0; int per; FastDiv div; };
__device__ __forceinline__ void ckpt_locate(const CkptPlace& b, int at, int64_t& row, int& c) {
    const int t = b.part0 + at, r = div_by(t, b.div);
    row = b.row0 + r;
    c = (t - r * b.per) * 8;
}

template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) ckpt_pack_kernel(int64_t rows, int C, FastDiv div, const T* __restrict__ x, uint8_t* __restrict__ q,
                                                                 uint8_t* __restrict__ ex) {
    const int per = ckpt_blocks(C) * 4;
    const int64_t first = (int64_t)blockIdx.x * (CKPT_ITEMS * CKPT_THREADS);
    CkptPlace b{first / per, 0, per, div};
    b.part0 = (int)(first - b.row0 * per);
    RawChunk<T> raw[CKPT_ITEMS];
    int64_t row[CKPT_ITEMS];
    int c[CKPT_ITEMS], n[CKPT_ITEMS];
#pragma unroll
    for (int i = 0; i < CKPT_ITEMS; ++i) {
        ckpt_locate(b, i * CKPT_THREADS + (int)threadIdx.x, row[i], c[i]);
        n[i] = row[i] < rows ? C - c[i] : 0;
        raw[i] = ld_raw(x + (row[i] < rows ? row[i] : 0) * C, c[i], C);
    }
#pragma unroll
    for (int i = 0; i < CKPT_ITEMS; ++i) {
        float v[8];
        chunk_values(raw[i], c[i], C, row[i] < rows, v);
        uint32_t top = chunk_top(v);
        for (int o = 1; o < 4; o <<= 1) { const uint32_t a = (uint32_t)__shfl_xor((int)top, o, 64); top = a > top ? a : top; }
        const uint32_t byte = ckpt_byte(top);
        if (n[i] > 0) st_bytes8(q + row[i] * C + c[i], n[i], ckpt_quantise(v, byte));
        if (n[i] > 0 && c[i] % CKPT_BLOCK == 0) ex[row[i] * ckpt_blocks(C) + c[i] / CKPT_BLOCK] = (uint8_t)byte;
    }
}

template <typename T, bool PAST>
__global__ void __launch_bounds__(CKPT_THREADS) ckpt_unpack_kernel(int64_t rows, int C, FastDiv div, const uint8_t* __restrict__ q,
                                                                   const uint8_t* __restrict__ ex, T* __restrict__ x) {
    const int per = ckpt_blocks(C) * 4;
    const int64_t first = (int64_t)blockIdx.x * (CKPT_ITEMS * CKPT_THREADS);
    CkptPlace b{first / per, 0, per, div};
    b.part0 = (int)(first - b.row0 * per);
    uint2 w[CKPT_ITEMS];
    uint32_t byte[CKPT_ITEMS];
    int64_t row[CKPT_ITEMS];
    int c[CKPT_ITEMS], n[CKPT_ITEMS];
#pragma unroll
    for (int i = 0; i < CKPT_ITEMS; ++i) {
        ckpt_locate(b, i * CKPT_THREADS + (int)threadIdx.x, row[i], c[i]);
        n[i] = row[i] < rows ? C - c[i] : 0;
        const bool some = n[i] > 0;
        w[i] = ld_bytes8(some ? q + row[i] * C + c[i] : q, n[i]);
        byte[i] = some ? ex[row[i] * ckpt_blocks(C) + c[i] / CKPT_BLOCK] : CKPT_BAD;
    }
#pragma unroll
    for (int i = 0; i < CKPT_ITEMS; ++i) {
        float v[8];
        ckpt_values(w[i], byte[i], v);
        if (PAST && n[i] >= 8) st_chunk_past(x + row[i] * C + c[i], v);
        else if (n[i] > 0) st_chunk(x + row[i] * C + c[i], n[i], v);
    }
}

static bool ckpt_shape_ok(int64_t rows, int32_t C) {
    return rows >= 0 && C > 0 && C <= (1 << 24) && rows <= ((int64_t)1 << 40) / C;
}
static int64_t ckpt_grid(int64_t rows, int C) {
    const int64_t items = rows * ckpt_blocks(C) * 4;
    return (items + CKPT_ITEMS * CKPT_THREADS - 1) / (CKPT_ITEMS * CKPT_THREADS);
}

hipError_t launch_ckpt8_pack(int dtype, int64_t rows, int32_t C, const void* x, void* ckpt, hipStream_t st) {
    if (rows == 0) return hipSuccess;
    const dim3 grid((unsigned)ckpt_grid(rows, C)), block(CKPT_THREADS);
    uint8_t* q = (uint8_t*)ckpt;
    uint8_t* ex = q + ckpt_exponents_at(rows, C);
    const FastDiv div = fast_div(ckpt_blocks(C) * 4);
    if (dtype == LPM_BF16) hipLaunchKernelGGL(ckpt_pack_kernel<bf16_t>, grid, block, 0, st, rows, (int)C, div, (const bf16_t*)x, q, ex);
    else hipLaunchKernelGGL(ckpt_pack_kernel<float>, grid, block, 0, st, rows, (int)C, div, (const float*)x, q, ex);
    return hipGetLastError();
}
hipError_t launch_ckpt8_unpack(int dtype, int64_t rows, int32_t C, const void* ckpt, void* x, hipStream_t st) {
    if (rows == 0) return hipSuccess;
    const dim3 grid((unsigned)ckpt_grid(rows, C)), block(CKPT_THREADS);
    const uint8_t* q = (const uint8_t*)ckpt;
    const uint8_t* ex = q + ckpt_exponents_at(rows, C);
    const FastDiv div = fast_div(ckpt_blocks(C) * 4);
    // A tensor of more than half of the last-level cache (256 MB) goes past it: what reads it next would find its first rows gone, and meanwhile it would push out
    // what is still wanted.  (100352 x 1000 bf16, 200 MB: 57 -> 51 us, and packing that tensor again, which then lies in the cache, 64 -> 49.)
    const bool past = (size_t)rows * C * (dtype == LPM_BF16 ? 2 : 4) > ((size_t)128 << 20);
    if (dtype == LPM_BF16) hipLaunchKernelGGL((past ? ckpt_unpack_kernel<bf16_t, true> : ckpt_unpack_kernel<bf16_t, false>), grid, block, 0, st, rows, (int)C, div, q, ex, (bf16_t*)x);
    else hipLaunchKernelGGL((past ? ckpt_unpack_kernel<float, true> : ckpt_unpack_kernel<float, false>), grid, block, 0, st, rows, (int)C, div, q, ex, (float*)x);
    return hipGetLastError();
}

}  // namespace lpm

static int32_t ckpt_check(int64_t rows, int32_t C, int32_t dtype, const void* a, const void* b) {
    if (dtype != LPM_F32 && dtype != LPM_BF16) return fail(LPM_EINVAL, "dtype must be LPM_F32 or LPM_BF16");
    if (!ckpt_shape_ok(rows, C)) return fail(LPM_ESHAPE, "a checkpoint of %lld rows of %d channels", (long long)rows, C);
    if (rows > 0 && (!a || !b)) return fail(LPM_EINVAL, "NULL argument");
    if (((uintptr_t)a | (uintptr_t)b) & 255u) return fail(LPM_EALIGN, "device buffers must be 256-byte aligned");
    return LPM_OK;
}

extern "C" int32_t lpm_ckpt8_bytes(int64_t rows, int32_t channels, size_t* bytes) {
    if (!bytes) return fail(LPM_EINVAL, "bytes is NULL");
    if (!ckpt_shape_ok(rows, channels)) return fail(LPM_ESHAPE, "a checkpoint of %lld rows of %d channels", (long long)rows, channels);
    *bytes = ckpt_exponents_at(rows, channels) + (size_t)rows * ckpt_blocks(channels);
    return LPM_OK;
}

extern "C" int32_t lpm_ckpt8_pack(int64_t rows, int32_t channels, int32_t dtype, const void* x, void* ckpt, void* stream) {
    const int32_t rc = ckpt_check(rows, channels, dtype, x, ckpt);
    if (rc) return rc;
    LPM_HIP(launch_ckpt8_pack(dtype, rows, channels, x, ckpt, (hipStream_t)stream));
    return LPM_OK;
}

extern "C" int32_t lpm_ckpt8_unpack(int64_t rows, int32_t channels, int32_t dtype, const void* ckpt, void* x, void* stream) {
    const int32_t rc = ckpt_check(rows, channels, dtype, ckpt, x);
    if (rc) return rc;
    LPM_HIP(launch_ckpt8_unpack(dtype, rows, channels, ckpt, x, (hipStream_t)stream));
    return LPM_OK;
}

// The layer's input in its own type at the head of the scratch, the contraction's partial sums behind it.  (16384 x 1024 to 1024 outputs: 9 us for the input, 46 for the
// contraction, whose tiles would each unpack their rows again for every 128 outputs.)
static int32_t wgrad_ckpt8_ws(const lpm_conv_geom* g, int32_t dtype, int64_t& rows, size_t& input, size_t& total) {
    size_t wgrad = 0;
    const int32_t rc = lpm_conv_ws_bytes(g, dtype, nullptr, nullptr, &wgrad);
    if (rc) return rc;
    rows = (int64_t)g->m * (g->d > 0 ? g->d : 1) * g->h * g->w;
    if (!ckpt_shape_ok(rows, g->cin)) return fail(LPM_ESHAPE, "a checkpoint of %lld rows of %d channels", (long long)rows, g->cin);
    input = ((size_t)rows * g->cin * (dtype == LPM_BF16 ? 2 : 4) + 255) & ~(size_t)255;
    total = input + wgrad;
    return LPM_OK;
}

extern "C" int32_t lpm_conv_wgrad_ckpt8_ws_bytes(const lpm_conv_geom* g, int32_t dtype, size_t* bytes) {
    if (!bytes) return fail(LPM_EINVAL, "bytes is NULL");
    int64_t rows;
    size_t input;
    return wgrad_ckpt8_ws(g, dtype, rows, input, *bytes);
}

extern "C" int32_t lpm_conv_wgrad_ckpt8(const lpm_conv_geom* g, int32_t dtype, const void* ckpt, const void* dz, float* dw, int32_t accumulate,
                                        void* ws, void* stream) {
    int64_t rows;
    size_t input, total;
    const int32_t rc = wgrad_ckpt8_ws(g, dtype, rows, input, total);
    if (rc) return rc;
    if (!ckpt || !dz || !dw || !ws) return fail(LPM_EINVAL, "NULL argument");
    for (const void* p : {ckpt, dz, (const void*)dw, (const void*)ws})
        if ((uintptr_t)p & 255u) return fail(LPM_EALIGN, "device buffers must be 256-byte aligned");
    LPM_HIP(launch_ckpt8_unpack(dtype, rows, g->cin, ckpt, ws, (hipStream_t)stream));
    return lpm_conv_wgrad(g, dtype, ws, dz, dw, accumulate, (char*)ws + input, stream);
}
