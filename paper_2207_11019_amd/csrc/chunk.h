// Eight consecutive channels of a row, and the 8-bit form in which a checkpoint keeps them.
#pragma once
#include "elem.h"
#include <cstring>
#include <type_traits>

namespace lpm {

// Rows of any channel count start anywhere: the accesses are 16 (8) bytes wide and aligned to an element only, which global memory takes.
__device__ __forceinline__ void ld_chunk(const float* p, float (&v)[8]) { __builtin_memcpy(v, p, 32); }
__device__ __forceinline__ void ld_chunk(const bf16_t* p, float (&v)[8]) {
    uint32_t w[4];
    __builtin_memcpy(w, p, 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(w[e] << 16); v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
}
__device__ __forceinline__ void st_chunk(float* p, const float (&v)[8]) { __builtin_memcpy(p, v, 32); }
__device__ __forceinline__ void st_chunk(bf16_t* p, const float (&v)[8]) {
    const uint32_t w[4] = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    __builtin_memcpy(p, w, 16);
}
// ... past the caches
__device__ __forceinline__ void st_chunk_past(float* p, const float (&v)[8]) {
    typedef float f4 __attribute__((ext_vector_type(4)));
    typedef f4 at_element __attribute__((aligned(4)));
    const f4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    __builtin_nontemporal_store(a, reinterpret_cast<at_element*>(p));
    __builtin_nontemporal_store(b, reinterpret_cast<at_element*>(p + 4));
}
__device__ __forceinline__ void st_chunk_past(bf16_t* p, const float (&v)[8]) {
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    typedef u4 at_element __attribute__((aligned(2)));
    const u4 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    __builtin_nontemporal_store(w, reinterpret_cast<at_element*>(p));
}
// ... the first n of them (n may be negative or more than eight)
template <typename T> __device__ __forceinline__ void st_chunk(T* p, int n, const float (&v)[8]) {
    if (n >= 8) { st_chunk(p, v); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < n) st(p, e, v[e]);
}

// A chunk as it lies in memory, for loads that are asked for long before they are used: what converts it waits for it.
template <typename T> struct RawChunk { uint32_t w[2 * sizeof(T)]; };
// Chunk c (a multiple of eight) of a row of C channels.  Where the row ends inside it, its last eight channels are loaded (shift_chunk puts them in place); of
// chunks behind the end, the row's first.
template <typename T> __device__ __forceinline__ RawChunk<T> ld_raw(const T* row, int c, int C) {
    RawChunk<T> r;
    if (C >= 8) {
        __builtin_memcpy(r.w, row + (c >= C ? 0 : c + 8 > C ? C - 8 : c), 8 * sizeof(T));
    } else {
        T e[8] = {};
#pragma unroll
        for (int k = 0; k < 8; ++k) if (k < C) e[k] = row[k];
        __builtin_memcpy(r.w, e, sizeof r.w);
    }
    return r;
}
__device__ __forceinline__ void raw_values(const RawChunk<float>& r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r.w[e]);
}
__device__ __forceinline__ void raw_values(const RawChunk<bf16_t>& r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(r.w[e] << 16); v[2 * e + 1] = __uint_as_float(r.w[e] & 0xffff0000u); }
}
// v[e] = v[e + s], zeros behind
__device__ __forceinline__ void shift_chunk(float (&v)[8], int s) {
#pragma unroll
    for (int b = 1; b < 8; b <<= 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = s & b ? (e + b < 8 ? v[e + b] : 0.f) : v[e];
}
// the values of chunk c as ld_raw brought it; zeros behind the row's end, and everywhere where it is not `there`
template <typename T> __device__ __forceinline__ void chunk_values(const RawChunk<T>& r, int c, int C, bool there, float (&v)[8]) {
    raw_values(r, v);
    if (C % 8 && C > 8) shift_chunk(v, c < C && c + 8 > C ? c + 8 - C : 0);
    if (!there || c >= C)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
}

// Sum of a value over groups of G lanes (4 to 64), the nearest by exchanges inside the vector unit
template <int G> __device__ __forceinline__ float group_sum(float v) {
#ifdef __HIP__
    auto dpp = [](float x, auto ctrl) __attribute__((always_inline)) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v += dpp(v, std::integral_constant<int, 0xb1>());                    // lane ^ 1
    v += dpp(v, std::integral_constant<int, 0x4e>());                    // lane ^ 2
    if (G >= 8) v += dpp(v, std::integral_constant<int, 0x141>());       // the other four of eight
    if (G >= 16) v += dpp(v, std::integral_constant<int, 0x140>());      // the other eight of sixteen
    if (G >= 32) v += __shfl_xor(v, 16, 64);
    if (G >= 64) v += __shfl_xor(v, 32, 64);
#else
    for (int o = 1; o < G; o <<= 1) v += __shfl_xor(v, o, 64);
#endif
    return v;
}

// ---- checkpoints in 8 bits ----
// A block is CKPT_BLOCK consecutive channels of a row (the last of a row may be shorter): k is the least integer >= -126 with
// max|x| 2^-k <= 127, an element is q = rint(x 2^-k) in int8, ties to even, and stands for q 2^k.  A power of two and eight bits: scaling is exact, and so
// is what comes back, in bfloat16 too -- the only rounding is that to a whole q, at most half a step of 1/127 to 1/63.5 of the block's
// largest element.  Kept are the q and the byte k + 127; byte 255: the block holds an infinity or a NaN and comes back as NaN.
constexpr int CKPT_BLOCK = 32;
constexpr uint32_t CKPT_BAD = 255;
__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }      // -126 <= k <= 127
// the byte of a block whose largest magnitude has these bits
__device__ __forceinline__ uint32_t ckpt_byte(uint32_t top) {
    if (top >= 0x7f800000u) return CKPT_BAD;
    const int k = (int)(top >> 23) - 127 - ((top & 0x7fffffu) <= 0x7e0000u ? 6 : 5);      // 127 = 1.984375 * 2^6
    return (uint32_t)((k < -126 ? -126 : k) + 127);
}
__device__ __forceinline__ uint32_t chunk_top(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) { const uint32_t a = __float_as_uint(v[e]) & 0x7fffffffu; m = a > m ? a : m; }
    return m;
}
// eight elements as bytes; of a bad block, zeros
__device__ __forceinline__ uint2 ckpt_quantise(const float (&v)[8], uint32_t byte) {
    const float up = pow2(byte == CKPT_BAD ? 0 : 127 - (int)byte);
    uint32_t w[2] = {0, 0};
    if (byte != CKPT_BAD) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= ((uint32_t)(int)rintf(v[e] * up) & 0xffu) << (8 * (e & 3));
    }
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void ckpt_values(uint2 q, uint32_t byte, float (&v)[8]) {
    const float step = byte == CKPT_BAD ? __uint_as_float(0x7fc00000u) : pow2((int)byte - 127);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)((e < 4 ? q.x : q.y) >> (8 * (e & 3))) * step;
}
__device__ __forceinline__ uint2 ld_bytes8(const uint8_t* p, int n) {
    uint2 q = make_uint2(0, 0);
    if (n >= 8) { __builtin_memcpy(&q, p, 8); return q; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < n) (e < 4 ? q.x : q.y) |= (uint32_t)p[e] << (8 * (e & 3));
    return q;
}
__device__ __forceinline__ void st_bytes8(uint8_t* p, int n, uint2 q) {
    if (n >= 8) { __builtin_memcpy(p, &q, 8); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < n) p[e] = (uint8_t)((e < 4 ? q.x : q.y) >> (8 * (e & 3)));
}
// where the bytes k + 127 of a checkpoint lie: behind the rows' q, on a 256-byte boundary, ckpt_blocks(channels) to a row
__host__ __device__ inline int ckpt_blocks(int channels) { return (channels + CKPT_BLOCK - 1) / CKPT_BLOCK; }
__host__ __device__ inline size_t ckpt_exponents_at(int64_t rows, int channels) { return ((size_t)rows * channels + 255) & ~(size_t)255; }

}  // namespace lpm
