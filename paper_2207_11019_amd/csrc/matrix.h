// Operands of the 32x32 matrix instructions as 16-byte chunks: eight bfloat16 or four floats of a row.
#pragma once
#include "elem.h"
#include <cstring>

namespace lpm {

typedef float mm_f16 __attribute__((ext_vector_type(16)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 mm_bf8;
typedef unsigned int mm_u2 __attribute__((ext_vector_type(2)));
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short mm_s4;

#ifdef __HIP__
#define LPM_MM_INLINE __forceinline__
#else                     // (a CPU build's frames would hold every product's temporaries)
#define LPM_MM_INLINE __attribute__((noinline))
#endif

// What a lane holds: of both operands, row (column) lane % 32 and of every 2 * EPC terms of the sum the EPC that belong to its half lane / 32;
// of the result, column lane % 32 and rows (r & 3) + 8 (r >> 2) + 4 (lane / 32), r = 0 .. 15.
template <typename T> struct Mm;
template <> struct Mm<bf16_t> {
    static constexpr int EPC = 8;
    static __device__ LPM_MM_INLINE mm_f16 mul(uint4 a, uint4 b, mm_f16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mm_bf8, a), __builtin_bit_cast(mm_bf8, b), c, 0, 0, 0);
    }
    // EPC values of the result as an operand of the next product
    static __device__ __forceinline__ uint4 pack(const float* v) {
        return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
    static __device__ __forceinline__ uint4 scale(uint4 v, float f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = pack_bf16x2(__uint_as_float(w[k] << 16) * f, __uint_as_float(w[k] & 0xffff0000u) * f);
        return make_uint4(r[0], r[1], r[2], r[3]);
    }
    // The LDS transpose read: lane i of 16 receives element i % 4 of the four-element pieces that lanes 4j + i/4 point at, j = 0 .. 3.
    static __device__ LPM_MM_INLINE uint2 read4(const unsigned char* p) {
#ifdef __HIP__
        return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) mm_s4*)(p)));
#else       // the same by lane exchanges
        unsigned e[4];
        const int lane = threadIdx.x & 63;
        for (int j = 0; j < 4; ++j) {
            const unsigned char* q = __shfl(p, (lane & ~15) + 4 * j + (lane & 15) / 4, 64);
            uint16_t w;
            __builtin_memcpy(&w, q + 2 * (lane & 3), 2);
            e[j] = w;
        }
        (void)__shfl(0, 0, 64);
        return make_uint2(e[0] | e[1] << 16, e[2] | e[3] << 16);
#endif
    }
    // Operand whose rows are the channels 32 t .. 32 t + 31 of a tile's rows in LDS (R: bytes of a row, and where a row's chunks lie) and whose terms are its
    // rows, in the order in which a result lies over the lanes: those of half g are 4 g + (0 .. 3) and 8 + 4 g + (0 .. 3); place() does not
    // differ between rows 8 apart.  column: where the lane reads, from the first of the rows on.
    template <typename R> static __device__ __forceinline__ int column(int t, int lane) {
        const int row = 4 * (lane >> 5) + ((lane >> 2) & 3);
        return row * R::ROW + (((4 * t + ((lane >> 3) & 2) + ((lane >> 1) & 1)) ^ R::place(row)) * 16 + (lane & 1) * 8);
    }
    template <typename R> static __device__ LPM_MM_INLINE uint4 columns(const unsigned char* tile, int at) {
        const uint2 a = read4(tile + at), b = read4(tile + at + 8 * R::ROW);
        return make_uint4(a.x, a.y, b.x, b.y);
    }
};
template <> struct Mm<float> {
    static constexpr int EPC = 4;
    static __device__ LPM_MM_INLINE mm_f16 mul(uint4 a, uint4 b, mm_f16 c) {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint4 pack(const float* v) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
    static __device__ __forceinline__ uint4 scale(uint4 v, float f) {
        return make_uint4(__float_as_uint(__uint_as_float(v.x) * f), __float_as_uint(__uint_as_float(v.y) * f), __float_as_uint(__uint_as_float(v.z) * f),
                          __float_as_uint(__uint_as_float(v.w) * f));
    }
    // ... the rows of half g: 4 g + (0 .. 3), whose places differ from the first one's by a constant in the chunk's bits
    template <typename R> static __device__ __forceinline__ int column(int t, int lane) {
        const int row = 4 * (lane >> 5);
        return row * R::ROW + (((8 * t + ((lane & 31) >> 2)) ^ R::place(row)) * 16 + (lane & 3) * 4);
    }
    template <typename R> static __device__ LPM_MM_INLINE uint4 columns(const unsigned char* tile, int at) {
        unsigned v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const unsigned*>(tile + k * R::ROW + (at ^ (R::place(k) * 16)));
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
};

// 2^x for x <= 0 or so: one instruction (a result below 2^-126 is 0)
__device__ __forceinline__ float exp2_fast(float x) {
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_exp2f(x);
#else
    return exp2f(x);
#endif
}

}  // namespace lpm
