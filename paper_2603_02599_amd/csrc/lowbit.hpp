// What the operators on 8- and 4-bit floats share.
#pragma once
#include "common.hpp"

namespace sun {

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
    const u32x4_s w = *reinterpret_cast<const u32x4_s*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
}

// Eight 32-bit values as their three planes.  What is not finite has its value in the first plane and zeros in the others.
__device__ __forceinline__ void three_planes(const float (&v)[8], bf16x8 (&planes)[3]) {
    u32x4_s w[3];
    float r[8];
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        r[i] = v[i];
        finite &= fabsf(v[i]) < INFINITY;
    }
    auto cut = [](float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); };
    auto plane = [&](int p) {   // the upper halves of two values a word
#pragma unroll
        for (int j = 0; j < 4; ++j) w[p][j] = __builtin_amdgcn_perm(__float_as_uint(r[2 * j + 1]), __float_as_uint(r[2 * j]), 0x07060302u);
    };
    if (!finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (v[i] != v[i]) r[i] = __uint_as_float(0x7fc00000u);   // a not-a-number that its upper half says
    }
    plane(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = cut(r[i]);
    if (!finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(fabsf(v[i]) < INFINITY)) r[i] = 0.f;
    }
    plane(1);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = cut(r[i]);
    plane(2);
#pragma unroll
    for (int p = 0; p < 3; ++p) planes[p] = __builtin_bit_cast(bf16x8, w[p]);
}

// Eight e4m3 codes times a power of two, exact
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t w0, uint32_t w1, float scale = 1.f) {
    struct { bf16x2_t v[4]; } r;
    r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false);
    r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
    r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false);
    r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
    return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ float power(uint32_t word, int byte) { return __uint_as_float(((word >> (8 * byte)) & 255u) << 23); }
// x with its lower 16 bits off; what is left of a finite x is exact
__device__ __forceinline__ float upper(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ float below(float x) {
    const float r = x - upper(x);
    return fabsf(x) < INFINITY ? r : 0.f;
}

// What is stored of a weighted sum v, the weights' sum and the largest score: zeros where there is no token
__device__ __forceinline__ float kv8_quotient(float v, float sum, float top) { return sum == 0.f && top == -INFINITY ? 0.f : v / sum; }

static __device__ u32x4_s g_zeros = {0, 0, 0, 0};   // what lanes are given whose place in memory is not there

// Requests from memory straight into LDS, the address a lane's own: 16 bytes a lane (lane i's land at lds_byte + 16 i), or a byte, which
// lands as a word (at lds_byte + 4 i).  Whoever reads the place waits for vmcnt and the barrier by hand.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 is a reserved register, see lds_dma16
__device__ __forceinline__ void lds_fetch16(const void* p, uint32_t lds_byte) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_byte), "v"(p) : "memory", "m0");
}
__device__ __forceinline__ void lds_fetch1(const void* p, uint32_t lds_byte) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, off" ::"s"(lds_byte), "v"(p) : "memory", "m0");
}
#pragma clang diagnostic pop

}  // namespace sun
