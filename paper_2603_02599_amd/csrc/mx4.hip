// Microscaled 4-bit floats: 32 consecutive columns of a row share a power of two 2^(s - 127), s a byte, and each value is an e2m1 code
// (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), as in the Open Compute Project's microscaling formats 1.0.  Codes are two a
// byte, the even column in the low half.
#include <math.h>

#include "kernels.hpp"

namespace sun {

constexpr int kMxBlock = 32;

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
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    *reinterpret_cast<u32x4_s*>(p) = u32x4_s{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}

// A lane takes eight columns, four lanes a block: reads and writes are contiguous over the wave.  The matrix is contiguous, so
// rows do not matter.  The converter rounds to the nearest even code and stops at 6.
template <class T>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const T* w, int64_t octets, uint32_t* codes, uint8_t* scales) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t u0 = (int64_t)blockIdx.x * 256; u0 < octets; u0 += stride) {
        const int64_t u = u0 + threadIdx.x;
        float x[8];
        load8(w + min(u, octets - 1) * 8, x);
        float top = 0.f;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            top = fmaxf(top, fabsf(x[i]));
            bad |= !(fabsf(x[i]) < INFINITY);
        }
        if (bad) top = INFINITY;
        top = fmaxf(top, lane_xor<1>(top));
        top = fmaxf(top, lane_xor<2>(top));
        int byte = max((int)(__float_as_uint(top) >> 23) - 2, 0);   // floor(log2) - 2, + 127; the subnormals' is 0 either way
        const float scale = byte ? __uint_as_float((uint32_t)byte << 23) : 0x1p-127f;
        uint32_t c = 0;
        if (top < INFINITY) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
        } else {
            byte = 255;
        }
        if (u < octets) {
            codes[u] = c;
            if ((u & 3) == 0) scales[u >> 2] = (uint8_t)byte;
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint32_t* codes, const uint8_t* scales, int64_t octets, T* out) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < octets; u += stride) {
        const uint32_t c = codes[u];
        const int byte = scales[u >> 2];
        const float scale = byte == 255 ? NAN : byte ? __uint_as_float((uint32_t)byte << 23) : 0x1p-127f;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t k = (c >> (4 * i)) & 15u, mag = k & 7u;
            // codes 2 to 7 are (1 + m / 2) 2^(e - 1); 1 is a half
            float v = mag >= 2 ? __uint_as_float((126u + (mag >> 1)) << 23 | (mag & 1u) << 22) : mag ? 0.5f : 0.f;
            if (k & 8u) v = -v;
            x[i] = v * scale;
        }
        store8(out + u * 8, x);
    }
}

static unsigned octet_grid(int64_t octets) { return (unsigned)std::min<int64_t>((octets + 255) / 256, 256 * 32); }

hipError_t launch_mx4_quantize(const void* w, bool f32, int64_t rows, int64_t cols, void* codes, void* scales, hipStream_t st) {
    const int64_t octets = rows * (cols / 8);
    if (f32) hipLaunchKernelGGL(mx4_quantize_kernel<float>, dim3(octet_grid(octets)), dim3(256), 0, st, (const float*)w, octets, (uint32_t*)codes, (uint8_t*)scales);
    else hipLaunchKernelGGL(mx4_quantize_kernel<uint16_t>, dim3(octet_grid(octets)), dim3(256), 0, st, (const uint16_t*)w, octets, (uint32_t*)codes, (uint8_t*)scales);
    return hipGetLastError();
}
hipError_t launch_mx4_dequantize(const void* codes, const void* scales, bool f32, int64_t rows, int64_t cols, void* out, hipStream_t st) {
    const int64_t octets = rows * (cols / 8);
    if (f32) hipLaunchKernelGGL(mx4_dequantize_kernel<float>, dim3(octet_grid(octets)), dim3(256), 0, st, (const uint32_t*)codes, (const uint8_t*)scales, octets, (float*)out);
    else hipLaunchKernelGGL(mx4_dequantize_kernel<uint16_t>, dim3(octet_grid(octets)), dim3(256), 0, st, (const uint32_t*)codes, (const uint8_t*)scales, octets, (uint16_t*)out);
    return hipGetLastError();
}

// ---------------------------------------------------------------- product
//
// out[b, n] = sum_k x[b, k] W[n, k].  A code times its power of two is a bf16 number, so the product runs on the bf16 matrix cores with 32-bit
// sums.  bf16 activations enter as they are, 32-bit ones as three planes of 8 bits each (x cut off behind the upper 16 bits of its
// representation, what is left likewise, and the rest): exact, at three times the operations.
struct Mx4Args {
    const uint8_t *codes, *scales;
    const uint16_t* x;     // planes of [rows][ld_x], plane bytes apart
    int64_t ld_x, plane, ld_out;
    int N, K, rows;
    void* out;
};

// 32-bit activations as their three planes; a lane takes eight
__global__ __launch_bounds__(256) void mx4_planes_kernel(const float* x, int64_t ld_x, int rows, int K, uint16_t* planes, int64_t plane) {
    const int64_t octets = (int64_t)rows * (K / 8), stride = (int64_t)gridDim.x * 256;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < octets; u += stride) {
        const int64_t row = u / (K / 8), k = u % (K / 8) * 8;
        float v[8];
        load8(x + row * ld_x + k, v);
        u32x4_s w[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t word[3] = {0, 0, 0};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float r = v[2 * j + e];
                if (r != r) r = __uint_as_float(0x7fc00000u);   // a not-a-number that its upper bits say
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    const uint32_t top = __float_as_uint(r) & 0xffff0000u;
                    word[p] |= e ? top : top >> 16;
                    r = fabsf(r) < INFINITY ? r - __uint_as_float(top) : 0.f;
                }
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) w[p][j] = word[p];
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4_s*>(planes + p * plane + row * K + k) = w[p];
    }
}

__device__ __forceinline__ bf16x8 mx4_values(uint32_t w, float scale) {
    struct { bf16x2_t v[4]; } r;
    r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return __builtin_bit_cast(bf16x8, r);
}
// the converter reads the power's exponent field: all ones is not-a-number
__device__ __forceinline__ float mx4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

template <class T>
__device__ __forceinline__ void store_as(T* p, float v) {
    if constexpr (sizeof(T) == 4) *p = v;
    else *p = f32_to_bf16_bits(v);
}

// Sixteen columns and 16 * RB rows a workgroup, the blocks of k dealt to its four waves, whose sums meet in LDS.  Lane (c = lane % 16,
// g = lane / 16) holds column c's block 4 i + g of codes, one 16-byte load, which are four 16 x 16 x 32 products.
template <class T, int P, int RB>
__global__ __launch_bounds__(256) void mx4_linear_kernel(Mx4Args a) {
    __shared__ float sums[4][16 * RB][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16, row0 = blockIdx.y * (16 * RB);
    const int64_t n = min(n0 + c16, a.N - 1);
    const int blocks = a.K / kMxBlock;
    f32x4 acc[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i = wave; i * 4 < blocks; i += 4) {
        const int blk = i * 4 + g, at = min(blk, blocks - 1);
        u32x4_s code = *reinterpret_cast<const u32x4_s*>(a.codes + (n * blocks + at) * 16);
        float scale = mx4_scale(a.scales[n * blocks + at]);
        if (blk >= blocks) code = u32x4_s{0, 0, 0, 0}, scale = 1.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x8 w = mx4_values(code[j], scale);
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const int64_t row = min(row0 + 16 * r + c16, a.rows - 1);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    u32x4_s x = *reinterpret_cast<const u32x4_s*>(a.x + p * a.plane + row * a.ld_x + at * 32 + j * 8);
                    if (blk >= blocks) x = u32x4_s{0, 0, 0, 0};
                    acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, x), acc[r], 0, 0, 0);
                }
            }
        }
    }
    // register i: column 4 g + i, row c
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][16 * r + c16][4 * g + i] = acc[r][i];
    __syncthreads();
    for (int u = threadIdx.x; u < 16 * RB * 16; u += 256) {
        const int r = u >> 4, c = u & 15;
        if (row0 + r < a.rows && n0 + c < a.N)
            store_as((T*)a.out + (row0 + r) * a.ld_out + n0 + c, ((sums[0][r][c] + sums[1][r][c]) + sums[2][r][c]) + sums[3][r][c]);
    }
}

size_t mx4_linear_workspace(int N, int K, int rows, bool x_f32) {
    return x_f32 ? (size_t)3 * rows * K * 2 : 0;   // planes of 32-bit activations
}

template <class T, int P>
static hipError_t multiply(const Mx4Args& a, hipStream_t st) {
    const dim3 grid((a.N + 15) / 16, (a.rows + 63) / 64);
    if (a.rows <= 16) hipLaunchKernelGGL((mx4_linear_kernel<T, P, 1>), dim3(grid.x, 1), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((mx4_linear_kernel<T, P, 4>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_mx4_linear(const Mx4Linear& m, void* workspace, hipStream_t st) {
    Mx4Args a{m.codes, m.scales, (const uint16_t*)m.x, m.ld_x, 0, m.ld_out, m.N, m.K, m.rows, m.out};
    if (m.x_f32) {
        a.x = (const uint16_t*)workspace;
        a.ld_x = m.K;
        a.plane = (int64_t)m.rows * m.K;
        hipLaunchKernelGGL(mx4_planes_kernel, dim3(octet_grid((int64_t)m.rows * (m.K / 8))), dim3(256), 0, st, (const float*)m.x, m.ld_x, m.rows, m.K,
                           (uint16_t*)workspace, a.plane);
        if (hipError_t e = hipGetLastError()) return e;
        return m.out_f32 ? multiply<float, 3>(a, st) : multiply<uint16_t, 3>(a, st);
    }
    return m.out_f32 ? multiply<float, 1>(a, st) : multiply<uint16_t, 1>(a, st);
}

}  // namespace sun
