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
// A lane takes eight columns, four lanes a block: reads and writes are contiguous over the wave.  The matrix is contiguous, so
// rows do not matter.  A workgroup has R runs of 256 octets under way.  The converter rounds to the nearest even code and stops at 6.
// Memory bounds it: 28672 x 4096 in bf16 (297 MB in and out) 48 us, 6.2 TB/s.
template <class T, int R>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const T* w, int64_t octets, uint32_t* codes, uint8_t* scales) {
    const int64_t stride = (int64_t)gridDim.x * 256 * R;
    for (int64_t u0 = (int64_t)blockIdx.x * 256 * R; u0 < octets; u0 += stride) {
        float x[R][8];
#pragma unroll
        for (int r = 0; r < R; ++r) load8(w + min(u0 + r * 256 + threadIdx.x, octets - 1) * 8, x[r]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t u = u0 + r * 256 + threadIdx.x;
            float top = 0.f;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                top = fmaxf(top, fabsf(x[r][i]));
                bad |= !(fabsf(x[r][i]) < INFINITY);
            }
            if (bad) top = INFINITY;
            top = fmaxf(top, lane_xor<1>(top));
            top = fmaxf(top, lane_xor<2>(top));
            int byte = max((int)(__float_as_uint(top) >> 23) - 2, 0);   // floor(log2) - 2, + 127; the subnormals' is 0 either way
            const float scale = byte ? __uint_as_float((uint32_t)byte << 23) : 0x1p-127f;
            uint32_t c = 0;
            if (top < INFINITY) {
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[r][0], x[r][1], scale, 0);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[r][2], x[r][3], scale, 1);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[r][4], x[r][5], scale, 2);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[r][6], x[r][7], scale, 3);
            } else {
                byte = 255;
            }
            if (u < octets) {
                codes[u] = c;
                if ((u & 3) == 0) scales[u >> 2] = (uint8_t)byte;
            }
        }
    }
}

// A lane takes sixteen bytes of the output, so that a wave's store is a KiB without gaps, which is what stores past the caches need.  Memory bounds it:
// 28672 x 4096 in bf16 44 to 48 us, 6.2 to 6.7 TB/s.
template <class T, int R, bool STREAM>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* codes, const uint8_t* scales, int64_t units, T* out) {
    constexpr int E = 16 / (int)sizeof(T);   // values of a unit
    typedef std::conditional_t<E == 8, uint32_t, uint16_t> Codes;
    const int64_t stride = (int64_t)gridDim.x * 256 * R;
    for (int64_t u0 = (int64_t)blockIdx.x * 256 * R + threadIdx.x; u0 < units; u0 += stride) {
        uint32_t code[R];
        int byte[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t u = min(u0 + r * 256, units - 1);
            code[r] = reinterpret_cast<const Codes*>(codes)[u];
            byte[r] = scales[u / (kMxBlock / E)];
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (u0 + r * 256 >= units) break;
            const float scale = byte[r] == 255 ? NAN : byte[r] ? __uint_as_float((uint32_t)byte[r] << 23) : 0x1p-127f;
            float x[E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t k = (code[r] >> (4 * i)) & 15u, mag = k & 7u;
                // codes 2 to 7 are (1 + m / 2) 2^(e - 1); 1 is a half
                float v = mag >= 2 ? __uint_as_float((126u + (mag >> 1)) << 23 | (mag & 1u) << 22) : mag ? 0.5f : 0.f;
                if (k & 8u) v = -v;
                x[i] = v * scale;
            }
            u32x4_s w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (E == 8) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
                else w[i] = __float_as_uint(x[i]);
            }
            u32x4_s* to = reinterpret_cast<u32x4_s*>(out) + u0 + r * 256;
            if constexpr (STREAM) __builtin_nontemporal_store(w, to);
            else *to = w;
        }
    }
}

// One run to a workgroup while there are few, which then start at once: 2048 x 2048 3.8 / 5.1 us, with four runs 4.4 / 5.7; four where the
// matrix is large: the values of 28672 x 4096 in bf16 72 -> 58 us.
constexpr int64_t kMxFewUnits = 1 << 20;
static unsigned unit_grid(int64_t units, int runs) { return (unsigned)std::min<int64_t>((units + 256 * runs - 1) / (256 * runs), 1 << 16); }
// Values that the memory-side cache cannot hold beside what they are made from leave past it: those of 28672 x 4096 in bf16 (62 MB to 235)
// 58 -> 51 us, and the matrix that is read next is still there.  Smaller ones stay in it for whoever reads them.
constexpr int64_t kMxStreamBytes = (int64_t)256 << 20;

template <class T>
static hipError_t quantize(const T* w, int64_t octets, void* codes, void* scales, hipStream_t st) {
    if (octets <= kMxFewUnits) hipLaunchKernelGGL((mx4_quantize_kernel<T, 1>), dim3(unit_grid(octets, 1)), dim3(256), 0, st, w, octets, (uint32_t*)codes, (uint8_t*)scales);
    else hipLaunchKernelGGL((mx4_quantize_kernel<T, 4>), dim3(unit_grid(octets, 4)), dim3(256), 0, st, w, octets, (uint32_t*)codes, (uint8_t*)scales);
    return hipGetLastError();
}
template <class T>
static hipError_t dequantize(const void* codes, const void* scales, int64_t values, T* out, hipStream_t st) {
    const int64_t units = values / (16 / (int)sizeof(T));
    const uint8_t *c = (const uint8_t*)codes, *s = (const uint8_t*)scales;
    if (units <= kMxFewUnits) hipLaunchKernelGGL((mx4_dequantize_kernel<T, 1, false>), dim3(unit_grid(units, 1)), dim3(256), 0, st, c, s, units, out);
    else if (values * (int64_t)sizeof(T) + values / 2 <= kMxStreamBytes)
        hipLaunchKernelGGL((mx4_dequantize_kernel<T, 4, false>), dim3(unit_grid(units, 4)), dim3(256), 0, st, c, s, units, out);
    else hipLaunchKernelGGL((mx4_dequantize_kernel<T, 4, true>), dim3(unit_grid(units, 4)), dim3(256), 0, st, c, s, units, out);
    return hipGetLastError();
}

hipError_t launch_mx4_quantize(const void* w, bool f32, int64_t rows, int64_t cols, void* codes, void* scales, hipStream_t st) {
    return f32 ? quantize((const float*)w, rows * (cols / 8), codes, scales, st) : quantize((const uint16_t*)w, rows * (cols / 8), codes, scales, st);
}
hipError_t launch_mx4_dequantize(const void* codes, const void* scales, bool f32, int64_t rows, int64_t cols, void* out, hipStream_t st) {
    return f32 ? dequantize(codes, scales, rows * cols, (float*)out, st) : dequantize(codes, scales, rows * cols, (uint16_t*)out, st);
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
    float* part;           // [splits][rows][N], where k is split
    bool wide;             // four columns of out may be stored at once
    int splits;
};

// Eight 32-bit activations as their three planes.  What is not finite has its value in the first plane and zeros in the others.
__device__ __forceinline__ void mx4_planes(const float (&v)[8], bf16x8 (&planes)[3]) {
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

// The planes of 32-bit activations for more than sixteen rows, once for all workgroups.  A lane takes eight.  150 x 13824: 6 us.
__global__ __launch_bounds__(256) void mx4_planes_kernel(const float* x, int64_t ld_x, int rows, int K, uint16_t* planes, int64_t plane) {
    const int64_t octets = (int64_t)rows * (K / 8), stride = (int64_t)gridDim.x * 256;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < octets; u += stride) {
        const int64_t row = u / (K / 8), k = u % (K / 8) * 8;
        float v[8];
        load8(x + row * ld_x + k, v);
        bf16x8 w[3];
        mx4_planes(v, w);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<bf16x8*>(planes + p * plane + row * K + k) = w[p];
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

__device__ u32x4_s g_mx4_zeros = {0, 0, 0, 0};   // what lanes behind the last column are given

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

// Four consecutive columns of one row
template <class T>
__device__ __forceinline__ void store_quad(const Mx4Args& a, T* out, int64_t ld, bool wide, int64_t row, int n, const f32x4& v) {
    T* p = out + row * ld + n;
    if (wide && n + 3 < a.N) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(p) = v;
        else *reinterpret_cast<uint2*>(p) = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < a.N) store_as(p + i, v[i]);
}

// Up to sixteen rows: reading the weights is what costs, and latency where they are few: 6144 x 4096 at one row (13.4 MB) takes 5.5 us, of which about four are a launch
// and one request's way; 28672 x 4096 at one row 13.1 us (4.8 TB/s) while the memory-side cache holds the matrix and 17.3 where it is read from memory, at 16 18.1 and 23.1.
// In 32 bits 26.3 and 40.8: every workgroup cuts all sixteen places into planes.  Rows of x are read a lane a row, which the address unit takes line by line.
// 16 * NT columns a workgroup, the chunks of 128 k dealt to its eight waves, whose sums meet in LDS.  A wave has U chunks under
// way at a time: their codes and powers go into LDS (see the next kernel for the order), its activations straight into the operand's registers: a
// row that is not there is not asked for.  32-bit activations are cut into their planes here.
constexpr int kFewWaves = 8;
template <class T, class X, int NT, int U>
__global__ __launch_bounds__(64 * kFewWaves) void mx4_few_kernel(Mx4Args a) {
    constexpr int P = sizeof(X) == 4 ? 3 : 1, WAVE = U * NT * 1280, SUMS = 16 * (16 * NT + 1) * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kFewWaves * (WAVE > SUMS ? WAVE : SUMS)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * (16 * NT), row16 = lane >> 2, piece = (lane & 3) ^ (lane >> 4);
    const int blocks = a.K / kMxBlock, chunks = (blocks + 3) / 4;
    const uint8_t* mine = lds + wave * WAVE;
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds + wave * WAVE;
    const X* xr = (const X*)a.x + (int64_t)min(c16, a.rows - 1) * a.ld_x;
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = wave; i0 < chunks; i0 += kFewWaves * U) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what the last chunks' operands were read from is written again
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int chunk = i0 + u * kFewWaves;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int64_t at = (int64_t)min(n0 + 16 * t + row16, a.N - 1) * blocks + chunk * 4;
                lds_fetch16(chunk * 4 + piece < blocks ? (const void*)(a.codes + (at + piece) * 16) : &g_mx4_zeros, to + (u * NT + t) * 1024);
                lds_fetch1(chunk * 4 + (lane & 3) < blocks ? (const void*)(a.scales + at + (lane & 3)) : &g_mx4_zeros, to + U * NT * 1024 + (u * NT + t) * 256);
            }
        }
        u32x4_s x[U][4][P == 3 ? 2 : 1];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int blk = (i0 + u * kFewWaves) * 4 + g;
            const bool on = c16 < a.rows && blk < blocks;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int h = 0; h < (P == 3 ? 2 : 1); ++h) {
                    x[u][j][h] = u32x4_s{0, 0, 0, 0};
                    if (on) x[u][j][h] = *reinterpret_cast<const u32x4_s*>(xr + blk * 32 + j * 8 + h * 4);
                }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the wave's codes and powers have landed; no other wave reads them
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * kFewWaves >= chunks) break;
            u32x4_s w[NT];
            float scale[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                w[t] = *reinterpret_cast<const u32x4_s*>(mine + (u * NT + t) * 1024 + (c16 * 4 + (g ^ (c16 >> 2))) * 16);
                scale[t] = mx4_scale(*reinterpret_cast<const uint32_t*>(mine + U * NT * 1024 + (u * NT + t) * 256 + (c16 * 4 + g) * 4));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8 planes[P];
                if constexpr (P == 3) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(x[u][j][e >> 2][e & 3]);
                    mx4_planes(v, planes);
                } else {
                    planes[0] = __builtin_bit_cast(bf16x8, x[u][j][0]);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const bf16x8 v = mx4_values(w[t][j], scale[t]);
#pragma unroll
                    for (int p = 0; p < P; ++p) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, planes[p], acc[t], 0, 0, 0);
                }
            }
        }
    }
    // register i of tile t: column 16 t + 4 g + i, row c
    __syncthreads();
    float* sums = reinterpret_cast<float*>(lds);
    constexpr int LD = 16 * NT + 1;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[(wave * 16 + c16) * LD + 16 * t + 4 * g + i] = acc[t][i];
    __syncthreads();
    for (int u = threadIdx.x; u < a.rows * 16 * NT; u += 64 * kFewWaves) {
        const int r = u / (16 * NT), c = u % (16 * NT);
        if (n0 + c >= a.N) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) v += sums[(w * 16 + r) * LD + c];
        store_as((T*)a.out + r * a.ld_out + n0 + c, v);
    }
}

// Some dozen rows, all in one workgroup, where reading the weights is what costs: 16 * RT rows and 16 * NT * WN columns a workgroup.  Of its eight waves WN share the columns, NT tiles
// each, WK have chunks of k of their own and WJ share the eighths of a block of 32; the sums of WK and WJ meet in LDS at the end.  Codes, powers and activations
// of ST - 1 steps are under way into LDS while one is computed on.  A step is a chunk of 128 k for each of WK, of one plane of the activations.
// 28672 x 4096 in bf16 at 32 / 64 / 128 rows: 17.7 / 23 to 25 / 33.7 us while the memory-side cache holds the weights' 62 MB, 21.5 / 26.4 / 38.6 from memory; in 32 bits 46 / 61 / 103.
// No unit bounds it (at 64 rows matrix cores 21 %, vector ALU 20 % busy, a wave waits 31 % of its time): one workgroup a compute unit, whose waves meet at each step, so that converting the
// codes (a conversion of two values takes a wave 4.4 cycles), requests (a KiB of activations or codes takes the address unit 20) and products come one after
// another, and 224 workgroups leave 32 of 256 units idle.  Rings apart for codes and activations with waves for each, a rotated start along k and deeper rings
// were no faster.
//
// A request reads 64 bytes of each of sixteen rows, four lanes side by side on a row (the address unit takes four neighbouring lanes on one line
// at a time; lanes on rows of their own take it four times as long).  In LDS the four pieces of row r are exchanged by r / 4, so that
// sixteen rows' pieces j, which is what an operand reads, lie on different banks.
template <class T, int P, int RT, int NT, int WN, int WK, int WJ, int ST>
__global__ __launch_bounds__(512) void mx4_stream_kernel(Mx4Args a) {
    static_assert(WN * WK * WJ == 8, "");
    constexpr int XF = RT * 4, CF = NT * WN;                    // operand fragments (1 KiB) of a chunk: activations, codes
    constexpr int C0 = XF * 1024, S0 = C0 + CF * 1024, CHUNK = S0 + CF * 256, STAGE = WK * CHUNK;
    constexpr int WC = WN * WJ, XW = XF / WC, CW = CF / WC;     // waves of a chunk, and what one requests of it
    constexpr int OPS = XW + 2 * CW, J = 4 / WJ;
    static_assert(XF % WC == 0 && CF % WC == 0 && OPS * (ST - 2) < 64 && ST * STAGE <= 160 * 1024 && WN * RT * NT * 1024 <= ST * STAGE, "");
    __shared__ __attribute__((aligned(16))) uint8_t lds[ST * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const int wn = wave % WN, wj = wave / WN % WJ, wk = wave / WC, wq = wave % WC;
    const int nb = blockIdx.x * (16 * CF), n0 = nb + wn * 16 * NT;
    const int blocks = a.K / kMxBlock, chunks = (blocks + 3) / 4;
    const int per = (chunks + gridDim.z - 1) / gridDim.z, c0 = blockIdx.z * per, c1 = min(chunks, c0 + per), steps = (c1 - c0 + WK - 1) / WK * P;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int row16 = lane >> 2, piece = (lane & 3) ^ (lane >> 4);   // what the lane requests of sixteen rows
    const uint8_t *code[CW], *power[CW];
#pragma unroll
    for (int t = 0; t < CW; ++t) {
        const int64_t at = (int64_t)min(nb + 16 * (wq * CW + t) + row16, a.N - 1) * blocks;
        code[t] = a.codes + (at + piece) * 16;
        power[t] = a.scales + at + (lane & 3);
    }
    const uint16_t* x[XW];
#pragma unroll
    for (int i = 0; i < XW; ++i) {
        const int f = wq * XW + i;   // row tile f / 4, block f % 4 of the chunk
        x[i] = a.x + (int64_t)min(16 * (f >> 2) + row16, a.rows - 1) * a.ld_x + (f & 3) * 32 + piece * 8;
    }
    int chunk = c0 + wk, plane = 0, fill = 0;   // what is requested next, and its place in the ring
    // Request i of OPS.  Behind the last chunk zeros are requested, so that every step has the same number of requests under way.
    auto request = [&](int i) {
        const uint32_t to = lds0 + fill * STAGE + wk * CHUNK;
        const int end = chunk < c1 ? blocks : 0;
        const bool full = chunk * 4 + 4 <= end;
        const void* src;
        if (i < XW) {
            const int f = wq * XW + i;
            src = x[i] + (plane * a.plane + (int64_t)chunk * 128);
            if (!full && chunk * 4 + (f & 3) >= end) src = &g_mx4_zeros;
            lds_fetch16(src, to + f * 1024);
        } else if (i < XW + CW) {
            src = code[i - XW] + (int64_t)chunk * 64;
            if (!full && chunk * 4 + piece >= end) src = &g_mx4_zeros;
            lds_fetch16(src, to + C0 + (wq * CW + i - XW) * 1024);
        } else {
            src = power[i - XW - CW] + chunk * 4;
            if (!full && chunk * 4 + (lane & 3) >= end) src = &g_mx4_zeros;
            lds_fetch1(src, to + S0 + (wq * CW + i - XW - CW) * 256);
        }
    };
    auto requested = [&]() {
        if (++plane == P) plane = 0, chunk += WK;
        if (++fill == ST) fill = 0;
    };
    f32x4 acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) {
#pragma unroll
        for (int i = 0; i < OPS; ++i) request(i);
        requested();
    }
    int at = 0;
    for (int s = 0; s < steps; ++s) {
        // The oldest step has landed for every wave, and every wave is done with the one before, whose place may be written again.
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(OPS * (ST - 2)) : "memory");
        const uint8_t* from = lds + at * STAGE + wk * CHUNK;
        uint32_t w[NT][J];
        float scale[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint8_t* p = from + C0 + (wn * NT + t) * 1024 + (c16 * 4 + (g ^ (c16 >> 2))) * 16 + wj * J * 4;
            if constexpr (J == 1) {
                w[t][0] = *reinterpret_cast<const uint32_t*>(p);
            } else {
                typedef uint32_t Words __attribute__((ext_vector_type(J)));
                const Words v = *reinterpret_cast<const Words*>(p);
#pragma unroll
                for (int j = 0; j < J; ++j) w[t][j] = v[j];
            }
            scale[t] = mx4_scale(*reinterpret_cast<const uint32_t*>(from + S0 + (wn * NT + t) * 256 + (c16 * 4 + g) * 4));
        }
        // The requests of the step that takes the place of the one before stand between the products: all in front of them, they keep the
        // address unit busy while the matrix cores wait.
        constexpr int GROUPS = J * RT, EACH = (OPS + GROUPS - 1) / GROUPS;
        auto rows_at = [&](int q) {   // operand of group q: row tile q % RT, eighth wj * J + q / RT of the blocks
            return *reinterpret_cast<const bf16x8*>(from + (q % RT * 4 + g) * 1024 + (c16 * 4 + ((wj * J + q / RT) ^ (c16 >> 2))) * 16);
        };
        bf16x8 b[GROUPS], v[J][NT];
        constexpr int AHEAD = 2;       // operands on their way from LDS
#pragma unroll
        for (int t = 0; t < NT; ++t) v[0][t] = mx4_values(w[t][0], scale[t]);
#pragma unroll
        for (int q = 0; q < min(AHEAD, GROUPS); ++q) b[q] = rows_at(q);
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
            if (q + AHEAD < GROUPS) b[q + AHEAD] = rows_at(q + AHEAD);
            __builtin_amdgcn_sched_barrier(0);   // left to itself the compiler reads an operand in front of its products and waits
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[q % RT][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[q / RT][t], b[q], acc[q % RT][t], 0, 0, 0);
            // the weights of the next eighth, a column tile at a time
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (q / RT + 1 < GROUPS / RT && t * RT / NT == q % RT) v[q / RT + 1][t] = mx4_values(w[t][q / RT + 1], scale[t]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = q * EACH; i < min(OPS, (q + 1) * EACH); ++i) request(i);
        }
        requested();
        if (++at == ST) at = 0;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is on its way into LDS any more
    if constexpr (WK * WJ > 1) {   // the sums of the waves that had other parts of k, in their order
        f32x4* sums = reinterpret_cast<f32x4*>(lds);
        const int part = wk * WJ + wj;
        for (int q = 1; q < WK * WJ; ++q) {
            __syncthreads();
            if (part == q) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int t = 0; t < NT; ++t) sums[((wn * RT + r) * NT + t) * 64 + lane] = acc[r][t];
            }
            __syncthreads();
            if (part == 0) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const f32x4 v = sums[((wn * RT + r) * NT + t) * 64 + lane];
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[r][t][i] += v[i];
                    }
            }
        }
        if (part > 0) return;
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = 16 * r + c16;
        if (row >= a.rows) continue;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int n = n0 + 16 * t + 4 * g;
            if (gridDim.z > 1) store_quad<float>(a, a.part + (int64_t)blockIdx.z * a.rows * a.N, a.N, a.N % 4 == 0, row, n, acc[r][t]);
            else store_quad<T>(a, (T*)a.out, a.ld_out, a.wide, row, n, acc[r][t]);
        }
    }
}

// Many rows, where the matrix cores are what is short: 28672 x 4096 at 2048 rows in bf16 takes 394 to 423 us from card to card, 1.14 to 1.22 PFLOP/s, the dense
// bf16 product of the library 400; 5120 x 13824 at 150 rows in 32 bits (three planes) 65 us and 15 for planes and joining.
// 16 * RT * WR rows and 16 * NT * WN columns a workgroup, a wave RT x NT tiles.  Activations,
// codes and powers go through LDS as above, the next step's on their way while one is computed on.  Two places for the activations; codes and powers,
// which a wave takes into registers when it enters the step, have one.
template <class T, int P, int RT, int NT, int WR, int WN>
__global__ __launch_bounds__(64 * WR * WN, 2) void mx4_tile_kernel(Mx4Args a) {
    constexpr int WAVES = WR * WN, XF = RT * WR * 4, XW = XF / WAVES, CF = NT * WN, CW = CF / WAVES;
    constexpr int C0 = 2 * XF * 1024, S0 = C0 + CF * 1024;
    static_assert(2 * CF / WAVES + XF / WAVES <= 4 * RT && XF % WAVES == 0 && CF % WAVES == 0 && S0 + CF * 256 <= 160 * 1024, "");
    __shared__ __attribute__((aligned(16))) uint8_t lds[S0 + CF * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    // Workgroups are dealt to the eight XCDs in turn.  An XCD gets the row tiles of every eighth column tile, whose codes it then reads once; those of the
    // last few column tiles are dealt evenly.
    const int col_tiles = (a.N + 16 * CF - 1) / (16 * CF), row_tiles = (a.rows + 16 * RT * WR - 1) / (16 * RT * WR);
    const int groups = col_tiles * a.splits, even = groups / 8 * row_tiles, rest = groups % 8 * row_tiles;
    const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3, late = xcd * ((rest + 7) / 8) + local - even;
    if (local >= even && late >= min(rest, (xcd + 1) * ((rest + 7) / 8))) return;
    const int group = local < even ? local / row_tiles * 8 + xcd : groups / 8 * 8 + late / row_tiles;
    const int row_tile = local < even ? local % row_tiles : late % row_tiles, col_tile = group % col_tiles, split = group / col_tiles;
    const int n0 = col_tile * (16 * CF), row0 = row_tile * (16 * RT * WR), wr = wave / WN, wn = wave % WN;
    const int blocks = a.K / kMxBlock, chunks = (blocks + 3) / 4;
    const int per = (chunks + a.splits - 1) / a.splits, c0 = split * per, steps = (min(chunks, c0 + per) - c0) * P;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int row16 = lane >> 2, piece = (lane & 3) ^ (lane >> 4);
    const uint8_t *code[CW], *power[CW];
#pragma unroll
    for (int t = 0; t < CW; ++t) {
        const int64_t at = (int64_t)min(n0 + 16 * (wave * CW + t) + row16, a.N - 1) * blocks;
        code[t] = a.codes + (at + piece) * 16;
        power[t] = a.scales + at + (lane & 3);
    }
    const uint16_t* x[XW];
#pragma unroll
    for (int i = 0; i < XW; ++i) {
        const int f = wave * XW + i;
        x[i] = a.x + (int64_t)min(row0 + 16 * (f >> 2) + row16, a.rows - 1) * a.ld_x + (f & 3) * 32 + piece * 8;
    }
    const int c1 = min(chunks, c0 + per);
    constexpr int OPS = 2 * CW + XW;
    int chunk = c0, plane = 0, fill = 0;
    auto request = [&](int i) {
        const int end = chunk < c1 ? blocks : 0;
        const bool full = chunk * 4 + 4 <= end;
        const void* src;
        if (i < CW) {
            src = code[i] + (int64_t)chunk * 64;
            if (!full && chunk * 4 + piece >= end) src = &g_mx4_zeros;
            lds_fetch16(src, lds0 + C0 + (wave * CW + i) * 1024);
        } else if (i < 2 * CW) {
            src = power[i - CW] + chunk * 4;
            if (!full && chunk * 4 + (lane & 3) >= end) src = &g_mx4_zeros;
            lds_fetch1(src, lds0 + S0 + (wave * CW + i - CW) * 256);
        } else {
            const int f = wave * XW + i - 2 * CW;
            src = x[i - 2 * CW] + (plane * a.plane + (int64_t)chunk * 128);
            if (!full && chunk * 4 + (f & 3) >= end) src = &g_mx4_zeros;
            lds_fetch16(src, lds0 + fill * (XF * 1024) + f * 1024);
        }
    };
    auto requested = [&]() {
        if (++plane == P) plane = 0, ++chunk;
        fill ^= 1;
    };
    f32x4 acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < OPS; ++i) request(i);
    requested();
    for (int s = 0; s < steps; ++s) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the step has landed for every wave
        u32x4_s w[NT];
        float scale[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            w[t] = *reinterpret_cast<const u32x4_s*>(lds + C0 + (wn * NT + t) * 1024 + (c16 * 4 + (g ^ (c16 >> 2))) * 16);
            scale[t] = mx4_scale(*reinterpret_cast<const uint32_t*>(lds + S0 + (wn * NT + t) * 256 + (c16 * 4 + g) * 4));
        }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");            // every wave has its codes, whose place is written next
        const uint8_t* from = lds + (s & 1) * (XF * 1024) + (wr * RT * 4 + g) * 1024 + c16 * 64;
        auto rows_at = [&](int q) { return *reinterpret_cast<const bf16x8*>(from + q % RT * 4096 + ((q / RT) ^ (c16 >> 2)) * 16); };
        constexpr int GROUPS = 4 * RT, AHEAD = 2, EACH = (2 * OPS + GROUPS - 1) / GROUPS;
        bf16x8 b[GROUPS], v[4][NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) v[0][t] = mx4_values(w[t][0], scale[t]);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) b[q] = rows_at(q);
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
            if (q + AHEAD < GROUPS) b[q + AHEAD] = rows_at(q + AHEAD);
            __builtin_amdgcn_sched_barrier(0);   // left to itself the compiler reads an operand in front of its products and waits
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[q % RT][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[q / RT][t], b[q], acc[q % RT][t], 0, 0, 0);
            // the weights of the next eighth, a column tile at a time
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (q / RT + 1 < GROUPS / RT && t * RT / NT == q % RT) v[q / RT + 1][t] = mx4_values(w[t][q / RT + 1], scale[t]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = q * EACH; i < min(OPS, (q + 1) * EACH); ++i) request(i);   // between the products, and early in the step
        }
        requested();
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is on its way into LDS any more
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = row0 + 16 * (wr * RT + r) + c16;
        if (row >= a.rows) continue;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int n = n0 + 16 * (wn * NT + t) + 4 * g;
            if (a.splits > 1) store_quad<float>(a, a.part + (int64_t)split * a.rows * a.N, a.N, a.N % 4 == 0, row, n, acc[r][t]);
            else store_quad<T>(a, (T*)a.out, a.ld_out, a.wide, row, n, acc[r][t]);
        }
    }
}

// out = sum of the parts along k, in their order
template <class T>
__global__ __launch_bounds__(256) void mx4_join_kernel(Mx4Args a, int splits) {
    const int64_t total = (int64_t)a.rows * a.N, stride = (int64_t)gridDim.x * 256;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += stride) {
        float v = a.part[u];
        for (int z = 1; z < splits; ++z) v += a.part[z * total + u];
        store_as((T*)a.out + u / a.N * a.ld_out + u % a.N, v);
    }
}

// How a product is dealt to workgroups.  Times in microseconds, measured on the 8B and 14B shapes' matrices with one plane of activations: a chunk
// of 128 k takes a streaming workgroup of 128 (64) columns 0.40 (0.28) with 32 rows, 0.60 (0.45) with 64, 0.90 (0.80) with 128; narrower ones were
// never faster.  A step of 128 k takes a tile of 256 columns and 32 * rt rows 0.9 + 0.275 * rt (3.1 with 256 rows), one or two of 128 x 128 on a
// compute unit 1.2 and 2.0.  A joining launch takes 4 and its parts' bytes at 4 TB/s.  Tiles of 160, 192 and 224 rows against 256 and 128 alone:
// 5120 x 13824 at 150 rows in 32 bits 95 -> 75 us, 14336 x 4096 at 1500 171 -> 149, 20000 x 5120 at 400 in 32 bits 267 -> 233; the
// worst that the estimate does is 28672 x 4096 at 192 rows, 57.5 -> 61.6.
constexpr int kMx4SplitRows = 1 << 17;   // more rows are never split along k
struct Mx4Plan {
    enum { FEW, STREAM, TILE } kind;
    int rt;        // row tiles of a wave
    int cols;      // columns of a workgroup
    int splits;    // along k
};
static Mx4Plan mx4_plan(int N, int K, int rows, int planes) {
    const int chunks = (K + 127) / 128;
    // Columns of a workgroup: the fewest that leave every compute unit one workgroup at most, 64 beyond.  32-bit activations of more than eight rows, whose cutting
    // each workgroup does again, take twice as many.  K 4096, with 16 / 32 / 64 columns: N 4096 at one row 4.3 / 5.1 / 6.8 us, N 6144 6.3 / 5.5 / 7.1, N 16384
    // 10.7 / 8.5 / 8.6 and at 16 rows 19 / 13.7 / 12.1; 16 rows in 32 bits, N 2048 14.9 / 12.3 / 14.4, N 6144 40 / 18.9 / 15.9.
    if (rows <= 16) {
        int cols = N <= 16 * 256 ? 16 : N <= 32 * 256 ? 32 : 64;
        if (planes > 1 && rows > 8) cols = std::min(2 * cols, 64);
        return Mx4Plan{Mx4Plan::FEW, 1, cols, 1};
    }
    Mx4Plan best{};
    double least = 1e30;
    auto consider = [&](auto kind, int rt, int cols, long long tiles, double step, double step2) {
        for (int want : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (want > 1 && (want > chunks / 4 || tiles >= 512 || rows > kMx4SplitRows)) break;
            const int per = (chunks + want - 1) / want, splits = (chunks + per - 1) / per;   // none of them empty
            if (splits != want) continue;
            const long long n = (tiles * splits + 255) / 256;   // workgroups of the busiest compute unit
            double t = (step2 > 0 ? n / 2 * step2 + n % 2 * step : n * step) * per * planes;
            if (splits > 1) t += 4 + (splits + 1) * (double)rows * N * 4 / 4e6;
            if (t < least) least = t, best = Mx4Plan{kind, rt, cols, splits};
        }
    };
    if (rows <= 128) {
        const int rt = rows <= 32 ? 2 : rows <= 64 ? 4 : 8;
        consider(Mx4Plan::STREAM, rt, 128, (N + 127) / 128, rt == 2 ? 0.40 : rt == 4 ? 0.60 : 0.90, 0);
        consider(Mx4Plan::STREAM, rt, 64, (N + 63) / 64, rt == 2 ? 0.28 : rt == 4 ? 0.45 : 0.80, 0);
    } else {
        for (int rt : {8, 7, 6, 5}) consider(Mx4Plan::TILE, rt, 256, (long long)((N + 255) / 256) * ((rows + 32 * rt - 1) / (32 * rt)), 0.9 + 0.275 * rt, 0);
        consider(Mx4Plan::TILE, 4, 128, (long long)((N + 127) / 128) * ((rows + 127) / 128), 1.2, 2.0);
    }
    return best;
}
static size_t align256(size_t v) { return (v + 255) / 256 * 256; }
size_t mx4_linear_workspace(int N, int K, int rows, bool x_f32) {
    const Mx4Plan p = mx4_plan(N, K, rows, x_f32 ? 3 : 1);
    if (p.kind == Mx4Plan::FEW) return 0;
    return (x_f32 ? align256((size_t)3 * rows * K * 2) : 0) + (p.splits > 1 ? (size_t)p.splits * rows * N * 4 : 0);
}
// No less than what any number of rows up to this takes.  Between two of the numbers at which tiles are added, more rows never ask for more parts (what
// joining costs grows with them), so the parts of the fewest of them and the size of the most are enough.
size_t mx4_linear_workspace_up_to(int N, int K, int rows) {
    size_t parts = 0;
    int from = 17;
    for (int64_t to = 32; from <= std::min(rows, kMx4SplitRows); from = (int)to + 1, to += to < 128 ? to : 32)
        for (int planes : {1, 3}) {
            const int s = mx4_plan(N, K, from, planes).splits;
            if (s > 1) parts = std::max(parts, (size_t)s * (size_t)std::min<int64_t>(to, rows) * N * 4);
        }
    return (rows > 16 ? align256((size_t)3 * rows * K * 2) : 0) + parts;
}

template <class T, class X>
static hipError_t multiply_few(const Mx4Args& a, int cols, hipStream_t st) {
    const dim3 grid((a.N + cols - 1) / cols), block(64 * kFewWaves);
    if (cols == 64) hipLaunchKernelGGL((mx4_few_kernel<T, X, 4, 2>), grid, block, 0, st, a);
    else if (cols == 32) hipLaunchKernelGGL((mx4_few_kernel<T, X, 2, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((mx4_few_kernel<T, X, 1, 4>), grid, block, 0, st, a);
    return hipGetLastError();
}

template <class T, int P>
static hipError_t multiply(const Mx4Args& a, const Mx4Plan& p, hipStream_t st) {
    if (p.kind == Mx4Plan::STREAM) {
        const dim3 grid((a.N + p.cols - 1) / p.cols, 1, p.splits);
        // RT, NT, WN, WK, WJ, ST
        const dim3 block(512);
        if (p.rt == 2 && p.cols == 128) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 2, 2, 4, 2, 1, 4>), grid, block, 0, st, a);
        else if (p.rt == 2) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 2, 2, 2, 2, 2, 4>), grid, block, 0, st, a);
        else if (p.rt == 4 && p.cols == 128) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 4, 2, 4, 2, 1, 3>), grid, block, 0, st, a);
        else if (p.rt == 4) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 4, 2, 2, 2, 2, 3>), grid, block, 0, st, a);
        else if (p.cols == 128) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 8, 2, 4, 1, 2, 3>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((mx4_stream_kernel<T, P, 8, 2, 2, 2, 2, 2>), grid, block, 0, st, a);
    } else {
        const long long groups = (long long)((a.N + p.cols - 1) / p.cols) * p.splits, rows = (a.rows + 32 * p.rt - 1) / (32 * p.rt);
        const dim3 grid((unsigned)(8 * (groups / 8 * rows + (groups % 8 * rows + 7) / 8)));
        if (p.rt == 8) hipLaunchKernelGGL((mx4_tile_kernel<T, P, 8, 4, 2, 4>), grid, dim3(512), 0, st, a);
        else if (p.rt == 7) hipLaunchKernelGGL((mx4_tile_kernel<T, P, 7, 4, 2, 4>), grid, dim3(512), 0, st, a);
        else if (p.rt == 6) hipLaunchKernelGGL((mx4_tile_kernel<T, P, 6, 4, 2, 4>), grid, dim3(512), 0, st, a);
        else if (p.rt == 5) hipLaunchKernelGGL((mx4_tile_kernel<T, P, 5, 4, 2, 4>), grid, dim3(512), 0, st, a);
        else hipLaunchKernelGGL((mx4_tile_kernel<T, P, 4, 4, 2, 2>), grid, dim3(256), 0, st, a);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if (p.splits > 1) {
        const int64_t total = (int64_t)a.rows * a.N;
        hipLaunchKernelGGL(mx4_join_kernel<T>, dim3((unsigned)std::min<int64_t>((total + 255) / 256, 8192)), dim3(256), 0, st, a, p.splits);
    }
    return hipGetLastError();
}

hipError_t launch_mx4_linear(const Mx4Linear& m, void* workspace, hipStream_t st) {
    const Mx4Plan p = mx4_plan(m.N, m.K, m.rows, m.x_f32 ? 3 : 1);
    const size_t out_size = m.out_f32 ? 4 : 2;
    Mx4Args a{m.codes, m.scales, (const uint16_t*)m.x, m.ld_x, 0, m.ld_out, m.N, m.K, m.rows, m.out, (float*)workspace,
              (uintptr_t)m.out % (4 * out_size) == 0 && m.ld_out % 4 == 0, p.splits};
    if (p.kind == Mx4Plan::FEW) {
        if (m.x_f32) return m.out_f32 ? multiply_few<float, float>(a, p.cols, st) : multiply_few<uint16_t, float>(a, p.cols, st);
        return m.out_f32 ? multiply_few<float, uint16_t>(a, p.cols, st) : multiply_few<uint16_t, uint16_t>(a, p.cols, st);
    }
    if (m.x_f32) {
        a.x = (const uint16_t*)workspace;
        a.ld_x = m.K;
        a.plane = (int64_t)m.rows * m.K;
        a.part = (float*)((char*)workspace + align256((size_t)3 * m.rows * m.K * 2));
        hipLaunchKernelGGL(mx4_planes_kernel, dim3(unit_grid((int64_t)m.rows * (m.K / 8), 1)), dim3(256), 0, st, (const float*)m.x, m.ld_x, m.rows, m.K,
                           (uint16_t*)workspace, a.plane);
        if (hipError_t e = hipGetLastError()) return e;
        return m.out_f32 ? multiply<float, 3>(a, p, st) : multiply<uint16_t, 3>(a, p, st);
    }
    return m.out_f32 ? multiply<float, 1>(a, p, st) : multiply<uint16_t, 1>(a, p, st);
}

}  // namespace sun
