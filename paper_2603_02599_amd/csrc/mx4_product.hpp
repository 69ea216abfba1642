// The products with microscaled 4-bit floats: kernels, and how a call comes to one.
#pragma once
#include "kernels.hpp"
#include "lowbit.hpp"

namespace sun {

constexpr int kMxBlock = 32;   // columns that share a power of two

struct Mx4Plan {
    enum { FEW, STREAM, TILE } kind;
    int rt;        // row tiles of a wave
    int cols;      // columns of a workgroup
    int splits;    // along k
};
Mx4Plan mx4_plan(int N, int K, int rows, int planes);
hipError_t launch_mx4_planes(const float* x, int64_t ld_x, int rows, int K, uint16_t* planes, int64_t plane, hipStream_t st);
static inline size_t align256(size_t v) { return (v + 255) / 256 * 256; }

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
    // behind the product, see Epilogue
    const uint8_t *up_codes, *up_scales;
    const void *bias, *residual;   // of the output's type
    int64_t ld_residual;
    int act;
    bool wide_in;          // and four of bias and residual be read
    bool out_f32;          // what out, bias and residual are, where the kernel's type does not say
};

// What happens to a sum before it is rounded and stored.  GATED: tiles of 16 columns are the gate's and the up projection's in turn, so that a lane has both sums of a
// column; N counts pairs, and parts along k are stored gate first, [rows][2 N].  The kernels are bound by what bounds them without: a pair of 14336 x 4096 at 1 / 64 / 2048 rows in
// bf16 takes 13.4 / 22 / 396 us (28672 x 4096 stored without one 13.1 / 22 / 394 to 423), of 13824 x 5120 at 150 in 32 bits 131, 5120 x 13824 at 333 with a residual 62.
enum Epilogue { PLAIN, FUSED, GATED };

// SiLU: x / (1 + e^-x).  GELU by tanh: x / (1 + e^(-2 u)), u = sqrt(2 / pi) (x + 0.044715 x^3).  GELU: with the normal distribution's upper tail Q at |x|, x - x Q and, below 0, x Q.
// Q = e^(-x^2 / 2) R, and R = t P(t) with t = 1 / (1 + 0.305 |x|) and P of degree 7, fitted for the least relative error where e^(-x^2 / 2) is a number of 32 bits: 1e-7, with the
// roundings of its evaluation 4e-7.  So small values keep their digits; a rational approximation of the error function that is good to an absolute 1.5e-7 left 0.16 % of the value off at -5 and 1 % at -8.
// A product's epilogue has them for up to 128 sums of a lane, so they are a few instructions each: an exponential's argument rounds once (GELU's three times), which takes
// |argument| 2^-24 of it.
template <int ACT>
__device__ __forceinline__ float mx4_activation(float x) {
    if constexpr (ACT == SUN_ACT_SILU) return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
    if constexpr (ACT == SUN_ACT_GELU_TANH)
        return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * __builtin_fmaf(x * x, -0.10294324f, -2.3022082f)));   // -2 log2(e) sqrt(2 / pi) (0.044715 x^2 + 1)
    if constexpr (ACT == SUN_ACT_GELU) {
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(x), 0.305f, 1.f));
        float c = __builtin_fmaf(t, 0.0366388746f, -0.152746111f);
        c = __builtin_fmaf(t, c, 0.185314938f);
        c = __builtin_fmaf(t, c, -0.0376206972f);
        c = __builtin_fmaf(t, c, 0.120840408f);
        c = __builtin_fmaf(t, c, 0.103473693f);
        c = __builtin_fmaf(t, c, 0.122458681f);
        c = __builtin_fmaf(t, c, 0.121640243f);
        c *= t * __builtin_amdgcn_exp2f(x * x * -0.72134752f);
        return x > 0.f ? __builtin_fmaf(-fminf(x, 100.f), c, x) : x * c;
    }
    return x;
}
template <class F>
__device__ __forceinline__ void mx4_with_activation(int act, F f) {
    if (act == SUN_ACT_SILU) f(std::integral_constant<int, SUN_ACT_SILU>{});
    else if (act == SUN_ACT_GELU) f(std::integral_constant<int, SUN_ACT_GELU>{});
    else if (act == SUN_ACT_GELU_TANH) f(std::integral_constant<int, SUN_ACT_GELU_TANH>{});
    else f(std::integral_constant<int, SUN_ACT_NONE>{});
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
// The same of bias or residual; 0 where there is none
__device__ __forceinline__ f32x4 load_quad(const Mx4Args& a, const void* p, int64_t at, int n) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (!p) return v;
    if (a.wide_in && n + 3 < a.N) {
        if (a.out_f32) return *reinterpret_cast<const f32x4*>((const float*)p + at);
        const uint2 w = *reinterpret_cast<const uint2*>((const uint16_t*)p + at);
        return f32x4{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < a.N) v[i] = a.out_f32 ? ((const float*)p)[at + i] : bf16_bits_to_f32(((const uint16_t*)p)[at + i]);
    return v;
}
// and behind an epilogue; `up` is of GATED alone
template <Epilogue E>
__device__ __forceinline__ void finish_quad(const Mx4Args& a, int64_t row, int n, f32x4 v, const f32x4& up) {
    f32x4 r;
    if constexpr (E == FUSED) {
        r = load_quad(a, a.residual, row * a.ld_residual + n, n);
        const f32x4 b = load_quad(a, a.bias, n, n);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += b[i];
    }
    mx4_with_activation(a.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = mx4_activation<decltype(act)::value>(v[i]);
    });
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = E == FUSED ? v[i] + r[i] : v[i] * up[i];
    if (a.out_f32) store_quad<float>(a, (float*)a.out, a.ld_out, a.wide, row, n, v);
    else store_quad<uint16_t>(a, (uint16_t*)a.out, a.ld_out, a.wide, row, n, v);
}
// A wave's tiles, the first row row0 and column n0 of the output; part: where k is split.  With an epilogue they go through LDS (the wave's own `lds`, PASS * NT KiB), `PASS` tiles of rows at a
// time: whole rows of the wave are then stored, and residuals read, side by side, and the epilogue's code stands there once for all tiles (in place
// it took the compiler four times as long).  In LDS a row's quads are exchanged among the sixteen rows, so that those of one row lie on different banks.
template <class T, Epilogue E, int RT, int NT, int PASS>
__device__ __forceinline__ void finish_tiles(const Mx4Args& a, float* part, int64_t row0, int n0, const f32x4 (&acc)[RT][NT], uint8_t* lds) {
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    if constexpr (E == PLAIN) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int64_t row = row0 + 16 * r + c16;
            if (row >= a.rows) continue;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (part) store_quad<float>(a, part, a.N, a.N % 4 == 0, row, n0 + 16 * t + 4 * g, acc[r][t]);
                else store_quad<T>(a, (T*)a.out, a.ld_out, a.wide, row, n0 + 16 * t + 4 * g, acc[r][t]);
            }
        }
    } else {
        constexpr int PAIR = E == GATED ? 2 : 1, QUADS = 4 * NT / PAIR;   // of a row
        auto place = [&](int r, int t, int row, int quad) { return lds + (r * NT + t) * 1024 + quad * 256 + ((row ^ (4 * (t / PAIR) + quad)) & 15) * 16; };
#pragma unroll
        for (int r0 = 0; r0 < RT; r0 += PASS) {
#pragma unroll
            for (int r = r0; r < (r0 + PASS < RT ? r0 + PASS : RT); ++r)
#pragma unroll
                for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(place(r - r0, t, c16, g)) = acc[r][t];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wave reads what its other lanes have written
            const int rows = (r0 + PASS < RT ? PASS : RT - r0) * 16;
#pragma unroll 1
            for (int u = lane; u < rows * QUADS; u += 64) {
                const int r = u / QUADS, q = u % QUADS, n = n0 + 4 * q;
                const int64_t row = row0 + 16 * r0 + r;
                if (row >= a.rows || n >= a.N) continue;
                const f32x4 v = *reinterpret_cast<const f32x4*>(place(r / 16, q / 4 * PAIR, r & 15, q & 3));
                f32x4 up = v;
                if constexpr (E == GATED) up = *reinterpret_cast<const f32x4*>(place(r / 16, q / 4 * PAIR + 1, r & 15, q & 3));
                if (part) {
                    store_quad<float>(a, part, PAIR * a.N, a.N % 4 == 0, row, n, v);
                    if constexpr (E == GATED) store_quad<float>(a, part + a.N, PAIR * a.N, a.N % 4 == 0, row, n, up);
                } else {
                    finish_quad<E>(a, row, n, v, up);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before it is written again
        }
    }
}
// and one column
template <Epilogue E>
__device__ __forceinline__ void finish_one(const Mx4Args& a, int64_t row, int n, float v, float up) {
    const int64_t at = row * a.ld_out + n;
    auto load = [&](const void* p, int64_t i) { return a.out_f32 ? ((const float*)p)[i] : bf16_bits_to_f32(((const uint16_t*)p)[i]); };
    float r = 0.f;
    if constexpr (E == FUSED) {
        if (a.residual) r = load(a.residual, row * a.ld_residual + n);
        if (a.bias) v += load(a.bias, n);
    }
    mx4_with_activation(a.act, [&](auto act) { v = mx4_activation<decltype(act)::value>(v); });
    v = E == FUSED ? v + r : v * up;
    if (a.out_f32) store_as((float*)a.out + at, v);
    else store_as((uint16_t*)a.out + at, v);
}
// Row `row` of the 16 of stacked tile `tile`, counted from the workgroup's first column n: of the gate's and the up matrix in turn, or of the one that there is
template <Epilogue E>
__device__ __forceinline__ int64_t tile_row(const Mx4Args& a, int n, int tile, int row) {
    return min(n + 16 * (E == GATED ? tile >> 1 : tile) + row, a.N - 1);
}
template <Epilogue E>
__device__ __forceinline__ const uint8_t* tile_codes(const Mx4Args& a, int tile) { return E == GATED && (tile & 1) ? a.up_codes : a.codes; }
template <Epilogue E>
__device__ __forceinline__ const uint8_t* tile_scales(const Mx4Args& a, int tile) { return E == GATED && (tile & 1) ? a.up_scales : a.scales; }

// Up to sixteen rows: reading the weights is what costs, and latency where they are few: 6144 x 4096 at one row (13.4 MB) takes 5.5 us, of which about four are a launch
// and one request's way; 28672 x 4096 at one row 13.1 us (4.8 TB/s) while the memory-side cache holds the matrix and 17.3 where it is read from memory, at 16 18.1 and 23.1.
// In 32 bits 26.3 and 40.8: every workgroup cuts all sixteen places into planes.  Rows of x are read a lane a row, which the address unit takes line by line.
// 16 * NT columns a workgroup, the chunks of 128 k dealt to its eight waves, whose sums meet in LDS.  A wave has U chunks under
// way at a time: their codes and powers go into LDS (see the next kernel for the order), its activations straight into the operand's registers: a
// row that is not there is not asked for.  32-bit activations are cut into their planes here.
constexpr int kFewWaves = 8;
template <class T, class X, int NT, int U, Epilogue E>
__global__ __launch_bounds__(64 * kFewWaves) void mx4_few_kernel(Mx4Args a) {
    static_assert(E != GATED || NT % 2 == 0, "");
    constexpr int P = sizeof(X) == 4 ? 3 : 1, WAVE = U * NT * 1280, SUMS = 16 * (16 * NT + 1) * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kFewWaves * (WAVE > SUMS ? WAVE : SUMS)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    constexpr int COLS = E == GATED ? 8 * NT : 16 * NT;
    const int n0 = blockIdx.x * COLS, row16 = lane >> 2, piece = (lane & 3) ^ (lane >> 4);
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
                const int64_t at = tile_row<E>(a, n0, t, row16) * blocks + chunk * 4;
                lds_fetch16(chunk * 4 + piece < blocks ? (const void*)(tile_codes<E>(a, t) + (at + piece) * 16) : &g_zeros, to + (u * NT + t) * 1024);
                lds_fetch1(chunk * 4 + (lane & 3) < blocks ? (const void*)(tile_scales<E>(a, t) + at + (lane & 3)) : &g_zeros, to + U * NT * 1024 + (u * NT + t) * 256);
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
                    three_planes(v, planes);
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
    for (int u = threadIdx.x; u < a.rows * COLS; u += 64 * kFewWaves) {
        const int r = u / COLS, c = u % COLS, at = E == GATED ? c / 16 * 32 + c % 16 : c;
        if (n0 + c >= a.N) continue;
        float v = 0.f, up = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            v += sums[(w * 16 + r) * LD + at];
            if constexpr (E == GATED) up += sums[(w * 16 + r) * LD + at + 16];
        }
        if constexpr (E == PLAIN) store_as((T*)a.out + r * a.ld_out + n0 + c, v);
        else finish_one<E>(a, r, n0 + c, v, up);
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
template <class T, int P, int RT, int NT, int WN, int WK, int WJ, int ST, Epilogue E>
__global__ __launch_bounds__(512) void mx4_stream_kernel(Mx4Args a) {
    static_assert(WN * WK * WJ == 8 && WK * WJ > 1 && (E != GATED || NT % 2 == 0), "");
    constexpr int XF = RT * 4, CF = NT * WN;                    // operand fragments (1 KiB) of a chunk: activations, codes
    constexpr int C0 = XF * 1024, S0 = C0 + CF * 1024, CHUNK = S0 + CF * 256, STAGE = WK * CHUNK;
    constexpr int WC = WN * WJ, XW = XF / WC, CW = CF / WC;     // waves of a chunk, and what one requests of it
    constexpr int OPS = XW + 2 * CW, J = 4 / WJ;
    static_assert(XF % WC == 0 && CF % WC == 0 && OPS * (ST - 2) < 64 && ST * STAGE <= 160 * 1024 && WN * RT * NT * 1024 <= ST * STAGE, "");
    __shared__ __attribute__((aligned(16))) uint8_t lds[ST * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const int wn = wave % WN, wj = wave / WN % WJ, wk = wave / WC, wq = wave % WC;
    constexpr int TILE = E == GATED ? 8 : 16;                    // output columns of a tile
    const int nb = blockIdx.x * (TILE * CF), n0 = nb + wn * TILE * NT;
    const int blocks = a.K / kMxBlock, chunks = (blocks + 3) / 4;
    const int per = (chunks + gridDim.z - 1) / gridDim.z, c0 = blockIdx.z * per, c1 = min(chunks, c0 + per), steps = (c1 - c0 + WK - 1) / WK * P;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int row16 = lane >> 2, piece = (lane & 3) ^ (lane >> 4);   // what the lane requests of sixteen rows
    const uint8_t *code[CW], *power[CW];
#pragma unroll
    for (int t = 0; t < CW; ++t) {
        const int64_t at = tile_row<E>(a, nb, wq * CW + t, row16) * blocks;
        code[t] = tile_codes<E>(a, wq * CW + t) + (at + piece) * 16;
        power[t] = tile_scales<E>(a, wq * CW + t) + at + (lane & 3);
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
            if (!full && chunk * 4 + (f & 3) >= end) src = &g_zeros;
            lds_fetch16(src, to + f * 1024);
        } else if (i < XW + CW) {
            src = code[i - XW] + (int64_t)chunk * 64;
            if (!full && chunk * 4 + piece >= end) src = &g_zeros;
            lds_fetch16(src, to + C0 + (wq * CW + i - XW) * 1024);
        } else {
            src = power[i - XW - CW] + chunk * 4;
            if (!full && chunk * 4 + (lane & 3) >= end) src = &g_zeros;
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
    {   // the sums of the waves that had other parts of k, in their order
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
    // what is in LDS by now is the wave's own
    finish_tiles<T, E, RT, NT, RT>(a, gridDim.z > 1 ? a.part + (int64_t)blockIdx.z * a.rows * a.N * (E == GATED ? 2 : 1) : nullptr, 0, n0, acc, lds + wn * RT * NT * 1024);
}

// Many rows, where the matrix cores are what is short: 28672 x 4096 at 2048 rows in bf16 takes 394 to 423 us from card to card, 1.14 to 1.22 PFLOP/s, the dense
// bf16 product of the library 400; 5120 x 13824 at 150 rows in 32 bits (three planes) 65 us and 15 for planes and joining.
// 16 * RT * WR rows and 16 * NT * WN columns a workgroup, a wave RT x NT tiles.  Activations,
// codes and powers go through LDS as above, the next step's on their way while one is computed on.  Two places for the activations; codes and powers,
// which a wave takes into registers when it enters the step, have one.
template <class T, int P, int RT, int NT, int WR, int WN, Epilogue E>
__global__ __launch_bounds__(64 * WR * WN, 2) void mx4_tile_kernel(Mx4Args a) {
    constexpr int WAVES = WR * WN, XF = RT * WR * 4, XW = XF / WAVES, CF = NT * WN, CW = CF / WAVES;
    constexpr int C0 = 2 * XF * 1024, S0 = C0 + CF * 1024;
    static_assert(2 * CF / WAVES + XF / WAVES <= 4 * RT && XF % WAVES == 0 && CF % WAVES == 0 && S0 + CF * 256 <= 160 * 1024, "");
    __shared__ __attribute__((aligned(16))) uint8_t lds[S0 + CF * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    // Workgroups are dealt to the eight XCDs in turn.  An XCD gets the row tiles of every eighth column tile, whose codes it then reads once; those of the
    // last few column tiles are dealt evenly.
    constexpr int TILE = E == GATED ? 8 : 16;   // output columns of a tile
    const int col_tiles = (a.N + TILE * CF - 1) / (TILE * CF), row_tiles = (a.rows + 16 * RT * WR - 1) / (16 * RT * WR);
    const int groups = col_tiles * a.splits, even = groups / 8 * row_tiles, rest = groups % 8 * row_tiles;
    const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3, late = xcd * ((rest + 7) / 8) + local - even;
    if (local >= even && late >= min(rest, (xcd + 1) * ((rest + 7) / 8))) return;
    const int group = local < even ? local / row_tiles * 8 + xcd : groups / 8 * 8 + late / row_tiles;
    const int row_tile = local < even ? local % row_tiles : late % row_tiles, col_tile = group % col_tiles, split = group / col_tiles;
    const int n0 = col_tile * (TILE * CF), row0 = row_tile * (16 * RT * WR), wr = wave / WN, wn = wave % WN;
    const int blocks = a.K / kMxBlock, chunks = (blocks + 3) / 4;
    const int per = (chunks + a.splits - 1) / a.splits, c0 = split * per, steps = (min(chunks, c0 + per) - c0) * P;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int row16 = lane >> 2, piece = (lane & 3) ^ (lane >> 4);
    const uint8_t *code[CW], *power[CW];
#pragma unroll
    for (int t = 0; t < CW; ++t) {
        const int64_t at = tile_row<E>(a, n0, wave * CW + t, row16) * blocks;
        code[t] = tile_codes<E>(a, wave * CW + t) + (at + piece) * 16;
        power[t] = tile_scales<E>(a, wave * CW + t) + at + (lane & 3);
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
            if (!full && chunk * 4 + piece >= end) src = &g_zeros;
            lds_fetch16(src, lds0 + C0 + (wave * CW + i) * 1024);
        } else if (i < 2 * CW) {
            src = power[i - CW] + chunk * 4;
            if (!full && chunk * 4 + (lane & 3) >= end) src = &g_zeros;
            lds_fetch1(src, lds0 + S0 + (wave * CW + i - CW) * 256);
        } else {
            const int f = wave * XW + i - 2 * CW;
            src = x[i - 2 * CW] + (plane * a.plane + (int64_t)chunk * 128);
            if (!full && chunk * 4 + (f & 3) >= end) src = &g_zeros;
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
    if constexpr (E != PLAIN) __syncthreads();
    constexpr int PASS = (RT + 1) / 2;
    static_assert(E == PLAIN || WAVES * PASS * NT * 1024 <= S0 + CF * 256, "");
    finish_tiles<T, E, RT, NT, PASS>(a, a.splits > 1 ? a.part + (int64_t)split * a.rows * a.N * (E == GATED ? 2 : 1) : nullptr, row0 + 16 * wr * RT, n0 + TILE * wn * NT, acc,
                                     lds + wave * PASS * NT * 1024);
}

// out = sum of the parts along k, in their order: four columns a lane, up to eight parts on their way at a time
template <class T, Epilogue E>
__global__ __launch_bounds__(256) void mx4_join_kernel(Mx4Args a, int splits) {
    constexpr int PAIR = E == GATED ? 2 : 1;
    const int quads = (a.N + 3) / 4;
    const int64_t total = (int64_t)a.rows * quads, stride = (int64_t)gridDim.x * 256, part = (int64_t)a.rows * a.N * PAIR;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += stride) {
        const int64_t row = total >> 32 ? u / quads : (uint32_t)u / (uint32_t)quads;
        const int n = 4 * (int)(u - row * quads);
        const float* at = a.part + row * PAIR * a.N + n;
        f32x4 v = {0.f, 0.f, 0.f, 0.f}, up = v;
        int z = 0;
        auto parts = [&](auto count) {
            constexpr int Z = decltype(count)::value;
            f32x4 x[Z][PAIR];
#pragma unroll
            for (int i = 0; i < Z; ++i)
#pragma unroll
                for (int m = 0; m < PAIR; ++m) {
                    const float* p = at + (z + i) * part + m * a.N;
                    if (a.N % 4 == 0) x[i][m] = *reinterpret_cast<const f32x4*>(p);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[i][m][e] = n + e < a.N ? p[e] : 0.f;
                }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < Z; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = z + i == 0 ? x[i][0][e] : v[e] + x[i][0][e];
                    if constexpr (E == GATED) up[e] = z + i == 0 ? x[i][1][e] : up[e] + x[i][1][e];
                }
            z += Z;
        };
        while (z + 8 <= splits) parts(std::integral_constant<int, 8>{});
        if (z + 4 <= splits) parts(std::integral_constant<int, 4>{});
        if (z + 2 <= splits) parts(std::integral_constant<int, 2>{});
        if (z < splits) parts(std::integral_constant<int, 1>{});
        if constexpr (E == PLAIN) store_quad<T>(a, (T*)a.out, a.ld_out, a.wide, row, n, v);
        else finish_quad<E>(a, row, n, v, up);
    }
}

template <class T, class X, Epilogue E>
static hipError_t multiply_few(const Mx4Args& a, int cols, hipStream_t st) {
    if (E == GATED) cols = std::max(cols, 32);   // a tile of each matrix
    const int each = E == GATED ? cols / 2 : cols;
    const dim3 grid((a.N + each - 1) / each), block(64 * kFewWaves);
    if (cols == 64) hipLaunchKernelGGL((mx4_few_kernel<T, X, 4, 2, E>), grid, block, 0, st, a);
    else if (cols == 32) hipLaunchKernelGGL((mx4_few_kernel<T, X, 2, 2, E>), grid, block, 0, st, a);
    else if constexpr (E != GATED) hipLaunchKernelGGL((mx4_few_kernel<T, X, 1, 4, E>), grid, block, 0, st, a);
    return hipGetLastError();
}

template <class T, int P, Epilogue E>
static hipError_t multiply(const Mx4Args& a, const Mx4Plan& p, hipStream_t st) {
    const int each = E == GATED ? p.cols / 2 : p.cols;
    if (p.kind == Mx4Plan::STREAM) {
        const dim3 grid((a.N + each - 1) / each, 1, p.splits);
        // RT, NT, WN, WK, WJ, ST
        const dim3 block(512);
        if (p.rt == 2 && p.cols == 128) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 2, 2, 4, 2, 1, 4, E>), grid, block, 0, st, a);
        else if (p.rt == 2) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 2, 2, 2, 2, 2, 4, E>), grid, block, 0, st, a);
        else if (p.rt == 4 && p.cols == 128) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 4, 2, 4, 2, 1, 3, E>), grid, block, 0, st, a);
        else if (p.rt == 4) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 4, 2, 2, 2, 2, 3, E>), grid, block, 0, st, a);
        else if (p.cols == 128) hipLaunchKernelGGL((mx4_stream_kernel<T, P, 8, 2, 4, 1, 2, 3, E>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((mx4_stream_kernel<T, P, 8, 2, 2, 2, 2, 2, E>), grid, block, 0, st, a);
    } else {
        const long long groups = (long long)((a.N + each - 1) / each) * p.splits, rows = (a.rows + 32 * p.rt - 1) / (32 * p.rt);
        const dim3 grid((unsigned)(8 * (groups / 8 * rows + (groups % 8 * rows + 7) / 8)));
        if (p.rt == 8) hipLaunchKernelGGL((mx4_tile_kernel<T, P, 8, 4, 2, 4, E>), grid, dim3(512), 0, st, a);
        else if (p.rt == 7) hipLaunchKernelGGL((mx4_tile_kernel<T, P, 7, 4, 2, 4, E>), grid, dim3(512), 0, st, a);
        else if (p.rt == 6) hipLaunchKernelGGL((mx4_tile_kernel<T, P, 6, 4, 2, 4, E>), grid, dim3(512), 0, st, a);
        else if (p.rt == 5) hipLaunchKernelGGL((mx4_tile_kernel<T, P, 5, 4, 2, 4, E>), grid, dim3(512), 0, st, a);
        else hipLaunchKernelGGL((mx4_tile_kernel<T, P, 4, 4, 2, 2, E>), grid, dim3(256), 0, st, a);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if (p.splits > 1) {
        const int64_t total = (int64_t)a.rows * ((a.N + 3) / 4);
        hipLaunchKernelGGL((mx4_join_kernel<T, E>), dim3((unsigned)std::min<int64_t>((total + 255) / 256, 8192)), dim3(256), 0, st, a, p.splits);
    }
    return hipGetLastError();
}

// With an epilogue the kernels' type T says nothing: what out, bias and residual are is asked where they are read and stored.
template <Epilogue E>
static hipError_t linear(const Mx4Linear& m, void* workspace, hipStream_t st) {
    const Mx4Plan p = mx4_plan(E == GATED ? 2 * m.N : m.N, m.K, m.rows, m.x_f32 ? 3 : 1);
    const size_t out_size = m.out_f32 ? 4 : 2;
    typedef std::conditional_t<E == PLAIN, uint16_t, float> Bf16;   // no kernels that no call reaches
    auto quads = [&](const void* q, int64_t ld) { return (uintptr_t)q % (4 * out_size) == 0 && ld % 4 == 0; };
    Mx4Args a{m.codes, m.scales, (const uint16_t*)m.x, m.ld_x, 0, m.ld_out, m.N, m.K, m.rows, m.out, (float*)workspace, quads(m.out, m.ld_out), p.splits,
              m.up_codes, m.up_scales, m.bias, m.residual, m.ld_residual, m.act, quads(m.bias, 0) && quads(m.residual, m.ld_residual), m.out_f32};
    if (p.kind == Mx4Plan::FEW) {
        if (m.x_f32) return E == PLAIN && !m.out_f32 ? multiply_few<Bf16, float, E>(a, p.cols, st) : multiply_few<float, float, E>(a, p.cols, st);
        return E == PLAIN && !m.out_f32 ? multiply_few<Bf16, uint16_t, E>(a, p.cols, st) : multiply_few<float, uint16_t, E>(a, p.cols, st);
    }
    if (m.x_f32) {
        a.x = (const uint16_t*)workspace;
        a.ld_x = m.K;
        a.plane = (int64_t)m.rows * m.K;
        a.part = (float*)((char*)workspace + align256((size_t)3 * m.rows * m.K * 2));
        if (hipError_t e = launch_mx4_planes((const float*)m.x, m.ld_x, m.rows, m.K, (uint16_t*)workspace, a.plane, st)) return e;
        return E == PLAIN && !m.out_f32 ? multiply<Bf16, 3, E>(a, p, st) : multiply<float, 3, E>(a, p, st);
    }
    return E == PLAIN && !m.out_f32 ? multiply<Bf16, 1, E>(a, p, st) : multiply<float, 1, E>(a, p, st);
}

}  // namespace sun
