// Microscaled 4-bit floats: 32 consecutive columns of a row share a power of two 2^(s - 127), s a byte, and each value is an e2m1 code
// (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), as in the Open Compute Project's microscaling formats 1.0.  Codes are two a
// byte, the even column in the low half.
#include <math.h>

#include "mx4_product.hpp"

namespace sun {

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

// ---------------------------------------------------------------- product (mx4_product.hpp)

// The planes of 32-bit activations for more than sixteen rows, once for all workgroups.  A lane takes eight.  150 x 13824: 6 us.
__global__ __launch_bounds__(256) void mx4_planes_kernel(const float* x, int64_t ld_x, int rows, int K, uint16_t* planes, int64_t plane) {
    const int64_t octets = (int64_t)rows * (K / 8), stride = (int64_t)gridDim.x * 256;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < octets; u += stride) {
        const int64_t row = u / (K / 8), k = u % (K / 8) * 8;
        float v[8];
        load8(x + row * ld_x + k, v);
        bf16x8 w[3];
        three_planes(v, w);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<bf16x8*>(planes + p * plane + row * K + k) = w[p];
    }
}
hipError_t launch_mx4_planes(const float* x, int64_t ld_x, int rows, int K, uint16_t* planes, int64_t plane, hipStream_t st) {
    hipLaunchKernelGGL(mx4_planes_kernel, dim3(unit_grid((int64_t)rows * (K / 8), 1)), dim3(256), 0, st, x, ld_x, rows, K, planes, plane);
    return hipGetLastError();
}

// How a product is dealt to workgroups.  Times in microseconds, measured on the 8B and 14B shapes' matrices with one plane of activations: a chunk
// of 128 k takes a streaming workgroup of 128 (64) columns 0.40 (0.28) with 32 rows, 0.60 (0.45) with 64, 0.90 (0.80) with 128; narrower ones were
// never faster.  A step of 128 k takes a tile of 256 columns and 32 * rt rows 0.9 + 0.275 * rt (3.1 with 256 rows), one or two of 128 x 128 on a
// compute unit 1.2 and 2.0.  A joining launch takes 4 and its parts' bytes at 4 TB/s.  Tiles of 160, 192 and 224 rows against 256 and 128 alone:
// 5120 x 13824 at 150 rows in 32 bits 95 -> 75 us, 14336 x 4096 at 1500 171 -> 149, 20000 x 5120 at 400 in 32 bits 267 -> 233; the
// worst that the estimate does is 28672 x 4096 at 192 rows, 57.5 -> 61.6.
constexpr int kMx4SplitRows = 1 << 17;   // more rows are never split along k
Mx4Plan mx4_plan(int N, int K, int rows, int planes) {
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

hipError_t launch_mx4_linear(const Mx4Linear& m, void* workspace, hipStream_t st) {
    if (m.up_codes) return launch_mx4_gated(m, workspace, st);
    return m.bias || m.residual || m.act != SUN_ACT_NONE ? launch_mx4_fused(m, workspace, st) : linear<PLAIN>(m, workspace, st);
}

}  // namespace sun
