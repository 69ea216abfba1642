// The 8-bit paged cache: keys and values rotated, rounded and appended, and attention of one new token over them.
//
// A cached vector y of head_dim values is stored as e4m3 codes and one power of two: with e the smallest integer >= -100 for
// which the largest finite |y| is at most 448 * 2^e, code = e4m3(y * 2^-e) and the scale byte is e + 127.  Scaling by a power of
// two is exact, so a value has one rounding (2^-4 of itself at most, above the format's subnormals), and the power can be applied behind a
// product: to a key's score, and to a value's weight.
#include <float.h>
#include <math.h>

#include "kernels.hpp"
#include "lowbit.hpp"
#include "rows.hpp"

namespace sun {

void kv8_thetas(const sun_model_cfg& c, double* theta) {
    EmbedRope e{};
    e.d = c.head_dim, e.base = c.rope_base;
    e.rs = RopeScale{c.rope_scaling, c.rope_original_max_position, (double)c.rope_factor, (double)c.rope_low_freq_factor, (double)c.rope_high_freq_factor};
    for (int j = 0; j < c.head_dim / 2; ++j) theta[j] = rope_theta(e, j);
}

struct Kv8AppendArgs {
    uint8_t *codes, *scales;   // the layer's
    int64_t k_page, k_head, v_off, v_page, v_head, s_page, s_head, vs_off;
    Kv8Rows r;
    int n_pages, Hq, Hkv, row_blocks, parts;
    float eps;
    double theta[kKv8Half];
};

template <class T>
__device__ __forceinline__ void load4(const T* p, float (&x)[4]) {
    if constexpr (sizeof(T) == 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(p);
        x[0] = v[0], x[1] = v[1], x[2] = v[2], x[3] = v[3];
    } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        x[0] = bf16_lo(v.x), x[1] = bf16_hi(v.x), x[2] = bf16_lo(v.y), x[3] = bf16_hi(v.y);
    }
}
// Rows of an append from which a workgroup takes four: 4096 rows of a prompt in bf16 25 us, with one row a workgroup 30, in 32 bits with head norms
// 49 / 50; but 1024 rows 13.1 / 10.4 and 2048 14.5 / 15.2 in bf16, 21.9 / 20.1 in 32 bits (8B shape).
constexpr int kKv8ManyRows = 4096;

template <int O>
__device__ __forceinline__ double lane_xor_f64(double v) {
    const uint2 w = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, uint2{lane_xor<O>(w.x), lane_xor<O>(w.y)});
}
template <int LANES, class R>
__device__ __forceinline__ R lanes_sum(R v) {
    auto step = [](auto o, R a) {
        if constexpr (sizeof(R) == 8) return a + lane_xor_f64<decltype(o)::value>(a);
        else return a + lane_xor<decltype(o)::value>(a);
    };
    v = step(std::integral_constant<int, 1>{}, v);
    v = step(std::integral_constant<int, 2>{}, v);
    v = step(std::integral_constant<int, 4>{}, v);
    if constexpr (LANES == 16) v = step(std::integral_constant<int, 8>{}, v);
    return v;
}
// the magnitude that decides a vector's power: not-a-numbers and infinities do not count
__device__ __forceinline__ float finite_abs(float y) {
    const float a = fabsf(y);
    return a < INFINITY ? a : 0.f;
}
// e + 127 for the largest magnitude top; 448 = 1.75 * 2^8
__device__ __forceinline__ int entry_scale(float top) {
    const uint32_t b = __float_as_uint(top);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);   // a subnormal top is far below 448 * 2^-100
    return max(e, -100) + 127;
}
__device__ __forceinline__ uint32_t entry_codes(float a, float b, float c, float d, float inv) {
    const float x[4] = {a, b, c, d};
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(fabsf(x[i]) < INFINITY)) w = (w & ~(255u << (8 * i))) | (0x7fu << (8 * i));
    return w;
}
__device__ __forceinline__ float entry_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// Where a row's key and value go: the page, or -1 for a padding row or a position without a page.
__device__ __forceinline__ int row_page(const Kv8AppendArgs& a, int row, int pos) {
    if (pos < 0) return -1;
    const int req = a.r.requests[row], col = pos / kPageTokens;
    if (req < 0 || req >= a.r.n_requests || col >= a.r.max_pages) return -1;
    const int page = a.r.page_tables[(int64_t)req * a.r.max_pages + col];
    return page >= 0 && page < a.n_pages ? page : -1;
}

// Workgroups [0, row_blocks * parts): q and k of RG rows, head_dim / 8 lanes a head with four pairs each.  The rest: v of 16 rows, a wave
// a head, through LDS, where the dims of a row come to lie side by side as the pool has them.  Queries are computed in 32 bits; keys, which are
// rounded to few bits behind it, in 64 up to one rounding to 32, so that no code depends on the order of operations.
// Memory bounds many rows: 4096 of the 14B shape in 32 bits (q, k, v in, q and codes out: 209 MB) take 48 us, 4.4 TB/s read + written, a large copy's
// 4.95.  Few rows are bound by the chain position -> table -> store and the sine of the angle in 64 bits, which run beside the first loads: 64 rows of the 8B
// shape in bf16 (1.4 MB) take 5.1 us.
template <class T, int D, int RG>
__global__ __launch_bounds__(256) void kv8_append_kernel(Kv8AppendArgs a) {
    constexpr int LPH = D / 8;   // lanes per head
    __shared__ float2 turn[RG][D / 2];
    __shared__ uint32_t vcode[4][16][D / 4 + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int rows = a.r.rows;
    if ((int)blockIdx.x < a.row_blocks * a.parts) {
        const int row0 = ((int)blockIdx.x / a.parts) * RG, part = (int)blockIdx.x % a.parts;
        const int nq = a.r.q ? a.Hq : 0, heads = nq + a.Hkv, total = heads * min(RG, rows - row0);
        const int sub = lane % LPH, j0 = 4 * sub, group = tid / LPH;
        constexpr int GROUPS = 256 / LPH;
        // Vector `at` of the workgroup's rows; behind the last that one again, which is not stored
        struct Vec { int r, head, pos; bool live, is_q; };
        auto vec = [&](int at) {
            const int i = min(at, total - 1), r = i / heads, head = i % heads, pos = a.r.positions[row0 + r];
            return Vec{r, head, pos, at < total && pos >= 0, head < nq};
        };
        float x[4], y[4];
        auto load = [&](const Vec& v) {
            const int64_t row = row0 + v.r;
            const T* src = v.is_q ? (const T*)a.r.q + row * a.r.ld_q + v.head * D : (const T*)a.r.k + row * a.r.ld_k + (v.head - nq) * D;
            load4(src + j0, x);
            load4(src + D / 2 + j0, y);
        };
        Vec v = vec(part * GROUPS + group);
        load(v);   // on its way while the angles are computed
        if (tid < RG * (D / 2)) {
            const int r = tid / (D / 2), j = tid % (D / 2);
            const int pos = row0 + r < rows ? a.r.positions[row0 + r] : -1;
            if (pos >= 0) {
                double sine, cosine;
                sincos((double)pos * a.theta[j], &sine, &cosine);
                turn[r][j] = float2{(float)cosine, (float)sine};
            }
        }
        __syncthreads();
        for (int base = part * GROUPS; base < total; base += a.parts * GROUPS) {   // the same for all lanes, which read one another
            if (base != part * GROUPS) {
                v = vec(base + group);
                load(v);
            }
            const int r = v.r, head = v.head, row = row0 + r, pos = v.pos;
            const bool live = v.live, is_q = v.is_q;
            const T* gain = (const T*)(is_q ? a.r.q_norm : a.r.k_norm);
            float gx[4], gy[4];
            if (gain) {
                load4(gain + j0, gx);
                load4(gain + D / 2 + j0, gy);
            }
            float2 cs[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) cs[i] = turn[r][j0 + i];
            float qa[4], qb[4], ka[4], kb[4];
            if (__any(is_q)) {
                float scale = 1.f;
                if (gain) {
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) ss += x[i] * x[i] + y[i] * y[i];
                    scale = 1.f / sqrtf(lanes_sum<LPH>(ss) / (float)D + a.eps);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float u = gain ? x[i] * scale * gx[i] : x[i], w = gain ? y[i] * scale * gy[i] : y[i];
                    qa[i] = u * cs[i].x - w * cs[i].y;
                    qb[i] = w * cs[i].x + u * cs[i].y;
                }
            }
            if (__any(!is_q)) {
                double scale = 1.0;
                if (gain) {
                    double ss = 0.0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) ss += (double)x[i] * (double)x[i] + (double)y[i] * (double)y[i];
                    scale = 1.0 / sqrt(lanes_sum<LPH>(ss) / (double)D + (double)a.eps);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double u = gain ? x[i] * scale * gx[i] : (double)x[i], w = gain ? y[i] * scale * gy[i] : (double)y[i];
                    ka[i] = (float)(u * cs[i].x - w * cs[i].y);
                    kb[i] = (float)(w * cs[i].x + u * cs[i].y);
                }
            }
            float top = 0.f;
            if (!is_q) {
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(finite_abs(ka[i]), finite_abs(kb[i])));
            }
            top = fmaxf(top, lane_xor<1>(top));
            top = fmaxf(top, lane_xor<2>(top));
            top = fmaxf(top, lane_xor<4>(top));
            if constexpr (LPH == 16) top = fmaxf(top, lane_xor<8>(top));
            if (!live) continue;
            if (is_q) {
                T* dst = (T*)a.r.q_out + ((int64_t)row * a.Hq + head) * D + j0;
                if constexpr (sizeof(T) == 4) {
                    *reinterpret_cast<f32x4*>(dst) = f32x4{qa[0], qa[1], qa[2], qa[3]};
                    *reinterpret_cast<f32x4*>(dst + D / 2) = f32x4{qb[0], qb[1], qb[2], qb[3]};
                } else {
                    *reinterpret_cast<uint2*>(dst) = uint2{pack_bf16(qa[0], qa[1]), pack_bf16(qa[2], qa[3])};
                    *reinterpret_cast<uint2*>(dst + D / 2) = uint2{pack_bf16(qb[0], qb[1]), pack_bf16(qb[2], qb[3])};
                }
                continue;
            }
            const int page = row_page(a, row, pos);
            if (page < 0) continue;
            const int byte = entry_scale(top), slot = pos % kPageTokens, kvh = head - nq;
            const float inv = entry_inverse(byte);
            uint8_t* dst = a.codes + page * a.k_page + kvh * a.k_head + slot * D + j0;
            *reinterpret_cast<uint32_t*>(dst) = entry_codes(ka[0], ka[1], ka[2], ka[3], inv);
            *reinterpret_cast<uint32_t*>(dst + D / 2) = entry_codes(kb[0], kb[1], kb[2], kb[3], inv);
            if (sub == 0) a.scales[page * a.s_page + kvh * a.s_head + slot] = (uint8_t)byte;
        }
        return;
    }
    // ---- v: lane (row lane / 4, quarter lane % 4) of 16 rows
    // Few rows: the four waves of a workgroup have one head, and each stores a quarter of what all four have; a head each otherwise.
    constexpr bool SHARED = RG == 1;
    const int blk = (int)blockIdx.x - a.row_blocks * a.parts, per = SHARED ? a.Hkv : (a.Hkv + 3) / 4;
    const int row0 = (blk / per) * 16, head = SHARED ? blk % per : (blk % per) * 4 + wave;
    const int share = SHARED ? wave : 0, shares = SHARED ? 4 : 1;
    if (head >= a.Hkv) return;   // a wave is by itself from here on
    constexpr int E = 16 / (int)sizeof(T), NL = D / (4 * E);   // values of a load, loads of a lane
    const int r = lane >> 2, quarter = lane & 3, row = min(row0 + r, rows - 1);
    const int pos = row0 + r < rows ? a.r.positions[row] : -1;
    const int page = row_page(a, row, pos);
    const T* src = (const T*)a.r.v + row * a.r.ld_v + head * D + quarter * E;
    float x[NL][E];
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int h = 0; h < E; h += 4) {
            float v[4];
            load4(src + i * 4 * E + h, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][h + e] = v[e];
        }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) top = fmaxf(top, finite_abs(x[i][e]));
    top = fmaxf(top, lane_xor<1>(top));
    top = fmaxf(top, lane_xor<2>(top));
    const int byte = entry_scale(top);
    const float inv = entry_inverse(byte);
    uint8_t* vbase = a.codes + a.v_off + head * a.v_head;
    if (page >= 0 && quarter == 0 && share == 0) a.scales[a.vs_off + page * a.s_page + head * a.s_head + pos % kPageTokens] = (uint8_t)byte;
    uint32_t* mine = &vcode[wave][r][0];
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int h = 0; h < E; h += 4)
            mine[(i * 4 * E + quarter * E + h) / 4] = entry_codes(x[i][h], x[i][h + 1], x[i][h + 2], x[i][h + 3], inv);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // a wave's LDS operations are in order, and other waves use other places
    const uint8_t* got = reinterpret_cast<const uint8_t*>(&vcode[wave][0][0]);
    constexpr int LDR = (D / 4 + 1) * 4;
    // Sixteen rows that are consecutive positions of one request and have their pages leave in groups of four tokens, others byte by byte:
    // lanes side by side on dims, 16 bytes apart.
    const int pos0 = __builtin_amdgcn_readfirstlane(pos), req = row0 + r < rows ? a.r.requests[row] : -1;
    const int req0 = __builtin_amdgcn_readfirstlane(req), count = min(16, rows - row0);
    if (!__all(r >= count || (page >= 0 && req == req0 && pos == pos0 + r))) {
        for (int i = share; i < count; i += shares) {
            const int pg = __shfl(page, i * 4), slot = __shfl(pos, i * 4) & (kPageTokens - 1);
            if (pg < 0) continue;
            uint8_t* dst = vbase + pg * a.v_page + slot;
            for (int dim = lane; dim < D; dim += 64) dst[dim * kPageTokens] = got[i * LDR + dim];
        }
        return;
    }
    for (int quad = (pos0 >> 2) + share; quad <= (pos0 + count - 1) >> 2; quad += shares) {
        const int t0 = quad * 4 - pos0;   // row of the quad's first token
        const int pg = __shfl(page, min(max(t0, 0), count - 1) * 4);
        uint8_t* dst = vbase + pg * a.v_page + (quad & 3) * 4;
        for (int dim = lane; dim < D; dim += 64) {
            uint32_t w = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) w |= (uint32_t)got[min(max(t0 + b, 0), count - 1) * LDR + dim] << (8 * b);
            if (t0 >= 0 && t0 + 3 < count) {
                *reinterpret_cast<uint32_t*>(dst + dim * kPageTokens) = w;
            } else {
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (t0 + b >= 0 && t0 + b < count) dst[dim * kPageTokens + b] = (uint8_t)(w >> (8 * b));
            }
        }
    }
}

struct Kv8AppendGrid {
    bool many;                             // rows by fours
    int64_t row_blocks, parts, v_blocks;   // workgroups of q and k are row_blocks * parts
};
// A row's heads are shared by as many workgroups as keep one pass each, while there are few rows: 64 / 256 rows of the 8B shape 5.8 / 6.6 us with one
// a row, 5.1 / 6.5 shared, but 600 rows 12.6 and 16.8.
static Kv8AppendGrid append_grid(const sun_model_cfg& c, const Kv8Rows& r) {
    const int64_t rows = r.rows, windows = (rows + 15) / 16, lanes = c.head_dim / 8;
    if (rows >= kKv8ManyRows) return Kv8AppendGrid{true, (rows + 3) / 4, 1, windows * ((c.n_kv_heads + 3) / 4)};
    const int64_t passes = (((r.q ? c.n_q_heads : 0) + (int64_t)c.n_kv_heads) * lanes + 255) / 256;
    return Kv8AppendGrid{false, rows, rows <= 256 ? passes : 1, windows * c.n_kv_heads};
}
int64_t kv8_append_groups(const sun_model_cfg& c, const Kv8Rows& r) {
    const Kv8AppendGrid g = append_grid(c, r);
    return g.row_blocks * g.parts + g.v_blocks;
}

template <class T, int D>
static hipError_t append(const Kv8AppendArgs& a, bool many, int64_t groups, hipStream_t st) {
    if (many) hipLaunchKernelGGL((kv8_append_kernel<T, D, 4>), dim3((unsigned)groups), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kv8_append_kernel<T, D, 1>), dim3((unsigned)groups), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv8_append(const Kv8Pool& pool, int layer, const Kv8Rows& r, bool f32, hipStream_t st) {
    const sun_model_cfg& c = pool.cfg;
    const sun_kv8_layout& L = pool.lay;
    Kv8AppendArgs a{};
    a.codes = pool.base + L.k_off + layer * L.k_layer;
    a.scales = pool.base + L.ks_off + layer * L.s_layer;
    a.k_page = L.k_page, a.k_head = L.k_head;
    a.v_off = L.v_off - L.k_off, a.v_page = L.v_page, a.v_head = L.v_head;
    a.s_page = L.s_page, a.s_head = L.s_head, a.vs_off = L.vs_off - L.ks_off;
    a.r = r;
    a.n_pages = (int)L.n_pages, a.Hq = c.n_q_heads, a.Hkv = c.n_kv_heads;
    a.eps = c.rms_eps;
    for (int j = 0; j < c.head_dim / 2; ++j) a.theta[j] = pool.theta[j];
    const Kv8AppendGrid g = append_grid(c, r);
    a.row_blocks = (int)g.row_blocks, a.parts = (int)g.parts;
    const int64_t groups = kv8_append_groups(c, r);
    if (f32) return c.head_dim == 128 ? append<float, 128>(a, g.many, groups, st) : append<float, 64>(a, g.many, groups, st);
    return c.head_dim == 128 ? append<uint16_t, 128>(a, g.many, groups, st) : append<uint16_t, 64>(a, g.many, groups, st);
}

// ---------------------------------------------------------------- attention of one new token
//
// A workgroup takes a chunk of one request's tokens for one KV head; its four waves walk it 64 tokens (four pages) a step, in turn, and
// their results meet in LDS.  With lanes (c = lane % 16, g = lane / 16):
//   scores  S^T = K Q^T, 16 x 16 x 32: row m of tile t (0..3) is token 4 t + m % 4 of page m / 4, so that lane (c, g) gets the scores
//           of head c and all sixteen tokens of page g: 4 t + i from register i of tile t.
//   output  O = P V: the same lane is P's operand for the tokens of page g, and V [dim][token] gives lane (dim, g) those tokens in one load.
// No value moves between lanes on the way.  Heads are at most eight, so the operands' sixteen places hold two of an operand's
// planes: a weight p is carried as bf16(p) and bf16 of the rest (16 bits together, 24 with a third plane for 32-bit calls), and a 32-bit
// query as three truncations of 8 bits, which are exact.  Codes become bf16 exactly.  Powers of two are applied to scores and weights.
// The running maximum and sum are in 32 bits; the sum is over the weights before they are split.
// A step's keys are requested when the step before has its scores, its values when that has its output, page numbers a step ahead of both.
// Reading the cache bounds it.  24 requests of the 14B shape of 2048 to 32768 tokens in bf16 (951 MB): 167 us and 4.7 for joining, 5.5 TB/s; 256 of the 8B shape with a window of
// 1500 in 32 bits (656 MB): 119 us, 5.5 TB/s.  One request of 8191 tokens has two steps' latency and a second launch: 8.1 and 3.2 us for 17 MB.
// Against a wave a chunk, four that share one have a quarter of the partial results; keys by whole token rows and past the caches took 24 long requests from
// 176 to 170 us, values past the caches from 204 to 196.

constexpr int kKv8Step = 64;
constexpr int kKv8Waves = 4;
constexpr int kKv8MinChunk = kKv8Step * kKv8Waves, kKv8MaxChunk = 2048;

// Tokens of a chunk: a power of two that gives about 512 of them (two a compute unit) over the batch if all requests were like this one.  It depends on the
// request's own length, the batch size and the heads, so a request's result does not depend on its batch-mates.  At least a step of each wave.  At most
// 2048: with 512 / 1024 / 2048 the 256 requests with the window took 163 / 148 / 128 us, with 1024 / 2048 the 24 long ones 204 / 190.
constexpr int kKv8Chunks = 512;
__host__ __device__ inline int kv8_chunk(int span, int batch, int Hkv) {
    const long long target = (long long)span * Hkv * batch / kKv8Chunks;
    int ch = kKv8MinChunk;
    while (ch < kKv8MaxChunk && 2 * ch <= target) ch *= 2;
    return ch;
}

struct Kv8AttnArgs {
    const uint8_t *codes, *scales;
    int64_t k_page, k_head, v_off, v_page, v_head, s_page, s_head, vs_off;
    const void* q;
    const int32_t *page_tables, *n_tokens;
    void* out;
    float* partial;     // [batch][chunks][Hq][D], behind them (maximum in powers of two, sum) pairs [batch][chunks][Hq]
    int batch, max_pages, n_pages, Hq, Hkv, window, chunks;
    float c;            // log2(e) / sqrt(D)
};

struct Kv8Span {
    int first, n, chunk, chunks;   // first token of the first page, end, tokens of a chunk, chunks (0: nothing to attend to)
    int lo;
};
__device__ __forceinline__ Kv8Span kv8_span(const Kv8AttnArgs& a, int b) {
    Kv8Span s;
    const long long cap = (long long)a.max_pages * kPageTokens;
    s.n = (int)min((long long)max(a.n_tokens[b], 0), cap);
    s.lo = a.window > 0 ? max(0, s.n - a.window) : 0;
    s.first = s.lo / kPageTokens * kPageTokens;
    const int span = s.n - s.first;
    s.chunk = kv8_chunk(span, a.batch, a.Hkv);
    s.chunks = (span + s.chunk - 1) / s.chunk;
    return s;
}

template <int D>
struct Kv8Parts {   // of the waves
    float o[kKv8Waves][kMaxGroup][D];
    float2 ml[kKv8Waves][kMaxGroup];
};

// Chunk ci of request b, KV head `head`.
template <class T, int D>
__device__ __forceinline__ void kv8_attend(const Kv8AttnArgs& a, int b, int head, int ci, Kv8Parts<D>& parts) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NH = D / 64, NB = D / 16;   // loads of a key's quarter, dim blocks of the output
    auto& part_o = parts.o;
    auto& part_ml = parts.ml;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const Kv8Span s = kv8_span(a, b);
    const int G = a.Hq / a.Hkv;
    if (ci >= s.chunks) {
        if (ci == 0)   // nothing to attend to
            for (int i = threadIdx.x; i < G * D; i += 64 * kKv8Waves) store_as((T*)a.out + ((int64_t)b * a.Hq + head * G) * D + i, 0.f);
        return;
    }
    const int begin = s.first + ci * s.chunk + wave * kKv8Step, end = min(s.n, s.first + (ci + 1) * s.chunk);
    const int32_t* table = a.page_tables + (int64_t)b * a.max_pages;

    // Keys of 128 dims are read in whole token rows, 128 bytes by a pair of lanes c, c ^ 1 and the four g: register h of both is token 2 (c / 2) + h,
    // the even lane has dims 16 g .. of it and the odd one 64 + 16 g .., and they exchange before the scores.  Half rows (each lane its own token) cannot be streamed
    // past the caches without loss.  Keys of 64 dims are whole rows as they are.
    const bool odd = c16 & 1;
    const uint8_t* kb = a.codes + head * a.k_head + 16 * g + (NH == 2 ? (c16 & 2) * D + (odd ? 64 : 0) : (c16 & 3) * D);
    const uint8_t* vb = a.codes + a.v_off + head * a.v_head + c16 * kPageTokens;
    const uint8_t* sb = a.scales + head * a.s_head;
    // Pages of a step: of the lane's key row and of the lane's sixteen tokens.  One that is not there is read as page 0, and left out.
    struct Pages { int k, v; };
    auto pages_at = [&](int tok) {
        const int col = tok / kPageTokens;
        return Pages{table[min(col + (c16 >> 2), a.max_pages - 1)], table[min(col + g, a.max_pages - 1)]};
    };
    auto usable = [&](int page) { return (unsigned)page < (unsigned)a.n_pages; };
    u32x4_s kr[4][NH], vr[NB], ks, vs;
    bool there;                           // whether the lane's page of tokens is
    auto request_k = [&](Pages p) {
        const uint8_t* kp = kb + (int64_t)(usable(p.k) ? p.k : 0) * a.k_page;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int h = 0; h < NH; ++h) kr[t][h] = load_stream(reinterpret_cast<const u32x4_s*>(kp + (4 * t + (NH == 2 ? h : 0)) * D));
        there = usable(p.v);
        ks = *reinterpret_cast<const u32x4_s*>(sb + (int64_t)(there ? p.v : 0) * a.s_page);
    };
    auto request_v = [&](Pages p) {
        const int64_t page = usable(p.v) ? p.v : 0;
        vs = *reinterpret_cast<const u32x4_s*>(sb + a.vs_off + page * a.s_page);
#pragma unroll
        for (int i = 0; i < NB; ++i) vr[i] = load_stream(reinterpret_cast<const u32x4_s*>(vb + page * a.v_page + i * 16 * kPageTokens));
    };

    constexpr int STRIDE = kKv8Step * kKv8Waves;
    bf16x8 q0[NH][2], q2[F32 ? NH : 1][2];
    auto load_q = [&]() {   // operand column c, dims 64 h + 16 g + 8 u .. + 7
        const int hd = c16 & 7;
        const T* qp = (const T*)a.q + ((int64_t)b * a.Hq + head * G + min(hd, G - 1)) * D + 16 * g;
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if constexpr (F32) {
                    u32x4_s w0, w2;
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        uint32_t bits0 = 0, bits2 = 0;
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float x = hd < G ? qp[64 * h + 8 * u + 2 * p + e] : 0.f;
                            if (x != x) x = __uint_as_float(0x7fc00000u);   // one that its upper bits say
                            const float r1 = below(x), r2 = below(r1);
                            const float mine = c16 < 8 ? x : r1;
                            bits0 |= (__float_as_uint(mine) >> 16) << (16 * e);
                            bits2 |= (c16 < 8 ? __float_as_uint(r2) >> 16 : 0u) << (16 * e);
                        }
                        w0[p] = bits0;
                        w2[p] = bits2;
                    }
                    q0[h][u] = __builtin_bit_cast(bf16x8, w0);
                    q2[h][u] = __builtin_bit_cast(bf16x8, w2);
                } else {
                    u32x4_s w = *reinterpret_cast<const u32x4_s*>(qp + 64 * h + 8 * u);
                    if (hd >= G) w = u32x4_s{0, 0, 0, 0};
                    q0[h][u] = __builtin_bit_cast(bf16x8, w);
                }
            }
    };
    f32x4 o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    auto step = [&](int tok, auto more, Pages here) {   // more: a step at `here` follows
        float p[16];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            __builtin_amdgcn_sched_barrier(0);   // codes are converted where they are used: all at once they take twice the registers
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            if constexpr (NH == 2) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t r0 = kr[t][0][e], r1 = kr[t][1][e], got = lane_xor<1>(odd ? r0 : r1);
                    kr[t][0][e] = odd ? got : r0;
                    kr[t][1][e] = odd ? r1 : got;
                }
            }
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bf16x8 k = codes_to_bf16(kr[t][h][2 * u], kr[t][h][2 * u + 1]);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q0[h][u], acc, 0, 0, 0);
                    if constexpr (F32) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q2[h][u], acc, 0, 0, 0);
                }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = acc[i];
                if constexpr (F32) v += lane_xor<8>(v);
                p[4 * t + i] = v * power(ks[t], i);
            }
        }
        // tokens outside [lo, end) and of pages that are not there: no weight, and codes and powers that nobody wrote are not used
        const int at = tok + kPageTokens * g;
        const bool whole = __all(there && at >= s.lo && at + kPageTokens <= end);
        uint32_t live = 0xffff;
        if (!whole) {
            live = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool on = there && at + i >= s.lo && at + i < end;
                live |= (uint32_t)on << i;
                if (!on) p[i] = -INFINITY;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(more)::value) request_k(here);
        __builtin_amdgcn_sched_barrier(0);
        float top = p[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, p[i]);
        {
            float x = top, y = top;
            swap_rows<16>(x, y);
            top = fmaxf(x, y);
            x = y = top;
            swap_rows<32>(x, y);
            top = fmaxf(x, y);
        }
        if (__any(top > m)) {
            const float grown = fmaxf(top, m);
            const float scale = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - grown) * a.c);
            l *= scale;
            m = grown;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = __shfl(scale, (4 * g + i) & 7);
#pragma unroll
                for (int j = 0; j < NB; ++j) o[j][i] *= f;
            }
        }
        const float mc = m == -INFINITY ? 0.f : m * a.c;
        float w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], a.c, -mc));
            l += e;
            w[i] = e * power(vs[i >> 2], i & 3);
        }
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(live >> i & 1)) w[i] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t mask = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) mask |= (live >> (4 * j + e) & 1) ? 255u << (8 * e) : 0u;
#pragma unroll
                for (int i = 0; i < NB; ++i) vr[i][j] &= mask;
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            __builtin_amdgcn_sched_barrier(0);
            u32x4_s w0, w2;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = w[8 * u + 2 * j], y = w[8 * u + 2 * j + 1];
                const uint32_t hi = pack_bf16(x, y);
                const float rx = x - bf16_lo(hi), ry = y - bf16_hi(hi);
                const uint32_t lo = pack_bf16(rx, ry);
                w0[j] = c16 < 8 ? hi : lo;
                if constexpr (F32) w2[j] = c16 < 8 ? pack_bf16(rx - bf16_lo(lo), ry - bf16_hi(lo)) : 0u;
            }
            const bf16x8 p0 = __builtin_bit_cast(bf16x8, w0);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const bf16x8 v = codes_to_bf16(vr[i][2 * u], vr[i][2 * u + 1]);
                o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p0, v, o[i], 0, 0, 0);
                if constexpr (F32) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w2), v, o[i], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(more)::value) request_v(here);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (begin < end) {   // the last step apart: no register is asked for that is not used
        Pages next = pages_at(begin);
        request_k(next);
        request_v(next);
        next = pages_at(begin + STRIDE);
        load_q();
        int tok = begin;
        for (; tok + STRIDE < end; tok += STRIDE) {
            const Pages here = next;
            next = pages_at(tok + 2 * STRIDE);
            step(tok, std::true_type{}, here);
        }
        step(tok, std::false_type{}, next);
        // A head whose every score is minus infinity has weights 0 / 0, not-a-numbers, where one without a token has zeros: its maximum is finite from
        // here on, and its sum 0.  The tokens are looked for again, so that no step has to count them.
        if (__any(m == -INFINITY)) {
            bool any = false;
            for (tok = begin; tok < end; tok += STRIDE) {
                const int at = tok + kPageTokens * g;
                any |= max(at, s.lo) < min(at + kPageTokens, end) && usable(table[min(tok / kPageTokens + g, a.max_pages - 1)]);
            }
            if (__any(any) && m == -INFINITY) m = -FLT_MAX;
        }
    }
    // sums of the four pages' lanes, planes of the output, and both to LDS by the lanes of heads 4 g + i
    {
        float x = l, y = l;
        swap_rows<16>(x, y);
        l = x + y;
        x = y = l;
        swap_rows<32>(x, y);
        l = x + y;
    }
    if (lane < kMaxGroup) part_ml[wave][lane] = float2{m == -INFINITY ? -INFINITY : m * a.c, l};
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v = o[j][i] + lane_xor<32>(o[j][i]);
            if (g < 2) part_o[wave][4 * g + i][16 * j + c16] = v;
        }
    __syncthreads();
    const int64_t at0 = ((int64_t)b * a.chunks + ci) * a.Hq + head * G;
    for (int e = threadIdx.x; e < G * D; e += 64 * kKv8Waves) {
        const int hd = e / D, dim = e % D;
        float top = -INFINITY, sum = 0.f, v = 0.f;
#pragma unroll
        for (int w = 0; w < kKv8Waves; ++w) top = fmaxf(top, part_ml[w][hd].x);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < kKv8Waves; ++w) {
            const float2 ml = part_ml[w][hd];
            const float f = __builtin_amdgcn_exp2f(ml.x - ref);
            sum += f * ml.y;
            v += f * part_o[w][hd][dim];
        }
        if (s.chunks == 1) {
            store_as((T*)a.out + ((int64_t)b * a.Hq + head * G) * D + e, kv8_quotient(v, sum, top));
        } else {
            a.partial[at0 * D + e] = v;
            if (dim == 0) reinterpret_cast<float2*>(a.partial + (int64_t)a.batch * a.chunks * a.Hq * D)[at0 + hd] = float2{top, sum};
        }
    }
}

// A workgroup for every chunk that the table has room for: the ones behind a request's last end at once.
template <class T, int D>
__global__ __launch_bounds__(64 * kKv8Waves, 2) void kv8_attn_kernel(Kv8AttnArgs a) {
    __shared__ Kv8Parts<D> parts;
    const int rest = blockIdx.x / a.Hkv;
    kv8_attend<T, D>(a, rest % a.batch, blockIdx.x % a.Hkv, rest / a.batch, parts);
}

// The chunks that there are, dealt to a fixed number of workgroups, each of which counts them first (one of a request without a token, whose
// output is zeros).  Neighbours in the order of work are kKv8Apart-ths of the list apart: neighbouring chunks of one request at a time are
// slower (64 requests of 8192 tokens: 238 us so, 182 apart).
constexpr int kKv8Apart = 16;
template <class T, int D>
__global__ __launch_bounds__(64 * kKv8Waves, 2) void kv8_attn_dealt_kernel(Kv8AttnArgs a) {
    __shared__ Kv8Parts<D> parts;
    __shared__ int ends[kKv8MaxBatch], sums[kKv8Waves];   // chunks of the requests up to each
    constexpr int EACH = kKv8MaxBatch / (64 * kKv8Waves);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int count[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int b = (int)threadIdx.x * EACH + i;
        count[i] = b < a.batch ? max(kv8_span(a, b).chunks, 1) : 0;
        sum += count[i];
    }
    int before = sum;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int v = __shfl_up(before, o);
        if (lane >= o) before += v;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    before -= sum;
#pragma unroll
    for (int w = 0; w < kKv8Waves - 1; ++w) before += w < wave ? sums[w] : 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) ends[threadIdx.x * EACH + i] = before += count[i];
    __syncthreads();
    const int chunks = ends[a.batch - 1], stretch = (chunks + kKv8Apart - 1) / kKv8Apart, items = stretch * kKv8Apart * a.Hkv;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int place = item / a.Hkv, chunk = place % stretch * kKv8Apart + place / stretch;
        if (chunk >= chunks) continue;
        int lo = 0, hi = a.batch - 1;   // the first request whose chunks end behind this one
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (ends[mid] > chunk) hi = mid;
            else lo = mid + 1;
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        const int first = __builtin_amdgcn_readfirstlane(lo ? ends[lo - 1] : 0);
        kv8_attend<T, D>(a, lo, item % a.Hkv, chunk - first, parts);
        __syncthreads();   // `parts` is written again
    }
}

// out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c over a request's chunks, a workgroup a head: chunk c is wave c % 4's.  The first
// partials are requested before their weights are known.
template <class T, int D>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8AttnArgs a) {
    constexpr int W = 4, U = 8, E = D / 64;   // waves, a wave's partials under way at a time, dims of a lane
    __shared__ float part[W][D];
    __shared__ float sums[W];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq;
    const Kv8Span s = kv8_span(a, b);
    if (s.chunks < 2) return;
    const int64_t at0 = (int64_t)b * a.chunks * a.Hq + h;
    const float2* ml = reinterpret_cast<const float2*>(a.partial + (int64_t)a.batch * a.chunks * a.Hq * D);
    float2 p[U];
    float v[U][E];
    auto request = [&](int c0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = at0 + (int64_t)min(c0 + u * W, s.chunks - 1) * a.Hq;
            p[u] = ml[at];
#pragma unroll
            for (int j = 0; j < E; ++j) v[u][j] = a.partial[at * D + 64 * j + lane];
        }
    };
    request(wave);
    float top = -INFINITY;
    for (int c = lane; c < s.chunks; c += 64) top = fmaxf(top, ml[at0 + (int64_t)c * a.Hq].x);
    top = wave_max(top);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, o[E];
#pragma unroll
    for (int j = 0; j < E; ++j) o[j] = 0.f;
    for (int c0 = wave; c0 < s.chunks; c0 += U * W) {
        if (c0 != wave) request(c0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u * W >= s.chunks) break;
            const float w = __builtin_amdgcn_exp2f(p[u].x - ref);
            sum += w * p[u].y;
#pragma unroll
            for (int j = 0; j < E; ++j) o[j] += w * v[u][j];
        }
    }
#pragma unroll
    for (int j = 0; j < E; ++j) part[wave][64 * j + lane] = o[j];
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    const int dim = threadIdx.x;
    if (dim >= D) return;
    const float l = ((sums[0] + sums[1]) + sums[2]) + sums[3];
    const float r = ((part[0][dim] + part[1][dim]) + part[2][dim]) + part[3][dim];
    store_as((T*)a.out + ((int64_t)b * a.Hq + h) * D + dim, kv8_quotient(r, l, top));
}

int kv8_max_chunks(const sun_model_cfg& c, int batch, int max_pages, int window) {
    long long most = (long long)max_pages * kPageTokens;
    if (window > 0) most = std::min(most, (long long)window + kPageTokens - 1);
    most = std::min(most, 0x7fffffffll);
    // within one length of chunk the longest request has the most of them
    long long chunks = 1;
    const long long per = (long long)c.n_kv_heads * batch;
    for (int ch = kKv8MinChunk; ch <= kKv8MaxChunk; ch *= 2) {
        const long long last = ch == kKv8MaxChunk ? most : std::min(most, (2ll * ch * kKv8Chunks - 1) / per);   // the longest with chunks of at most ch
        if (last > 0) chunks = std::max(chunks, (last + ch - 1) / ch);
    }
    return (int)std::min(chunks, 0x7fffffffll);
}
size_t kv8_partial_floats(const sun_model_cfg& c, int batch, int chunks) {
    return chunks < 2 ? 0 : (size_t)batch * chunks * c.n_q_heads * (c.head_dim + 2);
}

// How chunks come to workgroups.  A workgroup behind a request's last chunk costs 1.25 ns, counting the chunks 1 us and more for each of the 512
// workgroups that are on the chip at a time.  64 requests of 500 tokens, table of 512 / 1024 / 1536 / 2048 / 8192 pages (2048 / 4096 / 6144 / 8192 / 32768
// workgroups): 24.5 / 26.2 / 28.3 / 30.6 / 58 us with a workgroup for each, 30.3 in all five dealt; 64 of 4096 tokens, 6144 / 8192 / 16384: 97.8 / 100.2 / 111
// and 101; 256 of 1000, 16384: 112 and 106; 24 of 2048 to 32768 tokens, 6144: 162 and 158.5.  One to 256 requests on 2 and 8 KV heads, lengths from a
// sixteenth of the table's to all of it: up to 8192 none of 64 is more than 1.5 % faster dealt and 50 are 2 to 30 % slower, at 12288 three of seven are
// faster.  Where one chunk a request is all there can be, none is behind the last: 1024 of 100 tokens 86 us, dealt 106.
constexpr int64_t kKv8Room = 8192;
constexpr int kKv8Dealt = 2048;   // 1024: 256 requests of up to 4000 tokens 170 -> 178 us, 256 of 300 52.7 -> 49.1

template <class T, int D>
static hipError_t attend(const Kv8AttnArgs& a, hipStream_t st) {
    const int64_t room = (int64_t)a.batch * a.Hkv * a.chunks;
    if (a.chunks == 1 || room <= kKv8Room) hipLaunchKernelGGL((kv8_attn_kernel<T, D>), dim3((unsigned)room), dim3(64 * kKv8Waves), 0, st, a);
    else hipLaunchKernelGGL((kv8_attn_dealt_kernel<T, D>), dim3(kKv8Dealt), dim3(64 * kKv8Waves), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.chunks > 1)
        hipLaunchKernelGGL((kv8_join_kernel<T, D>), dim3((unsigned)(a.batch * a.Hq)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv8_attention(const Kv8Pool& pool, int layer, int batch, const void* q, bool f32, const int32_t* page_tables, int max_pages,
                                const int32_t* n_tokens, int window, void* out, float* partial, hipStream_t st) {
    const sun_model_cfg& c = pool.cfg;
    const sun_kv8_layout& L = pool.lay;
    Kv8AttnArgs a{};
    a.codes = pool.base + L.k_off + layer * L.k_layer;
    a.scales = pool.base + L.ks_off + layer * L.s_layer;
    a.k_page = L.k_page, a.k_head = L.k_head;
    a.v_off = L.v_off - L.k_off, a.v_page = L.v_page, a.v_head = L.v_head;
    a.s_page = L.s_page, a.s_head = L.s_head, a.vs_off = L.vs_off - L.ks_off;
    a.q = q, a.page_tables = page_tables, a.n_tokens = n_tokens, a.out = out, a.partial = partial;
    a.batch = batch, a.max_pages = max_pages, a.n_pages = (int)L.n_pages;
    a.Hq = c.n_q_heads, a.Hkv = c.n_kv_heads, a.window = window;
    a.chunks = kv8_max_chunks(c, batch, max_pages, window);
    a.c = 1.4426950408889634f / sqrtf((float)c.head_dim);
    if (f32) return c.head_dim == 128 ? attend<float, 128>(a, st) : attend<float, 64>(a, st);
    return c.head_dim == 128 ? attend<uint16_t, 128>(a, st) : attend<uint16_t, 64>(a, st);
}

}  // namespace sun
