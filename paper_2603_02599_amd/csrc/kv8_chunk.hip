// Attention of a chunk of new tokens of each request over the 8-bit paged cache.
//
// A request's query rows times the G = Hq / Hkv query heads of a KV head are the "places" of a product: place v is row v / G, head v % G.  With S^T = K Q^T and
// O^T = V^T P^T on the 32x32x16 matrix instruction a lane has one place as its column throughout:
//   scores  S^T = K Q^T: lane (c, h) gets scores of place c and the tokens of rows 8 a + 4 h + e; the row's token is chosen as 16 h + 4 a + e, so a lane's sixteen
//           scores are those of one page's tokens in their order, and
//   output  O^T = V^T P^T: the same lane is P's operand for those tokens, V [dim][token] gives lane (dim, h) the page's sixteen in one read.
// No value moves between lanes but for the maximum of the two halves h.  Codes become bf16 exactly, a key's power is applied while its codes are converted (a lane has one
// token's), a value's power to its weight.  bf16 queries enter as they are, 32-bit ones as three planes of 8 bits, exact; a weight of the softmax is two planes
// (16 bits, as in the attention of single tokens: bf16 of it and bf16 of what is left) in bf16 calls, three (24 bits) in 32-bit ones.  With one plane, which is 8 bits, weights that are alike all round the
// same way, and an output is off by up to 2^-8 of itself beside its own rounding: 2048 of 8191 tokens took 266 us so against 352 with two.  Maximum, sum and output are in 32 bits, the sum over the weights before they
// are rounded.
// The reference that scores are taken against is raised to HEAD above the maximum when a score passes it, so that it is raised seldom and a weight is never above 1.
//
// What bounds it, 8B heads (32 and 8 of 128) in bf16: 2048 of 8191 tokens take 350 to 370 us from card to card, 0.65 to 0.69 PFLOP/s, and there vector instructions and products one after another.
// A wave converts a block's 128 codes a lane, half of them keys', and takes 16 exponentials, maxima, sums and roundings for its 24 products; a block of 32 tokens takes the two waves of a SIMD 3580 cycles,
// in which matrix cores are busy for 43 % and vector instructions, products' issue among them, active for 72 %.  Alone, a conversion measures 4.3 cycles, an exponential 8, others 3 and a product 34, in all 3400 for both waves: next to
// nothing runs beside anything, although two waves of independent products and multiply-adds do overlap (24 and 192 of each: 0.70 and 0.50 us alone, 0.85 together).  Products right behind their
// conversions, a conversion ahead, by dims or by halves of the tokens, scores in front of the weights and no priorities all take the same to 3 %.
// The matrix instruction for 8-bit operands would need no conversion, but adds products to 2^-13 of their largest, which loses scores' last bits.
// Four drafted tokens of 64 requests take 70 us, 333 MB at 4.8 TB/s, where reading alone takes 57.  32-bit calls multiply three times (14B heads, window 1000: 98 to 101 us, 67 of them the
// planes' products at the rate of a large product).  Short prompts are bound by what stands in front of a tile's first product, a chain of five loads, and by their longest tile.
#include <float.h>
#include <limits.h>
#include <math.h>

#include "kernels.hpp"
#include "lowbit.hpp"

namespace sun {

// A workgroup's share and what it takes.  128 places, 32 to each of four waves, with two workgroups on a compute unit (77 KB of LDS, up to 256 registers): one computes while the
// other waits.  Eight waves of 256 places, whose blocks are converted once for all of them in LDS, took 340 us for 2048 of 8191 tokens against 299 (with
// weights of one plane), three workgroups a compute unit need 168 registers, which is fewer than there are operands.
constexpr int kTile = 128;
constexpr int kFew = 32;             // requests of so many places at most: the four waves share them and take tokens in turn
constexpr int kWaves = 4;
// Parts of long caches, for 512 workgroups (384 / 512 / 768 / 1024: 24 requests with prompts among them 116 / 87 / 87 / 91 us, four drafted tokens of 64 requests 71 / 71 / 86 / 86, 14B heads
// in 32 bits 101 / 101 / 125 / 125, where each further part is written and joined and the workgroups do not come out even), of 512 tokens at least (256: 64 of 8191 tokens 36 us
// against 33, 512 of 512 23.6 against 23.4; 128: 4 of 8191 20 against 16).  All requests of a call may have as many, whatever their lengths, and with 512 groups of heads and tiles none has: measured
// with lengths within a factor of eight of each other.  One long cache among many short ones is read by the workgroups of its own tiles and heads alone.
constexpr int kMinSplit = 512;
constexpr int kMaxSplits = 64;
constexpr int kGroupsWanted = 512;

// Division by a number that the host knows: a product, and one more where what is left says so.  The dozen divisions in front of a tile's first request took it over a microsecond.
struct Divider {
    uint32_t d, m;   // m = min(2^32 / d, 2^32 - 1): the product's upper word is the quotient or one less
    static Divider of(int d) { return Divider{(uint32_t)d, d == 1 ? ~0u : (uint32_t)((1ull << 32) / d)}; }
    __device__ __forceinline__ int quotient(int v) const {
        const uint32_t q = __umulhi((uint32_t)v, m);
        return (int)(q + ((uint32_t)v - q * d >= d));
    }
};

struct ChunkArgs {
    const uint8_t *codes, *scales;
    int64_t k_page, k_head, v_off, v_head, s_page, s_head, vs_off;   // a page's keys and values lie as far apart as any page's
    const void* q;
    const int32_t *row_starts, *page_tables, *n_tokens;
    void* out;
    float* partial;      // [slot][slot_rows][D], behind them (reference in powers of two, sum) pairs [slot][slot_rows]
    int64_t slots;
    int batch, rows, max_pages, n_pages, Hq, Hkv, window, splits, slot_rows;
    bool sorted;
    Divider G, heads;    // query heads of a KV head, KV heads
    float c;             // log2(e) / sqrt(D)
};

// ---------------------------------------------------------------- what there is to do

struct ChunkRequest { int start, count, n, tiles, splits; };
__device__ __forceinline__ ChunkRequest chunk_request(const ChunkArgs& a, int b) {
    ChunkRequest r{0, 0, 0, 0, 1};
    if (b >= a.batch) return r;
    r.start = min(max(a.row_starts[b], 0), a.rows);
    r.count = max(min(a.row_starts[b + 1], a.rows) - r.start, 0);
    r.n = (int)min((long long)max(a.n_tokens[b], 0), (long long)a.max_pages * kPageTokens);
    const int places = r.count * a.G.d;
    r.tiles = places <= kFew ? places > 0 : (places + kTile - 1) / kTile;
    const long long first = a.window > 0 ? max((long long)r.n - r.count - a.window + 1, 0ll) : 0;
    r.splits = max(1, min(a.splits, (int)((r.n - first + kMinSplit - 1) / kMinSplit)));
    return r;
}

// Sums over the lanes up to each
__device__ __forceinline__ int lanes_before(int v) {
    const auto moved = [](int x, auto ctrl, auto rows) { return __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };   // 0 where nothing moves to
    typedef std::integral_constant<int, 0xf> All;
    v += moved(v, std::integral_constant<int, 0x111>{}, All{});   // from 1, 2, 4 and 8 lanes before, within rows of sixteen
    v += moved(v, std::integral_constant<int, 0x112>{}, All{});
    v += moved(v, std::integral_constant<int, 0x114>{}, All{});
    v += moved(v, std::integral_constant<int, 0x118>{}, All{});
    v += moved(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // a row's last lane to the row behind it
    v += moved(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // lane 31 to the upper half
    return v;
}

struct ChunkPlace {
    ChunkRequest r;
    int b, index;           // request (-1: behind the last), and which of its items or tiles
    long long items;        // of the requests in front
};
// Item `index` of all requests' (a tile's part; TILES: a tile).  The whole wave calls it.
template <bool TILES>
__device__ __forceinline__ ChunkPlace chunk_find(const ChunkArgs& a, long long index) {
    const int lane = threadIdx.x & 63;
    long long items = 0;
    int tiles = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        const ChunkRequest r = chunk_request(a, b0 + lane);
        int t = r.tiles, s = r.tiles * r.splits;
        t = lanes_before(t);
        s = lanes_before(s);
        const long long mine = TILES ? (long long)tiles + t : items + s;
        const uint64_t past = __ballot(mine > index);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
            ChunkPlace p;
            p.r = ChunkRequest{of(r.start), of(r.count), of(r.n), of(r.tiles), of(r.splits)};
            p.b = b0 + l;
            const int before_t = of(t) - p.r.tiles, before_s = of(s) - p.r.tiles * p.r.splits;
            p.items = items + before_s;
            p.index = (int)(index - (TILES ? (long long)tiles + before_t : p.items));
            return p;
        }
        tiles += __builtin_amdgcn_readlane(t, 63);
        items += __builtin_amdgcn_readlane(s, 63);
    }
    ChunkPlace none{};
    none.b = -1;
    return none;
}

// Tile `index` of all requests' in the order of their lengths in steps of 64 tokens, the longest first, where that gains: what starts last has to be short.  For up to kSorted requests,
// one a lane (a limit of the search, not of what gains), without parts, and few rounds of workgroups (the host decides); false where no request is long.  Against requests in turn: prompts of 583 to 1500 tokens 78 -> 76 us,
// four drafted tokens of 64 requests 74 -> 71, 128 of 1000 to 2500 of sixteen 117 -> 103, but 32 prompts of 128 34 -> 43, whose workgroups then all wait and all compute at the
// same time; sixteen prompts of 200 to 1700 (eight rounds) 284 and 280.  Finding a tile takes 2000 cycles, chunk_find 1300.  The whole wave calls it.
constexpr int kSorted = 64, kSortedFrom = 512, kSortedGroups = 2560;
__device__ __forceinline__ bool chunk_longest(const ChunkArgs& a, int index, ChunkPlace& p) {
    const ChunkRequest r = chunk_request(a, threadIdx.x & 63);
    const int G = a.G.d, base = max(r.n - r.count, 0), most = min(r.count, r.n), cap = a.window > 0 ? a.window / 64 + 2 : INT_MAX;
    auto longer = [&](int steps) {   // the lane's request's tiles that end behind so many steps
        const int rows = steps * 64 - base;
        return steps > cap || rows > most ? 0 : rows <= 0 ? r.tiles : r.tiles - (rows * G + kTile - 1) / kTile + 1;
    };
    auto sum = [](int v) { return __builtin_amdgcn_readlane(lanes_before(v), 63); };
    if (!__any(r.tiles && r.n >= kSortedFrom)) return false;
    p = ChunkPlace{};
    p.b = -1;
    const int total = sum(r.tiles);
    if (index >= total) return true;
    // Where all are on the chip at once, two workgroups a compute unit, the second half comes the other way round, so that a unit has a long and a short one
    const int half = (total + 1) / 2;
    if (total * a.Hkv <= 512 && index >= half) index = total - 1 - (index - half);
    int lo = 0, hi = a.max_pages / 4 + 2, in_front = 0;   // more than `index` tiles end behind lo, in_front behind hi and no more than `index`
    while (hi - lo > 1) {
        const int each = (hi - lo + 3) / 4;
        int at[3], n[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) at[i] = min(lo + (i + 1) * each, hi), n[i] = sum(longer(at[i]));
#pragma unroll
        for (int i = 2; i >= 0; --i)
            if (n[i] <= index) hi = at[i], in_front = n[i];
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (n[i] > index) lo = at[i];
    }
    index -= in_front;
    const int behind = longer(hi), mine = longer(lo) - behind, past = lanes_before(mine);
    const int l = __ffsll((unsigned long long)__ballot(past > index)) - 1;
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
    p.r = ChunkRequest{of(r.start), of(r.count), of(r.n), of(r.tiles), 1};
    p.b = l;
    p.index = of(r.tiles) - 1 - of(behind) - (index - (of(past) - of(mine)));
    return true;
}

// ---------------------------------------------------------------- attention of one part

// LDS: blocks of 32 tokens (two pages) of a KV head.  Keys [token][16-byte piece ^ key], values [page][dim][16 tokens], 256 bytes a page of powers (16 of keys, 16 of
// values), and a page's notes, which the wave that requested it writes when it has landed: the powers as floats, whether it is there, and which of its values are not numbers.
struct Notes {
    float powers[32];         // of values, and behind them of keys
    uint32_t there, odd;      // odd: `bad` is to be looked at
    uint32_t unused[14];
    uint16_t bad[128];        // of a dim: its tokens, a bit each
    __device__ bool plain() const { return there && !odd; }
};
template <int D>
struct Block {
    static constexpr int V = 32 * D, S = 64 * D, N = S + 512, BYTES = N + 2 * (int)sizeof(Notes), OPS = 2 * (D / 64) + 1;   // requests of a page
    __device__ static int key(int token) { return D == 128 ? (token & 3) | (token >> 2 & 4) : (token >> 1 & 1) | (token >> 3 & 2); }
    __device__ static const Notes& notes(const uint8_t* block, int half) { return reinterpret_cast<const Notes*>(block + N)[half]; }
};
__device__ __forceinline__ uint32_t not_a_number(uint32_t codes) { return ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }   // the upper bit of each that is
constexpr int kWideStages = 4;
template <int D>
struct ChunkLds {   // two workgroups on a compute unit
    static constexpr int WIDE = kWideStages * 2 * Block<D>::BYTES, FEW = kWaves * 2 * Block<D>::BYTES, SUMS = kWaves * 32 * (D / 2 + 4) * 4 + kWaves * 32 * 8;
    static constexpr int BYTES = WIDE;
    static_assert(WIDE >= FEW && WIDE >= SUMS && 2 * WIDE <= 160 * 1024, "");
};

// What lanes are given of a page that is not there: a block of keys, one of values, powers
static __device__ uint32_t g_no_page[512] = {};

// Requests of pages.  The addresses' lane parts are the same for all pages, so that a page takes scalar instructions alone.
template <int D>
struct PageRequests {
    const uint8_t *codes, *scales;   // the head's
    int64_t k_page, v_off, s_page;
    int n_pages;
    uint32_t k_lane[2], v_lane, s_lane;   // keys by half of the block
    uint32_t there;                       // bit i: whether the page that was requested i pages ago is

    __device__ __forceinline__ void init(const ChunkArgs& a, int head) {
        const int lane = threadIdx.x & 63;
        codes = a.codes + head * a.k_head;
        scales = a.scales + head * a.s_head;
        k_page = a.k_page, v_off = a.v_off + head * (a.v_head - a.k_head), s_page = a.s_page;
        n_pages = a.n_pages;
        constexpr int PIECES = D / 16;
        const int token = lane / PIECES;   // more tokens of a page have the same key
#pragma unroll
        for (int half = 0; half < 2; ++half) k_lane[half] = token * D + ((lane % PIECES) ^ Block<D>::key(kPageTokens * half + token)) * 16;
        v_lane = lane * 16;
        s_lane = (lane & 3) * 4 + (lane & 4 ? (uint32_t)a.vs_off : 0u);   // sixteen powers of keys, sixteen of values, again and again
        there = 0;
    }
    __device__ __forceinline__ void request(int page, int half, uint32_t block) {
        const uint8_t *k = (const uint8_t*)g_no_page, *v = k, *s = k;
        there <<= 1;
        if ((unsigned)page < (unsigned)n_pages) {
            k = codes + (uint64_t)(uint32_t)page * (uint32_t)k_page;   // a page of a layer is less than 2^32 bytes
            v = k + v_off;
            s = scales + (uint64_t)(uint32_t)page * (uint32_t)s_page;
            there |= 1;
        }
        lds_dma16<D / 64>(k, half ? k_lane[1] : k_lane[0], block + half * 16 * D);
        lds_dma16<D / 64>(v, v_lane, block + Block<D>::V + half * 16 * D);
        lds_dma4(s, there & 1 ? s_lane : 0u, block + Block<D>::S + half * 256);   // values' powers may lie further behind than what stands for a page is long
    }
    // Notes of a page that has landed, requested `ago` pages ago, whose first token is `at`.  Powers and values from token n on, which nobody has written, become zeros; where some places see
    // a token and others do not (`partly`), values that are not numbers are noted and become zeros: their product with a weight of 0 would not be.
    // A power of 255 is none: its token's values are all noted as no numbers, whoever sees them.
    __device__ __forceinline__ void note(uint8_t* block, int half, int ago, int at, int n, bool partly) const {
        const int lane = threadIdx.x & 63;
        Notes& notes = reinterpret_cast<Notes*>(block + Block<D>::N)[half];
        const uint8_t* s = block + Block<D>::S + half * 256;
        const uint32_t byte = lane < 32 && at + (lane & 15) < n ? s[lane ^ 16] : 0;   // keys behind values
        const uint32_t lost = (uint32_t)__ballot(byte == 255) & 0xffffu;   // tokens whose values have no power
        if (lane < 32) notes.powers[lane] = lost >> lane & 1 ? 0.f : __uint_as_float(byte << 23);
        bool any = false;
        if (partly || lost) {
#pragma unroll 1
            for (int dim = lane; dim < D; dim += 64) {
                u32x4_s* p = reinterpret_cast<u32x4_s*>(block + Block<D>::V + half * 16 * D + dim * 16);
                u32x4_s x = *p;
                uint32_t mask = lost;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int written = min(max(n - at - 4 * e, 0), 4);
                    x[e] &= written == 4 ? ~0u : (1u << (8 * written)) - 1;
                    const uint32_t bad = not_a_number(x[e]);
                    x[e] &= ~((bad >> 7) * 0xffu);
                    mask |= ((bad >> 7 & 1) | (bad >> 14 & 2) | (bad >> 21 & 4) | (bad >> 28 & 8)) << (4 * e);
                }
                any |= mask != 0;
                notes.bad[dim] = (uint16_t)mask;
                *p = x;
            }
        }
        const uint32_t odd = __any(any) ? 1u : 0u;
        if (lane == 0) notes.there = there >> ago & 1, notes.odd = odd;
    }
};

// A wave's 32 places: operands, and what has been summed up
template <class T, int D>
struct Places {
    static constexpr bool F32 = sizeof(T) == 4;
    // In powers of two: 0 / 6 / 10 take 2048 of 8191 tokens 384 / 372 / 368 us.  An exponential's argument, up to HEAD, rounds to 24 bits of itself, so 32-bit weights have less of it.
    static constexpr float HEAD = F32 ? 6.f : 10.f;
    static constexpr int P = F32 ? 3 : 1, W = F32 ? 3 : 2, KS = D / 16, NB = D / 32;   // planes of a query and of a weight, steps of 16 dims, blocks of 32 dims
    bf16x8 q[P][KS];
    f32x16 o[NB];
    float m, l;        // the reference in powers of two, the lane's half of the sum
    int lo, hi;        // positions that the lane's place sees: lo .. hi
    uint32_t had;      // not 0: one of them was there

    __device__ __forceinline__ void load(const ChunkArgs& a, const ChunkRequest& r, int head, int v) {
        const int G = a.G.d, h = (threadIdx.x & 63) >> 5;
        const bool on = v < r.count * G;
        const int row = on ? a.G.quotient(v) : 0, pos = r.n - r.count + row;
        hi = on ? pos : -1;
        lo = a.window > 0 ? max(pos - a.window + 1, 0) : 0;
        const T* p = (const T*)a.q + ((int64_t)(r.start + row) * a.Hq + head * G + (on ? v - row * G : 0)) * D + 16 * h;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if constexpr (F32) {
                float x[8];
                bf16x8 planes[3];
                load8(p + 32 * (s / 2) + 8 * (s % 2), x);
                three_planes(x, planes);
#pragma unroll
                for (int i = 0; i < 3; ++i) q[i][s] = planes[i];
            } else {
                q[0][s] = *reinterpret_cast<const bf16x8*>(p + 32 * (s / 2) + 8 * (s % 2));
            }
        }
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
        m = -INFINITY;
        l = 0.f;
        had = 0;
    }

    // A block's keys on their way into operands
    struct Keys {
        const uint8_t* at;
        int key;
        float scale;
        u32x4_s codes[KS / 2];
        __device__ __forceinline__ Keys(const uint8_t* block) {
            const int lane = threadIdx.x & 63, c = lane & 31, token = 16 * (c >> 2 & 1) + 4 * (c >> 3) + (c & 3);
            at = block + token * D;
            key = Block<D>::key(token) ^ (lane >> 5);
            scale = Block<D>::notes(block, token >> 4).powers[16 + (token & 15)];
        }
        __device__ __forceinline__ void read(int w) { codes[w] = *reinterpret_cast<const u32x4_s*>(at + ((2 * w) ^ key) * 16); }
    };
    __device__ __forceinline__ void scores(const Keys& k, int i, f32x16& out) const {   // one step of 16 dims
        const bf16x8 x = codes_to_bf16(k.codes[i >> 1][2 * (i & 1)], k.codes[i >> 1][2 * (i & 1) + 1], k.scale);
#pragma unroll
        for (int p = 0; p < P; ++p) out = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q[p][i], out, 0, 0, 0);
    }
    __device__ __forceinline__ f32x16 scores(const uint8_t* block) const {
        Keys k(block);
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        k.read(0);
#pragma unroll
        for (int w = 0; w < KS / 2; ++w) {
            if (w + 1 < KS / 2) k.read(w + 1);
            __builtin_amdgcn_sched_barrier(0);   // all at once they take the registers
            scores(k, 2 * w, s);
            scores(k, 2 * w + 1, s);
        }
        return s;
    }

    // The output's products with a block's values: two of 32 dims.  Nothing but the matrix cores is short here, so they go first (2048 of 8191 tokens 372 -> 368 us).
    typedef u32x4_s Weights[W][2];
    __device__ __forceinline__ u32x4_s values(const uint8_t* block, int j) const {
        const int lane = threadIdx.x & 63;
        return *reinterpret_cast<const u32x4_s*>(block + Block<D>::V + (lane >> 5) * 16 * D + (32 * j + (lane & 31)) * 16);
    }
    __device__ __forceinline__ void add(const u32x4_s& codes, const Weights& w, int j, int u) {
        const bf16x8 x = codes_to_bf16(codes[2 * u], codes[2 * u + 1]);
#pragma unroll
        for (int p = 0; p < W; ++p) o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, w[p][u]), o[j], 0, 0, 0);
    }
    __device__ __forceinline__ void add(const uint8_t* block, const Weights& w) {
        u32x4_s codes = values(block, 0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const u32x4_s now = codes;
            if (j + 1 < NB) codes = values(block, j + 1);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                __builtin_amdgcn_sched_barrier(0);
                add(now, w, j, u);
            }
        }
        __builtin_amdgcn_s_setprio(0);
    }

    // Scores s of the block of tokens at .. at + 31 into weights and the output; meanwhile, NEXT, the scores s2 of the block behind, products and weights in
    // turn.  whole: every place of the wave sees all of the tokens, and nothing has been taken out
    template <bool NEXT>
    __device__ __forceinline__ void step(const ChunkArgs& a, f32x16& s, const uint8_t* block, int at, bool whole, const uint8_t* behind, f32x16& s2) {
        const int h = (threadIdx.x & 63) >> 5;
        const Notes& notes = Block<D>::notes(block, h);
        Keys k(NEXT ? behind : block);
        if constexpr (NEXT) {
#pragma unroll
            for (int i = 0; i < KS / 2; ++i) k.read(i);
        }
        uint32_t live = 0xffff;   // tokens that the lane's place sees
        if (!whole) {
            const int mine = at + 16 * h, from = max(lo - mine, 0), to = min(hi - mine, 15);
            live = notes.there && from <= to ? (0xffffu >> (15 - to)) & (0xffffu << from) : 0u;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = live >> i & 1 ? s[i] : -INFINITY;
            if (__any(notes.odd != 0)) mark(block, live);
        }
        had |= live;
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        {
            float x = top, y = top;
            swap_rows<32>(x, y);
            top = fmaxf(x, y) * a.c;
        }
        if (__any(top > m)) {
            const float grown = top > m ? top + HEAD : m;
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - grown);
            m = grown;
            l *= f;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[j][i] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        Weights words;
        f32x4 vs;
        if constexpr (NEXT) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s2[i] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j % 2 == 0) vs = *reinterpret_cast<const f32x4*>(notes.powers + 2 * j);
            if constexpr (NEXT)
                if (j % (8 / KS) == 0) scores(k, j / (8 / KS), s2);
            float x[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * j + e], a.c, -ref));
            l += x[0] + x[1];
#pragma unroll
            for (int e = 0; e < 2; ++e) x[e] *= vs[(2 * j + e) & 3];
#pragma unroll
            for (int p = 0; p < W; ++p) {
                const uint32_t word = pack_bf16(x[0], x[1]);
                words[p][j >> 2][j & 3] = word;
                x[0] -= bf16_lo(word), x[1] -= bf16_hi(word);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        asm volatile("" : "+v"(l));   // summed here: left to itself the compiler sums later, all in a row
        add(block, words);
    }

    // Not-a-numbers among a block's values into the output of the places that see them
    __device__ __forceinline__ void mark(const uint8_t* block, uint32_t live) {
        const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
        const Notes &first = Block<D>::notes(block, 0), &second = Block<D>::notes(block, 1);
        const uint32_t seen0 = first.odd ? __shfl(live, c) : 0u, seen1 = second.odd ? __shfl(live, c + 32) : 0u;   // `bad` says nothing where a page is not odd
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int dim = 32 * j + 8 * (i >> 2) + 4 * h + (i & 3);
                if ((first.bad[dim] & seen0) | (second.bad[dim] & seen1)) o[j][i] = NAN;
                __builtin_amdgcn_sched_barrier(0);
            }
    }

    // The two halves' sums, and a reference that says whether there was a token
    __device__ __forceinline__ void close() {
        float x = l, y = l;
        swap_rows<32>(x, y);
        l = x + y;
        uint32_t u = had, w = had;
        swap_rows<32>(u, w);
        had = u | w;
        if (m == -INFINITY && had) m = -FLT_MAX;
    }
};

// What a weighted sum is multiplied with: 1 / the weights' sum, 0 where there is no token.  Weights are 2^-HEAD and more at the reference, so a sum is no less, or 0 where all
// scores are minus infinity, which leaves not-a-numbers.
__device__ __forceinline__ float chunk_factor(float sum, float top) { return sum == 0.f && top == -INFINITY ? 0.f : sum == 0.f ? NAN : 1.f / sum; }
template <class T>
__device__ __forceinline__ void store4(T* to, float a, float b, float c, float d) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(to) = f32x4{a, b, c, d};
    else *reinterpret_cast<uint2*>(to) = uint2{pack_bf16(a, b), pack_bf16(c, d)};
}

// The range of a tile's part
struct ChunkRange { int begin, end; };
__device__ __forceinline__ ChunkRange chunk_range(const ChunkArgs& a, const ChunkRequest& r, int places0, int places, int split, int step) {
    const int last = min(places0 + places, r.count * (int)a.G.d) - 1;
    const int hi = r.n - r.count + a.G.quotient(last) + 1, low = a.window > 0 ? max(r.n - r.count + a.G.quotient(places0) - a.window + 1, 0) : 0;
    const int first = low / kPageTokens * kPageTokens, span = max(hi - first, 0);
    const int per = ((r.splits == 1 ? span : (span + r.splits - 1) / r.splits) + step - 1) / step * step;
    const long long begin = first + (long long)split * per;
    return ChunkRange{(int)min(begin, (long long)max(hi, 0)), (int)min(begin + per, (long long)max(hi, 0))};
}

// Four waves of 32 places each over the same tokens, 64 a step: wave w requests the step's page w.
template <class T, int D>
__device__ __forceinline__ void chunk_wide(const ChunkArgs& a, const ChunkPlace& p, int head, int tile, int split, int64_t slot, uint8_t* lds) {
    static_assert(kWideStages == 4, "");
    constexpr int STAGE = 2 * Block<D>::BYTES, OPS = Block<D>::OPS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
    const int G = a.G.d, live = p.r.count * G;
    // Up to 64 places: two waves have the same ones, and one of a step's two blocks each (nine new tokens of 64 requests of 2000 99 -> 82 us, sixteen 99 -> 84)
    const bool pairs = live - tile * kTile <= 64;
    const int v0 = tile * kTile + 32 * (pairs ? wave & 1 : wave);
    const ChunkRange range = chunk_range(a, p.r, tile * kTile, kTile, split, 64);
    const int32_t* table = a.page_tables + (int64_t)p.b * a.max_pages;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    // positions from all_from to low are seen by all of the wave's places
    const int base = p.r.n - p.r.count, low = base + a.G.quotient(v0), high = base + a.G.quotient(min(v0 + 32, live) - 1);
    const int all_from = a.window > 0 ? max(high - a.window + 1, 0) : 0;
    // and the tile's positions from tile_from to tile_to by all of its places
    const int tile_to = base + a.G.quotient(tile * kTile), tile_from = a.window > 0 ? max(base + a.G.quotient(min((tile + 1) * kTile, live) - 1) - a.window + 1, 0) : 0;
    Places<T, D> w;
    auto page_at = [&](int token) { return token < range.end ? load_uniform(table + min(token / kPageTokens, a.max_pages - 1)) : -1; };
    int ahead = range.begin + wave * kPageTokens, fill = 0;
    int page = page_at(ahead);
    PageRequests<D> pages;
    pages.init(a, head);
    auto request = [&]() {
        pages.request(page, wave & 1, lds0 + fill * STAGE + (wave >> 1) * Block<D>::BYTES);
        ahead += 64;
        page = page_at(ahead);
        fill = fill + 1 & 3;
    };
    auto note = [&](int stage, int ago, int token) {
        pages.note(lds + stage * STAGE + (wave >> 1) * Block<D>::BYTES, wave & 1, ago, token + 16 * wave, p.r.n, token < tile_from || token + 63 > tile_to);
    };
    request();
    request();
    w.load(a, p.r, head, v0 + c);   // behind the requests, whose way it shares
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(OPS) : "memory");
    note(0, 1, range.begin);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    // A step: the one two behind it is requested in the place of the one two before it, with which all are done.  Between its blocks the next one has landed and is
    // noted, for all waves, and its first scores are computed with the second block.
    int at = 0;
    auto turn = [&](int token) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(OPS) : "memory");
        note(at + 1 & 3, 1, token + 64);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    if (v0 < live) {
        auto whole = [&](const uint8_t* block, int from) { return from >= all_from && from + 31 <= low && __all(Block<D>::notes(block, h).plain()); };
        // 32-bit queries and weights take the registers that scores ahead of their block need, and there the matrix cores are what is short
        constexpr bool NEXT = sizeof(T) == 2;
        f32x16 s, s2;
        if (pairs) {
            const int mine = wave >> 1;
            for (int token = range.begin; token < range.end; token += 64) {
                const uint8_t* block = lds + at * STAGE + mine * Block<D>::BYTES;
                request();
                s = w.scores(block);
                w.template step<false>(a, s, block, token + 32 * mine, whole(block, token + 32 * mine), nullptr, s2);
                turn(token);
                at = at + 1 & 3;
            }
        } else {
            s = w.scores(lds);
            for (int token = range.begin; token < range.end; token += 64) {
                const uint8_t *first = lds + at * STAGE, *second = first + Block<D>::BYTES;
                request();
                w.template step<NEXT>(a, s, first, token, whole(first, token), second, s2);
                turn(token);
                at = at + 1 & 3;
                if constexpr (!NEXT) s2 = w.scores(second);
                w.template step<NEXT>(a, s2, second, token + 32, whole(second, token + 32), lds + at * STAGE, s);
                if constexpr (!NEXT) s = w.scores(lds + at * STAGE);
            }
        }
    } else {   // requests for the others
        for (int token = range.begin; token < range.end; token += 64) {
            request();
            turn(token);
            at = at + 1 & 3;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    w.close();
    if (pairs) {   // the second of a pair gives the first what it has
        constexpr int NB = D / 32;
        float* sums = reinterpret_cast<float*>(lds) + (wave & 1) * (NB * 16 + 2) * 64 + lane;
        static_assert(2 * (NB * 16 + 2) * 256 <= ChunkLds<D>::BYTES, "");
        __syncthreads();   // every wave is done with what was there
        if (wave >= 2) {
            sums[0] = w.m, sums[64] = w.l;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(2 + 16 * j + i) * 64] = w.o[j][i];
        }
        __syncthreads();
        if (wave >= 2) return;
        const float m = sums[0], top = fmaxf(w.m, m), ref = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(w.m - ref), g = __builtin_amdgcn_exp2f(m - ref);
        w.m = top;
        w.l = w.l * f + sums[64] * g;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) w.o[j][i] = w.o[j][i] * f + sums[(2 + 16 * j + i) * 64] * g;
    }
    const int v = v0 + c;
    if (v < live) {
        if (p.r.splits == 1) {
            const int row = a.G.quotient(v);
            T* out = (T*)a.out + ((int64_t)(p.r.start + row) * a.Hq + head * G + v - row * G) * D;
            const float f = chunk_factor(w.l, w.m);
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x16& o = w.o[j];
                    store4(out + 32 * j + 8 * e + 4 * h, o[4 * e] * f, o[4 * e + 1] * f, o[4 * e + 2] * f, o[4 * e + 3] * f);
                }
        } else {
            const int64_t place = slot * a.slot_rows + v - tile * kTile;
            float* out = a.partial + place * D;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<f32x4*>(out + 32 * j + 8 * e + 4 * h) = f32x4{w.o[j][4 * e], w.o[j][4 * e + 1], w.o[j][4 * e + 2], w.o[j][4 * e + 3]};
            if (h == 0) reinterpret_cast<float2*>(a.partial + a.slots * a.slot_rows * D)[place] = float2{w.m, w.l};
        }
    }
}

// Up to 32 places: each wave has all of them, and every fourth 32 tokens, which it requests for itself.
template <class T, int D>
__device__ __forceinline__ void chunk_few(const ChunkArgs& a, const ChunkPlace& p, int head, int split, int64_t slot, uint8_t* lds) {
    constexpr int HALF = D / 2, LD = HALF + 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
    const int G = a.G.d, live = p.r.count * G;
    const ChunkRange range = chunk_range(a, p.r, 0, kFew, split, 32 * kWaves);
    const int32_t* table = a.page_tables + (int64_t)p.b * a.max_pages;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds + wave * 2 * Block<D>::BYTES;
    const int low = p.r.n - p.r.count, high = p.r.n - 1;
    const int all_from = a.window > 0 ? max(high - a.window + 1, 0) : 0;
    Places<T, D> w;
    auto page_at = [&](int token) { return token < range.end ? load_uniform(table + min(token / kPageTokens, a.max_pages - 1)) : -1; };
    int ahead = range.begin + 32 * wave, fill = 0;
    int page0 = page_at(ahead), page1 = page_at(ahead + kPageTokens);
    PageRequests<D> pages;
    pages.init(a, head);
    auto request = [&]() {
        pages.request(page0, 0, lds0 + fill * Block<D>::BYTES);
        pages.request(page1, 1, lds0 + fill * Block<D>::BYTES);
        ahead += 32 * kWaves;
        page0 = page_at(ahead), page1 = page_at(ahead + kPageTokens);
        fill ^= 1;
    };
    if (range.begin + 32 * wave < range.end) request();
    w.load(a, p.r, head, c);   // behind the request, whose way it shares
    for (int from = range.begin + 32 * wave; from < range.end; from += 32 * kWaves) {
        uint8_t* const block = lds + (wave * 2 + (fill ^ 1)) * Block<D>::BYTES;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what the block before was read from is written again
        request();
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * Block<D>::OPS) : "memory");
        const bool partly = from < all_from || from + 31 > low;
        pages.note(block, 0, 3, from, p.r.n, partly);
        pages.note(block, 1, 2, from + kPageTokens, p.r.n, partly);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        f32x16 s = w.scores(block), none;
        w.template step<false>(a, s, block, from, !partly && __all(Block<D>::notes(block, h).plain()), nullptr, none);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    w.close();
    float* sums = reinterpret_cast<float*>(lds);
    float2* ml = reinterpret_cast<float2*>(lds + kWaves * 32 * LD * 4);
#pragma unroll
    for (int part = 0; part < 2; ++part) {   // half of the dims at a time
        __syncthreads();   // every wave is done with what was there
#pragma unroll
        for (int j = 0; j < HALF / 32; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x16& o = w.o[part * (HALF / 32) + j];
                *reinterpret_cast<f32x4*>(sums + (wave * 32 + c) * LD + 32 * j + 8 * e + 4 * h) = f32x4{o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]};
            }
        if (h == 0) ml[wave * 32 + c] = float2{w.m, w.l};
        __syncthreads();
        for (int u = threadIdx.x; u < live * (HALF / 4); u += 64 * kWaves) {
            const int v = u / (HALF / 4), d = u % (HALF / 4) * 4;
            float top = -INFINITY, sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kWaves; ++i) top = fmaxf(top, ml[i * 32 + v].x);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const float2 y = ml[i * 32 + v];
                const float f = __builtin_amdgcn_exp2f(y.x - ref);
                const f32x4 o = *reinterpret_cast<const f32x4*>(sums + (i * 32 + v) * LD + d);
                sum += f * y.y;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] += f * o[e];
            }
            if (p.r.splits == 1) {
                const int row = a.G.quotient(v);
                T* to = (T*)a.out + ((int64_t)(p.r.start + row) * a.Hq + head * G + v - row * G) * D + part * HALF + d;
                const float f = chunk_factor(sum, top);
                store4(to, x[0] * f, x[1] * f, x[2] * f, x[3] * f);
            } else {
                const int64_t place = slot * a.slot_rows + v;
                *reinterpret_cast<f32x4*>(a.partial + place * D + part * HALF + d) = f32x4{x[0], x[1], x[2], x[3]};
                if (part == 0 && d == 0) reinterpret_cast<float2*>(a.partial + a.slots * a.slot_rows * D)[place] = float2{top, sum};
            }
        }
    }
}

template <class T, int D>
__global__ __launch_bounds__(64 * kWaves, 2) void kv8_chunk_kernel(ChunkArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ChunkLds<D>::BYTES];
    // No loop over items: what it keeps in scalar registers has others spilled (with weights of one plane four drafted tokens of 64 requests 69 -> 66.5 us, 14B heads in 32 bits 103 -> 99)
    const int item = a.heads.quotient(blockIdx.x), head = blockIdx.x - item * a.Hkv;
    ChunkPlace p;
    const bool sorted = a.sorted && chunk_longest(a, item, p);
    if (!sorted) p = chunk_find<false>(a, item);
    if (p.b < 0) return;
    // The longest first.  Where all of a request's are on the chip at once, two workgroups a compute unit, the second half comes the other way round, so that a unit has a long and a
    // short one (2048 of 8191 tokens 380 -> 368 us).
    const int turn = p.r.splits == 1 ? p.index : p.index / p.r.splits, split = p.index - turn * p.r.splits, half = (p.r.tiles + 1) / 2;
    const bool paired = p.r.tiles * p.r.splits * a.Hkv <= 512;
    const int tile = sorted ? p.index : paired && turn >= half ? turn - half : p.r.tiles - 1 - turn;
    const int64_t slot = (p.items + (int64_t)tile * p.r.splits + split) * a.Hkv + head;
    if (p.r.splits > 1 && slot >= a.slots) return;   // row starts that are none could name more
    if (p.r.count * (int)a.G.d <= kFew) chunk_few<T, D>(a, p, head, split, slot, lds);
    else chunk_wide<T, D>(a, p, head, tile, split, slot, lds);
}

// out = sum over a tile's parts, four dims a lane; its places are dealt to gridDim.y workgroups.  Memory's latency is what bounds it: with eight parts on their way and eight places a
// workgroup 4 of 8191 tokens (32 parts) take 32 -> 16 us with their attention, 8 of 32768 (64) 101 -> 28, against one part and four times the places.
template <class T, int D>
__global__ __launch_bounds__(256) void kv8_chunk_join_kernel(ChunkArgs a) {
    const int G = a.G.d, item = a.heads.quotient(blockIdx.x), head = blockIdx.x - item * a.Hkv;
    const ChunkPlace p = chunk_find<true>(a, item);
    if (p.b < 0 || p.r.splits == 1) return;
    const int tile = p.index, places = p.r.count * G <= kFew ? kFew : kTile, live = min(p.r.count * G - tile * places, places);
    const int64_t slot = (p.items + (int64_t)tile * p.r.splits) * a.Hkv + head;
    if (slot + (int64_t)(p.r.splits - 1) * a.Hkv >= a.slots) return;
    const float2* ml = reinterpret_cast<const float2*>(a.partial + a.slots * a.slot_rows * D);
    constexpr int LANES = D / 4;   // of a place
    const int64_t step = (int64_t)a.Hkv * a.slot_rows;
    for (int i = blockIdx.y * (256 / LANES) + threadIdx.x / LANES; i < live; i += gridDim.y * (256 / LANES)) {
        const int64_t at0 = slot * a.slot_rows + i;
        const int d = threadIdx.x % LANES * 4;
        float top = -INFINITY, sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
        int s0 = 0;
        auto parts = [&](auto n) {   // so many of them, all on their way before the first is waited for
            constexpr int N = decltype(n)::value;
            float2 y[N];
            f32x4 o[N];
#pragma unroll
            for (int s = 0; s < N; ++s) {
                const int64_t at = at0 + (s0 + s) * step;
                y[s] = ml[at];
                o[s] = *reinterpret_cast<const f32x4*>(a.partial + at * D + d);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < N; ++s) {
                const float grown = fmaxf(top, y[s].x), ref = grown == -INFINITY ? 0.f : grown;
                const float f = __builtin_amdgcn_exp2f(top - ref), g = __builtin_amdgcn_exp2f(y[s].x - ref);
                top = grown;
                sum = sum * f + y[s].y * g;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = x[e] * f + o[s][e] * g;
            }
            s0 += N;
        };
        while (s0 + 8 <= p.r.splits) parts(std::integral_constant<int, 8>{});
        if (s0 + 4 <= p.r.splits) parts(std::integral_constant<int, 4>{});
        if (s0 + 2 <= p.r.splits) parts(std::integral_constant<int, 2>{});
        if (s0 < p.r.splits) parts(std::integral_constant<int, 1>{});
        const int v = tile * places + i, row = a.G.quotient(v);
        const float f = chunk_factor(sum, top);
        store4((T*)a.out + ((int64_t)(p.r.start + row) * a.Hq + head * G + v - row * G) * D + d, x[0] * f, x[1] * f, x[2] * f, x[3] * f);
    }
}

// ---------------------------------------------------------------- the call

static int64_t chunk_tiles(const sun_model_cfg& c, int batch, int rows) {   // no fewer than there can be
    const int G = c.n_q_heads / c.n_kv_heads;
    return (int64_t)rows * G / kTile + std::min(batch, rows);
}
static int chunk_splits(const sun_model_cfg& c, int batch, int rows, int max_pages) {
    const int64_t groups = chunk_tiles(c, batch, rows) * c.n_kv_heads, longest = ((int64_t)max_pages * kPageTokens + kMinSplit - 1) / kMinSplit;
    return (int)std::max<int64_t>(1, std::min<int64_t>({kMaxSplits, longest, (kGroupsWanted + groups - 1) / groups}));
}
static int chunk_slot_rows(const sun_model_cfg& c, int rows) {
    return (int)std::min<int64_t>(kTile, ((int64_t)rows * (c.n_q_heads / c.n_kv_heads) + 31) / 32 * 32);
}
static size_t chunk_bytes(const sun_model_cfg& c, int64_t slots, int slot_rows) { return (size_t)slots * slot_rows * (c.head_dim + 2) * 4; }

int64_t kv8_chunk_groups(const sun_model_cfg& c, int batch, int rows) { return chunk_tiles(c, batch, rows) * c.n_kv_heads; }
size_t kv8_chunk_workspace(const sun_model_cfg& c, int batch, int rows, int max_pages) {
    const int splits = chunk_splits(c, batch, rows, max_pages);
    return splits == 1 ? 0 : chunk_bytes(c, chunk_tiles(c, batch, rows) * c.n_kv_heads * splits, chunk_slot_rows(c, rows));
}
// No less than what any fewer rows of any fewer requests take: g workgroups without parts are given ceil(wanted / g) of them each at most, fewer than wanted + g in all
size_t kv8_chunk_workspace_up_to(const sun_model_cfg& c, int batch, int rows, int max_pages) {
    const int64_t groups = kv8_chunk_groups(c, batch, rows), splits = std::min<int64_t>(kMaxSplits, ((int64_t)max_pages * kPageTokens + kMinSplit - 1) / kMinSplit);
    if (splits == 1) return 0;
    return chunk_bytes(c, std::min<int64_t>(groups * splits, kGroupsWanted + std::min<int64_t>(groups, kGroupsWanted)), chunk_slot_rows(c, rows));
}

template <class T, int D>
static hipError_t chunk_attend(const ChunkArgs& a, int64_t tiles, hipStream_t st) {
    const unsigned grid = (unsigned)(tiles * a.splits * a.Hkv);   // not 2^23: parts are for fewer than kGroupsWanted groups
    hipLaunchKernelGGL((kv8_chunk_kernel<T, D>), dim3(grid), dim3(64 * kWaves), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    // Workgroups of a joined tile: a pass of eight places each where tiles are few (64 of 8191 tokens 36 -> 33 us against four of them), four where every further one would look for
    // its tile again (1024 of 8191 tokens 211 us, with sixteen 216)
    const int64_t joining = std::min<int64_t>(a.slot_rows / 8, std::max<int64_t>(4, 1024 / (tiles * a.Hkv)));
    if (a.splits > 1) hipLaunchKernelGGL((kv8_chunk_join_kernel<T, D>), dim3((unsigned)(tiles * a.Hkv), (unsigned)joining), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv8_chunk_attention(const Kv8Pool& pool, int layer, int batch, int rows, const void* q, bool f32, const int32_t* row_starts, const int32_t* page_tables,
                                      int max_pages, const int32_t* n_tokens, int window, void* out, float* partial, hipStream_t st) {
    const sun_model_cfg& c = pool.cfg;
    const sun_kv8_layout& L = pool.lay;
    ChunkArgs a{};
    a.codes = pool.base + L.k_off + layer * L.k_layer;
    a.scales = pool.base + L.ks_off + layer * L.s_layer;
    a.k_page = L.k_page, a.k_head = L.k_head;
    a.v_off = L.v_off - L.k_off, a.v_head = L.v_head;
    a.s_page = L.s_page, a.s_head = L.s_head, a.vs_off = L.vs_off - L.ks_off;
    a.q = q, a.row_starts = row_starts, a.page_tables = page_tables, a.n_tokens = n_tokens, a.out = out, a.partial = partial;
    a.batch = batch, a.rows = rows, a.max_pages = max_pages, a.n_pages = (int)L.n_pages;
    a.Hq = c.n_q_heads, a.Hkv = c.n_kv_heads, a.window = std::min(window, 1 << 30);   // no cache is longer, and positions less a window fit 32 bits
    a.G = Divider::of(c.n_q_heads / c.n_kv_heads), a.heads = Divider::of(c.n_kv_heads);
    a.splits = chunk_splits(c, batch, rows, max_pages);
    a.slot_rows = chunk_slot_rows(c, rows);
    const int64_t tiles = chunk_tiles(c, batch, rows);
    a.sorted = a.splits == 1 && batch > 1 && batch <= kSorted && tiles * a.Hkv <= kSortedGroups;
    a.slots = a.splits > 1 ? tiles * a.Hkv * a.splits : 0;
    a.c = 1.4426950408889634f / sqrtf((float)c.head_dim);
    if (f32) return c.head_dim == 128 ? chunk_attend<float, 128>(a, tiles, st) : chunk_attend<float, 64>(a, tiles, st);
    return c.head_dim == 128 ? chunk_attend<uint16_t, 128>(a, tiles, st) : chunk_attend<uint16_t, 64>(a, tiles, st);
}

}  // namespace sun
