// What the two kernels of the attention of ragged rows share: the call, the
// tiles of columns, what a column sees, and how the parts of a tile meet.
#pragma once

#include "md_arrive.h"
#include "md_decode.h"
#include "md_device.h"

namespace md {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A column's maximum is only followed when it has grown by more than this
// (base 2): weights then reach 2^8 and their sums 2^8 times a row's length,
// far inside float32 and bf16, and most steps leave the sums unscaled.
constexpr float kSlack = 8.0f;

struct PromptCall {
    int S, L, Hq, Hkv, G, P, Pshift, MP, NP, aligned, layer;
    size_t page_elems;
    const uint16_t* k_pool;
    const uint8_t* region;
    const int32_t* page_table;
    const int32_t* n_pages;
    const int32_t* n_tokens;
    const uint8_t* page_format;
    int32_t* status;
    const int32_t* row_start;
    const int32_t* row_slot;
    int n_rows;
    const void* q;
    int64_t q_stride;
    void* out;
    int64_t out_stride;
    float* lse;
    int q_f32, out_bf16, window, sinks;
    const uint16_t* v_pool;
    const uint8_t* v_codes;
    const float* v_scale;
    int units;       // parts that all tiles should come to, if they are fewer,
    int least_units; // and those that they may be cut into besides one each if not
    int32_t* count;  // [parts] arrivals of a tile's, at its first (zero between launches)
    float* part;     // [parts][columns][kPartWords] partial results
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((__vector_size__(4)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// acc plus both bf16 values of a word.
__device__ __forceinline__ float add_pair(uint32_t w, float acc) {
    typedef __bf16 bf16x2 __attribute__((__vector_size__(4)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3F803F80u), acc, false);
}

// The larger, or the sum, of both half-waves' values.
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Partial results cross workgroups of different XCDs, whose L2s are not
// coherent within a launch: 64-bit words, written through and read past them.
typedef unsigned long long u64;
__device__ __forceinline__ void put2(float* p, float a, float b) {
    const u64 w = (u64)__float_as_uint(a) | ((u64)__float_as_uint(b) << 32);
    __hip_atomic_store(reinterpret_cast<u64*>(p), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Tokens among 16 slots' region codes before the holes.
__device__ __forceinline__ int tokens_before_holes(const uint8_t* region) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(region);
    int n = 0;
#pragma unroll
    for (int i = 3; i >= 0; --i)
#pragma unroll
        for (int b = 3; b >= 0; --b)
            if (((w[i] >> (8 * b)) & 0xFFu) != (uint32_t)kHole) n = max(n, 4 * i + b + 1);
    return n;
}

__device__ __forceinline__ int wave_max_i(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o));
    return v;
}

// A row's result divided by its sum; nothing seen gives zeros.
__device__ __forceinline__ float inverse(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }
__device__ __forceinline__ float log_sum(float m, float l) { return (m + log2f(l)) * 0.69314718055994530942f; }

// What a lane knows of block `base + lane` of the list that a tile walks.
struct Block {
    int64_t tile;      // elements before its tile in the pools of keys and values
    int at;            // slot of its first token
    int live;          // its tokens, 0 .. 16
    int coded;         // 8-bit keys
    int ks, vs;        // scales of keys and values (float bits)
};

// Where a workgroup is: a tile of kCols columns of one session and KV head, and
// its part of the tile's blocks.
struct TileAt {
    int s, kv;
    int split, splits;
    int slot, apart;      // place of the tile's first part among all, and what follows to the next
    int col;              // its first column in the session
    int row_lo, rows;     // the session's rows
    int nt;               // and its slots in use
};

// The parts are of one size over all sessions, so that a session three times as
// long as another has three times as many and all end together (cut into the same
// number, 16 sessions of 2,048 to 8,192 tokens, 16 rows of 4 columns, 8-bit values
// took 92 us instead of 76).  A group is 8
// blocks; a part has at least kLeastGroups, what joining it costs.
constexpr int kGroup = 128, kLeastGroups = 4;

constexpr int kRun = 4;   // parts in a row on one XCD
// Workgroups for `parts` parts of each KV head.
inline unsigned grid_of(int64_t parts, int Hkv) {
    const int64_t runs = (parts + kRun - 1) / kRun * Hkv;
    return (unsigned)((runs + 7) / 8 * 8 * kRun);
}

// A session's parts follow one another, tile by tile and then part by part;
// pref: LDS, [S + 1] parts before.  False where there is nothing to do.
template <int kThreads, int kCols>
__device__ __forceinline__ bool find_tile(const PromptCall& c, int* scan_lds, int* pref, TileAt& t, int& status) {
    const int tid = threadIdx.x;
    bool broken = false;   // (rows of several sessions, or more than there are, would make more tiles than the grid has)
    auto tiles_of = [&](int s) {
        if (s >= c.S) return 0;
        const int lo = c.row_start[s], hi = c.row_start[s + 1];
        broken |= lo < 0 || lo > hi || hi > c.n_rows;
        return broken ? 0 : (int)(((int64_t)(hi - lo) * c.G + kCols - 1) / kCols);
    };
    auto groups_of = [&](int s) {   // (about: where a window lies over rows of any order is not known here)
        int n = s < c.S ? max(c.n_tokens[s], 0) : 0;
        if (c.window > 0) n = (int)min((int64_t)n, (int64_t)c.window + c.sinks + 64);
        return min((int)(((int64_t)n + kGroup - 1) / kGroup), 1 << 20);
    };
    int share = 0;
    if (c.units > 0) {   // (then tiles Hkv < 2^11)
        int all = 0, most = 0;
        for (int k = 0; k < c.S; k += kThreads) {
            const int tiles = tiles_of(k + tid), of[2] = {tiles * groups_of(k + tid), tiles};
            int ex[2], total[2];
            block_exclusive_scan_n<2>(of, scan_lds, ex, total);
            all += total[0];
            most += total[1];
        }
        // (with their short last parts they are no more than fit the card at once: a
        // second round of a few cost a tenth to a fifth of the call)
        const int units = max(c.units - most * c.Hkv, c.least_units);
        if (units > 0) share = max(kLeastGroups, (all * c.Hkv + units - 1) / units);
    }
    int before = 0;
    for (int k = 0; k < c.S; k += kThreads) {
        const int s = k + tid;
        int n = tiles_of(s);
        if (share > 0) n *= max(1, (groups_of(s) + share - 1) / share);
        int total;
        const int ex = block_exclusive_scan(n, scan_lds, &total);
        if (s < c.S) pref[s] = before + ex;
        before += total;
    }
    if (tid == 0) pref[c.S] = before;
    if (__syncthreads_or(broken ? 1 : 0)) {
        if (tid == 0) atomicOr(c.status, MD_DEV_BAD_ROW);
        return false;
    }
    // runs of kRun parts of a KV head, which tend to read the same tokens, on one
    // of the eight XCDs (workgroup i is on XCD i % 8), the longest of a session first
    const int at = blockIdx.x >> 3, run = at / kRun * 8 + (blockIdx.x & 7);
    t.kv = run % c.Hkv;
    const int unit = uni(before) - 1 - (run / c.Hkv * kRun + at % kRun);
    if (unit < 0) return false;
    t.s = uni(find_session(pref, c.S, unit));
    t.row_lo = uni(c.row_start[t.s]);
    t.rows = uni(c.row_start[t.s + 1]) - t.row_lo;
    const int first = uni(pref[t.s]), tiles = (int)(((int64_t)t.rows * c.G + kCols - 1) / kCols);
    t.split = (unit - first) / tiles;
    t.splits = (uni(pref[t.s + 1]) - first) / tiles;
    t.col = (unit - first) % tiles * kCols;
    t.slot = (unit - t.split * tiles) * c.Hkv + t.kv;
    t.apart = tiles * c.Hkv;
    const int np = uni(c.n_pages[t.s]);
    t.nt = uni(c.n_tokens[t.s]);
    const bool ok = np == 0 ? t.nt == 0 : np > 0 && np <= c.MP && t.nt > (np - 1) * c.P && t.nt <= np * c.P;
    if (!ok) {
        status |= kDevCorrupt;
        t.nt = 0;
    }
    return true;
}

// Blocks of each of the tile's parts (whole groups), of the n that it sees.
__device__ __forceinline__ int share_of(const TileAt& t, int n) {
    constexpr int per = kGroup / 16;
    const int groups = (n + per - 1) / per;
    return per * max(t.splits > 1 ? kLeastGroups : 1, (groups + t.splits - 1) / t.splits);
}

// A lane's column.
struct Column {
    bool mine;      // there is one
    int own;        // slot of its row (-1: it sees nothing)
    int64_t row;
    int head;
};

__device__ __forceinline__ Column column_of(const PromptCall& c, const TileAt& t, int col, int& status) {
    Column x;
    x.mine = col < t.rows * c.G;
    x.row = t.row_lo + (x.mine ? col / c.G : 0);
    x.head = t.kv * c.G + (x.mine ? col % c.G : 0);
    x.own = -1;
    if (x.mine) {
        const int slot = c.row_slot != nullptr ? c.row_slot[x.row] : t.nt - (t.rows - (int)(x.row - t.row_lo));
        if (slot >= 0 && slot < t.nt) x.own = slot; else status |= MD_DEV_BAD_ROW;
    }
    return x;
}

// Dims 16 kk + 8 h .. of a column's query as bf16 terms.
template <int TERMS>
__device__ __forceinline__ void query_terms(const PromptCall& c, const Column& x, int kk, u32x4 (&w)[TERMS]) {
    const int64_t at = x.row * c.q_stride + x.head * kHeadDim + 8 * (lane_id() >> 5) + 16 * kk;
#pragma unroll
    for (int t = 0; t < TERMS; ++t) w[t] = u32x4{0u, 0u, 0u, 0u};
    if (!x.mine) return;
    if (TERMS == 1 || !c.q_f32) {
        w[0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(c.q) + at);
    } else {
        const f32x4* from = reinterpret_cast<const f32x4*>(static_cast<const float*>(c.q) + at);
        const f32x4 y[2] = {from[0], from[1]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[3], b[3];
            split3(y[i >> 1][2 * (i & 1)], a[0], a[1], a[2]);
            split3(y[i >> 1][2 * (i & 1) + 1], b[0], b[1], b[2]);
#pragma unroll
            for (int t = 0; t < TERMS; ++t) w[t][i] = a[t] | (b[t] << 16);
        }
    }
}

// The blocks that some column sees, whose rows' slots run from lo to hi (hi < 0:
// none): the first tokens', then from the window's first slot to the last row's.
struct Seen {
    int win;        // slots a row looks back
    int low, first; // the first block behind the first tokens', and how many are theirs
    int n_blocks;
    __device__ __forceinline__ int block(int i) const { return i < first ? i : i + low - first; }
};

__device__ __forceinline__ Seen seen_of(const PromptCall& c, int lo, int hi) {
    Seen x;
    x.win = c.window > 0 ? c.window : 0x7FFFFFFF;
    x.low = hi < 0 ? 0 : max(0, lo - x.win + 1) >> 4;
    x.first = min((min(c.sinks, hi + 1) + 15) >> 4, x.low);   // (window 0: low is 0)
    x.n_blocks = hi < 0 ? 0 : x.first + (hi >> 4) + 1 - x.low;
    return x;
}

__device__ __forceinline__ int page_of(const PromptCall& c, const TileAt& t, const Seen& x, int i) {
    return c.page_table[(size_t)t.s * c.MP + ((16 * x.block(min(i, x.n_blocks - 1))) >> c.Pshift)];
}

// Block i of the list (any i; behind the last: page 0, which there is, without
// a token), whose page is p.
template <bool QT, bool V8>
__device__ __forceinline__ Block block_at(const PromptCall& c, const TileAt& t, const Seen& x, size_t row_elems, int i, int p,
                                          int& status) {
    Block b{(int64_t)row_elems, 0, 0, 0, 0x3F800000, 0};
    if (i >= x.n_blocks) return b;
    const int per = c.P >> 4, blk = x.block(i), sub = blk & (per - 1);
    b.at = 16 * blk;
    if ((unsigned)p >= (unsigned)c.NP) {
        status |= kDevCorrupt;
        return b;
    }
    b.tile = (int64_t)((size_t)p * c.page_elems + row_elems + (size_t)sub * 16 * kHeadDim);
    b.live = min(16, t.nt - b.at);
    if (c.aligned) b.live = min(b.live, tokens_before_holes(c.region + (size_t)p * c.P + 16 * sub));
    if constexpr (QT) {
        b.coded = c.page_format[p] != 0;
        if (b.coded) b.ks = *reinterpret_cast<const int*>(c.k_pool + b.tile + 1024);
    }
    if constexpr (V8)
        if (b.live > 0) b.vs = reinterpret_cast<const int*>(c.v_scale)[(((size_t)p * c.L + c.layer) * c.Hkv + t.kv) * (size_t)per + sub];
    return b;
}

__device__ __forceinline__ int lane_int(int x, int i) { return __builtin_amdgcn_readlane(x, i); }
__device__ __forceinline__ float lane_float(int x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(x, i)); }
__device__ __forceinline__ int64_t lane_tile(const Block& b, int i) {
    return (int64_t)((uint64_t)(uint32_t)lane_int((int)(uint32_t)b.tile, i) |
                     ((uint64_t)(uint32_t)lane_int((int)(b.tile >> 32), i) << 32));
}

// Whether a scale of values can go through the weights' exponents and out of
// their sums again, with room for weights from 2^-30 to 2^8.  A column that sees
// values with another (or none: NaN) is summed again.
__device__ __forceinline__ bool scale_fits(float s) { return s > 0x1p-96f && s < 0x1p96f; }

// Whether some column of the wave may hold what it does not see: a value that is
// not finite in a block that not every column sees in full, which reaches the
// others as 0 times it, or a scale that does not fit, which every column that sees
// it lacks.  A column without either that is not finite sees a value that is not,
// and stays.  (Telling costs a look at the blocks that some column does not see in
// full; without it every column that sees such a value would be summed again.
// 2,048 rows of 16 heads take 75 us, with a NaN in the first token 93; in the last
// but eight 2,960, where one workgroup's columns are summed again.)  describe(i): what lanes know of blocks i .. i + 63 of the wave's `count`.
template <bool V8, typename F>
__device__ __forceinline__ bool reached_unseen(const PromptCall& c, const Seen& x, int smin, int smax, int count, F&& describe) {
    for (int i = 0; i < count; i += 64) {
        const Block b = describe(i);
        const bool mine = i + lane_id() < count && b.live > 0;
        if constexpr (V8) {
            const float vs = __int_as_float(b.vs);
            if (__any(mine && vs == vs && vs != 0.0f && !scale_fits(vs))) return true;
        }
        const bool full = (b.live == 16) & (b.at + 15 <= smin) & ((b.at > smax - x.win) | (b.at + 15 < c.sinks));
        for (uint64_t left = __ballot(mine && !full); left != 0; left &= left - 1) {
            const int k = __ffsll((unsigned long long)left) - 1;
            const int64_t tile = lane_tile(b, k);
            const int k4 = lane_int(b.live, k) - 4 * (lane_id() >> 4);   // tokens of this lane's four that there are
            bool odd = false;
            if constexpr (V8) {
                const uint32_t there = k4 >= 4 ? ~0u : k4 <= 0 ? 0u : (1u << (8 * k4)) - 1u;
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(c.v_codes + tile + 1024 * a + 16 * lane_id());
#pragma unroll
                    for (int e = 0; e < 4; ++e) {   // a byte of 0x7F or 0xFF
                        const uint32_t y = ~(w[e] | 0x80808080u) | ~there;
                        odd |= ((y - 0x01010101u) & ~y & 0x80808080u) != 0;
                    }
                }
            } else {
                const uint32_t m0 = k4 >= 2 ? ~0u : k4 == 1 ? 0xFFFFu : 0u, m1 = k4 >= 4 ? ~0u : k4 == 3 ? 0xFFFFu : 0u;
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(c.v_pool + tile + 512 * a + 8 * lane_id());
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t y = w[e] & (e & 1 ? m1 : m0);
                        odd |= (y & 0x7F80u) == 0x7F80u || (y & 0x7F800000u) == 0x7F800000u;
                    }
                }
            }
            if (__any(odd)) return true;
        }
    }
    return false;
}

constexpr int kAgainWords = kHeadDim + 64;   // of column_again's LDS

// One column's sum of weighted values again (dims e and e + 1, e = 2 lane), from
// `count` blocks of which describe(k) tells 64 lanes, 64 tokens at a time: a
// lane's token's weight, then all tokens' values for its dims.  For values that
// are not finite, which reach, as 0 times them, the columns of their product that
// do not see them.  lds: the wave's own.
template <bool QT, bool V8, typename F>
__device__ __forceinline__ float2 column_again(const PromptCall& c, const Seen& x, int own, float top, int64_t row, int head,
                                               int count, float* lds, F&& describe) {
    const int lane = lane_id(), e = 2 * lane;
    const int64_t at_q = row * c.q_stride + head * kHeadDim + e;
    float q0, q1, y0 = 0.0f, y1 = 0.0f;
    if (c.q_f32) {
        q0 = static_cast<const float*>(c.q)[at_q];
        q1 = static_cast<const float*>(c.q)[at_q + 1];
    } else {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(c.q) + at_q);
        q0 = bf16_lo(w);
        q1 = bf16_hi(w);
    }
    lds[e] = q0;
    lds[e + 1] = q1;
    float* const weight = lds + kHeadDim;
    Block b{};
    for (int i = 0; i < count; i += 4) {
        if ((i & 63) == 0) b = describe(i);
        // ---- lane 16 k + t: token t of block i + k
        const int k = lane >> 4, t = lane & 15, of = (i & 63) + k;
        const int at = __shfl(b.at, of) + t, all = __shfl(b.live, of), live = i + k < count ? all : 0;
        const int64_t tile = (int64_t)((uint64_t)(uint32_t)__shfl((int)(uint32_t)b.tile, of) |
                                       ((uint64_t)(uint32_t)__shfl((int)(b.tile >> 32), of) << 32));
        const int coded_of = __shfl(b.coded, of);
        const bool coded = QT && coded_of != 0;
        const float ks = QT ? __int_as_float(__shfl(b.ks, of)) : 1.0f;
        const bool sees = t < live && at <= own && (at > own - x.win || at < c.sinks);
        const uint64_t seen = __ballot(sees);
        if (seen == 0) continue;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        float dot = 0.0f;
        if (sees) {
#pragma unroll 8
            for (int j = 0; j < 16; ++j) {   // dims 8 j ..
                u32x4 w;
                if (coded) {   // codes (a, g, t): dims 64 a + 8 g .. and 64 a + 32 + 8 g ..
                    const u32x4 z = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(c.k_pool + tile) +
                                                                    1024 * (j >> 3) + 16 * (t + 16 * (j & 3)));
                    w = j & 4 ? codes_to_bf16<1>(z) : codes_to_bf16<0>(z);
                } else {
                    w = *reinterpret_cast<const u32x4*>(c.k_pool + tile + 128 * j + 8 * t);
                }
#pragma unroll
                for (int z = 0; z < 4; ++z)
                    dot = fmaf(lds[8 * j + 2 * z], bf16_lo(w[z]), fmaf(lds[8 * j + 2 * z + 1], bf16_hi(w[z]), dot));
            }
        }
        weight[lane] = sees ? hw_exp2(dot * ks * kLogitScale - top) : 0.0f;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        // ---- this lane's dims of the blocks' tokens, four at a time
        for (int k = 0; k < 4; ++k) {
            const uint32_t mask = (uint32_t)(seen >> (16 * k)) & 0xFFFFu;
            if (mask == 0) continue;
            const int64_t tile = lane_tile(b, (i & 63) + k);
            const float vs = V8 ? lane_float(b.vs, (i & 63) + k) : 1.0f;
            u32x2 v0[4], v1[4];   // bf16 values of tokens 4 g .. of dims e and e + 1
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                if constexpr (V8) {
                    const uint8_t* v = c.v_codes + tile + (e / 64) * 1024 + g * 256 + (e % 16) * 16 + ((e / 16) % 4) * 4;
                    const uint32_t a = *reinterpret_cast<const uint32_t*>(v), z = *reinterpret_cast<const uint32_t*>(v + 16);
                    v0[g] = u32x2{codes_pair_to_bf16<false>(a), codes_pair_to_bf16<true>(a)};
                    v1[g] = u32x2{codes_pair_to_bf16<false>(z), codes_pair_to_bf16<true>(z)};
                } else {
                    const uint16_t* v = c.v_pool + tile + (e / 32) * 512 + g * 128 + (e % 16) * 8 + ((e / 16) % 2) * 4;
                    v0[g] = *reinterpret_cast<const u32x2*>(v);
                    v1[g] = *reinterpret_cast<const u32x2*>(v + 8);
                }
            }
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const float w = weight[16 * k + z];
                const uint32_t a = v0[z >> 2][(z >> 1) & 1], d = v1[z >> 2][(z >> 1) & 1];
                const float n0 = fmaf(w, vs * (z & 1 ? bf16_hi(a) : bf16_lo(a)), y0);
                const float n1 = fmaf(w, vs * (z & 1 ? bf16_hi(d) : bf16_lo(d)), y1);
                const bool counts = (mask >> z) & 1u;
                y0 = counts ? n0 : y0;
                y1 = counts ? n1 : y1;
            }
        }
    }
    return make_float2(y0, y1);
}

// Eight threads share a column: dims 4 j + 32 i .. of thread j (i: y's), and its
// log sum with the first.
__device__ __forceinline__ void write_column(const PromptCall& c, int64_t row, int head, int j, const f32x4 (&y)[4], float m, float l,
                                             float lw) {
    const float inv = inverse(lw);
    const int64_t to = row * c.out_stride + head * kHeadDim + 4 * j;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x4 z = y[i] * inv;
        if (c.out_bf16)
            *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(c.out) + to + 32 * i) = u32x2{pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3])};
        else
            *reinterpret_cast<f32x4*>(static_cast<float*>(c.out) + to + 32 * i) = z;
    }
    if (c.lse != nullptr && j == 0) c.lse[row * c.Hq + head] = log_sum(m, l);
}

// The partial results of a tile's part: [kCols][kPartWords], a column's sums of
// weighted values, then m, l and the sum that divides them.
template <int kCols>
__device__ __forceinline__ float* part_of(const PromptCall& c, const TileAt& t, int split) {
    return c.part + ((size_t)t.slot + (size_t)split * t.apart) * kCols * kPartWords;
}

// The tile's parts meet in the workgroup that comes last; all of this one's
// stores were issued before.  sh_last: LDS.
template <int W, int kCols>
__device__ __forceinline__ void join_parts(const PromptCall& c, const TileAt& t, int parts, int* sh_last) {
    int32_t* const count = c.count + t.slot;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) *sh_last = arrive_last(count, arrive(count), parts) ? 1 : 0;
    __syncthreads();
    if (*sh_last == 0) return;
    // The parts were stored past every cache, and are read as ordinary memory
    // behind what this workgroup may have cached of it: 16 bytes a lane, several
    // parts' under way (past the caches, 8 bytes a lane, a wave a
    // column: 86 us instead of 54 for 5 rows over 8 sessions of 24,000 tokens).
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    const int cols = min(kCols, t.rows * c.G - t.col);
    const int j = threadIdx.x & 7;
    const size_t apart = (size_t)t.apart * kCols * kPartWords;
    for (int k = threadIdx.x >> 3; k < cols; k += 8 * W) {
        const float* const p = part_of<kCols>(c, t, 0) + (size_t)k * kPartWords;
        float M = -INFINITY, lsum = 0.0f, wsum = 0.0f;
        auto meet = [&](float m, float l, float w) {
            const float mn = fmaxf(M, m);
            const float fa = mn == -INFINITY ? 0.0f : hw_exp2(M - mn), fb = mn == -INFINITY ? 0.0f : hw_exp2(m - mn);
            lsum = lsum * fa + l * fb;
            wsum = wsum * fa + w * fb;
            M = mn;
        };
#pragma unroll 4
        for (int z = j; z < parts; z += 8) {
            const f32x4 st = *reinterpret_cast<const f32x4*>(p + z * apart + kHeadDim);
            meet(st[0], st[1], st[2]);
        }
#pragma unroll
        for (int x = 1; x < 8; x *= 2) {
            const float m = __shfl_xor(M, x), l = __shfl_xor(lsum, x), w = __shfl_xor(wsum, x);
            meet(m, l, w);
        }
        f32x4 y[4] = {};
        const float top = M == -INFINITY ? 0.0f : M;
#pragma unroll 4
        for (int z = 0; z < parts; ++z) {
            const float f = hw_exp2(p[z * apart + kHeadDim] - top);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(p + z * apart + 4 * j + 32 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[i][e] = fmaf(v[e], f, y[i][e]);
            }
        }
        const int g = t.col + k;
        write_column(c, t.row_lo + g / c.G, t.kv * c.G + g % c.G, j, y, M, lsum, wsum);
    }
}

constexpr int kFewTile = 32;   // columns of a workgroup of the narrow kernel

// A kernel, and the columns and threads of its workgroups.
struct RowsKernel {
    const void* fn;
    int cols, threads;
};
RowsKernel few_kernel(bool all, bool exact, bool keys8, bool values8);   // md_few.hip; all: a CU's eight waves

}  // namespace md
