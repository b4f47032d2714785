// gfx950 kernel of the attention of ragged rows (a prompt, a chunk of one, a
// few tokens to verify) over the paged cache.
//
//   out_h = sum_i softmax_i(q_h . k_i / sqrt(d)) v_i   over the slots i that the row sees
//
// in one pass over the keys and values: a running maximum m and sum l of the
// weights 2^(x - m) for each column, a (row, query head) pair of one KV head.
// All products run on the matrix cores in 32 x 32 tiles, transposed, so that a
// lane keeps to one column throughout (n = lane & 31, h = lane >> 5):
//   logits [32 tokens][32 columns] = K q^T: register i of lane (n, h) is token
//          8 (i / 4) + 4 h + i % 4
//   sums   [32 dims][32 columns] += V^T [32 dims][16 tokens] P^T: lane (n, h)
//          feeds tokens 4h .. 4h+3 and 8+4h .. 8+4h+3 of a block, the very
//          weights it has, so they never leave their registers
// A block of 16 tokens in LDS is laid out as in the pools, which gives every
// operand as whole 16-byte (keys) or two 8-byte words (values), without bank
// conflicts.
//
// What bounds it: the matrix cores for prompts (4 d operations per column and
// token), HBM for a few rows over a long cache.

#include <algorithm>

#include "md_arrive.h"
#include "md_decode.h"
#include "md_device.h"

namespace md {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kStep = 64;                  // tokens of a step: four blocks
constexpr int kStepBytes = kStep * kHeadDim * 2;
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
    int splits;      // parts of a tile's steps
    int32_t* count;  // [tiles Hkv] arrivals (zero between launches)
    float* part;     // [tiles Hkv splits][columns][kPartWords] partial results
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((__vector_size__(4)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The other half-wave's value (lane ^ 32).
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
__device__ __forceinline__ float2 get2(const float* p) {
    const u64 w = __hip_atomic_load(reinterpret_cast<const u64*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
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
    int phys, at;      // page; slot of the block's first token
    int live;          // its tokens, 0 .. 16
    int coded;         // 8-bit keys
    float ks, vs;      // scales of keys and values
};

// A workgroup takes the tile's columns 4 waves x 32 CT, whose waves share each
// step of 64 tokens through LDS; the next step's loads are under way while this
// one is worked on.  TERMS: bf16 terms of queries and weights (1: bf16 in and
// out; 3: exact).
template <int TERMS, int CT, bool QT, bool V8>
__global__ void __launch_bounds__(kThreads, 1) k_rows_attend(PromptCall c) {
    constexpr int kCols = kWaves * 32 * CT;
    __shared__ __align__(16) uint8_t kl[2][kStepBytes];
    __shared__ __align__(16) uint8_t vl[2][kStepBytes];
    __shared__ int scan_lds[17];
    __shared__ int range_lds[2][kWaves];
    __shared__ int sh_last;
    extern __shared__ int pref[];   // [S + 1] tiles of the sessions before
    const int tid = threadIdx.x, lane = lane_id(), wv = uni(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const int per = c.P >> 4;
    int status = 0;
    // ---- this workgroup's tile
    int before = 0;
    for (int k = 0; k < c.S; k += kThreads) {
        const int s = k + tid;
        int tiles = 0;
        if (s < c.S) {
            const int lo = c.row_start[s], hi = c.row_start[s + 1];
            if (lo >= 0 && lo <= hi && hi <= c.n_rows) tiles = ((hi - lo) * c.G + kCols - 1) / kCols;
        }
        int total;
        const int ex = block_exclusive_scan(tiles, scan_lds, &total);
        if (s < c.S) pref[s] = before + ex;
        before += total;
    }
    if (tid == 0) pref[c.S] = before;
    __syncthreads();
    const int kv = blockIdx.x % c.Hkv, rest = blockIdx.x / c.Hkv;
    const int split = rest % c.splits;
    const int tile = uni(before) - 1 - rest / c.splits;   // the longest of a session first
    if (tile < 0) return;
    const int s = uni(find_session(pref, c.S, tile));
    const int row_lo = uni(c.row_start[s]), rows = uni(c.row_start[s + 1]) - row_lo;
    const int np = uni(c.n_pages[s]);
    int nt = uni(c.n_tokens[s]);
    const bool ok = np == 0 ? nt == 0 : np > 0 && np <= c.MP && nt > (np - 1) * c.P && nt <= np * c.P;
    if (!ok) {
        status |= kDevCorrupt;
        nt = 0;
    }
    // ---- the wave's columns and their queries
    const int col0 = (tile - uni(pref[s])) * kCols + wv * 32 * CT;
    int own[CT];          // slot of the column's row (-1: it sees nothing)
    int64_t row_of[CT];   // -1: not a column
    int head_of[CT];
    u32x4 qf[TERMS][CT][8];
    int smin = 0x7FFFFFFF, smax = -1;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int col = col0 + 32 * ct + n;
        const bool mine = col < rows * c.G;
        const int r = mine ? col / c.G : 0;
        head_of[ct] = kv * c.G + (mine ? col % c.G : 0);
        row_of[ct] = mine ? row_lo + r : -1;
        own[ct] = -1;
        if (mine) {
            const int slot = c.row_slot != nullptr ? c.row_slot[row_lo + r] : nt - (rows - r);
            if (slot >= 0 && slot < nt) own[ct] = slot; else status |= MD_DEV_BAD_ROW;
        }
        if (own[ct] >= 0) {
            smin = min(smin, own[ct]);
            smax = max(smax, own[ct]);
        }
        const int64_t at = (mine ? row_of[ct] : (int64_t)row_lo) * c.q_stride + head_of[ct] * kHeadDim + 8 * h;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
            if constexpr (TERMS == 1) {
                qf[0][ct][kk] = mine ? *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(c.q) + at + 16 * kk)
                                     : u32x4{0u, 0u, 0u, 0u};
            } else if (!c.q_f32) {
                qf[0][ct][kk] = mine ? *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(c.q) + at + 16 * kk)
                                     : u32x4{0u, 0u, 0u, 0u};
                qf[1][ct][kk] = qf[2][ct][kk] = u32x4{0u, 0u, 0u, 0u};
            } else {
                f32x4 x[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
                if (mine) {
                    const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(c.q) + at + 16 * kk);
                    x[0] = p[0];
                    x[1] = p[1];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t a[3], b[3];
                    split3(x[i >> 1][2 * (i & 1)], a[0], a[1], a[2]);
                    split3(x[i >> 1][2 * (i & 1) + 1], b[0], b[1], b[2]);
#pragma unroll
                    for (int k = 0; k < 3; ++k) qf[k % TERMS][ct][kk][i] = a[k] | (b[k] << 16);
                }
            }
        }
    }
    smin = uni(-wave_max_i(-smin));
    smax = uni(wave_max_i(smax));
    if (lane == 0) {
        range_lds[0][wv] = smin;
        range_lds[1][wv] = smax;
    }
    __syncthreads();
    int gmin = range_lds[0][0], gmax = range_lds[1][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        gmin = min(gmin, range_lds[0][w]);
        gmax = max(gmax, range_lds[1][w]);
    }
    gmin = uni(gmin);
    gmax = uni(gmax);
    // ---- the blocks that some column sees: the first tokens', then from the
    // window's first slot to the last row's
    const int win = c.window > 0 ? c.window : 0x7FFFFFFF;
    const int low = gmax < 0 ? 0 : max(0, gmin - win + 1) >> 4;
    const int first = min((min(c.sinks, gmax + 1) + 15) >> 4, low);   // (window 0: low is 0)
    const int n_blocks = gmax < 0 ? 0 : first + (gmax >> 4) + 1 - low;
    const int steps = (n_blocks + 3) >> 2;
    const int share = (steps + c.splits - 1) / c.splits;
    const int parts = steps == 0 ? 1 : (steps + share - 1) / share;
    if (split >= parts) {
        if (status != 0) atomicOr(c.status, status);
        return;
    }
    const int begin = split * share, end = min(steps, begin + share);

    const size_t row_elems = ((size_t)c.layer * c.Hkv + kv) * c.P * kHeadDim;
    auto describe = [&](int base) {
        Block b{0, 0, 0, 0, 1.0f, 0.0f};
        const int i = base + lane;
        if (i >= n_blocks) return b;
        const int blk = i < first ? i : i + low - first;
        b.at = 16 * blk;
        const int p = c.page_table[(size_t)s * c.MP + (b.at >> c.Pshift)];
        if ((unsigned)p >= (unsigned)c.NP) {
            status |= kDevCorrupt;
            return b;
        }
        const int sub = blk & (per - 1);
        b.phys = p;
        b.live = min(16, nt - b.at);
        if (c.aligned) b.live = min(b.live, tokens_before_holes(c.region + (size_t)p * c.P + 16 * sub));
        if constexpr (QT) {
            b.coded = c.page_format[p] != 0;
            if (b.coded)
                b.ks = *reinterpret_cast<const float*>(c.k_pool + (size_t)p * c.page_elems + row_elems + (size_t)sub * 16 * kHeadDim + 1024);
        }
        if constexpr (V8)
            if (b.live > 0) b.vs = c.v_scale[(((size_t)p * c.L + c.layer) * c.Hkv + kv) * (size_t)per + sub];
        return b;
    };
    Block mine = describe(4 * begin), ahead = describe(4 * begin + 64);
    auto of = [&](int x, int i) { return __builtin_amdgcn_readlane(x, i); };
    auto off = [&](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };

    // ---- a step's loads, and their way into LDS
    u32x4 rk[4], rv[4];
    auto load = [&](int j, const Block& d) {
        const int i0 = (4 * (j - begin)) & 63;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const size_t at = (size_t)of(d.phys, i0 + b) * c.page_elems + row_elems +
                              (size_t)((of(d.at, i0 + b) >> 4) & (per - 1)) * 16 * kHeadDim;
            const uint8_t* kp = reinterpret_cast<const uint8_t*>(c.k_pool + at);
            const bool coded = QT && of(d.coded, i0 + b) != 0;
            rk[b] = *reinterpret_cast<const u32x4*>(kp + 16 * (coded ? tid & 127 : tid));
            const uint8_t* vp = V8 ? c.v_codes + at : reinterpret_cast<const uint8_t*>(c.v_pool + at);
            rv[b] = *reinterpret_cast<const u32x4*>(vp + 16 * (V8 ? tid & 127 : tid));
        }
    };
    auto store = [&](int j, const Block& d, int buf) {
        const int i0 = (4 * (j - begin)) & 63;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            uint8_t* kb = kl[buf] + 4096 * b;
            uint8_t* vb = vl[buf] + 4096 * b;
            if (QT && of(d.coded, i0 + b) != 0) {
                // codes (a, g, t): dims 64 a + 8 g .. and 64 a + 32 + 8 g .. of token t
                if (tid < 128) {
                    uint8_t* to = kb + 2048 * (tid >> 6) + 16 * (tid & 63);
                    *reinterpret_cast<u32x4*>(to) = codes_to_bf16<0>(rk[b]);
                    *reinterpret_cast<u32x4*>(to + 1024) = codes_to_bf16<1>(rk[b]);
                }
            } else {
                *reinterpret_cast<u32x4*>(kb + 16 * tid) = rk[b];
            }
            // a slot without a token may hold anything, and 0 times an infinity
            // or NaN is NaN: its values become 0
            const int live = of(d.live, i0 + b);
            const int k4 = live - 4 * ((tid >> 4) & 3);
            const uint32_t m0 = k4 >= 2 ? 0xFFFFFFFFu : k4 == 1 ? 0x0000FFFFu : 0u;
            const uint32_t m1 = k4 >= 4 ? 0xFFFFFFFFu : k4 == 3 ? 0x0000FFFFu : 0u;
            if constexpr (V8) {
                if (tid < 128) {   // codes (a, g, m): words of dims 64 a + 16 i + m
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t x = rv[b][2 * i], y = rv[b][2 * i + 1];
                        *reinterpret_cast<u32x4*>(vb + 2048 * (tid >> 6) + 1024 * i + 16 * (tid & 63)) =
                            u32x4{codes_pair_to_bf16<false>(x) & m0, codes_pair_to_bf16<true>(x) & m1,
                                  codes_pair_to_bf16<false>(y) & m0, codes_pair_to_bf16<true>(y) & m1};
                    }
                }
            } else {
                *reinterpret_cast<u32x4*>(vb + 16 * tid) = rv[b] & u32x4{m0, m1, m0, m1};
            }
        }
    };

    // (the sums that lse tells of, and those of the weights as the products get
    // them, by which a result is divided: rounding a weight then moves it between
    // values, and does not scale the result)
    float m[CT], l[CT], lw[CT];
    f32x16 o[CT][4];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = -INFINITY;
        l[ct] = lw[ct] = 0.0f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[ct][d][i] = 0.0f;
    }
    if (begin < end) {
        load(begin, mine);
        store(begin, mine, 0);
        lds_sync();
    }
    for (int j = begin; j < end; ++j) {
        const int buf = (j - begin) & 1, i0 = (4 * (j - begin)) & 63;
        const Block now = mine;
        if (i0 == 60) {   // the next step's blocks are the next lot's
            mine = ahead;
            ahead = describe(4 * (j + 1) + 64);
        }
        const bool more = j + 1 < end;
        if (more) load(j + 1, mine);
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            const int b0 = i0 + 2 * sub;
            int at[2], live[2];
            bool any = false, all = true;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                at[b] = of(now.at, b0 + b);
                live[b] = of(now.live, b0 + b);
                any |= live[b] > 0 && at[b] <= smax && (at[b] + 15 > smin - win || at[b] < c.sinks);
                all &= live[b] == 16 && at[b] + 15 <= smin && (at[b] > smax - win || at[b] + 15 < c.sinks);
            }
            if (!any) continue;   // (no column of the wave sees any of it)
            f32x16 x[CT];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[ct][i] = 0.0f;
            const uint8_t* kb = kl[buf] + 8192 * sub + 4096 * (n >> 4) + 16 * (n & 15) + 256 * h;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                const bf16x8 a = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(kb + 512 * kk));
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t)
                        x[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, qf[t][ct][kk]), x[ct], 0, 0, 0);
            }
            float sc[2] = {kLogitScale, kLogitScale}, vs[2] = {1.0f, 1.0f}, rs[2] = {1.0f, 1.0f};
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if constexpr (QT) sc[b] *= off(now.ks, b0 + b);
                if constexpr (V8) {
                    vs[b] = off(now.vs, b0 + b);
                    if (vs[b] == 0.0f) vs[b] = 1.0f;   // (all its values are 0)
                    rs[b] = 1.0f / vs[b];
                }
            }
            uint32_t pw[TERMS][CT][8];   // the weights, two to a word
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[ct][i] *= sc[i >> 3];
                if (!all) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int t = 8 * ((i >> 2) & 1) + 4 * h + (i & 3), at_t = at[i >> 3] + t;
                        const bool sees = t < live[i >> 3] && at_t <= own[ct] && (at_t > own[ct] - win || at_t < c.sinks);
                        x[ct][i] = sees ? x[ct][i] : -INFINITY;
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, x[ct][i]);
                mx = max_halves(mx);
                if (__any(mx > m[ct] + kSlack || (m[ct] == -INFINITY && mx > -INFINITY))) {
                    const float mn = fmaxf(m[ct], mx);
                    const float f = mn == -INFINITY ? 1.0f : hw_exp2(m[ct] - mn);
                    l[ct] *= f;
                    lw[ct] *= f;
#pragma unroll
                    for (int d = 0; d < 4; ++d) o[ct][d] *= f;
                    m[ct] = mn;
                }
                const float ms = m[ct] == -INFINITY ? 0.0f : m[ct];
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    float a = hw_exp2(x[ct][i] - ms), b = hw_exp2(x[ct][i + 1] - ms);
                    l[ct] += a + b;
                    if constexpr (V8) {
                        a *= vs[i >> 3];
                        b *= vs[i >> 3];
                    }
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) {
                        const uint32_t w = pack_bf16(a, b);
                        pw[t][ct][i >> 1] = w;
                        if constexpr (TERMS == 1) {
                            lw[ct] = fmaf(bf16_lo(w) + bf16_hi(w), rs[i >> 3], lw[ct]);
                        } else {
                            a -= bf16_lo(w);
                            b -= bf16_hi(w);
                        }
                    }
                }
            }
            // words 4 b .. 4 b + 3: block b's tokens 4h .. 4h+3, 8+4h .. 8+4h+3
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint8_t* vb = vl[buf] + 8192 * sub + 4096 * b + 256 * h + 16 * (n & 15) + 8 * (n >> 4);
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const u32x2 lo = *reinterpret_cast<const u32x2*>(vb + 1024 * d), hi = *reinterpret_cast<const u32x2*>(vb + 1024 * d + 512);
                    const bf16x8 a = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                        for (int t = 0; t < TERMS; ++t)
                            o[ct][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                a, __builtin_bit_cast(bf16x8, u32x4{pw[t][ct][4 * b], pw[t][ct][4 * b + 1], pw[t][ct][4 * b + 2],
                                                                    pw[t][ct][4 * b + 3]}),
                                o[ct][d], 0, 0, 0);
                }
            }
        }
        if (more) store(j + 1, mine, buf ^ 1);
        lds_sync();
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        l[ct] = add_halves(l[ct]);
        lw[ct] = TERMS == 1 ? add_halves(lw[ct]) : l[ct];
    }
    // ---- A value that is not finite reaches, as 0 times it, the columns of its
    // step that do not see it.  Those with a finite sum and a result that is not
    // are worked out again, token by token: here, where it costs nothing else.
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        float z = lw[ct] * 0.0f;   // NaN unless everything is finite
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) z = fmaf(o[ct][d][i], 0.0f, z);
        z = add_halves(z);
        uint32_t bad = (uint32_t)__ballot(row_of[ct] >= 0 && own[ct] >= 0 && l[ct] * 0.0f == 0.0f && z != 0.0f);
        if (bad == 0) continue;
        float* const y_lds = reinterpret_cast<float*>(kl[0]) + kHeadDim * wv;
        const int e = 2 * lane;   // this lane's dims: e and e + 1
        while (bad != 0) {
            const int who = __ffs(bad) - 1;
            bad &= bad - 1;
            const int own_slot = of(own[ct], who), head = of(head_of[ct], who);
            const float top = off(m[ct], who);
            const int64_t q_at = (row_lo + (int64_t)((col0 + 32 * ct + who) / c.G)) * c.q_stride + head * kHeadDim + e;
            float q0, q1, y0 = 0.0f, y1 = 0.0f;
            if (c.q_f32) {
                q0 = static_cast<const float*>(c.q)[q_at];
                q1 = static_cast<const float*>(c.q)[q_at + 1];
            } else {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(c.q) + q_at);
                q0 = bf16_lo(w);
                q1 = bf16_hi(w);
            }
            for (int i = 4 * begin; i < min(n_blocks, 4 * end); ++i) {
                if (((i - 4 * begin) & 63) == 0) mine = describe(i);
                const int at = of(mine.at, (i - 4 * begin) & 63), live = of(mine.live, (i - 4 * begin) & 63);
                const size_t tile_at = (size_t)of(mine.phys, (i - 4 * begin) & 63) * c.page_elems + row_elems +
                                       (size_t)((at >> 4) & (per - 1)) * 16 * kHeadDim;
                const bool coded = QT && of(mine.coded, (i - 4 * begin) & 63) != 0;
                const float ks = off(mine.ks, (i - 4 * begin) & 63), vs = off(mine.vs, (i - 4 * begin) & 63);
                for (int t = 0; t < live; ++t) {
                    if (at + t > own_slot || (at + t <= own_slot - win && at + t >= c.sinks)) continue;
                    uint32_t kw;
                    if (coded)
                        kw = codes_pair_to_bf16<false>(*reinterpret_cast<const uint16_t*>(
                            reinterpret_cast<const uint8_t*>(c.k_pool + tile_at) + 1024 * (e / 64) + 16 * (t + 16 * ((e / 8) % 4)) +
                            8 * ((e / 32) % 2) + e % 8));
                    else
                        kw = *reinterpret_cast<const uint32_t*>(c.k_pool + tile_at + (e / 8) * 128 + t * 8 + e % 8);
                    const float x = wave_sum(fmaf(q0, bf16_lo(kw), q1 * bf16_hi(kw))) * ks * kLogitScale;
                    const float w = hw_exp2(x - top);
                    if constexpr (V8) {
                        const uint8_t* v = c.v_codes + tile_at + (e / 64) * 1024 + (t / 4) * 256 + (e % 16) * 16 + ((e / 16) % 4) * 4 + t % 4;
                        const uint32_t pair = codes_pair_to_bf16<false>((uint32_t)v[0] | ((uint32_t)v[16] << 8));
                        y0 = fmaf(w, vs * bf16_lo(pair), y0);
                        y1 = fmaf(w, vs * bf16_hi(pair), y1);
                    } else {
                        const uint16_t* v = c.v_pool + tile_at + (e / 32) * 512 + (t / 4) * 128 + (e % 16) * 8 + ((e / 16) % 2) * 4 + t % 4;
                        y0 = fmaf(w, bf16_lo(v[0]), y0);
                        y1 = fmaf(w, bf16_lo(v[8]), y1);
                    }
                }
            }
            y_lds[e] = y0;
            y_lds[e + 1] = y1;
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
            if (n == who) {
                lw[ct] = l[ct];
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[ct][d][i] = y_lds[32 * d + 8 * (i >> 2) + 4 * h + (i & 3)];
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
        }
    }

    if (status != 0) atomicOr(c.status, status);
    // ---- register i of o[ct][d]: dim 32 d + 8 (i / 4) + 4 h + i % 4
    auto write4 = [&](int64_t row, int head, int dim, f32x4 y) {
        const int64_t at = row * c.out_stride + head * kHeadDim + dim;
        if (c.out_bf16)
            *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(c.out) + at) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
        else
            *reinterpret_cast<f32x4*>(static_cast<float*>(c.out) + at) = y;
    };
    if (parts == 1) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            if (row_of[ct] < 0) continue;
            const float inv = inverse(lw[ct]);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    write4(row_of[ct], head_of[ct], 32 * d + 2 * i + 4 * h,
                           f32x4{o[ct][d][i], o[ct][d][i + 1], o[ct][d][i + 2], o[ct][d][i + 3]} * inv);
            if (c.lse != nullptr && h == 0) c.lse[row_of[ct] * c.Hq + head_of[ct]] = log_sum(m[ct], l[ct]);
        }
        return;
    }
    // ---- the tile's parts meet in the workgroup that comes last
    const int unit = tile * c.Hkv + kv;
    float* const part0 = c.part + (size_t)unit * c.splits * kCols * kPartWords;
    float* const part = part0 + (size_t)split * kCols * kPartWords;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        if (row_of[ct] < 0) continue;
        float* p = part + (size_t)(wv * 32 * CT + 32 * ct + n) * kPartWords;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 2) put2(p + 32 * d + 8 * (i >> 2) + 4 * h + (i & 3), o[ct][d][i], o[ct][d][i + 1]);
        if (h == 0) {
            put2(p + kHeadDim, m[ct], l[ct]);
            put2(p + kHeadDim + 2, lw[ct], 0.0f);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) sh_last = arrive_last(c.count + unit, arrive(c.count + unit), parts) ? 1 : 0;
    __syncthreads();
    if (sh_last == 0) return;
    const int cols = min(kCols, rows * c.G - (tile - uni(pref[s])) * kCols);
    for (int col = wv; col < cols; col += kWaves) {   // a wave a column, two dims a lane
        float M = -INFINITY, lsum = 0.0f, wsum = 0.0f, y0 = 0.0f, y1 = 0.0f;
        const float* p = part0 + (size_t)col * kPartWords;
#pragma unroll 4
        for (int z = 0; z < parts; ++z) {
            const float2 st = get2(p + (size_t)z * kCols * kPartWords + kHeadDim);
            const float ws = get2(p + (size_t)z * kCols * kPartWords + kHeadDim + 2).x;
            const float2 y = get2(p + (size_t)z * kCols * kPartWords + 2 * lane);
            const float mn = fmaxf(M, st.x);
            const float fa = mn == -INFINITY ? 0.0f : hw_exp2(M - mn), fb = mn == -INFINITY ? 0.0f : hw_exp2(st.x - mn);
            lsum = lsum * fa + st.y * fb;
            wsum = wsum * fa + ws * fb;
            y0 = y0 * fa + y.x * fb;
            y1 = y1 * fa + y.y * fb;
            M = mn;
        }
        const int g = (tile - uni(pref[s])) * kCols + col;
        const int64_t row = row_lo + g / c.G;
        const int head = kv * c.G + g % c.G;
        const float inv = inverse(wsum);
        const int64_t at = row * c.out_stride + head * kHeadDim + 2 * lane;
        if (c.out_bf16) *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(c.out) + at) = pack_bf16(y0 * inv, y1 * inv);
        else *reinterpret_cast<float2*>(static_cast<float*>(c.out) + at) = make_float2(y0 * inv, y1 * inv);
        if (c.lse != nullptr && lane == 0) c.lse[row * c.Hq + head] = log_sum(M, lsum);
    }
}

template <int TERMS, int CT>
const void* prompt_kernel(bool keys8, bool values8) {
    return keys8 ? (values8 ? reinterpret_cast<const void*>(&k_rows_attend<TERMS, CT, true, true>)
                            : reinterpret_cast<const void*>(&k_rows_attend<TERMS, CT, true, false>))
                 : (values8 ? reinterpret_cast<const void*>(&k_rows_attend<TERMS, CT, false, true>)
                            : reinterpret_cast<const void*>(&k_rows_attend<TERMS, CT, false, false>));
}

constexpr int kWideCols = kWaves * 64;    // columns of a tile, bf16 in and out
constexpr int kExactCols = kWaves * 32;   // and in three terms

// Parts that all tiles of a call may be cut into: a workgroup per CU.
int most_parts(int n_cu) { return n_cu; }

size_t count_words(int n_cu) { return ((size_t)n_cu + 63) / 64 * 64; }

}  // namespace

uint64_t rows_workspace(const Dims&, int n_cu) {
    return (count_words(n_cu) + (uint64_t)most_parts(n_cu) * kWideCols * kPartWords) * sizeof(float);
}

hipError_t launch_attend_rows(const Dims& dm, const View& v, const Scratch& sc, int n_cu, int layer, const md_rows_args& a,
                              hipStream_t st) {
    PromptCall c{};
    c.S = dm.S;
    c.L = dm.L;
    c.Hq = dm.Hq;
    c.Hkv = dm.Hkv;
    c.G = dm.G;
    c.P = dm.P;
    c.Pshift = dm.Pshift;
    c.MP = dm.MP;
    c.NP = dm.NP;
    c.aligned = dm.aligned;
    c.layer = layer;
    c.page_elems = (size_t)dm.LHkv * dm.P * kHeadDim;
    c.k_pool = v.k_pool;
    c.region = v.region;
    c.page_table = v.page_table;
    c.n_pages = v.n_pages;
    c.n_tokens = v.n_tokens;
    c.page_format = v.page_format;
    c.status = sc.status;
    c.row_start = a.rows.row_start;
    c.row_slot = a.rows.row_slot;
    c.n_rows = a.rows.n_rows;
    c.q = a.q;
    c.q_stride = a.q_stride;
    c.out = a.out;
    c.out_stride = a.out_stride;
    c.lse = a.lse;
    c.q_f32 = a.q_type == MD_F32;
    c.out_bf16 = a.out_type == MD_BF16;
    c.window = a.window;
    c.sinks = a.sinks;
    c.v_pool = a.values.v_pool;
    c.v_codes = a.values.v_codes;
    c.v_scale = a.values.v_scale;
    const bool exact = c.q_f32 || !c.out_bf16;
    const int cols = exact ? kExactCols : kWideCols;
    // the most tiles that rows can make, however they are spread over the sessions
    const int64_t tiles = (int64_t)a.rows.n_rows * dm.G / cols + std::min(dm.S, a.rows.n_rows);
    const int64_t steps = ((int64_t)dm.MP * dm.P + kStep - 1) / kStep;
    c.splits = (int)std::max<int64_t>(1, std::min<int64_t>(steps, most_parts(n_cu) / (tiles * dm.Hkv)));
    c.count = static_cast<int32_t*>(a.workspace);
    c.part = static_cast<float*>(a.workspace) + count_words(n_cu);
    void* args[] = {&c};
    const bool keys8 = dm.quant != 0, values8 = a.values.v_pool == nullptr;
    const void* fn = exact ? prompt_kernel<3, 1>(keys8, values8) : prompt_kernel<1, 2>(keys8, values8);
    return hipLaunchKernel(fn, dim3((unsigned)(tiles * dm.Hkv * c.splits)), dim3(kThreads), args,
                           (size_t)(dm.S + 1) * sizeof(int), st);
}

}  // namespace md
