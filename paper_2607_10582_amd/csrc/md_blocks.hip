// gfx950 kernels of block selection: bounds of each page's keys in 8 bits,
// and the pages whose bounds promise a query the largest logits.
//
// For keys k in a page with lo <= k <= hi elementwise, q . k is at most
//   sum_j max(q_j lo_j, q_j hi_j) = sum_{q_j > 0} q_j hi_j + sum_{q_j < 0} q_j lo_j,
// a product of (q-, q+) with (lo, hi) over 2 d elements.  Bounds and query
// are whole numbers times powers of two, so the product is an exact int32 sum
// on the matrix cores, whatever its order, and a float32 holds it (|sum| <=
// 128 * 127^2 < 2^24): the same pages come out of every way to compute it.
//
// What bounds them: the bounds read every key once (and write a sixteenth of
// that for pages of 16); the scores read 257 bytes per page and KV head, at
// 4.9 TB/s past the first 6 us; the choice is a chain of a few passes over one
// row's scores in registers (5 - 7 us; with the scores in the same launch,
// picked by the row's last workgroup, the two took 33 us against 27).

#include <algorithm>

#include "md_decode.h"
#include "md_device.h"

namespace md {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr int kBlkThreads = 256;
constexpr int kBoundBytes = 2 * kHeadDim;

// The least e in [kMinExp, kMaxExp] with amax <= 127 2^e (amax >= 0; from
// amax = 1.f 2^(E - 127): 127 2^(E - 133) is 1.984375 2^(E - 127)).
__device__ __forceinline__ int step_exp(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 133 + ((u & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
    return min(max(e, kMinExp), kMaxExp);
}

__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // |e| <= 126

// A pair of bf16 numbers in an int16 form that orders as they do (negative ones
// have their magnitude bits flipped; its own inverse).
__device__ __forceinline__ s16x2 ordered(s16x2 x) { return x ^ ((x >> 15) & (short)0x7FFF); }
// (through a parameter: a bit cast of a vector's element takes the vector's first one)
__device__ __forceinline__ s16x2 ordered(uint32_t w) { return ordered(__builtin_bit_cast(s16x2, w)); }

__device__ __forceinline__ s16x2 min2(s16x2 a, s16x2 b) { return __builtin_elementwise_min(a, b); }
__device__ __forceinline__ s16x2 max2(s16x2 a, s16x2 b) { return __builtin_elementwise_max(a, b); }

// A word of the lane whose index differs in bit 0 (quad_perm 1,0,3,2) or bit 1 (2,3,0,1).
template <int BIT>
__device__ __forceinline__ s16x2 from_pair(s16x2 x) {
    return __builtin_bit_cast(s16x2, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), BIT == 0 ? 0xB1 : 0x4E, 0xf,
                                                                 0xf, false));
}

// Largest of the 64 lanes' values, in every lane: rotations within rows of 16,
// then the rows' last lanes passed on (masked lanes meet their own value).
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_max(float v) {
    const int x = __float_as_int(v);
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(x, x, CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_max_dpp(float v) {
    v = dpp_max<0x128, 0xf>(v);
    v = dpp_max<0x124, 0xf>(v);
    v = dpp_max<0x122, 0xf>(v);
    v = dpp_max<0x121, 0xf>(v);
    v = dpp_max<0x142, 0xa>(v);   // row_bcast:15 into rows 1, 3
    v = dpp_max<0x143, 0xc>(v);   // row_bcast:31 into rows 2, 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

constexpr int kBoundSpan = 64;   // tiles of a page one workgroup takes at most
static_assert(kBoundGroup == kBlkThreads / 64 && kBoundSpan % kBoundGroup == 0, "a step's workgroups keep a time each");

// Tiles (layer, KV head) of pages, `span` consecutive ones of a page per
// workgroup, its waves taking them in turn, the next one requested before the
// present one is worked on.  blockIdx.y: session, blockIdx.x: page of it (all
// pages; else the last one, and with the quantised tier the pages that became
// codes since the workgroup's last look: 16 us for 16 such pages of 32,768, 8
// for none, in launches by themselves) and span.  Lane 4 b + i of a wave has
// dims 8 b .. 8 b + 7 of tokens i, i + 4, i + 8, i + 12 of a block (its four
// loads), so that most of the search over the tokens needs no other lane.
template <bool QT>
__global__ void __launch_bounds__(kBlkThreads) k_bounds(Dims dm, View v, Scratch sc, CodeTimes ct, int all, int span,
                                                        int8_t* __restrict__ bounds, int8_t* __restrict__ bound_exp) {
    __shared__ __align__(16) uint32_t staged[kBoundSpan * kBoundBytes / 4];
    __shared__ int8_t staged_exp[kBoundSpan];
    const int s = blockIdx.y;
    const int spans = (dm.LHkv + span - 1) / span;
    const int np = v.n_pages[s], nt = v.n_tokens[s];
    if (!counters_ok(np, nt, dm)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(sc.status, kDevCorrupt);
        return;
    }
    int page = all ? (int)blockIdx.x / spans : np - 1;
    const int row0 = ((int)blockIdx.x % spans) * span, row1 = min(dm.LHkv, row0 + span);
    if (page < 0 || page >= np) return;
    // ---- quantised tier: the pages that became codes since this workgroup
    // looked at the session last (its conversions come at one moment of a
    // step, which the look is before or behind; one before it counts as half a
    // step earlier).  Without the times of either every page of codes is due.
    bool due = false;
    uint32_t now = 0, seen = 0;
    uint32_t* looked = nullptr;
    if constexpr (QT) {
        if (ct.coded_at != nullptr) {
            looked = ct.looked + (size_t)s * bound_groups(dm) + row0 / kBoundGroup;
            const uint32_t last = ct.last[2 * s], pass = ct.last[2 * s + 1];
            now = code_time(sc);
            now -= pass == now ? 0u : 1u;
            if (all) {
                if (page == 0 && (int)threadIdx.x < (row1 - row0 + kBoundGroup - 1) / kBoundGroup)
                    looked[threadIdx.x] = now;
            } else {
                seen = *looked;
                due = last > seen;
            }
        } else {
            due = !all;
        }
    }
    constexpr int kWaves = kBlkThreads / 64;
    const int lane = lane_id(), b = lane >> 2, i4 = lane & 3;
    int from = 0, k = 0, n = 0;   // of the pages before `from` the n found due, k of which are taken
    auto next_due = [&] {
        __shared__ int found[kBlkThreads];
        __shared__ int sh_found;
        while (k == n) {
            if (from >= np - 1) return -1;
            __syncthreads();   // the pages found before are taken
            if (threadIdx.x == 0) sh_found = 0;
            __syncthreads();
            const int i = from + (int)threadIdx.x;
            if (i < np - 1) {
                const int p = v.page_table[(size_t)s * dm.MP + i];
                if ((unsigned)p < (unsigned)dm.NP && v.page_format[p] != 0 && (looked == nullptr || ct.coded_at[p] > seen))
                    found[atomicAdd(&sh_found, 1)] = i;
            }
            __syncthreads();
            from += kBlkThreads;
            k = 0;
            n = sh_found;
        }
        __syncthreads();   // what the page before staged is out
        return uni(found[k++]);
    };
    for (;;) {   // one page, or the last and each that is due
        const int p = v.page_table[(size_t)s * dm.MP + page];
        if ((unsigned)p >= (unsigned)dm.NP) {
            if (threadIdx.x == 0) atomicOr(sc.status, kDevCorrupt);
        } else {
            int row = row0 + uni(threadIdx.x >> 6);
            const int slots = min(dm.P, nt - page * dm.P), blocks = (slots + 15) >> 4;
            const bool codes = QT && v.page_format[p] != 0;
            // tokens of this lane that count: bit 4 k + j for token 16 k + 4 j + i4
            uint32_t live = 0;
            for (int k = 0; k < blocks; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int slot = 16 * k + 4 * j + i4;
                    if (slot < slots && (!dm.aligned || v.region[(size_t)p * dm.P + slot] != (uint8_t)kHole)) live |= 1u << (4 * k + j);
                }
            const bool whole = __all(live == (1u << (4 * blocks)) - 1u);
            const bool upper = i4 >= 2;   // after the search: lanes 2, 3 of four have the upper bounds
            const size_t tile = (size_t)dm.P * kHeadDim;
            const uint16_t* keys = v.k_pool + ((size_t)p * dm.LHkv + row) * tile;
            auto load = [&](const uint16_t* block, u32x4 (&w)[4]) {
                if (!codes) {
                    const u32x4* kp = reinterpret_cast<const u32x4*>(block) + 16 * b + i4;
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = kp[4 * j];
                } else {   // dims 8 b ..: 8 bytes of each token
                    const uint2* kp = reinterpret_cast<const uint2*>(block) + 128 * (b >> 3) + 2 * (i4 + 16 * (b & 3)) + ((b >> 2) & 1);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint2 c = kp[8 * j];
                        w[j] = codes_to_bf16<0>(u32x4{c.x, c.y, 0u, 0u});
                    }
                }
            };
            const s16x2 least = {-0x8000, -0x8000}, most = {0x7FFF, 0x7FFF};
            u32x4 w[4];
            if (row < row1) load(keys, w);
            for (; row < row1; row += kWaves) {
                s16x2 lo[4], hi[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    lo[x] = most;
                    hi[x] = least;
                }
                // The four lanes' ends meet, the largest complemented, so that both are
                // minima: lane i4 ends with the lower bounds (i4 < 2) or the negated
                // upper ones of dims 8 b + 4 (i4 & 1) .. + 3, infinities and NaNs as the
                // largest number of their sign.
                auto meet = [&](float (&z)[4]) {
                    s16x2 half[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) half[x] = min2(upper ? ~hi[x] : lo[x], from_pair<1>(upper ? lo[x] : ~hi[x]));
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const s16x2 all4 = min2(i4 & 1 ? half[2 + x] : half[x], from_pair<0>(i4 & 1 ? half[x] : half[2 + x]));
                        // (the complement of an ordered number is, but for a last bit that its
                        // own complement makes up for, its negative's: -1 - n)
                        const s16x2 c = max2(min2(all4, s16x2{0x7F7F, 0x7F7F}), s16x2{-0x7F80, -0x7F80});
                        const uint32_t u = __builtin_bit_cast(uint32_t, ordered(upper ? ~c : c)) ^ (upper ? 0x80008000u : 0u);
                        z[2 * x] = __uint_as_float(u << 16);
                        z[2 * x + 1] = __uint_as_float(u & 0xFFFF0000u);
                    }
                };
                float y[4] = {INFINITY, INFINITY, INFINITY, INFINITY};
                for (int k = 0; k < blocks; ++k) {
                    u32x4 now[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) now[j] = w[j];
                    const uint16_t* block = keys + (size_t)k * 16 * kHeadDim;
                    // (unconditional, like the attention's: behind the last block it reads that block again, out of the cache)
                    load(k + 1 < blocks ? block + 16 * kHeadDim : row + kWaves < row1 ? keys + kWaves * tile : block, w);
                    if (whole) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            s16x2 o[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[j] = ordered(now[j][x]);
                            lo[x] = min2(lo[x], min2(min2(o[0], o[1]), min2(o[2], o[3])));
                            hi[x] = max2(hi[x], max2(max2(o[0], o[1]), max2(o[2], o[3])));
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const bool count = (live >> (4 * k + j)) & 1u;
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                const s16x2 o = ordered(now[j][x]);
                                lo[x] = min2(lo[x], count ? o : most);
                                hi[x] = max2(hi[x], count ? o : least);
                            }
                        }
                    }
                    if (codes) {   // each block of codes has its own scale
                        const float scale = *reinterpret_cast<const float*>(reinterpret_cast<const uint8_t*>(block) + 2048);
                        const bool any = __any(((live >> (4 * k)) & 15u) != 0);
                        float z[4];
                        meet(z);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            if (any) y[x] = fminf(y[x], z[x] * scale);
                            lo[x] = most;
                            hi[x] = least;
                        }
                    }
                }
                if (!codes) meet(y);
                const int e = step_exp(wave_max_dpp(fmaxf(fmaxf(fabsf(y[0]), fabsf(y[1])), fmaxf(fabsf(y[2]), fabsf(y[3])))));
                const float unit = power2(-e);
                uint32_t word = 0;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    // (a number so small that the product becomes 0 still rounds outward)
                    float c = __builtin_amdgcn_fmed3f(floorf(y[x] * unit), -127.0f, y[x] < 0.0f ? -1.0f : 127.0f);
                    c = upper ? -c : c;
                    word |= ((uint32_t)(int)c & 0xFFu) << (8 * x);
                }
                staged[(row - row0) * (kBoundBytes / 4) + (upper ? kHeadDim / 4 : 0) + 2 * b + (i4 & 1)] = word;
                if (lane == 0) staged_exp[row - row0] = (int8_t)e;
                keys += kWaves * tile;
            }
            // The span's bounds go out at once, consecutive in memory (tile by tile as
            // they are found: 1,446 us against 1,412 for 7.5 GB of keys in pages of 64).
            // Few as they are, they cost HBM much: the same keys without them take
            // 1,225 us, 6.1 TB/s, and with them 1,603 in pages of 16, however they are
            // written (past the caches, or written through).
            __syncthreads();
            const size_t at = (size_t)p * dm.LHkv + row0;
            u32x4* out = reinterpret_cast<u32x4*>(bounds + at * kBoundBytes);
            for (int i = threadIdx.x; i < (row1 - row0) * (kBoundBytes / 16); i += kBlkThreads)
                out[i] = reinterpret_cast<const u32x4*>(staged)[i];
            if ((int)threadIdx.x < row1 - row0) bound_exp[at + threadIdx.x] = staged_exp[threadIdx.x];
        }
        if constexpr (QT) {
            if (due) page = next_due();
            if (due && page >= 0) continue;
        }
        break;
    }
    if (QT && due && looked != nullptr && threadIdx.x == 0) *looked = now;
}

// Order-preserving uint32 of a score.
__device__ __forceinline__ uint32_t score_key(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// Maximum, and sum, over the 16 lanes of a row (each lane gets it): rotations by
// 8, 4, 2, 1.
template <int STEP>
__device__ __forceinline__ float row_rotated(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + STEP, 0xf, 0xf, false));
}

__device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, row_rotated<8>(v));
    v = fmaxf(v, row_rotated<4>(v));
    v = fmaxf(v, row_rotated<2>(v));
    return fmaxf(v, row_rotated<1>(v));
}

__device__ __forceinline__ float row_sum16(float v) {
    v += row_rotated<8>(v);
    v += row_rotated<4>(v);
    v += row_rotated<2>(v);
    return v + row_rotated<1>(v);
}

struct BlockCall {
    int S, Hkv, G, P, MP, NP, LHkv, layer;
    const int32_t* page_table;
    const int32_t* n_pages;
    const int32_t* n_tokens;
    int32_t* status;
    const float* q;
    int64_t q_stride;
    const int8_t* bounds;
    const int8_t* bound_exp;
    int first, last, max_blocks;
    int32_t* blocks;
    int32_t* block_count;
    uint32_t* keys;      // [S Hkv][MP] scores in an order-preserving form
};

constexpr int kPickThreads = 1024;
constexpr int kPickPer = kMaxPages / kPickThreads;   // keys of one thread
constexpr int kBins = 2048;
constexpr int kWords = kMaxPages / 32;
constexpr int kRankAt = kPickThreads / 16;           // candidates ranked directly, 16 threads each

// The row's best keys, a workgroup: the first `first` and the last `last` pages
// and the best of the others, K in all (first + last <= K < np).  Thread i
// holds the keys of pages i, i + 1024 ...  A histogram
// over the range of the keys in question finds the bin that holds the K-th; it
// becomes the range (scores of one row share their leading bits, so that bins
// of fixed digits would mostly be a few full ones, whose counts the LDS adds
// one by one), until few are left in it, which are ranked against each other.
// Leaves a bit for each taken page in the first words of `bins`.
__device__ __forceinline__ void pick(const uint32_t (&key)[kPickPer], int np, int first, int last, int K, int* bins,
                                     int* lds) {
    __shared__ uint32_t sh_lo, sh_hi;
    __shared__ int sh_need, sh_count, sh_n;
    __shared__ uint32_t cand_key[kRankAt];
    __shared__ int cand_at[kRankAt];
    const int tid = threadIdx.x, lane = lane_id();
    const int from = first, to = np - last;   // pages that are chosen from
    auto chosen_from = [&](int i) { const int page = i * kPickThreads + tid; return page >= from && page < to; };
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
#pragma unroll
    for (int i = 0; i < kPickPer; ++i)
        if (chosen_from(i)) {
            lo = min(lo, key[i]);
            hi = max(hi, key[i]);
        }
    if (tid == 0) {
        sh_lo = 0xFFFFFFFFu;
        sh_hi = 0;
    }
    __syncthreads();
    lo = wave_min_u32(lo);
    hi = ~wave_min_u32(~hi);
    if (lane == 0) {
        atomicMin(&sh_lo, lo);
        atomicMax(&sh_hi, hi);
    }
    int need = K - first - last, count = to - from;   // keys to take from the range [lo, hi], and how many are in it
    for (;;) {
        bins[tid] = bins[tid + kPickThreads] = 0;
        __syncthreads();
        lo = sh_lo;
        hi = sh_hi;
        if (lo == hi || count <= kRankAt || need == 0) break;
        const int shift = max(0, 21 - __clz((int)(hi - lo)));   // (hi - lo) >> shift < 2^11
#pragma unroll
        for (int i = 0; i < kPickPer; ++i)
            if (chosen_from(i) && key[i] >= lo && key[i] <= hi) atomicAdd(&bins[(key[i] - lo) >> shift], 1);
        __syncthreads();
        // from the top bin down: thread i has bins 2047 - 2 i and the one below
        const int c0 = bins[kBins - 1 - 2 * tid], c1 = bins[kBins - 2 - 2 * tid];
        int total;
        const int before = block_exclusive_scan(c0 + c1, lds, &total);
        if (before < need && before + c0 + c1 >= need) {
            const bool upper = before + c0 >= need;
            const uint32_t bin = kBins - 1 - 2 * tid - (upper ? 0 : 1);
            sh_lo = lo + (bin << shift);
            sh_hi = lo + min(hi - lo, (bin << shift) + ((1u << shift) - 1));
            sh_need = need - before - (upper ? 0 : c0);
            sh_count = upper ? c0 : c1;
        }
        __syncthreads();
        need = sh_need;
        count = sh_count;
    }
    // Keys above the range are taken; of those in it, `need`: the largest, or
    // of equal ones the first.
    if (tid == 0) sh_n = 0;
    __syncthreads();
    const bool rank_them = need > 0 && count <= kRankAt;
    int taken = 0;
#pragma unroll
    for (int i = 0; i < kPickPer; ++i) {
        if (i * kPickThreads >= np) break;
        const int page = i * kPickThreads + tid;
        const bool free = chosen_from(i), in = free && need > 0 && key[i] >= lo && key[i] <= hi;
        bool take = page < np && (!free || (need > 0 && key[i] > hi));
        if (rank_them) {
            if (in) {
                const int at = atomicAdd(&sh_n, 1);
                cand_key[at] = key[i];
                cand_at[at] = page;
            }
        } else if (need > 0) {   // more equal keys than can be ranked: in page order
            int total;
            const int ex = block_exclusive_scan(in ? 1 : 0, lds, &total);
            take = take || (in && taken + ex < need);
            taken += total;
        }
        const uint64_t m = __ballot(take);
        if (lane < 2) bins[(i * kPickThreads + (tid & ~63)) / 32 + lane] = (int)(uint32_t)(m >> (32 * lane));
    }
    __syncthreads();
    if (rank_them) {   // thread 16 i + j counts candidates 4 j .. 4 j + 3 that go before the i-th
        const int i = tid >> 4;
        const uint32_t k = cand_key[i];
        const int at = cand_at[i];
        float rank = 0.0f;
#pragma unroll
        for (int x = 0; x < kRankAt / 16; ++x) {
            const int o = (tid & 15) * (kRankAt / 16) + x;
            rank += o < count && (cand_key[o] > k || (cand_key[o] == k && cand_at[o] < at)) ? 1.0f : 0.0f;
        }
        rank = row_sum16(rank);
        if ((tid & 15) == 0 && i < count && rank < (float)need) atomicOr(&bins[at >> 5], 1 << (at & 31));
    }
    __syncthreads();
}

__device__ __forceinline__ bool counts_ok(const BlockCall& c, int np, int nt) {
    return np == 0 ? nt == 0 : np > 0 && np <= c.MP && nt > (np - 1) * c.P && nt <= np * c.P;
}

// Scores of 32 pages of one (session, KV head) per wave, in two groups of 16,
// requested at once.  The waves of a workgroup take the KV heads of the same
// pages, whose bounds and exponents lie next to each other.  A load covers
// four pages' bounds whole (16 pages' 64-byte quarters, the operand's own
// order, took 25 us where this takes 21: 64 sessions of up to 4,096 pages, two
// KV heads, 72 MB), so the operands are put together through LDS.
constexpr int kScoreAt = 2;
constexpr int kScorePages = 16 * kScoreAt;

__global__ void __launch_bounds__(kBlkThreads) k_block_scores(BlockCall c) {
    __shared__ i32x4 lds[kBlkThreads / 64][16][17];
    i32x4 (&turned)[16][17] = lds[threadIdx.x >> 6];
    const int s = blockIdx.y;
    const int lane = lane_id(), h = lane & 15, g = lane >> 4;
    const int task = (int)blockIdx.x * (kBlkThreads / 64) + uni(threadIdx.x >> 6);
    const int kv = task % c.Hkv, p0 = task / c.Hkv * kScorePages, row = s * c.Hkv + kv;
    const int np = c.n_pages[s];
    if (p0 >= np || np <= c.max_blocks || !counts_ok(c, np, c.n_tokens[s])) return;
    // (the query first: it is turned into codes while the bounds are under way)
    f32x4 qv[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            qv[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (h < c.G)
                qv[j][i] = *reinterpret_cast<const f32x4*>(c.q + (int64_t)s * c.q_stride + (kv * c.G + h) * kHeadDim + 64 * j +
                                                           16 * g + 4 * i);
        }
    const int32_t* table = c.page_table + (size_t)s * c.MP;
    const int head = c.layer * c.Hkv + kv;
    bool bad = false;
    auto page_of = [&](int page) {
        int p = table[min(page, np - 1)];
        if ((unsigned)p >= (unsigned)c.NP) {
            bad = true;
            p = 0;
        }
        return (size_t)p * c.LHkv + head;
    };
    size_t at[kScoreAt][4], own[kScoreAt];
#pragma unroll
    for (int k = 0; k < kScoreAt; ++k) {
#pragma unroll
        for (int j = 0; j < 4; ++j) at[k][j] = page_of(p0 + 16 * k + 4 * j + g);
        own[k] = page_of(p0 + 16 * k + 4 * g + (h & 3));   // the page whose score this lane writes
    }
    i32x4 b[kScoreAt][4];
    int e[kScoreAt];
#pragma unroll
    for (int k = 0; k < kScoreAt; ++k) {
#pragma unroll
        for (int j = 0; j < 4; ++j) b[k][j] = reinterpret_cast<const i32x4*>(c.bounds + at[k][j] * kBoundBytes)[h];
        e[k] = c.bound_exp[own[k]];
    }
    if (__any(bad) && lane == 0) atomicOr(c.status, kDevCorrupt);
    // ---- the head's query in 8 bits: elements 64 j + 16 g .. + 15 of it
    i32x4 bq[4];   // against lo (0, 1) and hi (2, 3)
    int f;
    {
        float x[2][16];
        float amax = 0.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float a = qv[j][i / 4][i % 4];
                x[j][i] = a == a ? a : 0.0f;
                amax = fmaxf(amax, fabsf(x[j][i]));
            }
        amax = fmaxf(amax, __shfl_xor(amax, 16));
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        f = step_exp(amax);
        const float unit = power2(-f);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t lo = 0, hi = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int code = (int)fminf(fmaxf(rintf(x[j][4 * i + k] * unit), -127.0f), 127.0f);
                    lo |= ((uint32_t)min(code, 0) & 0xFFu) << (8 * k);
                    hi |= ((uint32_t)max(code, 0) & 0xFFu) << (8 * k);
                }
                bq[j][i] = (int)lo;
                bq[2 + j][i] = (int)hi;
            }
    }
    uint32_t* keys = c.keys + (size_t)row * c.MP;
#pragma unroll
    for (int k = 0; k < kScoreAt; ++k) {
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) turned[4 * j + g][h] = b[k][j];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(turned[h][4 * j + g], bq[j], acc, 0, 0, 0);
        __builtin_amdgcn_wave_barrier();
        float y[4];   // page 4 g + i: the best head's, short of the page's exponent
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = row_max(h < c.G ? ldexpf((float)acc[i], f) : -INFINITY);
        const float z = ldexpf((h & 2) ? ((h & 1) ? y[3] : y[2]) : ((h & 1) ? y[1] : y[0]), e[k]);
        const int page = p0 + 16 * k + 4 * g + h;
        if (h < 4 && page < np) keys[page] = score_key(z + 0.0f);
    }
}

// One workgroup per (session, KV head).
__global__ void __launch_bounds__(kPickThreads) k_block_pick(BlockCall c) {
    __shared__ int bins[kBins];
    __shared__ int lds[17];
    const int row = blockIdx.x, s = row / c.Hkv, tid = threadIdx.x;
    int np = c.n_pages[s];
    if (!counts_ok(c, np, c.n_tokens[s])) {
        if (tid == 0) atomicOr(c.status, kDevCorrupt);
        np = 0;
    }
    const int K = min(c.max_blocks, np);
    int32_t* out = c.blocks + (size_t)row * c.max_blocks;
    if (K == np) {   // every page: nothing to choose
        for (int i = tid; i < c.max_blocks; i += kPickThreads) out[i] = i < np ? i : -1;
        if (tid == 0) c.block_count[row] = K;
        return;
    }
    const uint32_t* keys = c.keys + (size_t)row * c.MP;
    uint32_t key[kPickPer];
#pragma unroll
    for (int i = 0; i < kPickPer; ++i) {
        key[i] = 0;
        if (i * kPickThreads < np) key[i] = keys[min(i * kPickThreads + tid, np - 1)];
    }
    pick(key, np, c.first, c.last, K, bins, lds);
    // ---- the taken pages in order, their places from the words' counts
    const uint32_t word = tid < kWords ? (uint32_t)bins[tid] : 0u;
    int total;
    int at = block_exclusive_scan(__popc(word), lds, &total);
    for (uint32_t w = word; w != 0; w &= w - 1) out[at++] = 32 * tid + __ffs((int)w) - 1;
    for (int i = K + tid; i < c.max_blocks; i += kPickThreads) out[i] = -1;
    if (tid == 0) c.block_count[row] = K;
}

}  // namespace

hipError_t launch_bounds(const Dims& dm, const View& v, const Scratch& sc, const CodeTimes& ct, int all, int8_t* bounds,
                         int8_t* bound_exp, hipStream_t st) {
    Dims d = dm;
    View vv = v;
    Scratch ss = sc;
    CodeTimes tt = ct;
    // every page: a workgroup walks all of one, or 64 tiles; the last pages: a tile per wave
    int span = all ? std::min(dm.LHkv, kBoundSpan) : kBoundGroup;
    void* args[] = {&d, &vv, &ss, &tt, &all, &span, &bounds, &bound_exp};
    const dim3 grid((unsigned)((dm.LHkv + span - 1) / span * (all ? dm.MP : 1)), (unsigned)dm.S);
    const void* fn = dm.quant ? reinterpret_cast<const void*>(&k_bounds<true>) : reinterpret_cast<const void*>(&k_bounds<false>);
    return hipLaunchKernel(fn, grid, dim3(kBlkThreads), args, 0, st);
}

uint64_t select_workspace(const Dims& dm) { return (uint64_t)dm.S * dm.Hkv * dm.MP * sizeof(uint32_t); }

hipError_t launch_blocks(const Dims& dm, const View& v, const Scratch& sc, int layer, const md_select_args& a,
                         hipStream_t st) {
    BlockCall c{};
    c.S = dm.S;
    c.Hkv = dm.Hkv;
    c.G = dm.G;
    c.P = dm.P;
    c.MP = dm.MP;
    c.NP = dm.NP;
    c.LHkv = dm.LHkv;
    c.layer = layer;
    c.page_table = v.page_table;
    c.n_pages = v.n_pages;
    c.n_tokens = v.n_tokens;
    c.status = sc.status;
    c.q = a.q;
    c.q_stride = a.q_stride;
    c.bounds = a.bounds;
    c.bound_exp = a.bound_exp;
    c.first = a.first;
    c.last = a.last;
    c.max_blocks = a.max_blocks;
    c.blocks = a.blocks;
    c.block_count = a.block_count;
    c.keys = static_cast<uint32_t*>(a.workspace);
    void* args[] = {&c};
    const unsigned rows = (unsigned)(dm.S * dm.Hkv);
    if (dm.MP > a.max_blocks) {   // else every page is taken
        const int tasks = (dm.MP + kScorePages - 1) / kScorePages * dm.Hkv, waves = kBlkThreads / 64;
        const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&k_block_scores),
                                             dim3((unsigned)((tasks + waves - 1) / waves), (unsigned)dm.S), dim3(kBlkThreads),
                                             args, 0, st);
        if (e != hipSuccess) return e;
    }
    return hipLaunchKernel(reinterpret_cast<const void*>(&k_block_pick), dim3(rows), dim3(kPickThreads), args, 0, st);
}

}  // namespace md
