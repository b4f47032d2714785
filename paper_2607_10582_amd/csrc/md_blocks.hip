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
// that for pages of 16); the scores read 257 bytes per page and KV head; the
// choice is a chain of a few passes over one row's scores in registers.

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

// bf16 pairs in an order-preserving int16 form and back (its own inverse):
// negative numbers have their magnitude bits flipped.
__device__ __forceinline__ s16x2 ordered(uint32_t w) {
    const s16x2 x = __builtin_bit_cast(s16x2, w);
    return x ^ ((x >> 15) & (short)0x7FFF);
}

__device__ __forceinline__ s16x2 min2(s16x2 a, s16x2 b) { return __builtin_elementwise_min(a, b); }

__device__ __forceinline__ s16x2 from_lane(s16x2 x, int mask) {
    return __builtin_bit_cast(s16x2, __shfl_xor(__builtin_bit_cast(int, x), mask));
}

// Minima and maxima over the 16 tokens of a block, whose token t and dims
// 32 j + 8 g + 2 k, + 1 lane (t, g) holds in x[0][j][k] (ordered), and their
// complement in x[1][j][k], so that both are minima.  A butterfly over the
// token bits in which each lane passes on the half it does not keep: lane
// (t, g) ends with the minimum (t < 8) or the complemented maximum of dims
// 32 ((t >> 1) & 3) + 8 g + 4 (t & 1) .. + 3, in two words.
__device__ __forceinline__ void reduce_tokens(s16x2 (&x)[2][4][4], int t, s16x2 (&out)[2]) {
    s16x2 a[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const s16x2 keep = t & 8 ? x[1][j][k] : x[0][j][k], give = t & 8 ? x[0][j][k] : x[1][j][k];
            a[j][k] = min2(keep, from_lane(give, 8));
        }
    s16x2 b[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const s16x2 keep = t & 4 ? a[2 + j][k] : a[j][k], give = t & 4 ? a[j][k] : a[2 + j][k];
            b[j][k] = min2(keep, from_lane(give, 4));
        }
    s16x2 d[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const s16x2 keep = t & 2 ? b[1][k] : b[0][k], give = t & 2 ? b[0][k] : b[1][k];
        d[k] = min2(keep, from_lane(give, 2));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const s16x2 keep = t & 1 ? d[2 + k] : d[k], give = t & 1 ? d[k] : d[2 + k];
        out[k] = min2(keep, from_lane(give, 1));
    }
}

// The four values of a lane after reduce_tokens, as numbers; infinities and
// NaNs of either sign become the largest float32.
__device__ __forceinline__ void as_numbers(const s16x2 (&w)[2], bool upper, float (&y)[4]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const s16x2 x = upper ? ~w[k] : w[k];
        const uint32_t u = __builtin_bit_cast(uint32_t, x ^ ((x >> 15) & (short)0x7FFF));
        y[2 * k] = __uint_as_float(u << 16);
        y[2 * k + 1] = __uint_as_float(u & 0xFFFF0000u);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if ((__float_as_uint(y[k]) & 0x7F800000u) == 0x7F800000u)
            y[k] = __uint_as_float(0x7F7FFFFFu | (__float_as_uint(y[k]) & 0x80000000u));
}

// One wave per (layer, KV head) tile of a page, four of them a workgroup;
// blockIdx.y: session, blockIdx.x: page of it (all) and group of tiles.
template <bool QT>
__global__ void __launch_bounds__(kBlkThreads) k_bounds(Dims dm, View v, Scratch sc, int all, int8_t* __restrict__ bounds,
                                                        int8_t* __restrict__ bound_exp) {
    const int s = blockIdx.y;
    const int groups = (dm.LHkv + 3) >> 2;
    const int np = v.n_pages[s], nt = v.n_tokens[s];
    if (!counters_ok(np, nt, dm)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(sc.status, kDevCorrupt);
        return;
    }
    const int page = all ? (int)blockIdx.x / groups : np - 1;
    const int row = ((int)blockIdx.x % groups) * 4 + (threadIdx.x >> 6);
    if (page < 0 || page >= np || row >= dm.LHkv) return;
    const int p = v.page_table[(size_t)s * dm.MP + page];
    if ((unsigned)p >= (unsigned)dm.NP) {
        atomicOr(sc.status, kDevCorrupt);
        return;
    }
    const int lane = lane_id(), t = lane & 15, g = lane >> 4;
    const size_t tile = ((size_t)p * dm.LHkv + row) * dm.P * kHeadDim;
    const int slots = min(dm.P, nt - page * dm.P);
    const uint8_t* region = v.region + (size_t)p * dm.P;
    const bool codes = QT && v.page_format[p] != 0;
    const s16x2 most = {0x7FFF, 0x7FFF};
    s16x2 x[2][4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) x[0][j][k] = x[1][j][k] = most;
    const bool upper = t >= 8;
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = upper ? -INFINITY : INFINITY;
    for (int b = 0; b < dm.P >> 4; ++b) {
        const int slot = 16 * b + t;
        const bool live = slot < slots && (!dm.aligned || region[slot] != (uint8_t)kHole);
        if (16 * b >= slots) break;
        const u32x4* kp = reinterpret_cast<const u32x4*>(v.k_pool + tile + (size_t)b * 16 * kHeadDim) + lane;
        u32x4 w[4];
        if (!codes) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = kp[64 * j];
        } else {
            const u32x4 c0 = kp[0], c1 = kp[64];
            w[0] = codes_to_bf16<0>(c0);
            w[1] = codes_to_bf16<1>(c0);
            w[2] = codes_to_bf16<0>(c1);
            w[3] = codes_to_bf16<1>(c1);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const s16x2 o = ordered(w[j][k]);
                if (live) {
                    x[0][j][k] = min2(x[0][j][k], o);
                    x[1][j][k] = min2(x[1][j][k], ~o);
                }
            }
        if (codes) {   // each block of codes has its own scale
            const float scale = *reinterpret_cast<const float*>(
                reinterpret_cast<const uint8_t*>(v.k_pool + tile + (size_t)b * 16 * kHeadDim) + 2048);
            const bool any = __any(live);
            s16x2 r[2];
            reduce_tokens(x, t, r);
            float z[4];
            as_numbers(r, upper, z);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (any) y[i] = upper ? fmaxf(y[i], z[i] * scale) : fminf(y[i], z[i] * scale);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) x[0][j][k] = x[1][j][k] = most;
        }
    }
    if (!codes) {
        s16x2 r[2];
        reduce_tokens(x, t, r);
        as_numbers(r, upper, y);
    }
    float amax = fmaxf(fmaxf(fabsf(y[0]), fabsf(y[1])), fmaxf(fabsf(y[2]), fabsf(y[3])));
    amax = wave_max(amax);
    const int e = step_exp(amax);
    const float unit = power2(-e);
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // (a key so small that the product becomes 0 still rounds outward)
        const float z = y[i] * unit;
        const float c = upper ? fmaxf(ceilf(z), y[i] > 0.0f ? 1.0f : -127.0f) : fminf(floorf(z), y[i] < 0.0f ? -1.0f : 127.0f);
        out |= ((uint32_t)(int)fminf(fmaxf(c, -127.0f), 127.0f) & 0xFFu) << (8 * i);
    }
    const size_t at = (size_t)p * dm.LHkv + row;
    // dims 32 ((t >> 1) & 3) + 8 g + 4 (t & 1) .. + 3 of lo (t < 8) or hi
    *reinterpret_cast<uint32_t*>(bounds + at * kBoundBytes + (upper ? kHeadDim : 0) + 32 * ((t >> 1) & 3) + 8 * g +
                                 4 * (t & 1)) = out;
    if (lane == 0) bound_exp[at] = (int8_t)e;
}

// Order-preserving uint32 of a score.
__device__ __forceinline__ uint32_t score_key(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// Scores of 64 pages of one (session, KV head) per workgroup, 16 per wave.
__global__ void __launch_bounds__(kBlkThreads) k_block_scores(Dims dm, View v, Scratch sc, int layer,
                                                              const float* __restrict__ q, int64_t q_stride,
                                                              const int8_t* __restrict__ bounds,
                                                              const int8_t* __restrict__ bound_exp,
                                                              uint32_t* __restrict__ keys) {
    const int s = blockIdx.x / dm.Hkv, kv = blockIdx.x % dm.Hkv;
    const int np = v.n_pages[s], nt = v.n_tokens[s];
    const int p0 = (int)blockIdx.y * 64 + (threadIdx.x >> 6) * 16;
    if (!counters_ok(np, nt, dm) || p0 >= np) return;
    const int lane = lane_id(), h = lane & 15, g = lane >> 4;
    // the head's query in 8 bits: elements 64 j + 16 g .. + 15 of it
    float x[2][16];
    float amax = 0.0f;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 a = {0.f, 0.f, 0.f, 0.f};
            if (h < dm.G)
                a = *reinterpret_cast<const f32x4*>(q + (int64_t)s * q_stride + (kv * dm.G + h) * kHeadDim + 64 * j + 16 * g +
                                                    4 * i);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[j][4 * i + k] = a[k] == a[k] ? a[k] : 0.0f;
                amax = fmaxf(amax, fabsf(x[j][4 * i + k]));
            }
        }
    amax = fmaxf(amax, __shfl_xor(amax, 16));
    amax = fmaxf(amax, __shfl_xor(amax, 32));
    const int f = step_exp(amax);
    const float unit = power2(-f);
    i32x4 bq[4];   // against lo (0, 1) and hi (2, 3)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t lo = 0, hi = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = (int)fminf(fmaxf(rintf(x[j][4 * i + k] * unit), -127.0f), 127.0f);
                lo |= ((uint32_t)min(c, 0) & 0xFFu) << (8 * k);
                hi |= ((uint32_t)max(c, 0) & 0xFFu) << (8 * k);
            }
            bq[j][i] = (int)lo;
            bq[2 + j][i] = (int)hi;
        }
    const int page = min(p0 + h, np - 1);
    int p = v.page_table[(size_t)s * dm.MP + page];
    if ((unsigned)p >= (unsigned)dm.NP) {
        atomicOr(sc.status, kDevCorrupt);
        p = 0;
    }
    const size_t at = (size_t)p * dm.LHkv + layer * dm.Hkv + kv;
    const i32x4* b = reinterpret_cast<const i32x4*>(bounds + at * kBoundBytes) + g;
    i32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[4 * j], bq[j], acc, 0, 0, 0);
    const int e = bound_exp[at];   // of page p0 + h
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // page p0 + 4 g + i, head h
        const int ep = __shfl(e, 4 * g + i);
        float y = h < dm.G ? ldexpf((float)acc[i], ep + f) : -INFINITY;
        y = fmaxf(y, __shfl_xor(y, 8));
        y = fmaxf(y, __shfl_xor(y, 4));
        y = fmaxf(y, __shfl_xor(y, 2));
        y = fmaxf(y, __shfl_xor(y, 1));
        if (h == 0 && p0 + 4 * g + i < np) keys[(size_t)blockIdx.x * dm.MP + p0 + 4 * g + i] = score_key(y + 0.0f);
    }
}

// One workgroup per (session, KV head): thread i holds the scores of eight
// pages 8 i .. 8 i + 7.  A radix select, eight bits at a time, finds the key
// of the last page to be taken and how many of those with that key are (the
// oldest); the taken pages' places come from prefix sums in page order.
__global__ void __launch_bounds__(kSelThreads) k_block_pick(Dims dm, View v, Scratch sc, md_select_args a,
                                                            const uint32_t* __restrict__ keys) {
    __shared__ int hist[256];
    __shared__ int lds[2 * 17];
    __shared__ int sh_bin, sh_need;
    const int s = blockIdx.x / dm.Hkv, tid = threadIdx.x;
    int np = v.n_pages[s];
    const int nt = v.n_tokens[s];
    if (!counters_ok(np, nt, dm)) {
        if (tid == 0) atomicOr(sc.status, kDevCorrupt);
        np = 0;
    }
    const int K = min(a.max_blocks, np);
    uint32_t key[kPerThread];
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const int page = tid * kPerThread + i;
        key[i] = 0;
        if (page < np) {
            key[i] = keys[(size_t)blockIdx.x * dm.MP + page];
            if (page < a.first || page >= np - a.last) key[i] = 0xFFFFFFFFu;
        }
    }
    uint32_t prefix = 0;
    int need = K;   // pages still to be found among those that share the prefix
    if (K < np) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kPerThread; ++i)
                if (tid * kPerThread + i < np && (shift == 24 || (key[i] >> (shift + 8)) == (prefix >> (shift + 8))))
                    atomicAdd(&hist[(key[i] >> shift) & 0xFFu], 1);
            __syncthreads();
            if (tid < 64) {   // from the top bin down: lane i has bins 255 - 4 i ..
                int c[4], sum = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    c[k] = hist[255 - (4 * tid + k)];
                    sum += c[k];
                }
                int before = wave_incl_sum(sum) - sum;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (before < need && before + c[k] >= need) {
                        sh_bin = 255 - (4 * tid + k);
                        sh_need = need - before;
                    }
                    before += c[k];
                }
            }
            __syncthreads();
            prefix |= (uint32_t)sh_bin << shift;
            need = sh_need;
            __syncthreads();
        }
    }
    // of the pages with the last key the first `need`
    int ties = 0, above = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const bool in = tid * kPerThread + i < np;
        ties += in && K < np && key[i] == prefix;
        above += in && (K == np || key[i] > prefix);
    }
    const int cnt[2] = {ties, above};
    int ex[2], tot[2];
    block_exclusive_scan_n<2>(cnt, lds, ex, tot);
    int tie = ex[0];
    int at = ex[1] + (K < np ? min(ex[0], need) : 0);
    int32_t* out = a.blocks + (size_t)blockIdx.x * a.max_blocks;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const int page = tid * kPerThread + i;
        if (page >= np) break;
        bool take = K == np || key[i] > prefix;
        if (!take && key[i] == prefix) take = tie++ < need;
        if (take) out[at++] = page;
    }
    for (int i = K + tid; i < a.max_blocks; i += kSelThreads) out[i] = -1;
    if (tid == 0) a.block_count[blockIdx.x] = K;
}

}  // namespace

hipError_t launch_bounds(const Dims& dm, const View& v, const Scratch& sc, int all, int8_t* bounds, int8_t* bound_exp,
                         hipStream_t st) {
    Dims d = dm;
    View vv = v;
    Scratch ss = sc;
    void* args[] = {&d, &vv, &ss, &all, &bounds, &bound_exp};
    const int groups = (dm.LHkv + 3) / 4;
    const dim3 grid((unsigned)(groups * (all ? dm.MP : 1)), (unsigned)dm.S);
    const void* fn = dm.quant ? reinterpret_cast<const void*>(&k_bounds<true>) : reinterpret_cast<const void*>(&k_bounds<false>);
    return hipLaunchKernel(fn, grid, dim3(kBlkThreads), args, 0, st);
}

uint64_t select_workspace(const Dims& dm) { return (uint64_t)dm.S * dm.Hkv * dm.MP * sizeof(uint32_t); }

hipError_t launch_blocks(const Dims& dm, const View& v, const Scratch& sc, int layer, const md_select_args& a,
                         hipStream_t st) {
    Dims d = dm;
    View vv = v;
    Scratch ss = sc;
    md_select_args aa = a;
    uint32_t* keys = static_cast<uint32_t*>(a.workspace);
    void* sargs[] = {&d, &vv, &ss, &layer, &aa.q, &aa.q_stride, &aa.bounds, &aa.bound_exp, &keys};
    const unsigned rows = (unsigned)(dm.S * dm.Hkv);
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&k_block_scores), dim3(rows, (unsigned)((dm.MP + 63) / 64)),
                                         dim3(kBlkThreads), sargs, 0, st);
    if (e != hipSuccess) return e;
    void* pargs[] = {&d, &vv, &ss, &aa, &keys};
    return hipLaunchKernel(reinterpret_cast<const void*>(&k_block_pick), dim3(rows), dim3(kSelThreads), pargs, 0, st);
}

}  // namespace md
