// gfx950 kernel of the attention of ragged rows where a session has few of them
// (a few tokens to verify, the end of a prompt) and for float32: the columns and
// products of md_prompt.hip, 32 columns a workgroup, whose waves take turns along
// the cache.
//
// TERMS: 1, bf16 in and out, whose weights are rounded to bf16 once and divided
// by the sum of what they were rounded to; 3, queries and weights as sums of three
// bf16 terms, which is exact in float32.
//
// Every wave works by itself, 32 tokens at a time: keys come from the pool in
// the order of the products' operands and stay in registers, values turn through
// a piece of LDS that is the wave's own, queries (their terms) are read from LDS
// by all.  The next tokens' bytes are under way while these are worked on, and
// no barrier holds a wave up.  The waves' results meet in LDS, a tile's parts in
// the workgroup that comes last.
//
// What bounds it: the bytes of keys and values for up to 32 columns a session, the
// products above.  5 rows of 6 columns over 8 sessions of 16,384 to 32,768 tokens
// in float32, with 8-bit values, take 48 us (the 155 MB alone, 22); 11 us of it are the same for a
// single session: finding the tile, the page, the first tokens, and the join.
// Through LDS, with a barrier a step and one wave of four at work, 130 us.

#include "md_prompt.h"

namespace md {

namespace {

constexpr int kRowWords = kHeadDim + 4;   // of a column's result in LDS

template <int W, int TERMS, bool QT, bool V8>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(2, 2))) k_rows_few(PromptCall c) {
    constexpr int kThreads = 64 * W;
    constexpr int kQueryBytes = TERMS * 8 * 1024, kValueBytes = 32 * kHeadDim * 2;
    constexpr int kResultBytes = W * kFewTile * kRowWords * 4;
    constexpr int kBytes = kQueryBytes + W * kValueBytes > kResultBytes ? kQueryBytes + W * kValueBytes : kResultBytes;
    __shared__ __align__(16) uint8_t lds[kBytes];   // queries and values, then the waves' results
    __shared__ int scan_lds[2 * 17];
    __shared__ int sh_last;
    extern __shared__ int pref[];   // [S + 1] tiles of the sessions before
    static_assert(8 / W * (kBytes + 256 + (kMaxSessions + 1) * 4) <= 160 * 1024, "eight waves a CU");
    const int tid = threadIdx.x, lane = lane_id(), wv = uni(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    int status = 0;
    TileAt t;
    if (!find_tile<kThreads, kFewTile>(c, scan_lds, pref, t, status)) return;
    // ---- the columns, the same for every wave, and their queries (asked for before
    // the first keys and values: behind them their wait is one for those too, 50 us
    // for 48.5 in the case above)
    const Column col = column_of(c, t, t.col + n, status);
    u32x4* const q_lds = reinterpret_cast<u32x4*>(lds);   // [TERMS][8][64]
#pragma unroll
    for (int y = 0; y < 8 / W; ++y) {
        const int kk = wv + y * W;
        u32x4 w[TERMS];
        query_terms<TERMS>(c, col, kk, w);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) q_lds[(k * 8 + kk) * 64 + lane] = w[k];
    }
    const int smin = uni(-wave_max_i(col.own >= 0 ? -col.own : -0x7FFFFFFF)), smax = uni(wave_max_i(col.own));
    const Seen seen = seen_of(c, smin, smax);
    const int halves = (seen.n_blocks + 1) >> 1;
    const int share = share_of(t, seen.n_blocks) >> 1;
    const int parts = halves == 0 ? 1 : (halves + share - 1) / share;
    if (t.split >= parts) {
        if (status != 0) atomicOr(c.status, status);
        return;
    }
    const int begin = t.split * share, end = min(halves, begin + share);
    const int count = max(0, (end - begin - wv + W - 1) / W);   // this wave's halves: begin + wv, + W ..
    __syncthreads();

    // ---- 32 halves at a time: lane 2 k + b knows of block b of the k-th
    const size_t row_elems = ((size_t)c.layer * c.Hkv + t.kv) * c.P * kHeadDim;
    auto describe = [&](int k) __attribute__((always_inline)) {
        const int half = begin + wv + (k + (lane >> 1)) * W;
        const int i = half < end ? 2 * half + (lane & 1) : seen.n_blocks;
        return block_at<QT, V8>(c, t, seen, row_elems, i, page_of(c, t, seen, i), status);
    };
    Block cur{};
    uint64_t full = 0;
    auto look = [&](int k) __attribute__((always_inline)) {
        cur = describe(k);
        full = __ballot((cur.live == 16) & (cur.at + 15 <= smin) & ((cur.at > smax - seen.win) | (cur.at + 15 < c.sinks)));
    };

    // ---- the next half's bytes
    constexpr int kVals = V8 ? 4 : 8;   // 16 bytes a lane each
    u32x4 rk[8], rv[kVals];
    auto tile_ptr = [](const void* pool, int64_t tile, int shift) {
        return (gbytes)(reinterpret_cast<uint64_t>(pool) + ((uint64_t)tile << shift));
    };
    auto load_keys = [&](const Block& d, int k) __attribute__((always_inline)) {
        // lane (n, h): token n % 16 of block n / 16, dims 16 kk + 8 h ..; codes (a, g, t) hold dims 64 a + 8 g .. and
        // 64 a + 32 + 8 g ..: the kk of the same a and kk % 2 come together
        const int64_t a = lane_tile(d, 2 * k), b = lane_tile(d, 2 * k + 1);
        const bool coded = QT && (n < 16 ? lane_int(d.coded, 2 * k) : lane_int(d.coded, 2 * k + 1)) != 0;
        const gbytes at = tile_ptr(c.k_pool, n < 16 ? a : b, 1) + 16 * (n & 15) + 256 * h;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
            uint32_t off = 512 * kk;
            if (QT && coded) off = kk < 4 ? 1024 * (kk >> 1) + 512 * (kk & 1) : 0;
            rk[kk] = *reinterpret_cast<gvec>(at + off);
        }
    };
    auto load_values = [&](const Block& d, int k) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < kVals; ++x) {   // block, then 1 KiB of it
            const int b = x / (kVals / 2), part = x % (kVals / 2);
            const gbytes at = tile_ptr(V8 ? (const void*)c.v_codes : (const void*)c.v_pool, lane_tile(d, 2 * k + b), V8 ? 0 : 1);
            rv[x] = *reinterpret_cast<gvec>(at + (uint32_t)(1024 * part + 16 * lane));
        }
    };
    uint8_t* const v_lds = lds + kQueryBytes + wv * kValueBytes;
    auto store_values = [&](int k) __attribute__((always_inline)) {
        uint8_t* const to = v_lds + 512 * ((lane >> 4) & 1) + 16 * (lane & 15) + 8 * (lane >> 5);
#pragma unroll
        for (int x = 0; x < kVals; ++x) {
            const int b = x / (kVals / 2), part = x % (kVals / 2);
            // (a slot without a token may hold anything, and 0 times an infinity or NaN is NaN)
            const int live = lane_int(cur.live, 2 * k + b);
            uint32_t m0 = 0xFFFFFFFFu, m1 = 0xFFFFFFFFu;
            if (live < 16) {
                const int k4 = live - 4 * (lane >> 4);
                m0 = k4 >= 2 ? 0xFFFFFFFFu : k4 == 1 ? 0x0000FFFFu : 0u;
                m1 = k4 >= 4 ? 0xFFFFFFFFu : k4 == 3 ? 0x0000FFFFu : 0u;
            }
            auto put = [&](int d, uint32_t p, uint32_t q, uint32_t r, uint32_t s) {   // dims 32 d + m, then 32 d + 16 + m
                *reinterpret_cast<u32x2*>(to + 4096 * b + 1024 * d) = u32x2{p & m0, q & m1};
                *reinterpret_cast<u32x2*>(to + 4096 * b + 1024 * d + 256) = u32x2{r & m0, s & m1};
            };
            if constexpr (V8) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    put(2 * part + y, codes_pair_to_bf16<false>(rv[x][2 * y]), codes_pair_to_bf16<true>(rv[x][2 * y]),
                        codes_pair_to_bf16<false>(rv[x][2 * y + 1]), codes_pair_to_bf16<true>(rv[x][2 * y + 1]));
            } else {
                put(part, rv[x][0], rv[x][1], rv[x][2], rv[x][3]);
            }
        }
    };

    float m = -INFINITY, l = 0.0f, lw = 0.0f;
    f32x16 o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    if (count > 0) {
        look(0);
        load_keys(cur, 0);
        load_values(cur, 0);
    }
    for (int i = 0; i < count; ++i) {
        const int k = i & 31;
        store_values(k);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        // what the lanes know of this half, before they may learn of the next lot
        int at[2], live[2];
        float ks[2] = {1.0f, 1.0f}, vs[2] = {1.0f, 1.0f};
        bool coded[2] = {false, false};
        const bool all = ((full >> (2 * k)) & 3) == 3;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            at[b] = lane_int(cur.at, 2 * k + b);
            live[b] = lane_int(cur.live, 2 * k + b);
            if (QT) coded[b] = lane_int(cur.coded, 2 * k + b) != 0;
            if (QT) ks[b] = lane_float(cur.ks, 2 * k + b);
            if (V8) vs[b] = lane_float(cur.vs, 2 * k + b);
        }
        // (unconditional: behind the last half its own bytes again, out of the cache)
        const int next = min(i + 1, count - 1);
        if ((next & 31) == 0 && next > i) look(next);
        load_values(cur, next & 31);
        if (QT) {
            const bool first = coded[0], second = coded[1];
            if (first || second) {
                const bool mine = n < 16 ? first : second;
                u32x4 w[4] = {rk[0], rk[1], rk[2], rk[3]};
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const u32x4 y = (kk >> 1) & 1 ? codes_to_bf16<1>(w[2 * (kk >> 2) + (kk & 1)])
                                                  : codes_to_bf16<0>(w[2 * (kk >> 2) + (kk & 1)]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) rk[kk][e] = mine ? y[e] : rk[kk][e];
                }
            }
        }
        float sc[2], rs[2], lg[2];
        bool lost[2];
        f32x16 x;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
#pragma unroll
            for (int y = 0; y < TERMS; ++y) {
                const f32x16 none = {};
                x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, rk[kk]),
                                                            __builtin_bit_cast(bf16x8, q_lds[(y * 8 + kk) * 64 + lane]),
                                                            kk == 0 && y == 0 ? none : x, 0, 0, 0);
            }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            sc[b] = kLogitScale;
            if constexpr (QT) {
                if (ks[b] > 0.0f && ks[b] < INFINITY) {
                    sc[b] *= ks[b];
                } else {   // (no factor for the -infinity of a token that is not seen)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[8 * b + e] *= ks[b];
                }
            }
            rs[b] = 1.0f;
            lg[b] = 0.0f;
            lost[b] = false;
            if constexpr (V8) {
                if (vs[b] == 0.0f) vs[b] = 1.0f;   // (all its values are 0)
                lost[b] = !scale_fits(vs[b]);
                if (lost[b]) vs[b] = 1.0f;
                rs[b] = 1.0f / vs[b];
                lg[b] = log2f(vs[b]);
            }
        }
        load_keys(cur, next & 31);
        if (!all) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int b = e >> 3, tk = 8 * ((e >> 2) & 1) + 4 * h + (e & 3), slot = at[b] + tk;
                const bool sees = (tk < live[b]) & (slot <= col.own) & ((slot > col.own - seen.win) | (slot < c.sinks));
                x[e] = sees ? x[e] : -INFINITY;
            }
        }
        float mb[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            mb[b] = x[8 * b];
#pragma unroll
            for (int e = 1; e < 8; ++e) mb[b] = fmaxf(mb[b], x[8 * b + e]);
        }
        const float mx = max_halves(fmaxf(mb[0] * sc[0], mb[1] * sc[1]));
        if (__any(mx > m + kSlack || (m == -INFINITY && mx > -INFINITY))) {
            const float mn = fmaxf(m, mx);
            const float f = mn == -INFINITY ? 1.0f : hw_exp2(m - mn);
            l *= f;
            lw *= f;
#pragma unroll
            for (int d = 0; d < 4; ++d) o[d] *= f;
            m = mn;
        }
        const float ms = m == -INFINITY ? 0.0f : m;
        uint32_t pw[TERMS][8];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const float shift = TERMS == 1 ? lg[b] - ms : -ms;
            float sum = 0.0f, wsum = 0.0f;
#pragma unroll
            for (int e = 8 * b; e < 8 * b + 8; e += 2) {
                float p = hw_exp2(fmaf(x[e], sc[b], shift)), q = hw_exp2(fmaf(x[e + 1], sc[b], shift));
                sum += p + q;
                if constexpr (TERMS != 1 && V8) {
                    p *= vs[b];
                    q *= vs[b];
                }
#pragma unroll
                for (int y = 0; y < TERMS; ++y) {
                    const uint32_t w = pack_bf16(p, q);
                    pw[y][e >> 1] = w;
                    if constexpr (TERMS == 1) {
                        wsum = add_pair(w, wsum);
                    } else {
                        p -= bf16_lo(w);
                        q -= bf16_hi(w);
                    }
                }
            }
            l = fmaf(sum, TERMS == 1 ? rs[b] : 1.0f, l);
            lw = fmaf(wsum, rs[b], lw);
            if (lost[b] && sum > 0.0f) lw = __uint_as_float(0x7FC00000u);   // (settled at the end)
        }
#pragma unroll
        for (int y = 0; y < 8; ++y) {   // block y / 4, dims 32 (y % 4) ..
            const bf16x8 a = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(v_lds + 1024 * y + 16 * lane));
            const int b = y >> 2, d = y & 3;
#pragma unroll
            for (int z = 0; z < TERMS; ++z)
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    a, __builtin_bit_cast(bf16x8, u32x4{pw[z][4 * b], pw[z][4 * b + 1], pw[z][4 * b + 2], pw[z][4 * b + 3]}), o[d], 0, 0, 0);
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
    l = add_halves(l);
    lw = add_halves(lw);
    if (TERMS != 1) lw += l;   // (0, or NaN)
    // A column without a row, or whose row's slot is not there, saw what its
    // neighbours see in full all the same; it has nothing.
    if (col.own < 0) {
        m = -INFINITY;
        l = lw = 0.0f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    }
    // ---- columns that a value reached which is not finite and which they do not see
    {
        float z = lw * 0.0f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) z = fmaf(o[d][i], 0.0f, z);
        z = add_halves(z);
        uint32_t bad = (uint32_t)__ballot(col.own >= 0 && l * 0.0f == 0.0f && z != 0.0f);
        auto blocks = [&](int i) __attribute__((always_inline)) { return describe(i >> 1); };
        if (bad != 0 && !reached_unseen<V8>(c, seen, smin, smax, 2 * count, blocks)) bad = 0;
        float* const y_lds = reinterpret_cast<float*>(v_lds);
        while (bad != 0) {
            const int who = __ffs(bad) - 1;
            bad &= bad - 1;
            const float2 y = column_again<QT, V8>(
                c, seen, lane_int(col.own, who), lane_float(__float_as_int(m), who), t.row_lo + (t.col + who) / c.G,
                lane_int(col.head, who), 2 * count, y_lds, blocks);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
            y_lds[2 * lane] = y.x;
            y_lds[2 * lane + 1] = y.y;
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
            if (n == who) {
                lw = l;
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] = y_lds[32 * d + 8 * (i >> 2) + 4 * h + (i & 3)];
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
        }
    }
    if (status != 0) atomicOr(c.status, status);
    // ---- the waves' results meet
    __syncthreads();
    float* const result = reinterpret_cast<float*>(lds);
    {
        float* to = result + (size_t)(wv * kFewTile + n) * kRowWords;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4*>(to + 32 * d + 2 * i + 4 * h) = f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
        if (h == 0) *reinterpret_cast<f32x4*>(to + kHeadDim) = f32x4{m, l, lw, 0.0f};
    }
    __syncthreads();
    // (eight threads a column: of eight waves, four take the columns)
    const int k = tid >> 3, j = tid & 7;   // column, and which of its dims
    const bool there = k < kFewTile && t.col + k < t.rows * c.G;
    float M = -INFINITY, lsum = 0.0f, wsum = 0.0f;
    f32x4 y[4] = {};
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const float* from = result + (size_t)(w * kFewTile + k % kFewTile) * kRowWords;
        const f32x4 st = *reinterpret_cast<const f32x4*>(from + kHeadDim);
        const float mn = fmaxf(M, st[0]);
        const float fa = mn == -INFINITY ? 0.0f : hw_exp2(M - mn), fb = mn == -INFINITY ? 0.0f : hw_exp2(st[0] - mn);
        lsum = lsum * fa + st[1] * fb;
        wsum = wsum * fa + st[2] * fb;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = y[i] * fa + *reinterpret_cast<const f32x4*>(from + 4 * j + 32 * i) * fb;
        M = mn;
    }
    if (parts == 1) {
        const int g = t.col + k;
        if (there) write_column(c, t.row_lo + g / c.G, t.kv * c.G + g % c.G, j, y, M, lsum, wsum);
        return;
    }
    if (there) {
        float* to = part_of<kFewTile>(c, t, t.split) + (size_t)k * kPartWords;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            put2(to + 4 * j + 32 * i, y[i][0], y[i][1]);
            put2(to + 4 * j + 32 * i + 2, y[i][2], y[i][3]);
        }
        if (j == 0) {
            put2(to + kHeadDim, M, lsum);
            put2(to + kHeadDim + 2, wsum, 0.0f);
        }
    }
    join_parts<W, kFewTile>(c, t, parts, &sh_last);
}

template <int W, int TERMS>
const void* kernel_of(bool keys8, bool values8) {
    return keys8 ? (values8 ? reinterpret_cast<const void*>(&k_rows_few<W, TERMS, true, true>)
                            : reinterpret_cast<const void*>(&k_rows_few<W, TERMS, true, false>))
                 : (values8 ? reinterpret_cast<const void*>(&k_rows_few<W, TERMS, false, true>)
                            : reinterpret_cast<const void*>(&k_rows_few<W, TERMS, false, false>));
}

}  // namespace

RowsKernel few_kernel(bool all, bool exact, bool keys8, bool values8) {
    return all ? RowsKernel{exact ? kernel_of<8, 3>(keys8, values8) : kernel_of<8, 1>(keys8, values8), kFewTile, 512}
               : RowsKernel{exact ? kernel_of<4, 3>(keys8, values8) : kernel_of<4, 1>(keys8, values8), kFewTile, 256};
}

}  // namespace md
