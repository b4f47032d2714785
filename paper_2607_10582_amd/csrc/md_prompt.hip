// gfx950 kernel of the attention of ragged rows (a prompt, a chunk of one) over
// the paged cache, bf16 in and out; md_few.hip has the one for few rows and for
// float32.
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
// Keys and values lie in LDS in the order of the products' operands, 16 bytes a
// lane side by side, which leaves 9% of the LDS's cycles to bank conflicts (in the
// order of the pools they were 36%).
//
// What bounds it: the matrix cores, 4 d operations per column and token.  A
// large library product does as many operations in 84% of the time: a prompt of
// 16,384 rows (16 query heads on 2) takes 1.08 ms, 1,020 TFLOP/s.  Without the weights it would take 0.89 ms, without the loads
// 1.02.

#include <algorithm>
#include <type_traits>

#include "md_prompt.h"

namespace md {

namespace {

constexpr int kStep = 64;                  // tokens of a step: four blocks
constexpr int kStepBytes = kStep * kHeadDim * 2;

// A workgroup takes a tile of 32 columns for each of its W waves, which share
// the steps of 64 tokens through LDS: keys of two steps, values of three.
// QT: pages may hold 8-bit keys; V8: the values are 8-bit codes, which widen to
// bf16 on their way into LDS, their scales going to the weights.
template <int W, bool QT, bool V8>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(W / 4, W / 4))) k_rows_attend(PromptCall c) {
    constexpr int kThreads = 64 * W;
    constexpr int kCols = W * 32;
    constexpr int kPer = kStepBytes / (16 * kThreads);   // 16-byte loads of a thread for a step's keys
    __shared__ __align__(16) uint8_t kl[2][kStepBytes];
    __shared__ __align__(16) uint8_t vl[3][kStepBytes];
    __shared__ int scan_lds[2 * 17];
    __shared__ int range_lds[2][W];
    __shared__ int sh_last;
    extern __shared__ int pref[];   // [S + 1] tiles of the sessions before
    const int tid = threadIdx.x, lane = lane_id(), wv = uni(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    int status = 0;
    TileAt t;
    if (!find_tile<kThreads, kCols>(c, scan_lds, pref, t, status)) return;
    // ---- the wave's columns and their queries
    Column x_col = column_of(c, t, t.col + wv * 32 + n, status);
    const bool mine = x_col.mine;
    const int own = x_col.own;
    int smin = own >= 0 ? own : 0x7FFFFFFF, smax = own;
    u32x4 qf[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
        u32x4 w[1];
        query_terms<1>(c, x_col, kk, w);
        qf[kk] = w[0];
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
    for (int w = 1; w < W; ++w) {
        gmin = min(gmin, range_lds[0][w]);
        gmax = max(gmax, range_lds[1][w]);
    }
    gmin = uni(gmin);
    gmax = uni(gmax);
    const Seen seen = seen_of(c, gmin, gmax);
    const int win = seen.win;
    const int steps = (seen.n_blocks + 3) >> 2;
    const int share = share_of(t, seen.n_blocks) >> 2;
    const int parts = steps == 0 ? 1 : (steps + share - 1) / share;
    if (t.split >= parts) {
        if (status != 0) atomicOr(c.status, status);
        return;
    }
    const int begin = t.split * share, end = min(steps, begin + share);

    const size_t row_elems = ((size_t)c.layer * c.Hkv + t.kv) * c.P * kHeadDim;
    auto describe = [&](int base, int p) __attribute__((always_inline)) {
        return block_at<QT, V8>(c, t, seen, row_elems, base + lane, p, status);
    };
    auto of = [](int x, int i) { return __builtin_amdgcn_readlane(x, i); };
    // Lanes know of 16 steps: kLot of them to work on, and the three behind
    // these that are on their way into LDS.  A bit for each block that every
    // column of the wave sees in full, that lacks tokens, that holds 8-bit keys;
    // four of them are step i's.
    constexpr int kLot = 13;
    Block cur = begin < end ? describe(4 * begin, page_of(c, t, seen, 4 * begin + lane)) : Block{}, next = cur;
    int next_page = 0;
    uint64_t full, part, coded;
    auto look = [&]() __attribute__((always_inline)) {
        const int at = cur.at;
        full = __ballot((cur.live == 16) & (at + 15 <= smin) & ((at > smax - win) | (at + 15 < c.sinks)));
        part = __ballot(cur.live < 16);
        coded = QT ? __ballot(cur.coded != 0) : 0;
    };
    look();
    auto bits = [](uint64_t of_blocks, int i) { return (uint32_t)(of_blocks >> (4 * i)) & 15u; };

    // ---- a step's loads, and their way into LDS
    // a thread's piece x is 16 bytes of the block (x W + its wave) / 4 (codes: / 2)
    u32x4 rk[kPer], rv[V8 ? (kPer + 1) / 2 : kPer];
    constexpr int kVals = V8 ? (kPer + 1) / 2 : kPer;
    // Where the thread's pieces go, once for all steps (kept as they are: taken
    // apart into what does not change they would cost the loop its registers).
    // Keys in LDS: [half][8 dims pairs][32 tokens] 16 bytes; values: [block][d / 32]
    // [tokens 4h .. and 8+4h ..][32 dims] 16 bytes.
    constexpr int kApart = W / 4;   // blocks between a thread's pieces
    const int c16 = tid & 255, c8 = tid & 127;
    uint32_t from = 16 * c16, from8 = 16 * c8;
    uint32_t key_at = 512 * (c16 >> 4) + 16 * (c16 & 15) + 256 * (tid >> 8);
    uint32_t key8_at = 4096 * (c16 >> 6) + 512 * ((c16 >> 4) & 3) + 16 * (c16 & 15) + 256 * (tid >> 8);
    uint32_t value_at = 512 * ((tid >> 4) & 1) + 16 * (tid & 15) + 8 * ((tid >> 5) & 1) +
                        (V8 ? 2048 * (c8 >> 6) + 4096 * (tid >> 7) : 1024 * (c16 >> 6) + 4096 * (tid >> 8));
    asm volatile("" : "+v"(from), "+v"(from8), "+v"(key_at), "+v"(key8_at), "+v"(value_at));
    // Requests piece x of the lot's step i.
    auto tile_ptr = [&](const void* pool, int i, int b, int shift) __attribute__((always_inline)) {
        const uint64_t t = (uint64_t)(uint32_t)of((int)(uint32_t)cur.tile, 4 * i + b) |
                           ((uint64_t)(uint32_t)of((int)(cur.tile >> 32), 4 * i + b) << 32);
        return (gbytes)(reinterpret_cast<uint64_t>(pool) + (t << shift));
    };
    auto load_key = [&](int i, int x) __attribute__((always_inline)) {
        const int b = (x * W + wv) >> 2;   // (uniform)
        const bool codes = QT && ((bits(coded, i) >> b) & 1) != 0;
        rk[x] = *reinterpret_cast<gvec>(tile_ptr(c.k_pool, i, b, 1) + (codes ? from8 : from));
    };
    auto load_value = [&](int i, int x) __attribute__((always_inline)) {
        if constexpr (V8) rv[x] = *reinterpret_cast<gvec>(tile_ptr(c.v_codes, i, (x * W + wv) >> 1, 0) + from8);
        else rv[x] = *reinterpret_cast<gvec>(tile_ptr(c.v_pool, i, (x * W + wv) >> 2, 1) + from);
    };
    auto store_key = [&](int i, int x, uint8_t* kbuf) __attribute__((always_inline)) {
        const int b = (x * W + wv) >> 2;
        // (block kApart x + tid / 256)
        uint8_t* to = kbuf + (kApart == 2 ? 8192 * x : 8192 * (x >> 1) + 256 * (x & 1));
        if (QT && ((bits(coded, i) >> b) & 1) != 0) {
            // codes (a, g, t): dims 64 a + 8 g .. and 64 a + 32 + 8 g .. of token t
            if (c16 < 128) {
                *reinterpret_cast<u32x4*>(to + key8_at) = codes_to_bf16<0>(rk[x]);
                *reinterpret_cast<u32x4*>(to + key8_at + 2048) = codes_to_bf16<1>(rk[x]);
            }
        } else {
            *reinterpret_cast<u32x4*>(to + key_at) = rk[x];
        }
    };
    // (four tokens 4g .. of dims m and 16 + m, g = (tid / 16) % 4, m = tid % 16)
    auto put_values = [&](uint8_t* to, u32x2 a, u32x2 b) __attribute__((always_inline)) {
        *reinterpret_cast<u32x2*>(to) = a;
        *reinterpret_cast<u32x2*>(to + 256) = b;
    };
    auto store_value = [&](int i, int x, uint8_t* vbuf) __attribute__((always_inline)) {
        const int b = (x * W + wv) >> (V8 ? 1 : 2);
        // a slot without a token may hold anything, and 0 times an infinity
        // or NaN is NaN: its values become 0
        uint32_t m0 = 0xFFFFFFFFu, m1 = 0xFFFFFFFFu;
        if (__builtin_expect((bits(part, i) >> b) & 1, 0)) {
            const int k4 = of(cur.live, 4 * i + b) - 4 * ((tid >> 4) & 3);
            m0 = k4 >= 2 ? 0xFFFFFFFFu : k4 == 1 ? 0x0000FFFFu : 0u;
            m1 = k4 >= 4 ? 0xFFFFFFFFu : k4 == 3 ? 0x0000FFFFu : 0u;
        }
        uint8_t* to = vbuf + value_at + (V8 ? 4096 * (W / 2) : 4096 * kApart) * x;
        if constexpr (V8) {   // codes (a, g, m): words of dims 64 a + 16 i + m
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const uint32_t u = rv[x][2 * y], v = rv[x][2 * y + 1];
                put_values(to + 1024 * y, u32x2{codes_pair_to_bf16<false>(u) & m0, codes_pair_to_bf16<true>(u) & m1},
                           u32x2{codes_pair_to_bf16<false>(v) & m0, codes_pair_to_bf16<true>(v) & m1});
            }
        } else {
            put_values(to, u32x2{rv[x][0] & m0, rv[x][1] & m1}, u32x2{rv[x][2] & m0, rv[x][3] & m1});
        }
    };

    // (the sums that lse tells of, and those of the weights as the products get
    // them, by which a result is divided: rounding a weight then moves it between
    // values, and does not scale the result)
    float m = -INFINITY, l = 0.0f, lw = 0.0f;
    f32x16 o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    // ---- A step is two halves of 32 tokens.  While a half's logits become
    // weights, the matrix cores work on its neighbours: the sums of the half
    // before and the logits of the half behind, product by product between the
    // weights' instructions.  (A wave alone issues one of those in 7 cycles, not
    // 4.  A wave pair that took turns, one's products beside the other's weights,
    // took 1.13 ms for 16,384 rows and left no room for what follows.)
    f32x16 x[2];
    uint32_t pw[2][8];   // weights, two to a word: 4 b .. are those of the half's block b
    // Sixteen operands from LDS and their products, kAhead reads under way: left
    // to itself the compiler has each product wait for its own.
    auto stream = [&](auto count, auto&& read, auto&& product, auto&& beside) {
        constexpr int N = decltype(count)::value, kAhead = 4;
        u32x4 a[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) a[i] = read(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            product(i, __builtin_bit_cast(bf16x8, a[i % kAhead]));
            if (i + kAhead < N) a[i % kAhead] = read(i + kAhead);
            beside(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    using std::integral_constant;
    const uint8_t* const k_lane = kl[0] + 16 * lane;
    const uint8_t* const v_lane = vl[0] + 16 * lane;
    auto key_part = [&](int u, uint32_t buf, int kk) { return *reinterpret_cast<const u32x4*>(k_lane + buf + 8192 * u + 1024 * kk); };
    auto value_part = [&](int u, uint32_t buf, int i) { return *reinterpret_cast<const u32x4*>(v_lane + buf + 8192 * u + 1024 * i); };
    auto logit = [&](int u, int kk, bf16x8 a) {
        const f32x16 none = {};
        x[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, qf[kk]), kk == 0 ? none : x[u], 0, 0, 0);
    };
    auto sum = [&](int u, int i, bf16x8 a) {   // block i / 4, dims 32 (i % 4) ..
        const int b = i >> 2, d = i & 3;
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            a, __builtin_bit_cast(bf16x8, u32x4{pw[u][4 * b], pw[u][4 * b + 1], pw[u][4 * b + 2], pw[u][4 * b + 3]}), o[d], 0, 0, 0);
    };
    auto nothing = [](int) {};
    // 8-bit keys and values: the keys' scale goes to the logits, the values' to
    // the weights (through the exponent where those are rounded to bf16 anyway)
    // and out of their sums again.
    float sc[2], vs[2], rs[2], lg[2], shift[2];
    bool lost[2] = {false, false};   // values whose scale is not taken so
    float mx;
    // A half's scales, what its columns see of it and their maxima: whether one
    // has grown enough to be followed.  i: the step's place in the lot.
    auto peak = [&](int u, int i) __attribute__((always_inline)) {
        const int i0 = 4 * i + 2 * u;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            sc[b] = kLogitScale;
            if constexpr (QT) {
                const float ks = __uint_as_float(of(cur.ks, i0 + b));
                if (__builtin_expect(ks > 0.0f && ks < INFINITY, 1)) {
                    sc[b] *= ks;
                } else {   // (no factor for the -infinity of a token that is not seen)
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[u][8 * b + k] *= ks;
                }
            }
            if constexpr (V8) {
                vs[b] = __uint_as_float(of(cur.vs, i0 + b));
                if (vs[b] == 0.0f) vs[b] = 1.0f;   // (all its values are 0)
                lost[b] = !scale_fits(vs[b]);
                if (lost[b]) vs[b] = 1.0f;
                rs[b] = __builtin_amdgcn_rcpf(vs[b]);
                lg[b] = log2f(vs[b]);
            }
        }
        if (__builtin_expect(((full >> i0) & 3) != 3, 0)) {
            int h4 = 4 * h, own_here = own;
            asm volatile("" : "+v"(h4), "+v"(own_here));   // (or the loop would carry 16 registers of what follows)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int at = of(cur.at, i0 + b), live = of(cur.live, i0 + b);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int t = 8 * (k >> 2) + h4 + (k & 3);
                    const bool sees = (t < live) & (at + t <= own_here) & ((at + t > own_here - win) | (at + t < c.sinks));
                    x[u][8 * b + k] = sees ? x[u][8 * b + k] : -INFINITY;
                }
            }
        }
        float mb[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const float y = fmaxf(fmaxf(x[u][8 * b], x[u][8 * b + 1]), x[u][8 * b + 2]);
            const float z = fmaxf(fmaxf(x[u][8 * b + 3], x[u][8 * b + 4]), x[u][8 * b + 5]);
            mb[b] = fmaxf(fmaxf(y, z), fmaxf(x[u][8 * b + 6], x[u][8 * b + 7]));
        }
        mx = max_halves(QT ? fmaxf(mb[0] * sc[0], mb[1] * sc[1]) : fmaxf(mb[0], mb[1]) * kLogitScale);
        return __any(mx > m + kSlack || (m == -INFINITY && mx > -INFINITY)) != 0;
    };
    // Follows the maxima, in whole steps: what was weighed before (the sums, and
    // the half before this one's weights, whose sums come later) moves by a
    // power of two, without a rounding.
    auto follow = [&](int last) __attribute__((always_inline)) {
        const float mn = fmaxf(m, ceilf(mx));
        const float f = mn == -INFINITY ? 1.0f : ldexpf(1.0f, (int)fmaxf(m - mn, -300.0f));
        l *= f;
        lw *= f;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= f;
#pragma unroll
        for (int k = 0; k < 8; ++k) pw[last][k] = pack_bf16(bf16_lo(pw[last][k]) * f, bf16_hi(pw[last][k]) * f);
        m = mn;
    };
    // The half's weights, pair by pair: begun, and a pair later finished.
    float p, q, all_sum, w_sum;
    auto finish = [&](int u, int k) __attribute__((always_inline)) {
        const int b = k >> 2;
        if ((k & 3) == 0) all_sum = w_sum = 0.0f;
        all_sum += p + q;
        uint32_t w = pack_bf16(p, q);
        asm volatile("" : "+v"(w));
        pw[u][k] = w;
        w_sum = add_pair(w, w_sum);
        if ((k & 3) != 3) return;
        if constexpr (V8) {
            l = fmaf(all_sum, rs[b], l);
            lw = fmaf(w_sum, rs[b], lw);
            if (lost[b] && all_sum > 0.0f) lw = __uint_as_float(0x7FC00000u);   // (settled at the end)
        } else {
            l += all_sum;
            lw += w_sum;
        }
    };
    auto pair = [&](int u, int k) __attribute__((always_inline)) {
        const int b = k >> 2;
        float y = hw_exp2(fmaf(x[u][2 * k], sc[b], shift[b])), z = hw_exp2(fmaf(x[u][2 * k + 1], sc[b], shift[b]));
        asm volatile("" : "+v"(y), "+v"(z));   // (here, between these products, not where they are used)
        if (k > 0) finish(u, k - 1);
        p = y;
        q = z;
    };
    constexpr int kPeak = 3;   // the product beside which a half's maxima are looked at
    // One half: its weights, beside the logits of the half behind it and the sums
    // of the one before it, both the other half of a step in LDS.  A half that no
    // column sees gets weights of 0 (two ways through here would keep the sums
    // in two places).
    auto half = [&](auto which, int i, uint32_t k_buf, uint32_t v_buf, auto&& beside) __attribute__((always_inline)) {
        constexpr int u = decltype(which)::value;
        // The sums come first: they need nothing of this half, whose logits are
        // the products just begun.  Its maxima are looked at beside them (moving
        // sums and weights by the same power of two is right between any two of
        // them), its eight pairs of weights spread over what is left.
        stream(integral_constant<int, 16>{},
               [&](int j) { return j < 8 ? value_part(1 - u, v_buf, j) : key_part(1 - u, k_buf, j - 8); },
               [&](int j, bf16x8 a) {
                   if (j < 8) sum(1 - u, j, a); else logit(1 - u, j - 8, a);
               },
               [&](int j) {
                   if (j == kPeak) {
                       if (__builtin_expect(peak(u, i), 0)) follow(1 - u);
                       const float ms = m == -INFINITY ? 0.0f : m;
#pragma unroll
                       for (int b = 0; b < 2; ++b) shift[b] = V8 ? lg[b] - ms : -ms;
                   }
                   constexpr int kLeft = 15 - kPeak;   // slots behind it
#pragma unroll
                   for (int k = 0; k < 8; ++k)
                       if (j == kPeak + 1 + k * kLeft / 8) pair(u, k);
                   if (!(j & 1)) beside(j >> 1);
               });
        finish(u, 7);
    };
    if (begin < end) {
        const int count = end - begin;
        auto load_keys = [&](int i) {
#pragma unroll
            for (int x = 0; x < kPer; ++x) load_key(i, x);
        };
        auto load_values = [&](int i) {
#pragma unroll
            for (int x = 0; x < kVals; ++x) load_value(i, x);
        };
        auto store_keys = [&](int i, uint32_t buf) {
#pragma unroll
            for (int x = 0; x < kPer; ++x) store_key(i, x, kl[0] + buf);
        };
        auto store_values = [&](int i, uint32_t buf) {
#pragma unroll
            for (int x = 0; x < kVals; ++x) store_value(i, x, vl[0] + buf);
        };
        // (behind the last step: page 0, which nobody looks at)
        load_keys(0);
        load_values(0);
        store_keys(0, 0);
        store_values(0, 0);
        load_keys(1);
        load_values(1);
        store_keys(1, kStepBytes);
        load_keys(2);
        lds_sync();
        // the step's keys; the values of the step before (weights of 0 at first, of
        // anything that was written), its own, and where the next one's go
        uint32_t k_now = 0, v_last = 0, v_now = 0, v_new = kStepBytes;
        auto turn = [&](int at, int& i) __attribute__((always_inline)) {
            if (__builtin_expect(i == kLot / 2 - 3, 0)) next_page = page_of(c, t, seen, 4 * (begin + at - i + kLot) + lane);   // in good time
            if (__builtin_expect(i == kLot / 2, 0)) next = describe(4 * (begin + at - i + kLot), next_page);
            if (__builtin_expect(i == kLot - 1, 0)) {
                cur = next;
                look();
                i = -1;
            }
            k_now = kStepBytes - k_now;
            v_last = v_now;
            v_now = v_new;
            v_new = v_new == 2 * kStepBytes ? 0 : v_new + kStepBytes;
        };
        if (smax >= 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) pw[1][k] = 0u;
            stream(integral_constant<int, 8>{}, [&](int j) { return key_part(0, 0, j); }, [&](int j, bf16x8 a) { logit(0, j, a); },
                   nothing);
            // A piece of the caches' bytes goes to LDS and the same one of the step
            // behind is requested a whole step before it goes: keys beside one half,
            // values beside the other (1.11 ms; all behind a half, 1.14).
            auto pieces = [](int k, int n, auto&& put, auto&& get) {
#pragma unroll
                for (int x = 0; x < n; ++x) {
                    if (k == (4 / n) * x) put(x);
                    if (k == 4 + (4 / n) * x) get(x);
                }
            };
            // Of a SIMD's two waves the older one goes first wherever both could,
            // and would wait for the other at every step's end: each gets one half
            // of the step to go first in (1.084 ms for 16,384 rows, 1.108 without).
            const bool younger = wv >= W / 2;
            auto go_first = [&](bool mine_now) __attribute__((always_inline)) {
                if (mine_now) __builtin_amdgcn_s_setprio(1); else __builtin_amdgcn_s_setprio(0);
            };
            for (int at = 0, i = 0; at < count; ++at, ++i) {   // i: the step's place in the lot
                go_first(!younger);
                half(integral_constant<int, 0>{}, i, k_now, v_last, [&](int k) {
                    pieces(k, kVals, [&](int x) { store_value(i + 1, x, vl[0] + v_new); }, [&](int x) { load_value(i + 2, x); });
                });
                lds_sync();   // (what all waves have read makes room)
                go_first(younger);
                half(integral_constant<int, 1>{}, i, kStepBytes - k_now, v_now, [&](int k) {
                    pieces(k, kPer, [&](int x) { store_key(i + 2, x, kl[0] + k_now); }, [&](int x) { load_key(i + 3, x); });
                });
                turn(at, i);
            }
            stream(integral_constant<int, 8>{}, [&](int j) { return value_part(1, v_last, j); },
                   [&](int j, bf16x8 a) { sum(1, j, a); }, nothing);
        } else {   // a wave without a column that sees anything helps with the loads
            for (int at = 0, i = 0; at < count; ++at, ++i) {
                store_values(i + 1, v_new);
                load_values(i + 2);
                lds_sync();
                store_keys(i + 2, k_now);
                load_keys(i + 3);
                turn(at, i);
            }
        }
        __syncthreads();
    }
    {   // (worked out again, not kept through the loop)
        int again = t.col + wv * 32 + n;
        asm volatile("" : "+v"(again));
        x_col.row = t.row_lo + (mine ? again / c.G : 0);
        x_col.head = t.kv * c.G + (mine ? again % c.G : 0);
    }
    const int64_t row = x_col.row;
    const int head = x_col.head;
    l = add_halves(l);
    lw = add_halves(lw);
    // A column without a row, or whose row's slot is not there, saw what its
    // neighbours see in full all the same; it has nothing.
    if (own < 0) {
        m = -INFINITY;
        l = lw = 0.0f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    }
    // ---- Columns with a finite sum and a result that is not: a value that is
    // not finite reached them unseen (here, where it costs nothing else)
    {
        float z = lw * 0.0f;   // NaN unless everything is finite
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) z = fmaf(o[d][i], 0.0f, z);
        z = add_halves(z);
        uint32_t bad = (uint32_t)__ballot(own >= 0 && l * 0.0f == 0.0f && z != 0.0f);
        auto blocks = [&](int i) __attribute__((always_inline)) {
            return describe(4 * begin + i, page_of(c, t, seen, 4 * begin + i + lane));
        };
        const int count = min(seen.n_blocks, 4 * end) - 4 * begin;
        if (bad != 0 && !reached_unseen<V8>(c, seen, smin, smax, count, blocks)) bad = 0;
        float* const y_lds = reinterpret_cast<float*>(kl[0]) + kAgainWords * wv;
        while (bad != 0) {
            const int who = __ffs(bad) - 1;
            bad &= bad - 1;
            const float2 y = column_again<QT, V8>(
                c, seen, of(own, who), lane_float(__float_as_int(m), who), t.row_lo + (t.col + wv * 32 + who) / c.G,
                of(head, who), count, y_lds, blocks);
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
    // ---- register i of o[d]: dim 32 d + 8 (i / 4) + 4 h + i % 4
    auto write4 = [&](int dim, f32x4 y) {
        const int64_t at = row * c.out_stride + head * kHeadDim + dim;
        if (c.out_bf16)
            *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(c.out) + at) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
        else
            *reinterpret_cast<f32x4*>(static_cast<float*>(c.out) + at) = y;
    };
    if (parts == 1) {
        if (!mine) return;
        const float inv = inverse(lw);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) write4(32 * d + 2 * i + 4 * h, f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]} * inv);
        if (c.lse != nullptr && h == 0) c.lse[row * c.Hq + head] = log_sum(m, l);
        return;
    }
    if (mine) {
        float* to = part_of<kCols>(c, t, t.split) + (size_t)(wv * 32 + n) * kPartWords;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 2) put2(to + 32 * d + 8 * (i >> 2) + 4 * h + (i & 3), o[d][i], o[d][i + 1]);
        if (h == 0) {
            put2(to + kHeadDim, m, l);
            put2(to + kHeadDim + 2, lw, 0.0f);
        }
    }
    join_parts<W, kCols>(c, t, parts, &sh_last);
}

template <int W>
const void* kernel_of(bool keys8, bool values8) {
    return keys8 ? (values8 ? reinterpret_cast<const void*>(&k_rows_attend<W, true, true>)
                            : reinterpret_cast<const void*>(&k_rows_attend<W, true, false>))
                 : (values8 ? reinterpret_cast<const void*>(&k_rows_attend<W, false, true>)
                            : reinterpret_cast<const void*>(&k_rows_attend<W, false, false>));
}

constexpr int kWideWaves = 8;                // of a workgroup, one a CU
constexpr int kWideCols = kWideWaves * 32;   // columns of its tile
// Columns a session up to which the narrow kernel is taken.  Both, in us:
//   columns                                        32      96      128-144    256-288
//   8 sessions of 16,384 - 32,768, 2 KV heads   46 / 56  63 / 74   86 / 99   130 / 142
//   16 of 2,048 - 8,192, 8 KV heads             78 / 114 114 / 121 131 / 124 199 / 228
//   the same with 8-bit values                  55 / 125 102 / 136 119 / 140 191 / 253
//   64 of 300 - 1,500, 8 KV heads               47 / 75  71 / 79   90 / 83   166 / 119
// One session is few tiles for the wide kernel, and up to 2,048 columns go to the
// narrow one: 1 of 16,384 tokens, 2 KV heads, 384 columns 32 / 106, 1,536 68 / 104,
// 6,144 200 / 156; 8,192 tokens, 8 KV heads, 2,048 columns 111 / 118,
// 8,192 384 / 284.  (Only the device knows the rows of each session: a long prompt
// beside many sessions without a row is taken for few rows of each, 942 for 700
// us with 8,192 rows of it.)  Between 144 and 288 columns a session the narrow
// kernel still is the faster one in three of the four, and by far the slower one
// in the fourth, of many short sessions: the limit is where that one turns.
constexpr int kFewCols = 128, kFewAll = 2048;
// Parts that the tiles of a call may come to, and their arrivals' words.
int most_parts(int n_cu) { return n_cu * (kWideCols / kFewTile); }
size_t count_words(int n_cu) { return ((size_t)most_parts(n_cu) + 63) / 64 * 64; }

}  // namespace

uint64_t rows_workspace(const Dims&, int n_cu) {
    return (count_words(n_cu) + (uint64_t)n_cu * kWideCols * kPartWords) * sizeof(float);
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
    const bool keys8 = dm.quant != 0, values8 = a.values.v_pool == nullptr;
    // Few columns a session (on average: only the device knows the rows of each)
    // are read past, many share what is in LDS.
    const int with_rows = std::min(dm.S, a.rows.n_rows);
    const bool few = exact || (int64_t)a.rows.n_rows * dm.G <= std::max<int64_t>((int64_t)kFewCols * with_rows, kFewAll);
    // the most tiles that rows can make, however they are spread over the sessions
    const int64_t tiles = (int64_t)a.rows.n_rows * dm.G / (few ? kFewTile : kWideCols) + with_rows;
    const bool all = 2 * tiles * dm.Hkv <= n_cu;
    const RowsKernel k = few ? few_kernel(all, exact, keys8, values8)
                             : RowsKernel{kernel_of<kWideWaves>(keys8, values8), kWideCols, 64 * kWideWaves};
    // Parts that are all on the card at once: one of eight waves a CU, or two of
    // four of the narrow kernel, where tiles fill half the card and the next one's
    // beginning hides behind another.  (5 rows over 8 sessions, 2 KV heads: 48 us
    // with eight, whose parts are half as many to join, 55 with four.)  Tiles that
    // fill the card three times over are balanced as they are.
    c.units = few ? (tiles * dm.Hkv < 6 * n_cu ? (all ? 1 : 2) * n_cu : 0) : tiles * dm.Hkv < n_cu ? n_cu : 0;
    c.least_units = few ? c.units / 2 : 0;
    c.count = static_cast<int32_t*>(a.workspace);
    c.part = static_cast<float*>(a.workspace) + count_words(n_cu);
    void* args[] = {&c};
    return hipLaunchKernel(k.fn, dim3(grid_of(tiles + c.units / dm.Hkv, dm.Hkv)), dim3((unsigned)k.threads), args,
                           (size_t)(dm.S + 1) * sizeof(int), st);
}

}  // namespace md
