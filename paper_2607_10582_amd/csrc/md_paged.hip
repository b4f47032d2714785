// gfx950 kernels of the attention of one new token over the paged cache.
//
//   out_h = sum_i softmax_i(q_h . k_i / sqrt(d)) v_i
//
// in one pass over a row (session, KV head): a wave keeps the running maximum
// m and sum l of its tokens' weights 2^(x - m) for the group's up to 16 query
// heads and scales its sums of weighted values down when the maximum grows.
// A row is split over its length into parts; their (m, l, sums) are joined as
// sum_p 2^(m_p - M) sums_p / sum_p 2^(m_p - M) l_p.
//
// Both products run on the matrix cores, transposed so that a lane keeps to
// one query head throughout (h = lane & 15, g = lane >> 4):
//   logits  [token][head] = K [16 tokens][128] q^T:  lane (h, g) gets tokens 4g .. 4g+3
//   sums    [dim][head]  += V^T [16 dims][32 tokens] P^T: lane (h, g) feeds the
//           weights of tokens 4g .. 4g+3 of two tiles, the very ones it got,
//           so the weights never leave their registers
// The value pool's layout holds, for lane (m, g), the four tokens 4g .. 4g+3 of
// dims 32 b + m and 32 b + 16 + m in 16 consecutive bytes, 64 lanes 1 KiB.
//
// What bounds it: the bytes of keys and values (G flops per byte); a call of a
// few hundred tokens by its chain of loads (counters, page table, keys).

#include <algorithm>

#include "md_arrive.h"
#include "md_decode.h"
#include "md_device.h"

namespace md {

namespace {

constexpr int kTokWaves = 4;
constexpr int kTokThreads = 64 * kTokWaves;
constexpr int kMinUnitSteps = kTokWaves;   // a step is two tiles of 16 tokens, whose values meet in one product of 32
constexpr int kJoin = 16;          // partial results that one workgroup joins

struct Desc {       // one 16-token tile, per lane
    int phys;       // page
    int live;       // tokens of it that count, 0 .. 16; -1: the new token
    int quant;      // its keys are 8-bit codes
};

struct Row {
    int s, kv, np, nt;   // session, KV head, pages and slots in use
    int tiles;           // 16-token tiles to walk
    bool ok;             // the session's counters are consistent
};

// Leading tokens among 16 slots' region codes (holes follow a page's last token).
__device__ __forceinline__ int tokens_before_holes(const uint8_t* region) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(region);
    int n = 0;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
        const uint32_t x = w[i];
#pragma unroll
        for (int b = 3; b >= 0; --b)
            if (((x >> (8 * b)) & 0xFFu) != (uint32_t)kHole) n = max(n, 4 * i + b + 1);
    }
    return n;
}

// Tile u of step t of a row: two tiles of its pages a step, then a step for
// the new token.
template <bool SPARSE, bool QT>
__device__ __forceinline__ Desc tile_desc(const Dims& dm, const View& v, const TokenCall& c, const Row& r, int step, int u,
                                          int& status) {
    Desc d{0, 0, 0};
    const int t = 2 * step + u;
    if (t >= r.tiles) {
        if (r.ok && c.new_k != nullptr && u == 0 && step == (r.tiles + 1) >> 1) d.live = -1;
        return d;
    }
    const int per = dm.P >> 4;
    int page = t >> (dm.Pshift - 4);
    const int sub = t & (per - 1);
    if constexpr (SPARSE) {
        const int32_t* list = c.blocks + ((size_t)r.s * dm.Hkv + r.kv) * c.max_blocks;
        const int o = page;
        page = list[o];
        if (page < 0 || page >= r.np || (o > 0 && page <= list[o - 1])) {
            status |= MD_DEV_BAD_BLOCK;
            return d;
        }
    }
    const int p = v.page_table[(size_t)r.s * dm.MP + page];
    if ((unsigned)p >= (unsigned)dm.NP) {
        status |= kDevCorrupt;
        return d;
    }
    d.phys = p;
    d.live = min(16, max(0, r.nt - (page * dm.P + 16 * sub)));
    if (dm.aligned) d.live = min(d.live, tokens_before_holes(v.region + (size_t)p * dm.P + 16 * sub));
    if constexpr (QT) d.quant = v.page_format[p];
    return d;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((__vector_size__(4)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

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

// A thread's share of a row's result: eight dims of one query head, 16
// threads a head.
struct Share {
    float m, l, y[8];
};

__device__ __forceinline__ float* part_at(const Dims& dm, const TokenCall& c, int unit, int slot, int hh) {
    return c.part + ((size_t)(2 * unit + slot) * dm.G + hh) * kPartWords;
}

__device__ __forceinline__ void part_store(float* p, int e8, const Share& r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) put2(p + 8 * e8 + 2 * i, r.y[2 * i], r.y[2 * i + 1]);
    if (e8 == 0) put2(p + kHeadDim, r.m, r.l);
}

__device__ __forceinline__ Share part_load(const float* p, int e8) {
    Share r;
    const float2 st = get2(p + kHeadDim);
    r.m = st.x;
    r.l = st.y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 w = get2(p + 8 * e8 + 2 * i);
        r.y[2 * i] = w.x;
        r.y[2 * i + 1] = w.y;
    }
    return r;
}

__device__ __forceinline__ void share_add(Share& a, const Share& b) {
    const float M = fmaxf(a.m, b.m);
    const float fa = M == -INFINITY ? 0.0f : hw_exp2(a.m - M), fb = M == -INFINITY ? 0.0f : hw_exp2(b.m - M);
    a.m = M;
    a.l = a.l * fa + b.l * fb;
#pragma unroll
    for (int i = 0; i < 8; ++i) a.y[i] = fmaf(b.y[i], fb, a.y[i] * fa);
}

__device__ __forceinline__ void write_out(const Dims& dm, const TokenCall& c, const Row& r, int hh, int e8, const Share& a) {
    const float inv = a.l > 0.0f ? 1.0f / a.l : a.l == 0.0f ? 0.0f : a.l;   // NaN stays NaN
    const int64_t at = (int64_t)r.s * c.out_stride + (r.kv * dm.G + hh) * kHeadDim + 8 * e8;
    if (c.out_bf16) {
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(c.out) + at) =
            u32x4{pack_bf16(a.y[0] * inv, a.y[1] * inv), pack_bf16(a.y[2] * inv, a.y[3] * inv),
                  pack_bf16(a.y[4] * inv, a.y[5] * inv), pack_bf16(a.y[6] * inv, a.y[7] * inv)};
    } else {
        f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(c.out) + at);
        o[0] = f32x4{a.y[0] * inv, a.y[1] * inv, a.y[2] * inv, a.y[3] * inv};
        o[1] = f32x4{a.y[4] * inv, a.y[5] * inv, a.y[6] * inv, a.y[7] * inv};
    }
    if (c.lse != nullptr && e8 == 0)
        c.lse[(size_t)r.s * dm.Hq + r.kv * dm.G + hh] = (a.m + log2f(a.l)) * 0.69314718055994530942f;
}

// The rows lie end to end on a line of steps of 32 tokens (sessions in order,
// each session's KV heads one after another), and a unit, one workgroup, takes
// an equal stretch of it, whatever the sessions' lengths: the whole of some
// rows and parts of at most two.  A row in several units is joined by the
// unit that finishes last: in groups of kJoin units by the last of each
// group, then the groups by the last of those (arrivals, no waits).
//
// Within a stretch of one row the four waves take steps in turn.  The keys of
// a wave's next step are requested as soon as this step's have been through
// the matrix cores, its values after this step's, so about 12 KiB per wave
// are under way at any time.  SPARSE: pages from the call's lists; QT: pages
// may hold 8-bit codes.
template <bool SPARSE, bool QT>
__global__ void __launch_bounds__(kTokThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
k_token(Dims dm, View v, Scratch sc, TokenCall c) {
    __shared__ __align__(16) u32x4 q_lds[3][4][64];
    __shared__ __align__(16) f32x4 acc_lds[kTokWaves][8][64];
    __shared__ float2 stat_lds[kTokWaves][16];
    __shared__ int pref[kMaxSessions + 1];
    __shared__ int scan_lds[17];
    __shared__ int sh_last;
    const int tid = threadIdx.x, lane = lane_id(), wv = tid >> 6;
    const int h = lane & 15, g = lane >> 4;
    const int per = dm.P >> 4;
    int status = 0;
    // ---- the line: steps of each session's rows
    {
        int before = 0;
        for (int b = 0; b < dm.S; b += kTokThreads) {
            const int s = b + tid;
            int n = 0;
            if (s < dm.S) {
                const int np = v.n_pages[s], nt = v.n_tokens[s];
                const bool ok = counters_ok(np, nt, dm);
                if (!ok) status = kDevCorrupt;
                const int tiles = !ok ? 0 : SPARSE ? min(c.max_blocks, np) * per : (nt + 15) >> 4;
                n = max(1, ((tiles + 1) >> 1) + (c.new_k != nullptr && ok ? 1 : 0));
            }
            int total;
            const int ex = block_exclusive_scan(n, scan_lds, &total);
            if (s < dm.S) pref[s] = before + ex;
            before += total;
        }
        if (tid == 0) pref[dm.S] = before;
        __syncthreads();
    }
    const int64_t T = (int64_t)pref[dm.S] * dm.Hkv;
    const int64_t per_unit = max((int64_t)kMinUnitSteps, (T + c.units - 1) / c.units);
    const int unit = blockIdx.x;
    int64_t pos = per_unit * unit;
    const int64_t end = min(T, pos + per_unit);
    if (unit != 0) status = 0;   // one unit reports the counters

    const size_t page_elems = (size_t)dm.LHkv * dm.P * kHeadDim;
    const int hh = tid >> 4, e8 = tid & 15;   // this thread's share of a result
    while (pos < end) {
        // ---- the row at pos and the stretch of it that this unit walks
        Row r;
        r.s = find_session(pref, dm.S, (int)(pos / dm.Hkv));
        const int steps = pref[r.s + 1] - pref[r.s];
        const int64_t at_s = (int64_t)pref[r.s] * dm.Hkv;
        r.kv = (int)((pos - at_s) / steps);
        const int64_t row0 = at_s + (int64_t)r.kv * steps;
        const int lo = (int)(pos - row0), hi = (int)min((int64_t)steps, end - row0);
        r.np = v.n_pages[r.s];
        r.nt = v.n_tokens[r.s];
        r.ok = counters_ok(r.np, r.nt, dm);
        if (!r.ok) r.np = r.nt = 0;
        r.tiles = (r.nt + 15) >> 4;
        if constexpr (SPARSE) {
            const int most = min(c.max_blocks, r.np);
            int n = c.block_count[(size_t)r.s * dm.Hkv + r.kv];
            if (n < 0 || n > most) {
                status |= MD_DEV_BAD_BLOCK;
                n = min(max(n, 0), most);
            }
            r.tiles = n * per;
        }
        // ---- the heads' queries: three bf16 terms, exactly; wave j has dims 32 j + 8 g ..
        f32x4 qa[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
        if (h < dm.G) {
            const f32x4* qp = reinterpret_cast<const f32x4*>(c.q + (int64_t)r.s * c.q_stride +
                                                             (r.kv * dm.G + h) * kHeadDim + 32 * wv + 8 * g);
            qa[0] = qp[0];
            qa[1] = qp[1];
        }
        const size_t tile_row = ((size_t)c.layer * dm.Hkv + r.kv) * dm.P * kHeadDim;   // elements into a page
        const int nw = max(0, (hi - lo - wv + kTokWaves - 1) / kTokWaves);   // this wave's steps: lo + wv + 4 i
        float m = -INFINITY, l = 0.0f;
        f32x4 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

        // descriptors of this wave's steps i .. i + 31: lane 2 k + u holds tile u of the k-th
        Desc d;
        auto describe = [&](int i) {
            const int mine = lo + wv + (i + (lane >> 1)) * kTokWaves;
            d = Desc{0, 0, 0};
            if (mine < hi) d = tile_desc<SPARSE, QT>(dm, v, c, r, mine, lane & 1, status);
        };
        u32x4 kt[2][4], vt[2][4];
        auto elem_at = [&](int i, int u) {
            const int phys = __builtin_amdgcn_readlane(d.phys, 2 * (i & 31) + u);
            const int t = 2 * (lo + wv + i * kTokWaves) + u;
            return (size_t)phys * page_elems + tile_row + (size_t)(t & (per - 1)) * 16 * kHeadDim;
        };
        auto load_k = [&](int i) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t* kp = reinterpret_cast<const uint8_t*>(v.k_pool + elem_at(i, u));
                const bool codes = QT && __builtin_amdgcn_readlane(d.quant, 2 * (i & 31) + u) != 0;
#pragma unroll
                for (int j = 0; j < 4; ++j)   // codes fill two loads; their scale sits at byte 2048
                    kt[u][j] = *reinterpret_cast<const u32x4*>(kp + (QT && j >= 2 && codes ? 2048 : 1024 * j + 16 * lane));
            }
        };
        auto load_v = [&](int i) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4* vp = reinterpret_cast<const u32x4*>(c.v_pool + elem_at(i, u)) + lane;
#pragma unroll
                for (int j = 0; j < 4; ++j) vt[u][j] = vp[64 * j];
            }
        };
        if (nw > 0) {
            describe(0);
            load_k(0);
            load_v(0);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t a[3], b[3];
                split3(qa[i >> 1][2 * (i & 1)], a[0], a[1], a[2]);
                split3(qa[i >> 1][2 * (i & 1) + 1], b[0], b[1], b[2]);
                w[i] = a[k] | (b[k] << 16);
            }
            q_lds[k][wv][lane] = w;
        }
        lds_sync();
        for (int i = 0; i < nw; ++i) {
            int live[2];
            float qsc[2] = {1.0f, 1.0f};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                live[u] = __builtin_amdgcn_readlane(d.live, 2 * (i & 31) + u);
                if constexpr (QT) {
                    if (__builtin_amdgcn_readlane(d.quant, 2 * (i & 31) + u)) {
                        qsc[u] = __uint_as_float(__builtin_amdgcn_readfirstlane(kt[u][2][0]));
                        kt[u][3] = codes_to_bf16<1>(kt[u][1]);
                        kt[u][2] = codes_to_bf16<0>(kt[u][1]);
                        kt[u][1] = codes_to_bf16<1>(kt[u][0]);
                        kt[u][0] = codes_to_bf16<0>(kt[u][0]);
                    }
                }
            }
            if (live[0] < 0) {   // the new token: every lane reads its dims, the other tokens count nothing
                const uint16_t* nk = c.new_k + (int64_t)r.s * c.kv_stride + r.kv * kHeadDim;
                const uint16_t* nv = c.new_v + (int64_t)r.s * c.kv_stride + r.kv * kHeadDim;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    kt[0][j] = *reinterpret_cast<const u32x4*>(nk + 32 * j + 8 * g);
                    vt[0][j] = u32x4{nv[32 * j + h], 0u, nv[32 * j + 16 + h], 0u};
                }
                live[0] = 1;
            }
            f32x4 x[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    const bf16x8 bq = __builtin_bit_cast(bf16x8, q_lds[k][j][lane]);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
                        x[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kt[u][j]), bq, x[u], 0, 0, 0);
                }
            if (i + 1 < nw) {
                if (((i + 1) & 31) == 0) describe(i + 1);
                load_k(i + 1);
            }
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    x[u][k] = 4 * g + k < live[u] ? x[u][k] * (QT ? kLogitScale * qsc[u] : kLogitScale) : -INFINITY;
                    mx = fmaxf(mx, x[u][k]);
                }
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            if (__any(mx > m)) {
                const float mn = fmaxf(m, mx);
                const float f = mn == -INFINITY ? 1.0f : hw_exp2(m - mn);
                l *= f;
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] *= f;
                m = mn;
            }
            const float ms = m == -INFINITY ? 0.0f : m;
            uint32_t ph[4], pl[4];   // weights as two bf16 terms
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float p[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    p[k] = hw_exp2(x[u][k] - ms);
                    l += p[k];
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t w = pack_bf16(p[2 * k], p[2 * k + 1]);
                    ph[2 * u + k] = w;
                    pl[2 * u + k] = pack_bf16(p[2 * k] - bf16_lo(w), p[2 * k + 1] - bf16_hi(w));
                }
                // a slot that does not count may hold anything, and 0 times
                // an infinity or NaN is NaN: its values become 0
                if (live[u] < 16) {
                    const int k4 = live[u] - 4 * g;   // tokens of this lane's four that count
                    const uint32_t m0 = k4 >= 2 ? 0xFFFFFFFFu : k4 == 1 ? 0x0000FFFFu : 0u;
                    const uint32_t m1 = k4 >= 4 ? 0xFFFFFFFFu : k4 == 3 ? 0x0000FFFFu : 0u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) vt[u][j] = vt[u][j] & u32x4{m0, m1, m0, m1};
                }
            }
            const bf16x8 bh = __builtin_bit_cast(bf16x8, u32x4{ph[0], ph[1], ph[2], ph[3]});
            const bf16x8 bl = __builtin_bit_cast(bf16x8, u32x4{pl[0], pl[1], pl[2], pl[3]});
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const bf16x8 a = __builtin_bit_cast(
                        bf16x8, u32x4{vt[0][j][2 * e], vt[0][j][2 * e + 1], vt[1][j][2 * e], vt[1][j][2 * e + 1]});
                    o[2 * j + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bh, o[2 * j + e], 0, 0, 0);
                    o[2 * j + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bl, o[2 * j + e], 0, 0, 0);
                }
            if (i + 1 < nw) load_v(i + 1);
        }
        // ---- the waves' results meet
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) stat_lds[wv][h] = make_float2(m, l);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc_lds[wv][i][lane] = o[i];
        lds_sync();
        Share mine{-INFINITY, 0.0f, {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int w = 0; w < kTokWaves; ++w) {
            const float2 st = stat_lds[w][hh];
            Share b{st.x, st.y, {}};
            // dim 8 e8 + i: tile e8 / 2, rows 8 (e8 & 1) + i, lane group (row / 4)
#pragma unroll
            for (int q4 = 0; q4 < 2; ++q4) {
                const f32x4 a = acc_lds[w][e8 >> 1][(2 * (e8 & 1) + q4) * 16 + hh];
#pragma unroll
                for (int i = 0; i < 4; ++i) b.y[4 * q4 + i] = a[i];
            }
            share_add(mine, b);
        }
        pos = row0 + hi;
        // ---- the row's other units
        const int first = (int)(row0 / per_unit), last = (int)((row0 + steps - 1) / per_unit);
        if (first == last) {
            if (hh < dm.G) write_out(dm, c, r, hh, e8, mine);
            lds_sync();   // the LDS is reused
            continue;
        }
        // A unit has at most two rows that others share: one begun before it
        // (slot 1) and one that goes on behind it (slot 0).
        const int i = unit - first, n = last - first + 1;
        auto slot_of = [&](int k) { return k == 0 ? 0 : 1; };
        if (hh < dm.G) part_store(part_at(dm, c, unit, slot_of(i), hh), e8, mine);
        auto arrived_last = [&](int* count, int want) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) sh_last = arrive_last(count, arrive(count), want) ? 1 : 0;
            __syncthreads();
            return sh_last != 0;
        };
        const int i0 = i / kJoin * kJoin, members = min(kJoin, n - i0);
        bool go = arrived_last(c.count + 2 * (first + i0) + slot_of(i0), members);
        if (go) {
            Share sum{-INFINITY, 0.0f, {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
            if (hh < dm.G) {
#pragma unroll 4
                for (int k = 0; k < members; ++k)
                    share_add(sum, part_load(part_at(dm, c, first + i0 + k, slot_of(i0 + k), hh), e8));
            }
            const int groups = (n + kJoin - 1) / kJoin;
            if (groups > 1) {
                if (hh < dm.G) part_store(part_at(dm, c, first + i0, slot_of(i0), hh), e8, sum);
                go = arrived_last(c.count + 2 * c.units + first, groups);
                if (go && hh < dm.G) {
                    sum = Share{-INFINITY, 0.0f, {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
#pragma unroll 4
                    for (int k = 0; k < groups; ++k)
                        share_add(sum, part_load(part_at(dm, c, first + k * kJoin, slot_of(k * kJoin), hh), e8));
                }
            }
            if (go && hh < dm.G) write_out(dm, c, r, hh, e8, sum);
        }
    }
    if (status != 0) atomicOr(sc.status, status);
}

}  // namespace

// Units: two workgroups per CU, fewer where the page tables' capacity leaves
// them less than a step per wave.
int attend_units(const Dims& dm, int n_cu) {
    const int64_t steps = (int64_t)dm.S * dm.Hkv * ((((int64_t)dm.MP * dm.P + 15) / 16 + 1) / 2 + 1);
    return (int)std::min<int64_t>(2 * n_cu, (steps + kMinUnitSteps - 1) / kMinUnitSteps);
}

// Counters (arrivals at each unit's two slots, and at a row's groups), then
// two partial results per unit.
static size_t count_words(int units) { return ((size_t)3 * units + 63) / 64 * 64; }

uint64_t attend_workspace(const Dims& dm, int n_cu) {
    const int u = attend_units(dm, n_cu);
    return (count_words(u) + (uint64_t)2 * u * dm.G * kPartWords) * sizeof(float);
}

void attend_carve(const Dims& dm, int n_cu, void* workspace, TokenCall* c) {
    c->units = attend_units(dm, n_cu);
    c->count = static_cast<int32_t*>(workspace);
    c->part = static_cast<float*>(workspace) + count_words(c->units);
}

hipError_t launch_token(const Dims& dm, const View& v, const Scratch& sc, const TokenCall& c, hipStream_t st) {
    Dims d = dm;
    View vv = v;
    Scratch ss = sc;
    TokenCall cc = c;
    void* args[] = {&d, &vv, &ss, &cc};
    const void* fn = c.blocks != nullptr ? (dm.quant ? reinterpret_cast<const void*>(&k_token<true, true>)
                                                     : reinterpret_cast<const void*>(&k_token<true, false>))
                                         : (dm.quant ? reinterpret_cast<const void*>(&k_token<false, true>)
                                                     : reinterpret_cast<const void*>(&k_token<false, false>));
    return hipLaunchKernel(fn, dim3((unsigned)c.units), dim3(kTokThreads), args, 0, st);
}

}  // namespace md
