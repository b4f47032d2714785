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
#include <type_traits>

#include "md_arrive.h"
#include "md_decode.h"
#include "md_device.h"

namespace md {

namespace {

// A step is two tiles of 16 tokens, whose values meet in one product of 32;
// a cell is two steps per wave or more.
constexpr int kMinWaveSteps = 2;
constexpr int kWideSteps = 64;       // even shares below this may be doubled for whole rows
constexpr int kStreamSteps = 8192;   // a line this long (128 MiB) is read past the caches
constexpr int kJoin = 8;             // partial results that one thread joins

__device__ __forceinline__ bool counts_ok(const TokenCall& c, int np, int nt) {
    return np == 0 ? nt == 0 : np > 0 && np <= c.MP && nt > (np - 1) * c.P && nt <= np * c.P;
}

// The kernel's LDS that grows with the sessions.
constexpr size_t session_bytes(int S) { return (size_t)(2 * S + 1) * sizeof(int); }

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
__device__ __forceinline__ Desc tile_desc(const TokenCall& c, const Row& r, int step, int u,
                                          int& status) {
    Desc d{0, 0, 0};
    const int t = 2 * step + u;
    if (t >= r.tiles) {
        if (r.ok && c.new_k != nullptr && u == 0 && step == (r.tiles + 1) >> 1) d.live = -1;
        return d;
    }
    const int per = c.P >> 4;
    int page = t >> (c.Pshift - 4);
    const int sub = t & (per - 1);
    if constexpr (SPARSE) {
        const int32_t* list = c.blocks + ((size_t)r.s * c.Hkv + r.kv) * c.max_blocks;
        const int o = page;
        page = list[o];
        // (by the entry before alone: the entries that count before a broken
        // one would take a pass over the list)
        if (page < 0 || page >= r.np || (o > 0 && page <= list[o - 1])) {
            status |= MD_DEV_BAD_BLOCK;
            return d;
        }
    }
    const int p = c.page_table[(size_t)r.s * c.MP + page];
    if ((unsigned)p >= (unsigned)c.NP) {
        status |= kDevCorrupt;
        return d;
    }
    d.phys = p;
    d.live = min(16, max(0, r.nt - (page * c.P + 16 * sub)));
    if (c.aligned) d.live = min(d.live, tokens_before_holes(c.region + (size_t)p * c.P + 16 * sub));
    if constexpr (QT) d.quant = c.page_format[p];
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

// A thread's share of a row's result: N dims of one query head.
template <int N>
struct Share {
    float m, l, y[N];
};

__device__ __forceinline__ float* part_at(const TokenCall& c, int cell, int slot, int hh) {
    return c.part + ((size_t)(2 * cell + slot) * c.G + hh) * kPartWords;
}

template <int N>
__device__ __forceinline__ void part_store(float* p, int part, const Share<N>& r) {
#pragma unroll
    for (int i = 0; i < N; i += 2) put2(p + N * part + i, r.y[i], r.y[i + 1]);
    if (part == 0) put2(p + kHeadDim, r.m, r.l);
}

template <int N>
__device__ __forceinline__ Share<N> part_load(const float* p, int part) {
    Share<N> r;
    const float2 st = get2(p + kHeadDim);
    r.m = st.x;
    r.l = st.y;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 w = get2(p + N * part + i);
        r.y[i] = w.x;
        r.y[i + 1] = w.y;
    }
    return r;
}

template <int N>
__device__ __forceinline__ Share<N> no_share() {
    Share<N> r;
    r.m = -INFINITY;
    r.l = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) r.y[i] = 0.0f;
    return r;
}

template <int N>
__device__ __forceinline__ void share_add(Share<N>& a, const Share<N>& b) {
    const float M = fmaxf(a.m, b.m);
    const float fa = M == -INFINITY ? 0.0f : hw_exp2(a.m - M), fb = M == -INFINITY ? 0.0f : hw_exp2(b.m - M);
    a.m = M;
    a.l = a.l * fa + b.l * fb;
#pragma unroll
    for (int i = 0; i < N; ++i) a.y[i] = fmaf(b.y[i], fb, a.y[i] * fa);
}

template <int N>
__device__ __forceinline__ void write_out(const TokenCall& c, const Row& r, int hh, int part, const Share<N>& a) {
    const float inv = a.l > 0.0f ? 1.0f / a.l : a.l == 0.0f ? 0.0f : a.l;   // NaN stays NaN
    const int64_t at = (int64_t)r.s * c.out_stride + (r.kv * c.G + hh) * kHeadDim + N * part;
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        if (c.out_bf16) {
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(c.out) + at + i) =
                u32x2{pack_bf16(a.y[i] * inv, a.y[i + 1] * inv), pack_bf16(a.y[i + 2] * inv, a.y[i + 3] * inv)};
        } else {
            *reinterpret_cast<f32x4*>(static_cast<float*>(c.out) + at + i) =
                f32x4{a.y[i] * inv, a.y[i + 1] * inv, a.y[i + 2] * inv, a.y[i + 3] * inv};
        }
    }
    if (c.lse != nullptr && part == 0)
        c.lse[(size_t)r.s * c.Hq + r.kv * c.G + hh] = (a.m + log2f(a.l)) * 0.69314718055994530942f;
}

// The rows lie end to end on a line of steps of 32 tokens (sessions in order,
// each session's KV heads one after another), which is cut into cells, one
// for each workgroup, whatever the sessions' lengths.  Where cells of the
// line's even share each (or of the shortest length) leave room for it, every
// row is cut by itself, into the fewest cells of at most that length (rows of
// equal length, mostly); short ones also where cells of twice that do (400
// rows of 300 - 700 tokens: 27 us whole against 31 cut evenly, 512 of about
// 1,000: 51 against 61); else the line is, and a cell holds the whole of some
// rows and parts of at most two.  A row in several cells is joined by the
// workgroup that finishes last: in groups of cells by the last of each
// group, then the groups by the last of those (arrivals, no waits).
//
// Within a cell's stretch of one row the waves take steps in turn.  The keys
// of a wave's next step are requested as soon as this step's have been through
// the matrix cores, its values after this step's, and the next stretch's first
// step before this one's results are put together: 12 KiB per wave under way,
// with which the CU's eight waves fill HBM (64 sessions of 32k tokens, two KV
// heads: 2.15 GB in 335 us, 6.4 TB/s; a second step in registers, or twelve
// waves, read no faster).  A load behind a branch would turn the wait for the
// values into one for the next keys too (421 against 407 us when it was
// taken out, 64 sessions of 2k - 64k tokens), and long lines are read past the
// caches (364 against 391 us; short ones the other way round: 54 MB that the
// cache still holds, 19 against 22 us).
// Small cells at the end of the line, claimed from a queue by whichever
// workgroup reads faster, cost more than they gave (390 us).
//
// What bounds short lines is the chain: counters, scan, page table, keys and
// values (3 - 6 us), results through LDS, and where a row is cut its parts
// through memory (4 us).
// SPARSE: pages from the call's lists; QT: pages may hold 8-bit codes.
template <int W, bool SPARSE, bool QT>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(2, 2)))
k_token(TokenCall c) {
    constexpr int kThreads = 64 * W;
    constexpr int N = 32 / W;              // dims of a thread's share, 4 W threads a head
    constexpr int kQ = W >= 4 ? 1 : 4 / W; // pieces of the query that a wave stages
    using Mine = Share<N>;
    __shared__ __align__(16) u32x4 q_lds[3][4][64];
    __shared__ __align__(16) f32x4 acc_lds[W][8][64];
    __shared__ float2 stat_lds[W][16];
    __shared__ int scan_lds[2 * 17];
    __shared__ int sh_last;
    extern __shared__ int session_lds[];
    int* held = session_lds;              // [S] slots in use (-1: counters inconsistent), which give the pages
    int* pref = held + c.S;               // [S + 1] steps of one row of the sessions before
    // (of rows cut by themselves only, whose one stretch begins before any result is there)
    int* cpref = reinterpret_cast<int*>(acc_lds);   // [S + 1] cells of one row of the sessions before
    int* wpref = cpref + c.S + 1;                   // [S + 1] the same, of cells twice as long
    static_assert(sizeof(acc_lds) >= 2 * (kMaxSessions + 1) * sizeof(int));
    static_assert(8 / W * (sizeof(q_lds) + sizeof(acc_lds) + sizeof(stat_lds) + sizeof(scan_lds) + sizeof(sh_last) +
                           session_bytes(kMaxSessions) + 1280) <= 160 * 1024,
                  "eight waves a CU, whatever the sessions (1,280: the LDS is given out in such pieces)");
    const int tid = threadIdx.x, lane = lane_id(), wv = uni(tid >> 6);
    const int h = lane & 15, g = lane >> 4;
    const int per = c.P >> 4;
    int status = 0;
    // ---- the line and its cells
    constexpr int kPer = kMaxSessions / kThreads;
    int n[kPer], before = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int s = k * kThreads + tid;
        n[k] = 0;
        if (k * kThreads >= c.S) break;
        if (s < c.S) {
            const int np = c.n_pages[s], nt = c.n_tokens[s];
            const bool ok = counts_ok(c, np, nt);
            if (!ok && blockIdx.x == 0) status = kDevCorrupt;
            held[s] = ok ? nt : -1;
            const int tiles = !ok ? 0 : SPARSE ? min(c.max_blocks, np) * per : (nt + 15) >> 4;
            n[k] = max(1, ((tiles + 1) >> 1) + (c.new_k != nullptr && ok ? 1 : 0));
        }
        int total;
        const int ex = block_exclusive_scan(n[k], scan_lds, &total);
        if (s < c.S) pref[s] = before + ex;
        before += total;
    }
    const int T = uni(before) * c.Hkv;
    const int big = max(kMinWaveSteps * W, (int)(((unsigned)T + c.units - 1) / (unsigned)c.units));
    // (cells of the even share and of twice that, by rows)
    int cells = 0, wide = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int s = k * kThreads + tid;
        if (k * kThreads >= c.S) break;
        const int of[2] = {(int)((unsigned)(n[k] + big - 1) / (unsigned)big),
                           (int)((unsigned)(n[k] + 2 * big - 1) / (unsigned)(2 * big))};
        int ex[2], total[2];
        block_exclusive_scan_n<2>(of, scan_lds, ex, total);
        if (s < c.S) {
            cpref[s] = cells + ex[0];
            wpref[s] = wide + ex[1];
        }
        cells += total[0];
        wide += total[1];
    }
    if (tid == 0) {
        pref[c.S] = before;
        cpref[c.S] = cells;
        wpref[c.S] = wide;
    }
    __syncthreads();
    if (uni(cells) * c.Hkv > c.units && big < kWideSteps) {
        cells = wide;
        cpref = wpref;
    }
    cells = uni(cells) * c.Hkv;
    const bool by_row = cells <= c.units;   // every row cut by itself
    const int cell = blockIdx.x;
    if (by_row ? cell >= cells : cell * big >= T) return;
    const int hh = tid / (4 * W), ep = tid % (4 * W);   // this thread's share of a result

    // ---- one stretch: steps lo .. hi - 1 of row r
    struct Stretch {
        Row r;
        int lo, hi;
        int first, count;   // the row's cells
        int next;           // the place on the line behind the stretch
    };
    // (past: reads past the caches, std::true_type or std::false_type)
    auto run = [&](auto past) {
        Desc d;
        u32x4 kt[2][4], vt[2][4];
        f32x4 qa[kQ][2];
        auto steps_of = [&](const Stretch& t) { return max(0, (t.hi - t.lo - wv + W - 1) / W); };
        // descriptors of this wave's steps i .. i + 31 (lo + wv + 4 i ..): lane 2 k + u holds tile u of the k-th
        auto describe = [&](const Stretch& t, int i) {
            const int mine = t.lo + wv + (i + (lane >> 1)) * W;
            d = Desc{0, 0, 0};
            if (mine < t.hi) d = tile_desc<SPARSE, QT>(c, t.r, mine, lane & 1, status);
        };
        auto elem_at = [&](const Stretch& t, int i, int u) {
            const int phys = __builtin_amdgcn_readlane(d.phys, 2 * (i & 31) + u);
            const int tile = 2 * (t.lo + wv + i * W) + u;
            return (size_t)phys * c.page_elems +
                   ((size_t)c.layer * c.Hkv + t.r.kv) * c.P * kHeadDim + (size_t)(tile & (per - 1)) * 16 * kHeadDim;
        };
        auto load_k = [&](const Stretch& t, int i) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const gbytes kp = uni_ptr(c.k_pool + elem_at(t, i, u));
                const bool codes = QT && __builtin_amdgcn_readlane(d.quant, 2 * (i & 31) + u) != 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {   // codes fill two loads; their scale sits at byte 2048
                    const gvec at = reinterpret_cast<gvec>(kp + (uint32_t)(QT && j >= 2 && codes ? 2048 : 1024 * j + 16 * lane));
                    kt[u][j] = past.value ? __builtin_nontemporal_load(at) : *at;
                }
            }
        };
        auto load_v = [&](const Stretch& t, int i) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const gbytes vp = uni_ptr(c.v_pool + elem_at(t, i, u));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const gvec at = reinterpret_cast<gvec>(vp + (uint32_t)(1024 * j + 16 * lane));
                    vt[u][j] = past.value ? __builtin_nontemporal_load(at) : *at;
                }
            }
        };
        // this cell's stretch at `pos` of the line, its query and this wave's
        // first step requested
        const int end = by_row ? 0 : min(T, (cell + 1) * big);
        auto begin = [&](int pos) {
            Stretch t;
            Row& r = t.r;
            const int* starts = by_row ? cpref : pref;   // by rows: pos is the cell
            r.s = uni(find_session(starts, c.S, (int)((unsigned)pos / (unsigned)c.Hkv)));
            const int length = uni(starts[r.s + 1] - starts[r.s]), at_s = uni(starts[r.s]) * c.Hkv;
            r.kv = (int)((unsigned)(pos - at_s) / (unsigned)length);
            const int row0 = at_s + r.kv * length;
            if (by_row) {
                const int steps = uni(pref[r.s + 1] - pref[r.s]);
                t.first = row0;
                t.count = length;
                const int i = pos - row0;   // (steps * count fits: at most 2^15 steps and a cell per workgroup)
                t.lo = (int)((unsigned)(steps * i) / (unsigned)length);
                t.hi = (int)((unsigned)(steps * (i + 1)) / (unsigned)length);
                t.next = end;
            } else {
                t.lo = pos - row0;
                t.hi = min(length, end - row0);
                t.first = (int)((unsigned)row0 / (unsigned)big);
                t.count = (int)((unsigned)(row0 + length - 1) / (unsigned)big) - t.first + 1;
                t.next = row0 + t.hi;
            }
            r.nt = uni(held[r.s]);
            r.ok = r.nt >= 0;
            r.nt = max(0, r.nt);
            r.np = (r.nt + c.P - 1) >> c.Pshift;   // (what counts_ok says of consistent ones)
            r.tiles = (r.nt + 15) >> 4;
            if constexpr (SPARSE) {
                const int most = min(c.max_blocks, r.np);
                int n = c.block_count[(size_t)r.s * c.Hkv + r.kv];
                if (n < 0 || n > most) {
                    status |= MD_DEV_BAD_BLOCK;
                    n = min(max(n, 0), most);
                }
                r.tiles = n * per;
            }
            // wave w stages dims 32 j + 8 g .. of the heads' queries, j = w, w + W ..
#pragma unroll
            for (int k = 0; k < kQ; ++k) {
                const int j = wv + k * W;
                qa[k][0] = qa[k][1] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (h < c.G && j < 4) {
                    const f32x4* qp = reinterpret_cast<const f32x4*>(c.q + (int64_t)r.s * c.q_stride +
                                                                     (r.kv * c.G + h) * kHeadDim + 32 * j + 8 * g);
                    qa[k][0] = qp[0];
                    qa[k][1] = qp[1];
                }
            }
            if (steps_of(t) > 0) {
                describe(t, 0);
                load_k(t, 0);
                load_v(t, 0);
            }
            return t;
        };

        Stretch t = begin(by_row ? cell : cell * big);
        for (bool more = true; more;) {
            // ---- the heads' queries: three bf16 terms, exactly
#pragma unroll
            for (int y = 0; y < kQ; ++y) {
                const int j = wv + y * W;
                if (j >= 4) break;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    u32x4 w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t a[3], b[3];
                        split3(qa[y][i >> 1][2 * (i & 1)], a[0], a[1], a[2]);
                        split3(qa[y][i >> 1][2 * (i & 1) + 1], b[0], b[1], b[2]);
                        w[i] = a[k] | (b[k] << 16);
                    }
                    q_lds[k][j][lane] = w;
                }
            }
            lds_sync();
            float m = -INFINITY, l = 0.0f;
            f32x4 o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int nw = steps_of(t);
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
                    const uint16_t* nk = c.new_k + (int64_t)t.r.s * c.kv_stride + t.r.kv * kHeadDim;
                    const uint16_t* nv = c.new_v + (int64_t)t.r.s * c.kv_stride + t.r.kv * kHeadDim;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        kt[0][j] = *reinterpret_cast<const u32x4*>(nk + 32 * j + 8 * g);
                        vt[0][j] = u32x4{nv[32 * j + h], 0u, nv[32 * j + 16 + h], 0u};
                    }
                    live[0] = 1;
                }
                // (the query terms are read from LDS in every step: kept over the
                // steps they would take 48 registers)
                asm volatile("" ::: "memory");
                u32x4 bq[4][3];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 3; ++k) bq[j][k] = q_lds[k][j][lane];
                __builtin_amdgcn_sched_barrier(0);   // all of them before the products, not each before its own
                f32x4 x[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 3; ++k)
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            x[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                __builtin_bit_cast(bf16x8, kt[u][j]), __builtin_bit_cast(bf16x8, bq[j][k]), x[u], 0, 0, 0);
                // (unconditional: loads behind a branch would make the wait for the
                // values one for these keys too; behind the last step it reads
                // that step's tiles again, out of the cache)
                const int nx = min(i + 1, nw - 1);
                if ((nx & 31) == 0 && nx > i) describe(t, nx);
                load_k(t, nx);
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
                uint32_t ph[4], pm[4], pl[4];   // weights as three bf16 terms
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
                        float a = p[2 * k], b = p[2 * k + 1];
                        uint32_t w = ph[2 * u + k] = pack_bf16(a, b);
                        a -= bf16_lo(w);
                        b -= bf16_hi(w);
                        w = pm[2 * u + k] = pack_bf16(a, b);
                        pl[2 * u + k] = pack_bf16(a - bf16_lo(w), b - bf16_hi(w));
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
                const bf16x8 bm = __builtin_bit_cast(bf16x8, u32x4{pm[0], pm[1], pm[2], pm[3]});
                const bf16x8 bl = __builtin_bit_cast(bf16x8, u32x4{pl[0], pl[1], pl[2], pl[3]});
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const bf16x8 a = __builtin_bit_cast(
                            bf16x8, u32x4{vt[0][j][2 * e], vt[0][j][2 * e + 1], vt[1][j][2 * e], vt[1][j][2 * e + 1]});
                        o[2 * j + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bh, o[2 * j + e], 0, 0, 0);
                        o[2 * j + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bm, o[2 * j + e], 0, 0, 0);
                        o[2 * j + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bl, o[2 * j + e], 0, 0, 0);
                    }
                load_v(t, nx);
            }
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (g == 0) stat_lds[wv][h] = make_float2(m, l);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc_lds[wv][i][lane] = o[i];
            // ---- the cell's next row is requested
            const Stretch done = t;
            more = t.next < end;
            if (more) t = begin(t.next);
            // ---- the waves' results meet
            lds_sync();
            Mine mine = no_share<N>();
#pragma unroll
            for (int w = 0; w < W; ++w) {   // dims N ep ..: tile (dim / 16), lane group (dim / 4) & 3
                Mine b;
                b.m = stat_lds[w][hh].x;
                b.l = stat_lds[w][hh].y;
#pragma unroll
                for (int x = 0; x < N; x += 4) {
                    const int e = N * ep + x;
                    const f32x4 a = acc_lds[w][e >> 4][((e >> 2) & 3) * 16 + hh];
#pragma unroll
                    for (int i = 0; i < 4; ++i) b.y[x + i] = a[i];
                }
                share_add(mine, b);
            }
            // ---- the row's other cells
            const int first = done.first, n = done.count;
            if (n == 1) {
                if (hh < c.G) write_out(c, done.r, hh, ep, mine);
                lds_sync();   // the LDS is reused
                continue;
            }
            // A cell has at most two rows that others share: one begun before it
            // (slot 1) and one that goes on behind it (slot 0).
            const int i = cell - first;
            auto slot_of = [&](int k) { return k == 0 ? 0 : 1; };
            if (hh < c.G) part_store(part_at(c, cell, slot_of(i), hh), ep, mine);
            auto arrived_last = [&](int* count, int want) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (tid == 0) sh_last = arrive_last(count, arrive(count), want) ? 1 : 0;
                __syncthreads();
                return sh_last != 0;
            };
            // The sum of n partial results, `step` cells apart: all threads load,
            // gp of each `heads` threads' groups a part of them, and the groups
            // meet in LDS.
            const int heads = c.G <= 1 ? 1 : c.G <= 2 ? 2 : c.G <= 4 ? 4 : c.G <= 8 ? 8 : 16;
            auto sum_parts = [&](int cell0, int k0, int step, int count) {
                Mine sum = no_share<N>();
                const int head = hh & (heads - 1), gp = 16 / heads;
                if (head < c.G) {
#pragma unroll 8
                    for (int k = hh / heads; k < count; k += gp)
                        share_add(sum, part_load<N>(part_at(c, cell0 + k * step, slot_of(k0 + k * step), head), ep));
                }
                // (the groups' sums reach the first one by halves, so that they fit the LDS of the waves' results)
                for (int half = gp / 2; half > 0; half /= 2) {
                    float* lds = reinterpret_cast<float*>(acc_lds) + (hh & (half * heads - 1)) * 4 * W * (N + 2) + ep * (N + 2);
                    lds_sync();
                    if (hh >= half * heads && hh < 2 * half * heads) {
                        lds[0] = sum.m;
                        lds[1] = sum.l;
#pragma unroll
                        for (int x = 0; x < N; ++x) lds[2 + x] = sum.y[x];
                    }
                    lds_sync();
                    if (hh < half * heads) {
                        Mine b;
                        b.m = lds[0];
                        b.l = lds[1];
#pragma unroll
                        for (int x = 0; x < N; ++x) b.y[x] = lds[2 + x];
                        share_add(sum, b);
                    }
                }
                return sum;
            };
            const int join = kJoin * 16 / heads;
            const int i0 = i / join * join, members = min(join, n - i0);
            bool go = arrived_last(c.count + 2 * (first + i0) + slot_of(i0), members);
            if (go) {
                Mine sum = sum_parts(first + i0, i0, 1, members);
                const int groups = (n + join - 1) / join;
                if (groups > 1) {
                    if (hh < c.G) part_store(part_at(c, first + i0, slot_of(i0), hh), ep, sum);
                    go = arrived_last(c.count + 2 * c.units + first, groups);
                    if (go) sum = sum_parts(first, 0, join, groups);
                }
                if (go && hh < c.G) write_out(c, done.r, hh, ep, sum);
            }
            lds_sync();   // the LDS is reused
        }
    };
    if (T >= kStreamSteps) run(std::true_type{}); else run(std::false_type{});
    if (status != 0) atomicOr(c.status, status);
}

template <int W>
const void* token_kernel(bool sparse, bool codes) {
    return sparse ? (codes ? reinterpret_cast<const void*>(&k_token<W, true, true>)
                           : reinterpret_cast<const void*>(&k_token<W, true, false>))
                  : (codes ? reinterpret_cast<const void*>(&k_token<W, false, true>)
                           : reinterpret_cast<const void*>(&k_token<W, false, false>));
}

}  // namespace

// Waves of a workgroup; there are eight waves a CU either way, fewer where the
// page tables' capacity leaves the workgroups less than the shortest cell.
// Four, as a rule.  Two where each CU has eight rows or more, most of them
// whole in one cell (4,096 rows of 5 - 60 tokens: 44 against 61 us, of about
// 1,000: 359 against 373); four of these workgroups fit a CU's LDS with any
// number of sessions (1,024 of 300 - 700 tokens, two KV heads: 123 us; 142
// where their words left room for three).  Eight where a few long rows are cut into half as
// many parts to join (two rows of 131k tokens: 37 against 41 us; 32 rows of
// 32k: 82 either way).  The length that the host knows is the page tables':
// short rows in a table for long ones pay for it (one session of 450 tokens,
// two KV heads: one cell of eight waves a row, 10.4 us, against two of four and
// their join, 9.9; of 1,700: 12.9 against 11.1).
static int attend_waves(const Dims& dm, int n_cu) {
    const int rows = dm.S * dm.Hkv;
    if (rows >= 8 * n_cu) return 2;
    return rows * 16 <= n_cu && (int64_t)dm.MP * dm.P >= 16384 ? 8 : 4;
}

static int attend_units(const Dims& dm, int n_cu) {
    const int W = attend_waves(dm, n_cu), shortest = kMinWaveSteps * W;
    const int64_t steps = (((int64_t)dm.MP * dm.P + 15) / 16 + 1) / 2 + 1;   // of a row
    const int64_t cells = (int64_t)dm.S * dm.Hkv * ((steps + shortest - 1) / shortest);
    return (int)std::min<int64_t>((int64_t)n_cu * 8 / W, cells);
}

// Counters (arrivals at each cell's two slots, and at a row's groups), then
// two partial results per cell.
static size_t count_words(int units) { return ((size_t)3 * units + 63) / 64 * 64; }

uint64_t attend_workspace(const Dims& dm, int n_cu) {
    const int u = attend_units(dm, n_cu);
    return (count_words(u) + (uint64_t)2 * u * dm.G * kPartWords) * sizeof(float);
}

bool attend_fits(const Dims& dm) {
    return (int64_t)dm.S * dm.Hkv * ((int64_t)dm.MP * dm.P / 32 + 2) < (int64_t)1 << 31;
}

hipError_t launch_token(const Dims& dm, const View& v, const Scratch& sc, int n_cu, int layer, const md_attend_args& a,
                        hipStream_t st) {
    TokenCall c{};
    c.S = dm.S;
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
    c.q = a.q;
    c.q_stride = a.q_stride;
    c.new_k = a.new_k;
    c.new_v = a.new_v;
    c.kv_stride = a.kv_stride;
    c.v_pool = a.v_pool;
    c.blocks = a.blocks;
    c.block_count = a.block_count;
    c.max_blocks = a.max_blocks;
    c.out_bf16 = a.out_type == MD_BF16;
    c.out = a.out;
    c.out_stride = a.out_stride;
    c.lse = a.lse;
    c.units = attend_units(dm, n_cu);
    c.count = static_cast<int32_t*>(a.workspace);
    c.part = static_cast<float*>(a.workspace) + count_words(c.units);
    void* args[] = {&c};
    const int W = attend_waves(dm, n_cu);
    const bool sparse = a.blocks != nullptr, codes = dm.quant != 0;
    const void* fn = W == 8 ? token_kernel<8>(sparse, codes) : W == 4 ? token_kernel<4>(sparse, codes)
                                                             : token_kernel<2>(sparse, codes);
    return hipLaunchKernel(fn, dim3((unsigned)c.units), dim3(64 * W), args, session_bytes(dm.S), st);
}

}  // namespace md
