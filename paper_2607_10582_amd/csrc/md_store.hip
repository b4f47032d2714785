// gfx950 kernels that move rows between a caller's arrays and the pools: keys
// and values of ragged rows in and out, and a step's values in 8 bits.
//
//   scale = max |v| / 448 over a block of 16 tokens and KV head,  code = e4m3(v / scale)
//
// Each moves a value once and turns it by a few operations, so long calls are
// bound by HBM, and a decode step's by the launch and its chain of loads
// (sessions' bounds, slot, page, bytes).  Rows in: 4 x 8,192 of two KV heads, 14.2
// us, 4.1 TB/s of reads and writes (14.8 where the open blocks are kept); 64 uneven
// chunks, 14.4.  Rows out: 16 x 32,768 into float32, 311 us, 4.4 TB/s (a copy of 4
// GiB runs at 4.8); 32 x 1,700, 26.8 us, 20.4 in a graph of such calls.  The values
// of a decode step of 32 sessions, 36 layers: 5.8 us from Python, 5.0 in a graph.

#include "md_decode.h"
#include "md_device.h"

namespace md {

namespace {

constexpr int kWaves = 4;          // waves per workgroup
constexpr float kTopCode = 448.0f; // the largest E4M3 value
constexpr int kPitch = kHeadDim + 8;   // elements between the tokens of a block in LDS

struct RowCall {
    int S, L, Hkv, P, Pshift, MP, NP, layer, quant;
    size_t page_elems;
    uint16_t* k_pool;
    const int32_t* page_table;
    const int32_t* n_pages;
    const int32_t* n_tokens;
    const uint8_t* page_format;
    int32_t* status;
    const int32_t* row_start;
    const int32_t* row_slot;
    int n_rows;
    md_values values;
    Held held;
    void* k;   // the caller's rows
    void* v;
    int64_t stride;
};

// Eight E4M3 codes of 8 floats (already divided by their scale).
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// v / scale, 0 where the scale is 0 or not a number.
__device__ __forceinline__ float in_scale(float v, float scale) { return scale > 0.0f ? v / scale : 0.0f; }

// The scale of a block whose largest magnitude has these bf16 bits (NaN for
// a value that is not finite: those have the largest bits).
__device__ __forceinline__ float scale_of(uint32_t top_bits) {
    return top_bits >= 0x7F80u ? __uint_as_float(0x7FC00000u) : __uint_as_float(top_bits << 16) / kTopCode;
}

__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) { return ~wave_min_u32(~v); }

// Largest magnitude bits among the two bf16 values of a word.
__device__ __forceinline__ uint32_t top_of(uint32_t w) { return max(w & 0x7FFFu, (w >> 16) & 0x7FFFu); }

// A block's codes out of LDS ([16 tokens][kPitch] bf16), lane (m, g): tokens
// 4g .. 4g+3 of dims 64 a + 16 i + m, in the pool's order.
__device__ __forceinline__ u32x4 block_codes(const uint16_t* x, int a, float scale) {
    const int m = lane_id() & 15, g = lane_id() >> 4;
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float q[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) q[t] = in_scale(bf16_value(x[(4 * g + t) * kPitch + 64 * a + 16 * i + m]), scale);
        w[i] = four_codes(q[0], q[1], q[2], q[3]);
    }
    return w;
}

// Orders a wave's LDS accesses before and behind it (the hardware takes them
// in order; this keeps the compiler from moving them).
__device__ __forceinline__ void wave_lds() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// What the wave's row `lane & 31` of rows r0 .. r0 + 31 is.
struct Span {
    int s, lo, hi, nt; // its session, that session's rows and slots in use
    int slot, prev;    // its slot, and that of the session's row before it (-1: its first)
    int edge;          // ENDS: the slot of the session's first row, from lane 32 on of its last one
    int phys, sub, t;  // page, block of it and token of the block
    bool mine;         // it is some session's row
    bool in;           // and its slot holds a token's place
};

template <bool ENDS>
__device__ __forceinline__ Span span_of(const RowCall& c, int r0, int& status) {
    const int lane = lane_id(), r = r0 + (lane & 31);
    Span x{};
    // the sessions that end at or before a row, for 32 rows at once
    int s = 0;
    bool broken = false;   // row_start does not ascend within the rows: nobody's rows
    for (int base = 0; base < c.S; base += 64) {
        int end = 0x7FFFFFFF;
        if (base + lane < c.S) {
            const int begin = c.row_start[base + lane];
            end = c.row_start[base + lane + 1];
            broken |= begin < 0 || begin > end || end > c.n_rows;
        }
#pragma unroll 8
        for (int i = 0; i < 32; ++i) {
            const int n = __popcll(__ballot(end <= r0 + i));
            if (i == (lane & 31)) s += n;
        }
    }
    x.s = min(s, c.S - 1);
    x.lo = c.row_start[x.s];
    x.hi = c.row_start[x.s + 1];
    broken = __any(broken);
    if (broken) status |= MD_DEV_BAD_ROW;
    x.mine = !broken && s < c.S && x.lo <= r && r < x.hi;
    if (!x.mine) return x;
    const int np = c.n_pages[x.s], nt = c.n_tokens[x.s];
    const bool ok = np == 0 ? nt == 0 : np > 0 && np <= c.MP && nt > (np - 1) * c.P && nt <= np * c.P;
    if (!ok) {
        status |= kDevCorrupt;
        return x;
    }
    x.nt = nt;
    x.slot = c.row_slot != nullptr ? c.row_slot[r] : nt - (x.hi - r);
    x.prev = r <= x.lo ? -1 : c.row_slot != nullptr ? c.row_slot[r - 1] : x.slot - 1;
    if constexpr (ENDS) {
        const int at = lane < 32 ? x.lo : x.hi - 1;
        x.edge = c.row_slot != nullptr ? c.row_slot[at] : nt - (x.hi - at);
    }
    x.in = x.slot >= 0 && x.slot < nt;
    if (!x.in) {
        status |= MD_DEV_BAD_ROW;
        return x;
    }
    x.phys = c.page_table[(size_t)x.s * c.MP + (x.slot >> c.Pshift)];
    if ((unsigned)x.phys >= (unsigned)c.NP) {
        status |= kDevCorrupt;
        x.in = false;
        x.phys = 0;
    }
    x.sub = (x.slot & (c.P - 1)) >> 4;
    x.t = x.slot & 15;
    return x;
}

__device__ __forceinline__ size_t tile_of(const RowCall& c, int phys, int sub, int kv) {
    return (size_t)phys * c.page_elems + ((size_t)c.layer * c.Hkv + kv) * c.P * kHeadDim + (size_t)sub * 16 * kHeadDim;
}
__device__ __forceinline__ size_t scale_at(const RowCall& c, int phys, int sub, int kv) {
    return (((size_t)phys * c.L + c.layer) * c.Hkv + kv) * (size_t)(c.P >> 4) + sub;
}

// A session's rows lo .. hi - 1, some of whose slots may not be there (outside
// of 0 .. nt - 1): these are passed over.  All of a wave call these together.
struct SessionRows {
    const int32_t* row_slot;
    int lo, hi, nt;
    __device__ __forceinline__ int slot(int r) const { return row_slot != nullptr ? row_slot[r] : nt - (hi - r); }
    __device__ __forceinline__ bool there(int slot) const { return slot >= 0 && slot < nt; }

    // The first of rows a .. b - 1 that is there and whose slot is not below
    // `least`; b if there is none.  256 rows a round trip.
    __device__ __forceinline__ int first_from(int a, int b, int least) const {
        for (int q = a; q < b; q += 256) {
            int x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = q + 64 * k + lane_id();
                x[k] = r < b ? slot(r) : -1;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint64_t found = __ballot(there(x[k]) && x[k] >= least);
                if (found != 0) return q + 64 * k + __ffsll((unsigned long long)found) - 1;
            }
        }
        return b;
    }

    // The same over all rows, of those that ascend: by 64 probes at a time.
    // The answer depends on the rows and on `least` alone, whatever the rows are.
    __device__ __forceinline__ int search(int least) const {
        int a = lo, b = hi;
        while (b - a > 256) {
            const int at = a + (int)((int64_t)(b - a) * lane_id() / 64), x = slot(at);
            const uint64_t above = __ballot(there(x) && x >= least);
            const int k = above != 0 ? __ffsll((unsigned long long)above) - 1 : 64;
            const uint64_t below = __ballot(there(x) && x < least) & (k < 64 ? (1ull << k) - 1ull : ~0ull);
            const int end = k < 64 ? __builtin_amdgcn_readlane(at, k) : b;
            const int begin = below != 0 ? __builtin_amdgcn_readlane(at, 63 - __clzll(below)) + 1 : a;
            const bool little = end - begin > (b - a) / 2;   // (the probes are not there)
            a = begin;
            b = end;
            if (little) break;
        }
        return first_from(a, b, least);
    }

    // The rows of the last block that rows up to `end` (not itself) reach.
    struct Block {
        int base;    // its first slot (-1: no row is there)
        int begin;   // its first row
        int from;    // lane m's: that of token m, or -1
        uint32_t have;
        // Its tokens up to the last one (0: some are missing).
        __device__ __forceinline__ int tokens() const { return (have & (have + 1)) == 0 ? __popc(have) : 0; }
    };
    __device__ __forceinline__ Block last_block(int end) const {
        Block b{-1, end, -1, 0};
        for (int q = end; q > lo; q -= 64) {
            const int r = q - 1 - lane_id(), x = r >= lo ? slot(r) : -1;
            uint64_t in = __ballot(there(x));
            while (in != 0) {
                const int i = __ffsll((unsigned long long)in) - 1, at = __builtin_amdgcn_readlane(x, i);
                in &= in - 1;
                if (b.base < 0) b.base = at & ~15;
                if ((at & ~15) != b.base) return b;
                b.begin = q - 1 - i;
                b.have |= 1u << (at & 15);
                if (b.from < 0 && (at & 15) == (lane_id() & 15)) b.from = b.begin;
            }
        }
        return b;
    }
};

// A wave takes 16 rows and one KV head: the groups of rows that begin among
// them, each the rows of one block.  A block has one group, whose first row is
// the one that a search of the session's rows for the block's first slot finds,
// so that no two waves write a block even where the slots do not ascend; rows
// whose slots are not there may lie anywhere between (the search by halves
// gives way to one that passes over them where it meets one).  Keys go as they
// come, 1 KiB of a block at a time; values turn in LDS, from rows of dims to
// dims of four tokens.  Six waves a SIMD: left to five by its registers, 16 x
// 32,768 rows with 8-bit values took 177 us instead of 171, by lists of slots 217
// instead of 207.
template <bool CODES>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(6))) k_write_rows(RowCall c) {
    __shared__ __align__(16) uint16_t turn[kWaves][16 * kPitch];
    const int lane = lane_id(), wv = threadIdx.x >> 6;
    const int64_t task = (int64_t)blockIdx.x * kWaves + wv;
    const int r0 = (int)(task / c.Hkv) * 16, kv = (int)(task % c.Hkv);
    if (r0 >= c.n_rows) return;
    int status = 0;
    const Span x = span_of<CODES>(c, r0, status);
    const int r = r0 + (lane & 31);
    // the slot of the session's row before it that is there, as far as these 32 rows
    // and the one in front of them tell (below 0: none)
    int prev = x.prev;
    if (__builtin_expect(__any(x.in && r > x.lo && (prev < 0 || prev >= x.nt)), 0)) {
        const uint32_t below = (uint32_t)__ballot(x.in) & ((1u << (lane & 31)) - 1u);
        const int j = below != 0 ? 31 - __clz(below) : 0;
        const int slot = __shfl(x.slot, j), s = __shfl(x.s, j), front = __builtin_amdgcn_readlane(x.prev, 0);
        prev = below != 0 && s == x.s ? slot : r0 > x.lo && front < x.nt ? front : -1;
    }
    const bool ascends = x.in && x.slot > prev;
    if (x.in && !ascends) status |= MD_DEV_BAD_ROW;
    bool leads = ascends && lane < 16 && (prev >> 4) != (x.slot >> 4);   // (below 0 is no block)
    bool odd = false;   // a row that is not there came into the search's way
    if (leads && c.row_slot != nullptr) {   // the first row that is not below the block
        int lo = x.lo, hi = x.hi;
        while (lo < hi && !odd) {
            const int mid = lo + (hi - lo) / 2, slot = c.row_slot[mid];
            odd = slot < 0 || slot >= x.nt;
            if (slot < (x.slot & ~15)) lo = mid + 1; else hi = mid;
        }
        leads = !odd && lo == r;
    }
    auto rows_of = [&](int i) {   // of lane i's session
        return SessionRows{c.row_slot, __builtin_amdgcn_readlane(x.lo, i), __builtin_amdgcn_readlane(x.hi, i),
                           __builtin_amdgcn_readlane(x.nt, i)};
    };
    for (uint64_t left = __ballot(odd); __builtin_expect(left != 0, 0); left &= left - 1) {
        const int i = __ffsll((unsigned long long)left) - 1;
        if (rows_of(i).search(__builtin_amdgcn_readlane(x.slot, i) & ~15) == r0 + i && lane == i) leads = true;
    }
    const bool coded = c.quant && x.in && c.page_format[x.phys] != 0;
    if (coded && c.k != nullptr) status |= MD_DEV_BAD_ROW;
    const uint32_t ascending = (uint32_t)__ballot(ascends);
    uint64_t todo = __ballot(leads);
    uint16_t* const buf = turn[wv];
    const int m = lane & 15, g = lane >> 4;
    while (todo != 0) {
        const int i = __ffsll((unsigned long long)todo) - 1;
        todo &= todo - 1;
        const int o = __builtin_amdgcn_readlane(x.t, i), phys = __builtin_amdgcn_readlane(x.phys, i);
        const int sub = __builtin_amdgcn_readlane(x.sub, i), s = __builtin_amdgcn_readlane(x.s, i);
        const int row = r0 + i, block = __builtin_amdgcn_readlane(x.slot, i) >> 4;
        const SessionRows rows = rows_of(i);
        const bool skip_k = c.quant && __builtin_amdgcn_readlane(coded ? 1 : 0, i);
        // the group's rows among the 32, up to the first that is there and in another block
        const bool same = x.in && x.s == s && (x.slot >> 4) == block;
        const uint32_t behind = 0xFFFFFFFFu << i;
        uint32_t mine = (uint32_t)__ballot(same) & behind;
        const uint32_t others = (uint32_t)__ballot(x.in && x.s == s && !same) & behind;
        bool more = others == 0 && rows.hi > r0 + 32;   // it may go on behind them
        if (others != 0) mine &= (others & -others) - 1u;
        // which tokens of the block it holds, and the row of lane m's token
        uint32_t have = 0;
        int from = row, top = -1;
        const int len = __popc(mine);
        if (__builtin_expect(mine >> i == (1u << (len & 31)) - 1u && len <= 16 &&
                             __builtin_amdgcn_readlane(x.t, i + len - 1) - o == len - 1 && (mine & ~ascending) == 0, 1)) {
            have = ((1u << len) - 1u) << o;
            from = row + m - o;
            top = o + len - 1;
        } else {
            for (uint32_t left = mine; left != 0; left &= left - 1) {   // those that ascend
                const int j = __ffs(left) - 1, t = __builtin_amdgcn_readlane(x.t, j);
                if (t <= top) continue;
                have |= 1u << t;
                if (m == t) from = r0 + j;
                top = t;
            }
        }
        for (int q = r0 + 32; __builtin_expect(more && q < rows.hi, 0);) {   // (only behind rows that are not there)
            q = rows.first_from(q, rows.hi, 0);
            if (q == rows.hi) break;
            const int slot = uni(rows.slot(q));
            more = (slot >> 4) == block;
            if (more && (slot & 15) > top) {
                top = slot & 15;
                have |= 1u << top;
                if (m == top) from = q;
            }
            ++q;
        }
        const bool last = others == 0 && (more || rows.hi <= r0 + 32);   // no row behind it is there
        // whether it is the session's first, and whether that starts with a block
        const int head = CODES ? __builtin_amdgcn_readlane(x.edge, i) : 0, tail = CODES ? __builtin_amdgcn_readlane(x.edge, i + 32) : 0;
        const bool ends = rows.there(head) && rows.there(tail);   // the session's first and last rows are there
        bool first = row == rows.lo, starts_block = (head & 15) == 0;
        if (CODES && __builtin_expect(!ends, 0)) {
            const int begin = uni(rows.first_from(rows.lo, row, 0));
            first = begin == row;
            starts_block = (uni(rows.slot(begin)) & 15) == 0;
        }
        // Where a token in front of the group's last one is not among the rows, it is
        // in the open block or the one before that, whichever is this one: the
        // session's first group looks, which alone may (the others' blocks are not
        // there yet).  Told of neither the open block is taken for it.
        const int id = phys * (c.P >> 4) + sub;
        const size_t open_at = CODES ? ((((size_t)s * c.L + c.layer) * c.Hkv + kv) * 16 + m) * kHeadDim + 8 * g : 0;
        uint16_t* const open = CODES ? c.values.v_open + open_at : nullptr;
        uint16_t* const before = CODES ? c.held.before + open_at : nullptr;
        int4* const held_at = CODES && c.held.at != nullptr
                                  ? reinterpret_cast<int4*>(c.held.at) + ((size_t)s * c.L + c.layer) * c.Hkv + kv : nullptr;
        const uint16_t* source = open;
        int known = first ? o : 0;   // tokens of it that count
        int4 held{-1, 0, -1, 0};
        if (held_at != nullptr) {
            if (first && (last || o > 0)) {
                held = *held_at;
                held = int4{uni(held.x), uni(held.y), uni(held.z), uni(held.w)};
            }
            known = 0;
            if (have != (2u << top) - 1u) {
                if (first && o > 0 && held.x == id) known = min(held.y, top);
                else if (first && o > 0 && held.z == id) known = min(held.w, top), source = before;
                if (known == 0) {   // what the block holds is not known: it stays
                    status |= MD_DEV_BAD_ROW;
                    have = 0;
                }
            }
        }
        const bool refused = have == 0;
        // lane (m, g): dims 8g .. of token m
        const bool has = (have >> m) & 1u;
        const int64_t at = (int64_t)from * c.stride + kv * kHeadDim + 8 * g;
        const size_t tile = tile_of(c, phys, sub, kv);
        if (c.k != nullptr && !skip_k && has) {
            const uint16_t* from = static_cast<const uint16_t*>(c.k) + at;
            uint16_t* to = c.k_pool + tile + 8 * lane;
            u32x4 w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const u32x4*>(from + 32 * j);
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x4*>(to + 512 * j) = w[j];
        }
        if (c.v == nullptr) continue;
        u32x4 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = u32x4{0u, 0u, 0u, 0u};
        if (has || (CODES && m < known)) {
            const uint16_t* from = has ? static_cast<const uint16_t*>(c.v) + at : source;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const u32x4*>(from + 32 * j);
        }
        wave_lds();
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x4*>(buf + m * kPitch + 32 * j + 8 * g) = w[j];
        wave_lds();
        if constexpr (CODES) {
            // The open block becomes the session's last one, and the one before it the
            // last but one, each by its own wave.  Where the rows go on inside a block,
            // the first block's wave alone has read them, and writes both: from the
            // rows, for blocks that are other waves'.
            auto keep = [&](uint16_t* to) {
#pragma unroll
                for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x4*>(to + 32 * j) = w[j];
            };
            auto keep_rows = [&](uint16_t* to, int from) {   // from: the row of token m, or -1
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u32x4 y{0u, 0u, 0u, 0u};
                    if (from >= 0)
                        y = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(c.v) + (int64_t)from * c.stride +
                                                            kv * kHeadDim + 8 * g + 32 * j);
                    *reinterpret_cast<u32x4*>(to + 32 * j) = y;
                }
            };
            auto id_of = [&](int slot) {
                return c.page_table[(size_t)s * c.MP + (slot >> c.Pshift)] * (c.P >> 4) + ((slot & (c.P - 1)) >> 4);
            };
            const bool alone = first && last;
            const bool second = others != 0 && ends && starts_block &&   // the last but one
                                __builtin_amdgcn_readlane(x.slot, __ffs(others | 0x80000000u) - 1) >> 4 == tail >> 4;
            if ((alone && !refused) || (last && !first && starts_block)) {
                int4 now{-1, 0, -1, 0};
                if (held_at != nullptr && alone) {
                    if (held.x == id) {
                        now = held;
                    } else if (o == 0 && block > 0 && held.z >= 0 && held.z == uni(id_of(16 * block - 1))) {
                        now = held;   // (the open one was taken back whole)
                    } else if (o == 0 && held.x >= 0) {   // a new block: the open one becomes the one before it
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            *reinterpret_cast<u32x4*>(before + 32 * j) = *reinterpret_cast<const u32x4*>(open + 32 * j);
                        now = int4{-1, 0, held.x, held.y};
                    }
                } else if (held_at != nullptr && !refused && !ends) {   // (else the last but one does this)
                    const SessionRows::Block b = rows.last_block(row);
                    if (b.tokens() > 0) {
                        keep_rows(before, b.from);
                        now = int4{-1, 0, id_of(b.base), b.tokens()};
                    }
                }
                if (!refused) {
                    keep(open);
                    now.x = id;
                    now.y = top + 1;
                }
                if (held_at != nullptr && lane == 0) {
                    reinterpret_cast<int2*>(held_at)[0] = int2{now.x, now.y};
                    if (alone || !ends) reinterpret_cast<int2*>(held_at)[1] = int2{now.z, now.w};
                }
            } else if (second && held_at != nullptr) {
                if (!refused) keep(before);
                if (lane == 0) reinterpret_cast<int2*>(held_at)[1] = refused ? int2{-1, 0} : int2{id, top + 1};
            } else if (first && o > 0 && !last) {
                const SessionRows::Block b = rows.last_block(rows.hi);
                keep_rows(open, b.from);
                if (held_at != nullptr) {
                    int4 now{-1, 0, -1, 0};
                    if (b.tokens() > 0) {
                        now = int4{id_of(b.base), b.tokens(), -1, 0};
                        const SessionRows::Block f = rows.last_block(b.begin);
                        if (f.base >> 4 == block) {   // this one
                            if (!refused) {
                                keep(before);
                                now.z = id;
                                now.w = top + 1;
                            }
                        } else if (f.tokens() > 0) {
                            keep_rows(before, f.from);
                            now.z = id_of(f.base);
                            now.w = f.tokens();
                        }
                    }
                    if (lane == 0) *held_at = now;
                }
            }
            if (refused) continue;
            uint32_t largest = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) largest = max(largest, top_of(w[j][k]));
            const float scale = scale_of(wave_max_u32(largest));
            uint8_t* to = c.values.v_codes + tile + 16 * lane;
#pragma unroll
            for (int a = 0; a < 2; ++a) *reinterpret_cast<u32x4*>(to + 1024 * a) = block_codes(buf, a, scale);
            if (lane == 0) c.values.v_scale[scale_at(c, phys, sub, kv)] = scale;
        } else {
            uint16_t* to = c.values.v_pool + tile + 8 * lane;
            const uint32_t quad = (have >> (4 * g)) & 15u;   // which of this lane's four tokens come
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint16_t y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = buf[(4 * g + (e & 3)) * kPitch + 32 * j + 16 * (e >> 2) + m];
                if (quad == 15u) {
                    *reinterpret_cast<u32x4*>(to + 512 * j) = u32x4{y[0] | (uint32_t)y[1] << 16, y[2] | (uint32_t)y[3] << 16,
                                                                    y[4] | (uint32_t)y[5] << 16, y[6] | (uint32_t)y[7] << 16};
                } else if (quad != 0u) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if ((quad >> (e & 3)) & 1u) to[512 * j + e] = y[e];
                }
            }
        }
    }
    if (status != 0) atomicOr(c.status, status);
}

template <bool F32>
__device__ __forceinline__ void put8(void* p, int64_t at, const float (&x)[8]) {
    if constexpr (F32) {
        f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(p) + at);
        o[0] = f32x4{x[0], x[1], x[2], x[3]};
        o[1] = f32x4{x[4], x[5], x[6], x[7]};
    } else {
        typedef __bf16 bf16x2 __attribute__((__vector_size__(4)));
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + at) = w;
    }
}

// Eight bf16 values (words) times a scale; the scale 1 changes nothing.
__device__ __forceinline__ void widen8(const u32x4& w, float scale, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16) * scale;
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u) * scale;
    }
}

// A wave takes 16 rows and one KV head.  Lane (m, g) fetches row m's key, 16
// bytes at a time (consecutive rows of a block make 1 KiB); the values' blocks
// come whole and turn in LDS, one for each run of rows of the same block.
template <bool CODES, bool F32>
__global__ void __launch_bounds__(64 * kWaves) k_read_rows(RowCall c) {
    __shared__ __align__(16) uint16_t turn[kWaves][16 * kPitch];
    const int lane = lane_id(), wv = threadIdx.x >> 6;
    const int64_t task = (int64_t)blockIdx.x * kWaves + wv;
    const int r0 = (int)(task / c.Hkv) * 16, kv = (int)(task % c.Hkv);
    if (r0 >= c.n_rows) return;
    int status = 0;
    Span x = span_of<false>(c, r0, status);
    const int m = lane & 15, g = lane >> 4;
    // lane (m, g) works on row m
    const int phys = __shfl(x.phys, m), sub = __shfl(x.sub, m), t = __shfl(x.t, m);
    const bool mine = __shfl(x.mine ? 1 : 0, m) != 0, in = __shfl(x.in ? 1 : 0, m) != 0;
    const int64_t at = (int64_t)(r0 + m) * c.stride + kv * kHeadDim + 8 * g;
    // values, a block at a time, the first one's requested before the keys (behind
    // them: 322 us for 311, 16 x 32,768 rows into float32)
    uint32_t left = (uint32_t)__ballot(in) & 0xFFFFu;
    bool here = false;
    float v_scale = 1.0f;
    u32x4 vw[CODES ? 2 : 4];
    auto load_values = [&]() __attribute__((always_inline)) {
        const int i = __ffs(left) - 1;
        const int p = __builtin_amdgcn_readlane(phys, i), b = __builtin_amdgcn_readlane(sub, i);
        here = in && phys == p && sub == b;
        left &= ~(uint32_t)__ballot(here);
        const size_t tile = tile_of(c, p, b, kv);
        if constexpr (CODES) {
            v_scale = c.values.v_scale[scale_at(c, p, b, kv)];
#pragma unroll
            for (int a = 0; a < 2; ++a) vw[a] = *reinterpret_cast<const u32x4*>(c.values.v_codes + tile + 1024 * a + 16 * lane);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) vw[j] = *reinterpret_cast<const u32x4*>(c.values.v_pool + tile + 512 * j + 8 * lane);
        }
    };
    bool more = c.v != nullptr && left != 0;
    if (more) load_values();
    if (c.k != nullptr && mine) {
        const uint16_t* tile = c.k_pool + tile_of(c, phys, sub, kv);
        u32x4 w[4];
        float scale = 1.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = u32x4{0u, 0u, 0u, 0u};
        if (in && c.quant && c.page_format[phys] != 0) {
            const uint8_t* b = reinterpret_cast<const uint8_t*>(tile);
            scale = *reinterpret_cast<const float*>(b + 2048);
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const u32x4 k = *reinterpret_cast<const u32x4*>(b + 1024 * a + 16 * (t + 16 * g));
                w[2 * a] = codes_to_bf16<0>(k);
                w[2 * a + 1] = codes_to_bf16<1>(k);
            }
        } else if (in) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const u32x4*>(tile + 512 * j + 8 * (16 * g + t));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float y[8];
            widen8(w[j], scale, y);
            put8<F32>(c.k, at + 32 * j, y);
        }
    }
    if (c.v != nullptr && mine && !in) {
        const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) put8<F32>(c.v, at + 32 * j, none);
    }
    uint16_t* const buf = turn[wv];
    while (more) {
        wave_lds();
        if constexpr (CODES) {
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int e = 0; e < 4; ++e) {   // word e: tokens 4g .. of dim 64 a + 16 e + m
                    const uint32_t lo = codes_pair_to_bf16<false>(vw[a][e]), hi = codes_pair_to_bf16<true>(vw[a][e]);
                    uint16_t* to = buf + 4 * g * kPitch + 64 * a + 16 * e + m;
                    to[0] = (uint16_t)lo;
                    to[kPitch] = (uint16_t)(lo >> 16);
                    to[2 * kPitch] = (uint16_t)hi;
                    to[3 * kPitch] = (uint16_t)(hi >> 16);
                }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {   // words 0, 1: tokens 4g .. of dim 32 j + m; 2, 3: of 32 j + 16 + m
                    uint16_t* to = buf + (4 * g + 2 * (e & 1)) * kPitch + 32 * j + 16 * (e >> 1) + m;
                    to[0] = (uint16_t)vw[j][e];
                    to[kPitch] = (uint16_t)(vw[j][e] >> 16);
                }
        }
        wave_lds();
        const bool mine_now = here;
        const float scale = v_scale;
        more = left != 0;
        if (more) load_values();
        if (mine_now) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float y[8];
                widen8(*reinterpret_cast<const u32x4*>(buf + t * kPitch + 32 * j + 8 * g), scale, y);
                put8<F32>(c.v, at + 32 * j, y);
            }
        }
    }
    if (status != 0) atomicOr(c.status, status);
}

// One wave per (session, layer, KV head), two dims a lane.  The scale can
// only grow within a block, and max and division keep their order under
// rounding: scale = max(scale before, |v|'s own), so a token that does not
// raise it costs its own 128 codes.  One that does has the block's codes
// written anew, from the open block's values; so has one behind tokens that were
// taken back, which the scale still knows of (HELD: they are told by what the
// blocks held).
template <bool HELD>
__global__ void __launch_bounds__(64 * kWaves) k_append_codes(Dims dm, View v, const uint16_t* __restrict__ new_v,
                                                              md_values values, Held kept, int32_t* status) {
    __shared__ __align__(16) uint16_t turn[kWaves][16 * kPitch];
    const int lane = lane_id(), wv = threadIdx.x >> 6, s = blockIdx.y;
    const int row = blockIdx.x * kWaves + wv;   // (layer, KV head)
    if (row >= dm.LHkv) return;
    const uint32_t mine = reinterpret_cast<const uint32_t*>(new_v)[((size_t)s * dm.LHkv + row) * (kHeadDim / 2) + lane];
    int4* const held_at = HELD ? reinterpret_cast<int4*>(kept.at) + (size_t)s * dm.LHkv + row : nullptr;
    int4 held{-1, 0, -1, 0};
    if constexpr (HELD) held = *held_at;
    const int np = v.n_pages[s], nt = v.n_tokens[s];
    if (!counters_ok(np, nt, dm) || np == 0) return;
    const int p = v.page_table[(size_t)s * dm.MP + np - 1];
    if ((unsigned)p >= (unsigned)dm.NP) return;
    const int slot = nt - 1 - (np - 1) * dm.P, o = slot & 15;
    if (v.t_ins[(size_t)p * dm.P + slot] != v.clock[s]) return;
    const size_t tile = ((size_t)p * dm.LHkv + row) * dm.P * kHeadDim + (size_t)(slot & ~15) * kHeadDim;
    float* const scale_p = values.v_scale + ((size_t)p * dm.LHkv + row) * (dm.P >> 4) + (slot >> 4);
    const size_t open_at = ((size_t)s * dm.LHkv + row) * 16 * (kHeadDim / 2) + lane;
    uint32_t* const open = reinterpret_cast<uint32_t*>(values.v_open) + open_at;
    const uint32_t* source = open;
    int known = o;          // tokens of the source that count
    bool again = false;     // the scale may know of tokens that are no more
    if constexpr (HELD) {
        uint32_t* const before = reinterpret_cast<uint32_t*>(kept.before) + open_at;
        const int id = p * (dm.P >> 4) + (slot >> 4);
        int4 now{id, o + 1, held.z, held.w};
        if (held.x == id) {
            again = held.y > o;
            known = min(o, held.y);
        } else if (o > 0 && held.z == id) {
            again = true;
            known = min(o, held.w);
            source = before;
            now.z = -1;
        } else if (o > 0) {   // what the block holds is not known: it stays
            if (lane == 0) atomicOr(status, MD_DEV_BAD_ROW);
            return;
        } else {              // a new block: the open one becomes the one before it
            int front = -1;   // (unless it was taken back whole)
            if (slot > 0) front = id - 1;
            else if (np > 1) front = v.page_table[(size_t)s * dm.MP + np - 2] * (dm.P >> 4) + (dm.P >> 4) - 1;
            if (held.z < 0 || held.z != front) {
                now.z = held.x;
                now.w = held.y;
                if (held.x >= 0) {
#pragma unroll
                    for (int t = 0; t < 16; ++t) before[t * (kHeadDim / 2)] = open[t * (kHeadDim / 2)];
                }
            }
        }
        if (lane == 0) *held_at = now;
    }
    const float scale_before = o > 0 ? *scale_p : 0.0f;
    uint32_t top = top_of(mine);
    uint8_t* const codes = values.v_codes + tile;
    float own_scale = scale_of(wave_max_u32(top));
    if (o > 0 && !again && (own_scale <= scale_before || scale_before != scale_before)) {
        open[o * (kHeadDim / 2)] = mine;
        const int e = 2 * lane;   // dims e and e + 1: neighbours m, m + 1 of the same 16
        const uint32_t w = four_codes(in_scale(bf16_value((uint16_t)mine), scale_before),
                                      in_scale(bf16_value((uint16_t)(mine >> 16)), scale_before), 0.0f, 0.0f);
        uint8_t* to = codes + (e / 64) * 1024 + (o / 4) * 256 + (e % 16) * 16 + ((e / 16) % 4) * 4 + o % 4;
        to[0] = (uint8_t)w;
        to[16] = (uint8_t)(w >> 8);
        return;
    }
    uint16_t* const buf = turn[wv];
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        uint32_t w = 0u;
        if (t < known) w = source[t * (kHeadDim / 2)];
        if (t == o) w = mine;
        if (again) top = max(top, top_of(w));
        if (t == o || again || (o == 0 && t > 0)) open[t * (kHeadDim / 2)] = w;
        *reinterpret_cast<uint32_t*>(buf + t * kPitch + 2 * lane) = w;
    }
    if (again) own_scale = scale_of(wave_max_u32(top));
    wave_lds();
#pragma unroll
    for (int a = 0; a < 2; ++a) *reinterpret_cast<u32x4*>(codes + 1024 * a + 16 * lane) = block_codes(buf, a, own_scale);
    if (lane == 0) *scale_p = own_scale;
}

RowCall row_call(const Dims& dm, const View& v, const Scratch& sc, int layer, const md_row_list& rows) {
    RowCall c{};
    c.S = dm.S;
    c.L = dm.L;
    c.Hkv = dm.Hkv;
    c.P = dm.P;
    c.Pshift = dm.Pshift;
    c.MP = dm.MP;
    c.NP = dm.NP;
    c.layer = layer;
    c.quant = dm.quant;
    c.page_elems = (size_t)dm.LHkv * dm.P * kHeadDim;
    c.k_pool = v.k_pool;
    c.page_table = v.page_table;
    c.n_pages = v.n_pages;
    c.n_tokens = v.n_tokens;
    c.page_format = v.page_format;
    c.status = sc.status;
    c.row_start = rows.row_start;
    c.row_slot = rows.row_slot;
    c.n_rows = rows.n_rows;
    return c;
}

hipError_t launch(const void* fn, RowCall& c, hipStream_t st) {
    const int64_t waves = ((int64_t)c.n_rows + 15) / 16 * c.Hkv;
    void* args[] = {&c};
    return hipLaunchKernel(fn, dim3((unsigned)((waves + kWaves - 1) / kWaves)), dim3(64 * kWaves), args, 0, st);
}

}  // namespace

static hipError_t launch_append(const void* fn, const Dims& dm, const View& v, int32_t* status, const uint16_t* new_v,
                                const md_values& values, const Held& held, hipStream_t st) {
    Dims d = dm;
    View vv = v;
    md_values w = values;
    Held b = held;
    void* args[] = {&d, &vv, &new_v, &w, &b, &status};
    const dim3 grid((unsigned)((dm.LHkv + kWaves - 1) / kWaves), (unsigned)dm.S);
    return hipLaunchKernel(fn, grid, dim3(64 * kWaves), args, 0, st);
}

hipError_t launch_append_codes(const Dims& dm, const View& v, const uint16_t* new_v, const md_values& values, hipStream_t st) {
    return launch_append(reinterpret_cast<const void*>(&k_append_codes<false>), dm, v, nullptr, new_v, values, Held{}, st);
}

hipError_t launch_append_held(const Dims& dm, const View& v, const Scratch& sc, const uint16_t* new_v, const md_values& values,
                              const Held& held, hipStream_t st) {
    return launch_append(reinterpret_cast<const void*>(&k_append_codes<true>), dm, v, sc.status, new_v, values, held, st);
}

hipError_t launch_write_held(const Dims& dm, const View& v, const Scratch& sc, int layer, const md_write_args& a,
                             const Held& held, hipStream_t st) {
    RowCall c = row_call(dm, v, sc, layer, a.rows);
    c.values = a.values;
    c.held = held;
    c.k = const_cast<uint16_t*>(a.k);
    c.v = const_cast<uint16_t*>(a.v);
    c.stride = a.stride;
    return launch(a.v != nullptr && a.values.v_pool == nullptr ? reinterpret_cast<const void*>(&k_write_rows<true>)
                                                               : reinterpret_cast<const void*>(&k_write_rows<false>), c, st);
}

hipError_t launch_write_rows(const Dims& dm, const View& v, const Scratch& sc, int layer, const md_write_args& a,
                             hipStream_t st) {
    return launch_write_held(dm, v, sc, layer, a, Held{}, st);
}

hipError_t launch_read_rows(const Dims& dm, const View& v, const Scratch& sc, int layer, const md_read_args& a, hipStream_t st) {
    RowCall c = row_call(dm, v, sc, layer, a.rows);
    c.values = a.values;
    c.k = a.k;
    c.v = a.v;
    c.stride = a.stride;
    const bool codes = a.v != nullptr && a.values.v_pool == nullptr, wide = a.type == MD_F32;
    const void* fn = codes ? (wide ? reinterpret_cast<const void*>(&k_read_rows<true, true>)
                                   : reinterpret_cast<const void*>(&k_read_rows<true, false>))
                           : (wide ? reinterpret_cast<const void*>(&k_read_rows<false, true>)
                                   : reinterpret_cast<const void*>(&k_read_rows<false, false>));
    return launch(fn, c, st);
}

}  // namespace md
