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

#include "md_decode.h"
#include "md_device.h"

namespace md {

namespace {

constexpr int kTokWaves = 4;
constexpr int kTokThreads = 64 * kTokWaves;
constexpr int kTilesPerStep = 2;   // tiles of 16 tokens whose values meet in one product of 32

struct Desc {       // one 16-token tile, per lane
    int phys;       // page
    int live;       // tokens of it that count, 0 .. 16; -1: the new token
    int quant;      // its keys are 8-bit codes
};

struct Row {
    int s, kv, np, nt;   // session, KV head, pages and slots in use
    int tiles;           // 16-token tiles to walk
    int count;           // list entries (sparse)
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

template <bool SPARSE, bool QT>
__device__ __forceinline__ Desc tile_desc(const Dims& dm, const View& v, const TokenCall& c, const Row& r, int t,
                                          int& status) {
    Desc d{0, 0, 0};
    if (t >= r.tiles) {
        if (t == r.tiles && c.new_k != nullptr) d.live = -1;
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

// One part of one row.  SPARSE: pages from the call's lists; QT: pages may
// hold 8-bit codes.
template <bool SPARSE, bool QT>
__global__ void __launch_bounds__(kTokThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
k_token(Dims dm, View v, Scratch sc, TokenCall c) {
    __shared__ __align__(16) f32x4 acc_lds[kTokWaves][8][64];
    __shared__ float2 stat_lds[kTokWaves][16];
    const int lane = lane_id(), wv = threadIdx.x >> 6;
    const int h = lane & 15, g = lane >> 4;
    Row r;
    r.s = blockIdx.x / dm.Hkv;
    r.kv = blockIdx.x % dm.Hkv;
    r.np = v.n_pages[r.s];
    r.nt = v.n_tokens[r.s];
    int status = 0;
    const bool ok = counters_ok(r.np, r.nt, dm);
    if (!ok) {
        status = kDevCorrupt;
        r.np = r.nt = 0;
    }
    if constexpr (SPARSE) {
        r.count = c.block_count[(size_t)r.s * dm.Hkv + r.kv];
        if (r.count < 0 || r.count > c.max_blocks) {
            status |= MD_DEV_BAD_BLOCK;
            r.count = min(max(r.count, 0), c.max_blocks);
        }
        r.tiles = ok ? r.count * (dm.P >> 4) : 0;
    } else {
        r.tiles = (r.nt + 15) >> 4;
    }
    const int all = r.tiles + (c.new_k != nullptr && ok ? 1 : 0);
    // this part's tiles, in steps of two; the waves take steps in turn
    const int steps = (all + kTilesPerStep - 1) / kTilesPerStep;
    const int part = blockIdx.y;
    const int s0 = (int)((int64_t)steps * part / c.splits), s1 = (int)((int64_t)steps * (part + 1) / c.splits);

    // the head's query: three bf16 terms, exactly
    u32x4 bq[3][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f32x4 a[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
        if (h < dm.G) {
            const f32x4* qp = reinterpret_cast<const f32x4*>(c.q + (int64_t)r.s * c.q_stride +
                                                             (r.kv * dm.G + h) * kHeadDim + 32 * j + 8 * g);
            a[0] = qp[0];
            a[1] = qp[1];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t t0[3], t1[3];
            split3(a[i >> 1][2 * (i & 1)], t0[0], t0[1], t0[2]);
            split3(a[i >> 1][2 * (i & 1) + 1], t1[0], t1[1], t1[2]);
#pragma unroll
            for (int k = 0; k < 3; ++k) bq[k][j][i] = t0[k] | (t1[k] << 16);
        }
    }

    const size_t tile_row = ((size_t)c.layer * dm.Hkv + r.kv) * dm.P * kHeadDim;   // elements into a page
    const size_t page_elems = (size_t)dm.LHkv * dm.P * kHeadDim;
    float m = -INFINITY, l = 0.0f;
    f32x4 o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int st0 = s0 + wv; st0 < s1; st0 += 32 * kTokWaves) {
        // descriptors of this wave's next 64 tiles: lane 2 k + u holds tile u of its k-th step
        const int mine = st0 + (lane >> 1) * kTokWaves;
        Desc d{0, 0, 0};
        if (mine < s1) d = tile_desc<SPARSE, QT>(dm, v, c, r, mine * kTilesPerStep + (lane & 1), status);
        const int n = min(32, (s1 - st0 + kTokWaves - 1) / kTokWaves);
        for (int k = 0; k < n; ++k) {
            u32x4 kt[2][4], vt[2][4];
            float qsc[2] = {1.0f, 1.0f};
            int live[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int phys = __builtin_amdgcn_readlane(d.phys, 2 * k + u);
                live[u] = __builtin_amdgcn_readlane(d.live, 2 * k + u);
                if (live[u] < 0) {   // the new token: every lane reads its dims, the other tokens count nothing
                    const uint16_t* nk = c.new_k + (int64_t)r.s * c.kv_stride + r.kv * kHeadDim;
                    const uint16_t* nv = c.new_v + (int64_t)r.s * c.kv_stride + r.kv * kHeadDim;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        kt[u][j] = *reinterpret_cast<const u32x4*>(nk + 32 * j + 8 * g);
                        vt[u][j] = u32x4{nv[32 * j + h], 0u, nv[32 * j + 16 + h], 0u};
                    }
                    live[u] = 1;
                } else {
                    const int t = (st0 + k * kTokWaves) * kTilesPerStep + u;
                    const size_t at = (size_t)phys * page_elems + tile_row + (size_t)(t & ((dm.P >> 4) - 1)) * 16 * kHeadDim;
                    const u32x4* kp = reinterpret_cast<const u32x4*>(v.k_pool + at) + lane;
                    const u32x4* vp = reinterpret_cast<const u32x4*>(c.v_pool + at) + lane;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        kt[u][j] = kp[64 * j];
                        vt[u][j] = vp[64 * j];
                    }
                    if constexpr (QT) {
                        if (__builtin_amdgcn_readlane(d.quant, 2 * k + u)) {
                            qsc[u] = *reinterpret_cast<const float*>(reinterpret_cast<const uint8_t*>(v.k_pool + at) + 2048);
                            kt[u][3] = codes_to_bf16<1>(kt[u][1]);
                            kt[u][2] = codes_to_bf16<0>(kt[u][1]);
                            kt[u][1] = codes_to_bf16<1>(kt[u][0]);
                            kt[u][0] = codes_to_bf16<0>(kt[u][0]);
                        }
                    }
                }
            }
            f32x4 x[2];
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        x[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kt[u][j]),
                                                                       __builtin_bit_cast(bf16x8, bq[i][j]), x[u], 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[u][i] = 4 * g + i < live[u] ? x[u][i] * (QT ? kLogitScale * qsc[u] : kLogitScale) : -INFINITY;
                    mx = fmaxf(mx, x[u][i]);
                }
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            if (__any(mx > m)) {
                const float mn = fmaxf(m, mx);
                const float f = mn == -INFINITY ? 1.0f : hw_exp2(m - mn);
                l *= f;
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] *= f;
                m = mn;
            }
            const float ms = m == -INFINITY ? 0.0f : m;
            uint32_t ph[4], pl[4];   // weights as two bf16 terms
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[i] = hw_exp2(x[u][i] - ms);
                    l += p[i];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t w = pack_bf16(p[2 * i], p[2 * i + 1]);
                    ph[2 * u + i] = w;
                    pl[2 * u + i] = pack_bf16(p[2 * i] - bf16_lo(w), p[2 * i + 1] - bf16_hi(w));
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
        }
    }
    if (status != 0) atomicOr(sc.status, status);

    // the waves' results meet
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) stat_lds[wv][h] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc_lds[wv][i][lane] = o[i];
    __syncthreads();
    const int hh = threadIdx.x >> 4, e8 = threadIdx.x & 15;   // head, dims 8 e8 .. 8 e8 + 7
    if (hh >= dm.G) return;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kTokWaves; ++w) M = fmaxf(M, stat_lds[w][hh].x);
    float L = 0.0f, y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kTokWaves; ++w) {
        const float2 st = stat_lds[w][hh];
        const float f = M == -INFINITY ? 0.0f : hw_exp2(st.x - M);
        L = fmaf(st.y, f, L);
        // dim 8 e8 + i: tile e8 / 2, rows 8 (e8 & 1) + i, lane group (row / 4)
#pragma unroll
        for (int q4 = 0; q4 < 2; ++q4) {
            const f32x4 a = acc_lds[w][e8 >> 1][(2 * (e8 & 1) + q4) * 16 + hh];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[4 * q4 + i] = fmaf(a[i], f, y[4 * q4 + i]);
        }
    }
    if (c.splits == 1) {
        const float inv = L > 0.0f ? 1.0f / L : L == 0.0f ? 0.0f : L;
        const int64_t at = (int64_t)r.s * c.out_stride + (r.kv * dm.G + hh) * kHeadDim + 8 * e8;
        if (c.out_bf16) {
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(c.out) + at) =
                u32x4{pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv),
                      pack_bf16(y[4] * inv, y[5] * inv), pack_bf16(y[6] * inv, y[7] * inv)};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) static_cast<float*>(c.out)[at + i] = y[i] * inv;
        }
        if (c.lse != nullptr && e8 == 0)
            c.lse[(size_t)r.s * dm.Hq + r.kv * dm.G + hh] = (M + log2f(L)) * 0.69314718055994530942f;
        return;
    }
    float* out = c.part + (((size_t)blockIdx.x * c.splits + part) * dm.G + hh) * kPartWords;
#pragma unroll
    for (int i = 0; i < 8; ++i) out[8 * e8 + i] = y[i];
    if (e8 == 0) {
        out[kHeadDim] = M;
        out[kHeadDim + 1] = L;
    }
}

// One workgroup per query head of a session: joins its row's parts.
__global__ void __launch_bounds__(kHeadDim) k_join(Dims dm, TokenCall c) {
    const int s = blockIdx.x / dm.Hq, head = blockIdx.x % dm.Hq;
    const int e = threadIdx.x;
    const float* p = c.part + (((size_t)s * dm.Hkv + head / dm.G) * c.splits * dm.G + head % dm.G) * kPartWords;
    const size_t stride = (size_t)dm.G * kPartWords;
    float M = -INFINITY;
    for (int i = 0; i < c.splits; ++i) M = fmaxf(M, p[i * stride + kHeadDim]);
    float L = 0.0f, y = 0.0f;
    for (int i = 0; i < c.splits; ++i) {
        const float f = M == -INFINITY ? 0.0f : hw_exp2(p[i * stride + kHeadDim] - M);
        L = fmaf(p[i * stride + kHeadDim + 1], f, L);
        y = fmaf(p[i * stride + e], f, y);
    }
    y *= L > 0.0f ? 1.0f / L : L == 0.0f ? 0.0f : L;
    const int64_t at = (int64_t)s * c.out_stride + (int64_t)head * kHeadDim + e;
    if (c.out_bf16) static_cast<__bf16*>(c.out)[at] = (__bf16)y;
    else static_cast<float*>(c.out)[at] = y;
    if (c.lse != nullptr && e == 0) c.lse[(size_t)s * dm.Hq + head] = (M + log2f(L)) * 0.69314718055994530942f;
}

}  // namespace

// Parts of a row: two workgroups per CU over all rows, none without at least
// eight tiles at the page table's capacity.
int attend_splits(const Dims& dm, int n_cu) {
    const int rows = dm.S * dm.Hkv;
    const int64_t tiles = (int64_t)dm.MP * dm.P / 16 + 1;
    const int64_t most = (tiles + 7) / 8;
    const int64_t want = (2 * n_cu + rows - 1) / rows;
    return (int)(want < most ? want : most);
}

uint64_t attend_workspace(const Dims& dm, int n_cu) {
    return (uint64_t)dm.S * dm.Hkv * attend_splits(dm, n_cu) * dm.G * kPartWords * sizeof(float);
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
    hipError_t e = hipLaunchKernel(fn, dim3((unsigned)(dm.S * dm.Hkv), (unsigned)c.splits), dim3(kTokThreads), args, 0, st);
    if (e != hipSuccess || c.splits == 1) return e;
    void* jargs[] = {&d, &cc};
    return hipLaunchKernel(reinterpret_cast<const void*>(&k_join), dim3((unsigned)(dm.S * dm.Hq)), dim3(kHeadDim), jargs, 0,
                           st);
}

}  // namespace md
