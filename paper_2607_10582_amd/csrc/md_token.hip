// gfx950 kernels that prepare a decode step's heads: norms of the query and
// key heads with the rotation by position in the same pass, and the values of
// the appended tokens.
//
// Norm and rotation read each element once and write it once, a few dozen
// operations in between, so a long prompt is bound by HBM and a decode step
// (a row per session) by the launch and one chain of loads.

#include <algorithm>
#include <type_traits>

#include "md_decode.h"
#include "md_device.h"

namespace md {

namespace {

constexpr int kRopeWaves = 4;   // waves per workgroup

struct RopeCall {
    const void* qkv;
    int64_t qkv_stride;
    const float* q_weight;
    const float* k_weight;
    const double* inv_freq;
    const int32_t* position;
    float* q_out;
    uint16_t* k_out;
    uint16_t* v_out;
    int64_t q_stride, kv_stride;
    float eps;
    int n_rows, rot, Hq, Hkv, heads;   // heads a row has to write: Hq + Hkv, + Hkv with v_out
    int parts;                         // waves per row
};

// Eight elements of a head (dims 8 m .. 8 m + 7 of lane m of 16) as float32.
template <int TYPE>
__device__ __forceinline__ void load8(const void* p, int64_t at, float (&x)[8]) {
    if constexpr (TYPE == MD_F32) {
        const f32x4* s = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
        const f32x4 a = s[0], b = s[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    } else {
        const u32x4 a = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == MD_BF16) {
                x[2 * i] = __uint_as_float(a[i] << 16);
                x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
            } else {
                x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)a[i]);
                x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(a[i] >> 16));
            }
        }
    }
}

// Round to bf16 (nearest, ties to even), two values in a word.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((__vector_size__(4)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    *reinterpret_cast<u32x4*>(p) = u32x4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]),
                                         bf16_pair(x[6], x[7])};
}

// Sum over the 16 lanes of a row (each lane gets it): rotations by 8, 4, 2, 1.
__device__ __forceinline__ float row_sum(float v) {
    auto add = [&](auto step) {
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + step, 0xf, 0xf, false));
    };
    add(std::integral_constant<int, 8>{});
    add(std::integral_constant<int, 4>{});
    add(std::integral_constant<int, 2>{});
    add(std::integral_constant<int, 1>{});
    return v;
}

// A wave takes one row, or one of `parts` of its heads, four heads at a time:
// 16 lanes a head, eight consecutive elements each (16-byte loads of 16-bit
// types).  Lane i works out the cosine and sine of frequency i once (in
// turns, reduced in float64: a float32 product of a position of a million is
// off by up to 0.03 radian, of ten millions by up to 0.5), and the row's heads share them through LDS.  The
// halves that turn together sit rot / 16 lanes apart.
template <int TYPE, bool PAIRS>
__global__ void __launch_bounds__(64 * kRopeWaves) k_norm_rope(RopeCall c, const int32_t* __restrict__ clock) {
    __shared__ __align__(16) float2 turn_lds[kRopeWaves][64];
    const int lane = lane_id(), wv = threadIdx.x >> 6;
    const int64_t task = (int64_t)blockIdx.x * kRopeWaves + wv;
    const int row = (int)(task / c.parts), part = (int)(task % c.parts);
    if (row >= c.n_rows) return;
    float2* turn = turn_lds[wv];
    const int half = c.rot / 2;
    const int m = lane & 15;
    float x[8];
    auto load_head = [&](int h) {
        load8<TYPE>(c.qkv, (int64_t)row * c.qkv_stride + (int64_t)min(h, c.heads - 1) * kHeadDim + 8 * m, x);
    };
    load_head(4 * part + (lane >> 4));   // under way while the angles are worked out
    if (lane < half) {
        const int pos = c.position != nullptr ? c.position[row] : clock[row];
        const double t = (double)pos * (c.inv_freq[lane] * 0.15915494309189533577);   // turns
        const float f = (float)(2.0 * (t - rint(t)));                                  // half turns in [-1, 1]
        float sn, cs;
        sincospif(f, &sn, &cs);
        turn[lane] = make_float2(cs, sn);
    }
    __builtin_amdgcn_wave_barrier();
    // frequencies of this lane's elements: dims 8 m + e, or pairs 4 m + e / 2
    const bool turns = 8 * m < c.rot;
    const bool upper = 8 * m >= half;
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = PAIRS ? 4 * m + e / 2 : (8 * m + e) - (upper ? half : 0);
        const float2 t = turns ? turn[i] : make_float2(1.0f, 0.0f);
        cs[e] = t.x;
        // the first of a pair loses the sine times the second, the second gains it times the first
        sn[e] = (PAIRS ? (e & 1) == 0 : !upper) ? -t.y : t.y;
    }
    const int partner = (lane & 48) | (turns ? (upper ? m - half / 8 : m + half / 8) : m);
    for (int h0 = 4 * part; h0 < c.heads; h0 += 4 * c.parts) {
        const int h = h0 + (lane >> 4);
        const bool ok = h < c.heads;
        if (h0 != 4 * part) load_head(h);
        const bool value = h >= c.Hq + c.Hkv;
        const float* w = h < c.Hq ? c.q_weight : c.k_weight;
        if (!value && w != nullptr) {
            float ss = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
            const float r = 1.0f / sqrtf(row_sum(ss) * (1.0f / kHeadDim) + c.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] * r * w[8 * m + e];
        }
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float o = PAIRS ? x[e ^ 1] : __shfl(x[e], partner);
            // elements that do not turn are passed on as they are (an infinite
            // neighbour would make 0 times it a NaN)
            y[e] = value || !turns ? x[e] : fmaf(x[e], cs[e], o * sn[e]);
        }
        if (!ok) continue;
        if (h < c.Hq) {
            f32x4* o = reinterpret_cast<f32x4*>(c.q_out + (int64_t)row * c.q_stride + h * kHeadDim + 8 * m);
            o[0] = f32x4{y[0], y[1], y[2], y[3]};
            o[1] = f32x4{y[4], y[5], y[6], y[7]};
        } else if (!value) {
            store8(c.k_out + (int64_t)row * c.kv_stride + (h - c.Hq) * kHeadDim + 8 * m, y);
        } else {
            store8(c.v_out + (int64_t)row * c.kv_stride + (h - c.Hq - c.Hkv) * kHeadDim + 8 * m, y);
        }
    }
}

// One workgroup per (session, 256 elements of the token's values).  The
// token that the step appended is the session's last, inserted at its clock;
// a session that took none has an older token there, or none at all.  Bound by
// the launch and the chain of counters, page table and insertion time: behind
// a step's observation 5.3 us for 32 sessions of 36 layers and two KV heads, 3.9
// for one of 28 (called again and again 3.5 and 3.0).
__global__ void __launch_bounds__(256) k_append_values(Dims dm, View v, const uint16_t* __restrict__ new_v,
                                                       uint16_t* __restrict__ v_pool) {
    const int s = blockIdx.y;
    const int np = v.n_pages[s], nt = v.n_tokens[s];
    if (!counters_ok(np, nt, dm) || np == 0) return;
    const int p = v.page_table[(size_t)s * dm.MP + np - 1];
    if ((unsigned)p >= (unsigned)dm.NP) return;
    const int t = nt - 1 - (np - 1) * dm.P;
    if (v.t_ins[(size_t)p * dm.P + t] != v.clock[s]) return;
    const int i = blockIdx.x * 256 + threadIdx.x;   // (layer, KV head, element)
    if (i >= dm.LHkv * kHeadDim) return;
    const int row = i / kHeadDim, e = i % kHeadDim;
    const size_t tile = ((size_t)p * dm.LHkv + row) * dm.P * kHeadDim;
    v_pool[tile + (size_t)(t & ~15) * kHeadDim + (e / 32) * 512 + ((t / 4) % 4) * 128 + (e % 16) * 8 +
           ((e / 16) % 2) * 4 + t % 4] = new_v[((size_t)s * dm.LHkv) * kHeadDim + i];
}

template <int TYPE>
const void* rope_kernel(bool pairs) {
    return pairs ? reinterpret_cast<const void*>(&k_norm_rope<TYPE, true>)
                 : reinterpret_cast<const void*>(&k_norm_rope<TYPE, false>);
}

}  // namespace

hipError_t launch_norm_rope(const Dims& dm, const View& v, const md_rope_args& a, int n_cu, hipStream_t st) {
    RopeCall c{};
    c.qkv = a.qkv;
    c.qkv_stride = a.qkv_stride;
    c.q_weight = a.q_weight;
    c.k_weight = a.k_weight;
    c.inv_freq = a.inv_freq;
    c.position = a.position;
    c.q_out = a.q_out;
    c.k_out = a.k_out;
    c.v_out = a.v_out;
    c.q_stride = a.q_stride;
    c.kv_stride = a.kv_stride;
    c.eps = a.eps;
    c.n_rows = a.n_rows;
    c.rot = a.rope_dims;
    c.Hq = dm.Hq;
    c.Hkv = dm.Hkv;
    c.heads = dm.Hq + dm.Hkv * (a.v_out != nullptr ? 2 : 1);
    // Few rows: a wave per four heads, so that the chain of loads is walked
    // once (32 rows of 20 heads: 3.3 us, a wave a row 5.7; 512: 4.4 and 6.7);
    // many: a wave per row, which works the angles out once (32,768 rows of 16
    // heads: 78 - 80 us either way, HBM at a copy's rate).
    const int64_t most = (c.heads + 3) / 4;
    c.parts = (int)std::max<int64_t>(1, std::min<int64_t>(most, 16 * (int64_t)n_cu / a.n_rows));
    const void* fn = a.qkv_type == MD_F32    ? rope_kernel<MD_F32>(a.interleaved != 0)
                     : a.qkv_type == MD_BF16 ? rope_kernel<MD_BF16>(a.interleaved != 0)
                                             : rope_kernel<MD_F16>(a.interleaved != 0);
    const int32_t* clock = v.clock;
    void* args[] = {&c, &clock};
    const int64_t tasks = (int64_t)a.n_rows * c.parts;
    return hipLaunchKernel(fn, dim3((unsigned)((tasks + kRopeWaves - 1) / kRopeWaves)), dim3(64 * kRopeWaves), args, 0, st);
}

hipError_t launch_append_values(const Dims& dm, const View& v, const uint16_t* new_v, uint16_t* v_pool,
                                hipStream_t st) {
    Dims d = dm;
    View vv = v;
    void* args[] = {&d, &vv, &new_v, &v_pool};
    const dim3 grid((unsigned)((dm.LHkv * kHeadDim + 255) / 256), (unsigned)dm.S);
    return hipLaunchKernel(reinterpret_cast<const void*>(&k_append_values), grid, dim3(256), args, 0, st);
}

}  // namespace md
