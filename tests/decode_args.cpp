// The decode operators' checks of their arguments, with a handle, on the host.
// The library's host layer is compiled in, handles are filled in by hand and
// the launchers only note what reached them, so no GPU and no HIP call is
// needed; built with AddressSanitizer and UndefinedBehaviorSanitizer
// (tests/test_decode_sanitizer.py).  Exit status 0 when every call returns what
// include/memdecay.h promises.
#include "../paper_2607_10582_amd/csrc/md_api.cpp"

#include <stdio.h>

static int fails = 0;
static int launched = 0;          // launches since the last look
static int current = 0, switches = 0;

// ---- what the host layer calls
extern "C" hipError_t hipGetDevice(int* d) {
    *d = current;
    return hipSuccess;
}
extern "C" hipError_t hipSetDevice(int d) {
    switches += d != current;
    current = d;
    return hipSuccess;
}

namespace md {
hipError_t launch_norm_rope(const Dims&, const View&, const md_rope_args&, int, hipStream_t) { return ++launched, hipSuccess; }
hipError_t launch_append_values(const Dims&, const View&, const uint16_t*, uint16_t*, hipStream_t) { return ++launched, hipSuccess; }
hipError_t launch_token(const Dims&, const View&, const Scratch&, int, int, const md_attend_args&, hipStream_t) {
    return ++launched, hipSuccess;
}
hipError_t launch_bounds(const Dims&, const View&, const Scratch&, const CodeTimes&, int, int8_t*, int8_t*, hipStream_t) {
    return ++launched, hipSuccess;
}
hipError_t launch_blocks(const Dims&, const View&, const Scratch&, int, const md_select_args&, hipStream_t) {
    return ++launched, hipSuccess;
}
uint64_t attend_workspace(const Dims&, int) { return 4096; }
uint64_t select_workspace(const Dims&) { return 8192; }
bool attend_fits(const Dims& dm) { return dm.MP < 8000; }
}  // namespace md

// A call, its status, and whether it may have launched anything.
#define EXPECT(call, want)                                                                                  \
    do {                                                                                                    \
        launched = switches = 0;                                                                            \
        current = 3;                                                                                        \
        const md_status got_ = (call);                                                                      \
        if (got_ != (want) || launched > (got_ == MD_OK) || current != 3 || switches != 2 * launched) {     \
            fprintf(stderr, "line %d: %s -> %d, expected %d (%d launches, device %d)\n", __LINE__, #call, got_, \
                    (int)(want), launched, current);                                                        \
            ++fails;                                                                                        \
        }                                                                                                   \
    } while (0)

alignas(256) static unsigned char mem[65536];   // addresses only: nothing reads them
template <class T>
static T* at(size_t byte) {
    return reinterpret_cast<T*>(mem + byte);
}

// `call` with one field changed at a time.
#define BAD(field, value)                  \
    do {                                   \
        auto b = a;                        \
        b.field = (value);                 \
        EXPECT(call(b), MD_E_INVALID);     \
    } while (0)
#define GOOD(field, value)                 \
    do {                                   \
        auto b = a;                        \
        b.field = (value);                 \
        EXPECT(call(b), MD_OK);            \
    } while (0)

int main() {
    md_handle_s handle{};
    md_handle h = &handle;
    handle.dm.L = 3;
    handle.dm.Hq = 12;
    handle.dm.Hkv = 2;
    handle.dm.S = 5;
    handle.dm.MP = 100;
    handle.n_cu = 256;
    handle.device = 0;

    {   // ---- md_norm_rope
        auto call = [&](const md_rope_args& b) { return md_norm_rope(h, &b); };
        md_rope_args a{};
        a.qkv = at<void>(0);
        a.qkv_stride = 16 * 128;
        a.qkv_type = MD_BF16;
        a.n_rows = 5;
        a.eps = 1e-6f;
        a.rope_dims = 128;
        a.inv_freq = at<double>(1024);
        a.q_out = at<float>(2048);
        a.q_stride = 12 * 128;
        a.k_out = at<uint16_t>(4096);
        a.v_out = at<uint16_t>(8192);
        a.kv_stride = 2 * 128;
        EXPECT(call(a), MD_OK);
        EXPECT(md_norm_rope(nullptr, &a), MD_E_INVALID);
        EXPECT(md_norm_rope(h, nullptr), MD_E_INVALID);
        BAD(qkv, nullptr);
        BAD(qkv, mem + 8);
        BAD(qkv_stride, 16 * 128 - 8);
        BAD(qkv_stride, 16 * 128 + 4);
        BAD(qkv_stride, INT64_MIN);
        BAD(qkv_type, -1);
        BAD(qkv_type, 3);
        BAD(n_rows, -1);
        BAD(n_rows, 4);                       // clocks of five sessions
        BAD(n_rows, 0);
        BAD(eps, -1.0f);
        BAD(eps, NAN);
        BAD(eps, INFINITY);
        BAD(rope_dims, -16);
        BAD(rope_dims, 8);
        BAD(rope_dims, 144);
        BAD(inv_freq, nullptr);
        BAD(inv_freq, at<double>(1028));
        BAD(q_weight, at<float>(2));
        BAD(k_weight, at<float>(2));
        BAD(position, at<int32_t>(2));
        BAD(interleaved, 2);
        BAD(interleaved, -1);
        BAD(q_out, nullptr);
        BAD(q_out, at<float>(2052));
        BAD(q_stride, 12 * 128 - 4);
        BAD(q_stride, 12 * 128 + 2);
        BAD(k_out, nullptr);
        BAD(k_out, at<uint16_t>(4098));
        BAD(v_out, at<uint16_t>(8194));
        BAD(kv_stride, 2 * 128 - 8);
        BAD(kv_stride, 2 * 128 + 4);
        GOOD(v_out, nullptr);
        GOOD(eps, 0.0f);
        GOOD(qkv_type, MD_F32);
        GOOD(qkv_type, MD_F16);
        GOOD(interleaved, 1);
        a.position = at<int32_t>(0);
        GOOD(n_rows, 1 << 30);
        launched = 0;
        a.n_rows = 0;
        EXPECT(call(a), MD_OK);               // nothing to do
        if (launched != 0) ++fails;
        a.rope_dims = 0;
        a.n_rows = 1;
        GOOD(inv_freq, nullptr);
    }
    {   // ---- md_append_values
        EXPECT(md_append_values(nullptr, at<uint16_t>(0), at<uint16_t>(0)), MD_E_INVALID);
        EXPECT(md_append_values(h, at<uint16_t>(0), at<uint16_t>(0)), MD_E_STATE);
        handle.fresh = true;
        EXPECT(md_append_values(h, at<uint16_t>(0), at<uint16_t>(4096)), MD_OK);
        EXPECT(md_append_values(h, nullptr, at<uint16_t>(0)), MD_E_INVALID);
        EXPECT(md_append_values(h, at<uint16_t>(0), nullptr), MD_E_INVALID);
        EXPECT(md_append_values(h, at<uint16_t>(2), at<uint16_t>(0)), MD_E_INVALID);
        EXPECT(md_append_values(h, at<uint16_t>(0), at<uint16_t>(8)), MD_E_INVALID);
        handle.dm.H = 1;
        EXPECT(md_append_values(h, at<uint16_t>(0), at<uint16_t>(0)), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
    }
    for (int sparse = 0; sparse < 2; ++sparse) {   // ---- md_attend_token
        int layer = 2;
        auto call = [&](const md_attend_args& b) { return md_attend_token(h, layer, &b); };
        md_attend_args a{};
        a.q = at<float>(0);
        a.q_stride = 12 * 128;
        a.new_k = at<uint16_t>(1024);
        a.new_v = at<uint16_t>(2048);
        a.kv_stride = 2 * 128;
        a.v_pool = at<uint16_t>(4096);
        a.out_type = MD_BF16;
        a.out = at<void>(8192);
        a.out_stride = 12 * 128;
        a.workspace = at<void>(16384);
        if (sparse) {
            a.blocks = at<int32_t>(20480);
            a.block_count = at<int32_t>(24576);
            a.max_blocks = 1;
        }
        EXPECT(call(a), MD_OK);
        EXPECT(md_attend_token(nullptr, 0, &a), MD_E_INVALID);
        EXPECT(md_attend_token(h, 0, nullptr), MD_E_INVALID);
        for (int bad : {-1, 3, INT32_MIN, INT32_MAX}) {
            layer = bad;
            EXPECT(call(a), MD_E_INVALID);
        }
        layer = 0;
        BAD(q, nullptr);
        BAD(q, at<float>(4));
        BAD(q_stride, 12 * 128 - 4);
        BAD(q_stride, 12 * 128 + 2);
        BAD(new_k, nullptr);
        BAD(new_v, nullptr);
        BAD(new_k, at<uint16_t>(1026));
        BAD(new_v, at<uint16_t>(2050));
        BAD(kv_stride, 2 * 128 - 8);
        BAD(kv_stride, 2 * 128 + 4);
        BAD(v_pool, nullptr);
        BAD(v_pool, at<uint16_t>(4098));
        BAD(out_type, MD_F16);
        BAD(out_type, -1);
        BAD(out, nullptr);
        BAD(out, mem + 8196);
        BAD(out_stride, 12 * 128 - 8);
        BAD(out_stride, 12 * 128 + 4);
        BAD(lse, at<float>(2));
        BAD(workspace, nullptr);
        BAD(workspace, mem + 8);
        GOOD(lse, at<float>(4));
        GOOD(out_type, MD_F32);
        GOOD(q_stride, INT64_MAX - 3);
        if (sparse) {
            BAD(blocks, nullptr);
            BAD(block_count, nullptr);
            BAD(blocks, at<int32_t>(20482));
            BAD(block_count, at<int32_t>(24578));
            BAD(max_blocks, 0);
            BAD(max_blocks, -1);
            BAD(max_blocks, md::kMaxPages + 1);
            GOOD(max_blocks, md::kMaxPages);
        } else {
            BAD(blocks, at<int32_t>(20480));
            BAD(block_count, at<int32_t>(24576));
            a.new_k = a.new_v = nullptr;
            GOOD(kv_stride, 0);
        }
        handle.dm.H = 1;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
        handle.dm.MP = 8000;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.MP = 100;
    }
    {   // ---- md_key_bounds
        EXPECT(md_key_bounds(h, 0, at<int8_t>(0), at<int8_t>(1)), MD_OK);
        EXPECT(md_key_bounds(h, 1, at<int8_t>(0), at<int8_t>(1)), MD_OK);
        EXPECT(md_key_bounds(nullptr, 0, at<int8_t>(0), at<int8_t>(1)), MD_E_INVALID);
        EXPECT(md_key_bounds(h, 2, at<int8_t>(0), at<int8_t>(1)), MD_E_INVALID);
        EXPECT(md_key_bounds(h, -1, at<int8_t>(0), at<int8_t>(1)), MD_E_INVALID);
        EXPECT(md_key_bounds(h, 0, nullptr, at<int8_t>(1)), MD_E_INVALID);
        EXPECT(md_key_bounds(h, 0, at<int8_t>(0), nullptr), MD_E_INVALID);
        EXPECT(md_key_bounds(h, 0, at<int8_t>(8), at<int8_t>(1)), MD_E_INVALID);
        handle.dm.H = 1;
        EXPECT(md_key_bounds(h, 0, at<int8_t>(0), at<int8_t>(1)), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
    }
    {   // ---- md_select_blocks
        int layer = 2;
        auto call = [&](const md_select_args& b) { return md_select_blocks(h, layer, &b); };
        md_select_args a{};
        a.q = at<float>(0);
        a.q_stride = 12 * 128;
        a.bounds = at<int8_t>(4096);
        a.bound_exp = at<int8_t>(8193);
        a.first = 1;
        a.last = 2;
        a.max_blocks = 3;
        a.blocks = at<int32_t>(12288);
        a.block_count = at<int32_t>(16384);
        a.workspace = at<void>(20480);
        EXPECT(call(a), MD_OK);
        EXPECT(md_select_blocks(nullptr, 0, &a), MD_E_INVALID);
        EXPECT(md_select_blocks(h, 0, nullptr), MD_E_INVALID);
        for (int bad : {-1, 3, INT32_MIN, INT32_MAX}) {
            layer = bad;
            EXPECT(call(a), MD_E_INVALID);
        }
        layer = 0;
        BAD(q, nullptr);
        BAD(q, at<float>(8));
        BAD(q_stride, 12 * 128 - 4);
        BAD(q_stride, 12 * 128 + 1);
        BAD(bounds, nullptr);
        BAD(bounds, at<int8_t>(4104));
        BAD(bound_exp, nullptr);
        BAD(first, -1);
        BAD(last, -1);
        BAD(first, 2);
        BAD(first, INT32_MAX);
        BAD(last, INT32_MAX);
        BAD(max_blocks, 2);
        BAD(max_blocks, 0);
        BAD(max_blocks, md::kMaxPages + 1);
        BAD(blocks, nullptr);
        BAD(blocks, at<int32_t>(12290));
        BAD(block_count, nullptr);
        BAD(block_count, at<int32_t>(16386));
        BAD(workspace, nullptr);
        BAD(workspace, mem + 4);
        GOOD(first, 0);
        GOOD(max_blocks, md::kMaxPages);
        handle.dm.H = 1;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
    }
    {   // ---- md_decode_workspace
        uint64_t n = 0, m = 0;
        EXPECT(md_decode_workspace(h, &n, &m), MD_OK);
        if (n != 4096 || m != 8192) ++fails;
        EXPECT(md_decode_workspace(nullptr, &n, &m), MD_E_INVALID);
        EXPECT(md_decode_workspace(h, nullptr, &m), MD_E_INVALID);
        EXPECT(md_decode_workspace(h, &n, nullptr), MD_E_INVALID);
    }
    if (fails == 0) printf("decode argument checks passed under the sanitizers\n");
    return fails == 0 ? 0 : 1;
}
