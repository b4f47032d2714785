// The row operators' checks of their arguments, with a handle, on the host.
// The library's host layer is compiled in, handles are filled in by hand and
// the launchers only note what reached them, so no GPU and no HIP call is
// needed; built with AddressSanitizer and UndefinedBehaviorSanitizer
// (tests/test_rows_host.py).  Exit status 0 when every call returns what
// include/memdecay.h promises.
#include "../paper_2607_10582_amd/csrc/md_api.cpp"

#include <stdio.h>

static int fails = 0;
static int launched = 0;   // launches since the last look
static int current = 0, switches = 0;

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
hipError_t launch_append_codes(const Dims&, const View&, const uint16_t*, const md_values&, hipStream_t) { return ++launched, hipSuccess; }
hipError_t launch_write_rows(const Dims&, const View&, const Scratch&, int, const md_write_args&, hipStream_t) { return ++launched, hipSuccess; }
hipError_t launch_read_rows(const Dims&, const View&, const Scratch&, int, const md_read_args&, hipStream_t) { return ++launched, hipSuccess; }
hipError_t launch_token_values(const Dims&, const View&, const Scratch&, int, int, const md_attend_args&, const md_values&, int, int,
                               hipStream_t) {
    return ++launched, hipSuccess;
}
hipError_t launch_attend_rows(const Dims&, const View&, const Scratch&, int, int, const md_rows_args&, hipStream_t) {
    return ++launched, hipSuccess;
}
uint64_t rows_workspace(const Dims&, int) { return 12288; }
bool attend_fits(const Dims& dm) { return dm.MP < 8000; }
}  // namespace md

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

// What every call with rows refuses.
template <class A, class C>
static void row_checks(const A& a, C& call, int32_t& layer) {
    EXPECT(call(a), MD_OK);
    for (int bad : {-1, 3, INT32_MIN, INT32_MAX}) {
        layer = bad;
        EXPECT(call(a), MD_E_INVALID);
    }
    layer = 0;
    BAD(rows.row_start, nullptr);
    BAD(rows.row_start, at<int32_t>(2));
    BAD(rows.row_slot, at<int32_t>(2));
    GOOD(rows.row_slot, at<int32_t>(4));
    BAD(rows.n_rows, -1);
    BAD(rows.n_rows, INT32_MIN);
    BAD(rows.reserved, 1);
    launched = 0;
    auto none = a;
    none.rows.n_rows = 0;
    EXPECT(call(none), MD_OK);
    if (launched != 0) ++fails;
}

// What every call with values refuses (written: the call writes them).
template <class A, class C>
static void value_checks(const A& a0, C& call, bool written) {
    A a = a0;
    a.values = md_values{at<uint16_t>(0), nullptr, nullptr, nullptr};
    EXPECT(call(a), MD_OK);
    BAD(values.v_pool, nullptr);
    BAD(values.v_pool, at<uint16_t>(8));
    BAD(values.v_codes, at<uint8_t>(0));   // both forms
    BAD(values.v_scale, at<float>(0));
    BAD(values.v_open, at<uint16_t>(0));
    a.values = md_values{nullptr, at<uint8_t>(0), at<float>(1024), at<uint16_t>(2048)};
    EXPECT(call(a), MD_OK);
    BAD(values.v_codes, nullptr);
    BAD(values.v_codes, at<uint8_t>(1));
    BAD(values.v_scale, nullptr);
    BAD(values.v_scale, at<float>(4));
    BAD(values.v_open, at<uint16_t>(2));
    if (written) BAD(values.v_open, nullptr); else GOOD(values.v_open, nullptr);
}

int main() {
    md_handle_s handle{};
    md_handle h = &handle;
    handle.dm.L = 3;
    handle.dm.Hq = 12;
    handle.dm.Hkv = 2;
    handle.dm.G = 6;
    handle.dm.S = 5;
    handle.dm.MP = 100;
    handle.n_cu = 256;
    const md_values codes{nullptr, at<uint8_t>(0), at<float>(1024), at<uint16_t>(2048)};
    const md_row_list rows{at<int32_t>(0), nullptr, 7, 0};
    int32_t layer = 2;

    {   // ---- md_append_codes
        struct Args { md_values values; };
        Args a{codes};
        auto call = [&](const Args& b) { return md_append_codes(h, at<uint16_t>(0), &b.values); };
        EXPECT(call(a), MD_E_STATE);
        handle.fresh = true;
        EXPECT(call(a), MD_OK);
        EXPECT(md_append_codes(nullptr, at<uint16_t>(0), &codes), MD_E_INVALID);
        EXPECT(md_append_codes(h, nullptr, &codes), MD_E_INVALID);
        EXPECT(md_append_codes(h, at<uint16_t>(2), &codes), MD_E_INVALID);
        EXPECT(md_append_codes(h, at<uint16_t>(0), nullptr), MD_E_INVALID);
        BAD(values.v_pool, at<uint16_t>(0));
        BAD(values.v_codes, nullptr);
        BAD(values.v_scale, at<float>(2));
        BAD(values.v_open, nullptr);
        handle.dm.H = 1;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
    }
    {   // ---- md_write_rows
        auto call = [&](const md_write_args& b) { return md_write_rows(h, layer, &b); };
        md_write_args a{};
        a.rows = rows;
        a.k = at<uint16_t>(0);
        a.v = at<uint16_t>(1024);
        a.stride = 2 * 128;
        a.values = codes;
        row_checks(a, call, layer);
        value_checks(a, call, true);
        EXPECT(md_write_rows(nullptr, 0, &a), MD_E_INVALID);
        EXPECT(md_write_rows(h, 0, nullptr), MD_E_INVALID);
        BAD(k, at<uint16_t>(2));
        BAD(v, at<uint16_t>(2));
        BAD(stride, 2 * 128 - 8);
        BAD(stride, 2 * 128 + 4);
        BAD(stride, INT64_MIN);
        GOOD(k, nullptr);
        GOOD(v, nullptr);
        a.k = nullptr;
        BAD(v, nullptr);
        a.k = at<uint16_t>(0);
        a.v = nullptr;
        GOOD(values, md_values{});   // no values, no pools
        handle.dm.H = 1;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
    }
    {   // ---- md_read_rows
        auto call = [&](const md_read_args& b) { return md_read_rows(h, layer, &b); };
        md_read_args a{};
        a.rows = rows;
        a.k = at<void>(0);
        a.v = at<void>(1024);
        a.stride = 2 * 128;
        a.type = MD_F32;
        a.values = codes;
        row_checks(a, call, layer);
        value_checks(a, call, false);
        EXPECT(md_read_rows(nullptr, 0, &a), MD_E_INVALID);
        EXPECT(md_read_rows(h, 0, nullptr), MD_E_INVALID);
        BAD(k, at<void>(8));
        BAD(v, at<void>(8));
        BAD(stride, 2 * 128 - 8);
        BAD(stride, 2 * 128 + 4);
        BAD(type, MD_F16);
        BAD(type, -1);
        GOOD(type, MD_BF16);
        GOOD(k, nullptr);
        a.k = nullptr;
        BAD(v, nullptr);
        handle.dm.H = 1;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
    }
    {   // ---- md_attend_values
        struct Args {
            md_attend_args t;
            md_values values;
            int32_t window, sinks;
        };
        auto call = [&](const Args& b) { return md_attend_values(h, layer, &b.t, &b.values, b.window, b.sinks); };
        Args a{};
        a.t.q = at<float>(0);
        a.t.q_stride = 12 * 128;
        a.t.out_type = MD_BF16;
        a.t.out = at<void>(8192);
        a.t.out_stride = 12 * 128;
        a.t.workspace = at<void>(16384);
        a.values = codes;
        EXPECT(call(a), MD_OK);
        value_checks(a, call, false);
        EXPECT(md_attend_values(nullptr, 0, &a.t, &codes, 0, 0), MD_E_INVALID);
        EXPECT(md_attend_values(h, 0, nullptr, &codes, 0, 0), MD_E_INVALID);
        EXPECT(md_attend_values(h, 0, &a.t, nullptr, 0, 0), MD_E_INVALID);
        EXPECT(md_attend_values(h, 3, &a.t, &codes, 0, 0), MD_E_INVALID);
        BAD(t.q, nullptr);
        BAD(t.q_stride, 12 * 128 + 2);
        BAD(t.new_k, at<uint16_t>(0));   // without its value
        BAD(t.blocks, at<int32_t>(0));   // without counts
        BAD(t.out_type, MD_F16);
        BAD(t.out_stride, 12 * 128 - 8);
        BAD(t.workspace, nullptr);
        BAD(window, -1);
        BAD(sinks, -1);
        GOOD(window, INT32_MAX);
        GOOD(sinks, INT32_MAX);
        GOOD(t.v_pool, at<uint16_t>(2));   // not looked at
        a.t.blocks = at<int32_t>(0);
        a.t.block_count = at<int32_t>(4);
        a.t.max_blocks = 4;
        EXPECT(call(a), MD_OK);
        a.window = 1;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        a.window = 0;
        handle.dm.MP = 8000;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.MP = 100;
        handle.dm.H = 1;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
    }
    {   // ---- md_attend_rows
        auto call = [&](const md_rows_args& b) { return md_attend_rows(h, layer, &b); };
        md_rows_args a{};
        a.rows = rows;
        a.q = at<void>(0);
        a.q_stride = 12 * 128;
        a.q_type = MD_BF16;
        a.out_type = MD_BF16;
        a.out = at<void>(8192);
        a.out_stride = 12 * 128;
        a.values = codes;
        a.workspace = at<void>(16384);
        row_checks(a, call, layer);
        value_checks(a, call, false);
        EXPECT(md_attend_rows(nullptr, 0, &a), MD_E_INVALID);
        EXPECT(md_attend_rows(h, 0, nullptr), MD_E_INVALID);
        BAD(q, nullptr);
        BAD(q, at<void>(8));
        BAD(q_stride, 12 * 128 - 8);
        BAD(q_stride, 12 * 128 + 4);
        BAD(q_type, MD_F16);
        BAD(out_type, MD_F16);
        BAD(out, nullptr);
        BAD(out, at<void>(8));
        BAD(out_stride, 12 * 128 - 8);
        BAD(out_stride, 12 * 128 + 4);
        BAD(lse, at<float>(2));
        BAD(window, -1);
        BAD(sinks, -1);
        BAD(workspace, nullptr);
        BAD(workspace, at<void>(8));
        GOOD(q_type, MD_F32);
        GOOD(out_type, MD_F32);
        GOOD(lse, at<float>(4));
        GOOD(window, INT32_MAX);
        GOOD(sinks, INT32_MAX);
        a.rows.n_rows = 300000000;   // times six heads a KV head and the sessions' tiles: below 2^31
        EXPECT(call(a), MD_OK);
        a.rows.n_rows = 400000000;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        a.rows.n_rows = 7;
        handle.dm.H = 1;
        EXPECT(call(a), MD_E_UNSUPPORTED);
        handle.dm.H = 0;
    }
    uint64_t bytes = 0;
    EXPECT(md_rows_workspace(nullptr, &bytes), MD_E_INVALID);
    EXPECT(md_rows_workspace(h, nullptr), MD_E_INVALID);
    EXPECT(md_rows_workspace(h, &bytes), MD_OK);
    if (bytes != 12288) ++fails;
    if (fails == 0) printf("row operators' argument checks passed under the sanitizers\n");
    return fails == 0 ? 0 : 1;
}
