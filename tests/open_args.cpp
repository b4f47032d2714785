// md_open_blocks on the host: its checks, and which launchers the calls that
// write reach with and without it.  Built like tests/rows_args.cpp, whose stubs
// and checks it takes (tests/test_rows_sessions_host.py).
#define main rows_main
#include "rows_args.cpp"
#undef main

static int held = 0;   // launches that got what the open blocks hold

namespace md {
hipError_t launch_append_held(const Dims&, const View&, const Scratch&, const uint16_t*, const md_values&, const Held& h, hipStream_t) {
    if (h.before != at<uint16_t>(4096) || h.at != at<int32_t>(8192)) ++fails;
    return ++held, ++launched, hipSuccess;
}
hipError_t launch_write_held(const Dims&, const View&, const Scratch&, int, const md_write_args&, const Held& h, hipStream_t) {
    if (h.before != at<uint16_t>(4096) || h.at != at<int32_t>(8192)) ++fails;
    return ++held, ++launched, hipSuccess;
}
}  // namespace md

int main() {
    md_handle_s handle{};
    md_handle h = &handle;
    handle.dm.L = 3;
    handle.dm.Hq = 12;
    handle.dm.Hkv = 2;
    handle.dm.S = 5;
    handle.fresh = true;
    const md_values codes{nullptr, at<uint8_t>(0), at<float>(1024), at<uint16_t>(2048)};
    md_write_args a{};
    a.rows = md_row_list{at<int32_t>(0), nullptr, 7, 0};
    a.k = a.v = at<uint16_t>(0);
    a.stride = 2 * 128;
    a.values = codes;
    auto writes = [&](int want) {   // how many of them reach the launchers with the blocks
        held = 0;
        EXPECT(md_write_rows(h, 0, &a), MD_OK);
        EXPECT(md_append_codes(h, at<uint16_t>(0), &codes), MD_OK);
        if (held != want) {
            fprintf(stderr, "%d launches with the blocks, expected %d\n", held, want);
            ++fails;
        }
    };
    auto call = [&](uint16_t* before, int32_t* at_) { return md_open_blocks(h, before, at_); };
    writes(0);
    EXPECT(call(at<uint16_t>(4096), nullptr), MD_E_INVALID);
    EXPECT(call(nullptr, at<int32_t>(8192)), MD_E_INVALID);
    EXPECT(call(at<uint16_t>(4098), at<int32_t>(8192)), MD_E_INVALID);
    EXPECT(call(at<uint16_t>(4096), at<int32_t>(8196)), MD_E_INVALID);
    EXPECT(md_open_blocks(nullptr, at<uint16_t>(4096), at<int32_t>(8192)), MD_E_INVALID);
    handle.dm.H = 1;
    EXPECT(call(at<uint16_t>(4096), at<int32_t>(8192)), MD_E_UNSUPPORTED);
    handle.dm.H = 0;
    writes(0);
    if (call(at<uint16_t>(4096), at<int32_t>(8192)) != MD_OK) ++fails;
    writes(2);
    held = 0;
    md_write_args b = a;   // bf16 values, and keys alone, have none
    b.values = md_values{at<uint16_t>(0), nullptr, nullptr, nullptr};
    EXPECT(md_write_rows(h, 0, &b), MD_OK);
    b = a;
    b.v = nullptr;
    EXPECT(md_write_rows(h, 0, &b), MD_OK);
    if (held != 0) ++fails;
    if (call(nullptr, nullptr) != MD_OK) ++fails;
    writes(0);
    if (fails == 0) printf("open blocks passed under the sanitizers\n");
    return fails == 0 ? 0 : 1;
}
