// Launchers of the decode operators: head preparation, attention over the
// paged cache, page bounds and page selection.
#pragma once

#include "md_internal.h"

namespace md {

constexpr int kMinExp = -100, kMaxExp = 100;   // exponents of bounds and query codes

// What one call of the attention over the cache reads and writes: the parts
// of the handle's dimensions and view that it needs (a few scalar registers,
// not three structs' worth), and the call's arrays.
struct TokenCall {
    int S, Hq, Hkv, G, P, Pshift, MP, NP, aligned;
    int layer;
    size_t page_elems;      // elements of a page's keys, and of its values
    const uint16_t* k_pool;
    const uint8_t* region;
    const int32_t* page_table;
    const int32_t* n_pages;
    const int32_t* n_tokens;
    const uint8_t* page_format;
    int32_t* status;
    const float* q;
    int64_t q_stride;
    const uint16_t* new_k;
    const uint16_t* new_v;
    int64_t kv_stride;
    const uint16_t* v_pool;
    const int32_t* blocks;
    const int32_t* block_count;
    int max_blocks;
    int out_bf16;
    void* out;
    int64_t out_stride;
    float* lse;
    int units;      // workgroups
    int32_t* count; // [3 units] arrivals (zero between launches)
    float* part;    // [units][2][G][kPartWords] partial results
};

// Partial result of one query head: unnormalised sums of the 128 dims, then
// the maximum (base 2) and the sum of the weights.
constexpr int kPartWords = kHeadDim + 4;

uint64_t attend_workspace(const Dims& dm, int n_cu);
// Whether the sessions' rows at the page tables' capacity can be counted in
// steps (int32).
bool attend_fits(const Dims& dm);
hipError_t launch_token(const Dims& dm, const View& v, const Scratch& sc, int n_cu, int layer, const md_attend_args& a,
                        hipStream_t st);

hipError_t launch_norm_rope(const Dims& dm, const View& v, const md_rope_args& a, int n_cu, hipStream_t st);
hipError_t launch_append_values(const Dims& dm, const View& v, const uint16_t* new_v, uint16_t* v_pool,
                                hipStream_t st);

// md_key_bounds after a step: tiles (layer, KV head) of one workgroup.
constexpr int kBoundGroup = 4;
inline __host__ __device__ int bound_groups(const Dims& dm) { return (dm.LHkv + kBoundGroup - 1) / kBoundGroup; }

// Quantised tier: when pages became codes, and when the bounds of their keys
// were last looked after.  Behind the handle's scratch, zero at first; NULL
// where there is no room or no md_key_bounds (offload tier).
struct CodeTimes {
    uint32_t* coded_at;   // [NP] each page's conversion (0: none)
    uint32_t* last;       // [S][2] each session's last conversion, and its last tier pass
    uint32_t* looked;     // [S][bound_groups] md_key_bounds' last look at the session, by its workgroup
};
size_t code_times_bytes(const Dims& dm);
CodeTimes code_times_carve(const Dims& dm, void* base);
// Time in half steps: twice the steps observed before the step's conversions,
// one more from then on.  This is the conversions'.
__device__ __forceinline__ uint32_t code_time(const Scratch& sc) { return 2u * (uint32_t)sc.counters[1] + 1u; }
// The quantised tier's pass that notes its conversions.
hipError_t launch_quant(const Dims& dm, const View& v, const Scratch& sc, const CodeTimes& ct, const int32_t* ev_serial,
                        const int32_t* ev_count, hipStream_t st);

hipError_t launch_bounds(const Dims& dm, const View& v, const Scratch& sc, const CodeTimes& ct, int all, int8_t* bounds,
                         int8_t* bound_exp, hipStream_t st);
uint64_t select_workspace(const Dims& dm);
hipError_t launch_blocks(const Dims& dm, const View& v, const Scratch& sc, int layer, const md_select_args& a,
                         hipStream_t st);

}  // namespace md
