// Internal interface between the host side of mla_prefill.h
// (mla_prefill_abi.cpp) and its kernels.  Not part of the public C ABI.
#pragma once

#include <cstdint>

#include <hip/hip_runtime_api.h>

#include "internal.h"

namespace mla {

// Position rotation, resolved (mla_rotation).
struct Rotation {
    const float* table;         // [num_positions][64]: 32 cosines, 32 sines
    int64_t num_positions;
    int32_t halves;             // pairs (i, i+32) instead of (2i, 2i+1)
};

// Norm and rotation on the way into a cache.  `append.positions` is always set;
// `append.prot` only under protection.
struct NormRopeArgs {
    AppendArgs append;
    Rotation rot;
    int32_t has_norm;
    const uint16_t* weight;     // bf16 [512] or null
    double eps;
    uint16_t* c_out;            // null: no dense rows
    int64_t c_out_stride;
    uint16_t* k_out;
    int64_t k_out_stride;
};

struct RopeArgs {
    Rotation rot;
    const uint16_t* q;
    int64_t q_stride_t, q_stride_h;
    const int32_t* positions;
    int32_t n, H;
    uint16_t* out;
    int64_t out_stride_t, out_stride_h;
};

struct GatherArgs {
    const uint8_t* cache;
    int64_t num_pages;
    const int32_t* block_table;
    int32_t max_pages;
    const int32_t* first;       // null: 0
    const int32_t* cu_rows;
    int32_t B, n;
    PageGeom g;                 // BF16: page_size and page_bytes only
    const int32_t* seq_lens;    // under protection
    const uint8_t* prot;
    int64_t num_prot;
    const int32_t* prot_slot;
    int32_t sink, recent;
    uint16_t* c_out;
    int64_t c_out_stride;
    uint16_t* k_out;
    int64_t k_out_stride;
};

// A work item of the expanded attention: the keys [key0, key1) of one sequence
// for one block of its query rows.  Row r of the block sees the keys below
// min(key1, seen0 + r).
struct PrefillItem {
    int32_t q_row;      // first query row (of the tensor)
    int32_t q_rows;     // rows of the block that exist
    int32_t kv_row;     // the sequence's first key row (of the tensor)
    int32_t key0, key1;
    int32_t seen0;
    int32_t part;       // partial block it writes; -1: the output itself
    int32_t seq;        // the sequence (the planner's own use)
};
// The merge of a block's partials, part0 .. part0 + num_parts - 1.
struct PrefillMerge {
    int32_t q_row, q_rows;
    int32_t part0, num_parts;
    int32_t seen0, kv_len;
    int32_t pad[2];
};
constexpr int kPrefillRecordInts = 8;
// Behind the records, where workgroups go through several items each (256 rows):
// int32 first[lists + 1], then the lists' entries, x = local head + heads * item (or
// ~x: the block's tiles are gone through from the last to the first), where
// a list is gone through by one workgroup on each XCD, for the heads of that XCD
// (heads = H / 8), or by one workgroup (heads = H) if the heads do not divide by 8.
constexpr int kListedRows = 256;
struct PrefillLists {
    int32_t lists, heads;
    int64_t entries;
};
inline PrefillLists prefill_lists(int64_t num_items, int32_t H, int32_t rows) {
    if (rows != kListedRows) return {0, 0, 0};
    const int32_t heads = H % 8 == 0 ? H / 8 : H, most = H % 8 == 0 ? 32 : 256;
    const int64_t entries = num_items * heads;
    return {static_cast<int32_t>(entries < most ? entries : most), heads, entries};
}
static_assert(sizeof(PrefillItem) == 4 * kPrefillRecordInts && sizeof(PrefillMerge) == sizeof(PrefillItem), "one record size");

constexpr int kNope = 128, kValue = 128;    // channels of a head's expanded keys and values
constexpr int kPrefillUnmasked = 1 << 30;   // seen0 of a non-causal item
constexpr int64_t kMaxHeadStride = int64_t(1) << 24;

struct HeadRows {
    const uint16_t* data;
    int64_t stride_t, stride_h;
};

struct PrefillArgs {
    const PrefillItem* items;
    const PrefillMerge* merges;
    const int32_t* first;       // lists (prefill_lists); null: an item of one head per workgroup
    int32_t num_items, num_merges, num_parts, H;
    int32_t rows;               // query rows of a workgroup
    int32_t part_rows;          // rows of a partial block: the most that a block with split keys has
    int32_t total_q, total_kv;
    HeadRows q_nope, q_rope, k_nope, k_rope, v;
    float scale_log2;           // softmax_scale * log2(e)
    uint16_t* out;
    int64_t out_stride_t, out_stride_h;
    float* lse;
    float* part_m;              // [num_parts][H][part_rows], log2 units
    float* part_l;
    float* part_o;              // [num_parts][H][part_rows][128], normalized
};

constexpr int kRowsPerWave = 32;
constexpr int64_t kPartRowBytes = kValue * 4 + 2 * 4;

hipError_t launch_norm_rope_append(const NormRopeArgs& a, bool lowbit, hipStream_t stream);
hipError_t launch_rope_queries(const RopeArgs& a, hipStream_t stream);
hipError_t launch_gather(const GatherArgs& a, bool lowbit, hipStream_t stream);
hipError_t launch_prefill(const PrefillArgs& a, hipStream_t stream);

}  // namespace mla
