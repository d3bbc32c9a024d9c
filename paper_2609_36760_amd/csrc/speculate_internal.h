// Internal interface between the host side of mla_speculate.h
// (mla_speculate_abi.cpp) and its kernels.  Not part of the public C ABI.
#pragma once

#include <cstdint>

#include <hip/hip_runtime_api.h>

#include "internal.h"

namespace mla {

constexpr int kMaxNodes = 64;       // of one sequence's tree: the bits of a mask

// Attention of trees.  In the base: s_q the most nodes of a sequence, seq_lens
// the contexts' lengths, shape 64 or 128 rows of four waves.
struct TreeArgs : DecodeArgs {
    const int32_t* cu_nodes;        // [B + 1] first node of every sequence
    const uint64_t* mask;           // [num_nodes] nodes of its sequence that a node sees
    int32_t num_nodes;              // rows of the node-indexed arrays
};

// Merge of its split partials (rows of a split: s_q * H).
struct TreeCombineArgs : CombineArgs {
    const int32_t* cu_nodes;
    int32_t num_nodes;
    int32_t num_splits;
};

// Verification of drafted tokens (verify.hip).
constexpr int kLogitChunk = 2048;               // logits of one wave's statistics
constexpr int32_t kMaxVocab = 1 << 21;
constexpr int logit_chunks(int32_t vocab) { return (vocab + kLogitChunk - 1) / kLogitChunk; }
struct ChunkStat {                              // of one chunk of a row
    double sum;                                 // of e^((l - max) / T); at temperature 0 the first index of the maximum
    float max;                                  // NaN or inf: the row cannot be used
    float unused;
};
struct VerifyArgs {
    const void* logits;
    int64_t logits_stride;
    int32_t fp32;                               // type of the logits
    int32_t vocab;
    const float* draft_probs;
    int64_t draft_stride;
    const int32_t* tokens;
    const int32_t* parents;
    const int32_t* cu_nodes;
    int32_t num_nodes, max_nodes, B;
    const float* temperature;
    const float* u_accept;
    const float* u_draw;
    int32_t* path;
    int32_t* out_tokens;
    float* logprobs;
    int32_t* keep;
    ChunkStat* stats;                           // [num_nodes][chunks]
    double* sums;                               // [B][chunks] of a shared pass
    int32_t* arrived;                           // [B] workgroups that have done their share of it
};

// Commit (commit.hip).
struct CommitArgs {
    uint8_t* const* caches;
    int32_t num_layers;
    int64_t num_pages;
    const int32_t* block_table;
    int32_t max_pages;
    const int32_t* ctx_lens;
    const int32_t* path;
    const int32_t* keep;
    int32_t max_nodes, B;
    int32_t* new_lens;
    PageGeom g;
    int32_t layers_each;                        // layers of a workgroup (set by the launch)
};

// Its workgroups go round the 8 XCDs in runs: the row blocks of a split where they
// are up to 8, else an even part of them of at most 8.
#if defined(__HIPCC__)
__host__ __device__
#endif
constexpr int tree_run(int row_blocks) {
    if (row_blocks <= 2) return 4;
    const int parts = (row_blocks + 7) / 8;
    return (row_blocks + parts - 1) / parts;
}
// Workgroups of its launch: padded to whole rounds of runs.
constexpr int64_t tree_workgroups(int64_t num_work, int64_t rows, int64_t rows_per_block) {
    const int64_t blocks = (rows + rows_per_block - 1) / rows_per_block, round = 8 * tree_run(static_cast<int>(blocks));
    return (num_work * blocks + round - 1) / round * round;
}

// The nodes of sequence b, kept inside the node-indexed arrays for any values.
struct NodeRange {
    int32_t first, count;
};
#if defined(__HIPCC__)
__host__ __device__
#endif
inline NodeRange node_range(const int32_t* cu_nodes, int32_t b, int32_t num_nodes, int32_t max_nodes) {
    const int32_t c0 = cu_nodes[b], c1 = cu_nodes[b + 1];
    const int32_t first = c0 < 0 ? 0 : c0 < num_nodes ? c0 : num_nodes;
    const int32_t end = c1 < first ? first : c1 < num_nodes ? c1 : num_nodes;
    return {first, end - first < max_nodes ? end - first : max_nodes};
}

hipError_t launch_tree_attn(CacheKind kind, const TreeArgs& a, hipStream_t stream);
hipError_t launch_tree_combine(const TreeCombineArgs& a, hipStream_t stream);
hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream);
hipError_t launch_commit(const CommitArgs& a, bool lowbit, hipStream_t stream);

}  // namespace mla
