// Host side of the C ABI declared in include/mla_speculate.h: argument
// validation, the choice of a split size, workspace layout and dispatch.
//
// This translation unit is plain C++ (it needs only the HIP runtime API
// types); every check below runs on the host before any HIP call is made.
#include "mla_speculate.h"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <exception>
#include <functional>
#include <queue>
#include <vector>

#include "abi_checks.h"
#include "internal.h"
#include "speculate_internal.h"

namespace {

using namespace mla::abi;

constexpr int64_t kMaxRows = int64_t{1} << 20;          // of one sequence: 32-bit byte offsets in the kernel
constexpr int64_t kMaxTokens = int64_t{1} << 30;        // of a sequence's page table
constexpr int64_t kPartialBytes = kDc * 2 + 2 * 4;      // of one row of a split
constexpr int32_t kMaxGridAxis = 65535;

bool sizes_ok(int32_t max_nodes, int32_t H) {
    return max_nodes >= 1 && max_nodes <= mla::kMaxNodes && H >= 1 && static_cast<int64_t>(max_nodes) * H <= kMaxRows;
}

int32_t rows_per_workgroup(int32_t max_nodes, int32_t H) {
    return static_cast<int64_t>(max_nodes) * H <= 64 ? 64 : mla::kDecodeRowsPerBlock;
}

// Whether n int32 at x and at y share memory.
bool overlap(const int32_t* x, const int32_t* y, int64_t n) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y), size = 4 * static_cast<uintptr_t>(n);
    return a < b ? b - a < size : a - b < size;
}

bool blocks_fit(int64_t blocks, int64_t threads) { return blocks * threads <= mla::kMaxDispatchItems; }

// Estimated time of a call, us: its work items on the compute units in the order of
// the launch (up to 64 sequences whole splits, then the last ones of the sequences,
// the longest first; past them sequence by sequence), and the merge.  rows: of every
// sequence.  The costs are those of low-bit caches.
double tree_cost(const int32_t* seq_lens, const std::vector<int64_t>& rows, int32_t rows_wg, int64_t split_tokens) {
    const double fixed = rows_wg == 64 ? 18.5 : 17.5, per_tile = rows_wg == 64 ? 1.25 : 1.6;
    const auto tiles = [](int64_t n) { return static_cast<double>((n + kTile - 1) / kTile); };
    struct Item { double time; int64_t blocks; };
    std::vector<Item> items, last;
    const bool sorted = rows.size() <= mla::kWaveThreads;
    double partial_rows = 0.0;
    for (size_t b = 0; b < rows.size(); ++b) {
        const int64_t own = rows[b], blocks = (own + rows_wg - 1) / rows_wg;
        const int64_t whole = seq_lens[b] / split_tokens, left = seq_lens[b] % split_tokens;
        if (whole > 0) items.push_back({fixed + per_tile * tiles(split_tokens), whole * blocks});
        if (left > 0) (sorted ? last : items).push_back({fixed + per_tile * tiles(left), blocks});
        if (seq_lens[b] > split_tokens) partial_rows += static_cast<double>(own * (whole + (left > 0 ? 1 : 0)));
    }
    std::sort(last.begin(), last.end(), [](const Item& x, const Item& y) { return x.time > y.time; });
    items.insert(items.end(), last.begin(), last.end());
    std::priority_queue<double, std::vector<double>, std::greater<double>> free;
    for (int i = 0; i < mla::kCus; ++i) free.push(0.0);
    double longest = 0.0;
    for (const Item& item : items)
        for (int64_t r = 0; r < item.blocks; ++r) {
            const double done = free.top() + item.time;
            free.pop();
            free.push(done);
            longest = std::max(longest, done);
        }
    // partials written and read at 4 TB/s beside the merge's launch
    return partial_rows == 0.0 ? longest : longest + 4.0 + 2.0 * partial_rows * kPartialBytes / 4e6;
}

// nodes: of every sequence, or NULL where they are not known.
int32_t split_size(const int32_t* seq_lens, const int32_t* nodes, int32_t B, int32_t max_nodes, int32_t H) {
    int64_t tokens = 0;
    int32_t longest = 0;
    for (int32_t b = 0; b < B; ++b) {
        tokens += seq_lens[b];
        longest = std::max(longest, seq_lens[b]);
    }
    if (B == 0) return 0;
    const int32_t rows_wg = rows_per_workgroup(max_nodes, H);
    const int64_t most = static_cast<int64_t>(max_nodes) * H, row_blocks = (most + rows_wg - 1) / rows_wg;
    constexpr int64_t kMostBlocks = 16 * mla::kCus;
    if (B * row_blocks >= kMostBlocks) return 0;
    // Without the nodes, sequences of one length are taken to have the most, others to be
    // a mixed batch: three guesses at who has an eighth to all of the rows, which say
    // little about single sizes, so that the smallest size within 4 % of the best one is
    // taken, whose items end closer together.  Ragged contexts behind equal trees pay for
    // that (128 heads: 8 x 4 nodes 107 us with their nodes given, 156 without; 24 x 4
    // 202, 231; 64 x 4 553, 636; 24 x 13 at 64 heads of one length but for a token 165,
    // 202), ragged ones behind ragged trees little (32 sequences of up to 8: 235, 255; 24
    // of up to 32: 676, 651).
    bool mixed = false;
    for (int32_t b = 1; b < B && nodes == nullptr; ++b) mixed = mixed || seq_lens[b] != seq_lens[0];
    std::vector<std::vector<int64_t>> guesses(mixed ? 3 : 1, std::vector<int64_t>(static_cast<size_t>(B)));
    for (size_t k = 0; k < guesses.size(); ++k)
        for (int32_t b = 0; b < B; ++b) {
            const int64_t eighths = mixed ? (int64_t{b} * 5 + 3 * static_cast<int64_t>(k) + 1) % 8 + 1 : 8;
            guesses[k][static_cast<size_t>(b)] = nodes != nullptr ? static_cast<int64_t>(nodes[b]) * H : (most * eighths + 7) / 8;
        }
    // unsplit, sizes of about a quarter more each time, and even parts of the longest
    // sequence, as long as there are not far more workgroups than compute units
    std::vector<int64_t> sizes{(int64_t{longest} + kTile - 1) / kTile * kTile};
    for (int64_t s = kTile; s < longest; s = (s + std::max<int64_t>(s / 4, 1) + kTile - 1) / kTile * kTile) sizes.push_back(s);
    for (int64_t parts = 2; parts <= 32; ++parts) sizes.push_back((longest + parts * kTile - 1) / (parts * kTile) * kTile);
    std::vector<double> times;
    for (size_t i = 0; i < sizes.size(); ++i) {
        const bool no = i > 0 && (sizes[i] >= longest || (tokens / sizes[i] + B) * row_blocks > kMostBlocks);
        double time = no ? HUGE_VAL : 0.0;
        for (size_t k = 0; !no && k < guesses.size(); ++k) time += tree_cost(seq_lens, guesses[k], rows_wg, sizes[i]);
        times.push_back(time);
    }
    const double best = *std::min_element(times.begin(), times.end());
    if (best == 0.0) return 0;          // no nodes at all
    size_t pick = sizes.size();
    for (size_t i = 0; i < sizes.size(); ++i)
        if (times[i] <= (mixed ? 1.04 : 1.0) * best && (pick == sizes.size() || sizes[i] < sizes[pick])) pick = i;
    return pick == 0 ? 0 : static_cast<int32_t>(sizes[pick]);
}

int32_t checked_split_size(const int32_t* seq_lens, const int32_t* nodes, int32_t B, int32_t max_nodes, int32_t H) {
    if (B < 0 || max_nodes < 1 || H < 1 || (B > 0 && seq_lens == nullptr)) return -MLA_EINVAL;
    if (!sizes_ok(max_nodes, H)) return -MLA_ENOTSUP;
    for (int32_t b = 0; b < B; ++b)
        if (seq_lens[b] < 1 || (nodes != nullptr && (nodes[b] < 0 || nodes[b] > max_nodes))) return -MLA_EINVAL;
    try {
        return split_size(seq_lens, nodes, B, max_nodes, H);
    } catch (const std::exception&) {       // no memory for the estimate: any size is a right one
        return 0;
    }
}

int tree_attn(const mla_cache_format* f, bool lowbit, const uint16_t* q_lat, const uint16_t* q_rope,
              const void* cache, int64_t num_pages, const int32_t* block_table, int32_t max_pages_per_seq,
              const int32_t* ctx_lens, const int32_t* cu_nodes, const uint64_t* tree_mask, int32_t num_nodes,
              int32_t max_nodes, int32_t B, int32_t H, float softmax_scale, int32_t split_tokens,
              const int32_t* split_indptr, int32_t num_splits, uint16_t* out, float* lse, void* workspace,
              int64_t workspace_bytes, hipStream_t stream) {
    const int st = lowbit ? check_lowbit_format(f) : check_shape(f);
    if (st != MLA_OK) return st;
    if (B < 0 || num_nodes < 0 || num_pages < 0 || max_pages_per_seq <= 0 || split_tokens < 0 || num_splits < 0 ||
        max_nodes < 1 || H < 1)
        return MLA_EINVAL;
    if (!std::isfinite(softmax_scale) || !(softmax_scale > 0.0f)) return MLA_EINVAL;
    if (!sizes_ok(max_nodes, H) || split_tokens % kTile != 0) return MLA_ENOTSUP;
    // positions in 32 bits, those of a split past the longest sequence too
    if (static_cast<int64_t>(max_pages_per_seq) * f->page_size > kMaxTokens || split_tokens > kMaxTokens) return MLA_ENOTSUP;
    if (B == 0 || num_nodes == 0) return MLA_OK;
    if (q_lat == nullptr || q_rope == nullptr || cache == nullptr || block_table == nullptr || ctx_lens == nullptr ||
        cu_nodes == nullptr || tree_mask == nullptr || out == nullptr || num_pages == 0)
        return MLA_EINVAL;
    if (!aligned(cache, 256)) return MLA_EINVAL;
    if (!aligned(q_lat, 16) || !aligned(q_rope, 16) || !aligned(out, 16)) return MLA_ENOTSUP;
    const int64_t rows = static_cast<int64_t>(max_nodes) * H;
    const int64_t num_work = split_tokens == 0 ? B : num_splits;
    const int32_t rows_wg = rows_per_workgroup(max_nodes, H);
    if (!blocks_fit(mla::tree_workgroups(num_work, rows, rows_wg), mla::kDecodeThreads)) return MLA_ENOTSUP;
    if (split_tokens != 0) {
        if (split_indptr == nullptr) return MLA_EINVAL;
        const int64_t need = mla_tree_workspace_bytes(num_splits, max_nodes, H);
        if (need < 0) return MLA_ENOTSUP;
        if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return MLA_EINVAL;
        if (!aligned(workspace, 16)) return MLA_ENOTSUP;
        if (!blocks_fit((B * rows + 7) / 8 * 8, mla::kCombineThreads)) return MLA_ENOTSUP;
    }
    mla::TreeArgs a{};
    a.shape = {rows_wg, 4};
    a.q_lat = q_lat;
    a.q_rope = q_rope;
    a.cache = static_cast<const uint8_t*>(cache);
    a.num_pages = num_pages;
    a.block_table = block_table;
    a.max_pages = max_pages_per_seq;
    a.seq_lens = ctx_lens;
    a.B = B;
    a.s_q = max_nodes;
    a.H = H;
    a.scale_log2 = softmax_scale * 1.4426950408889634f;
    a.split_tokens = split_tokens;
    a.split_indptr = split_indptr;
    a.num_work = static_cast<int32_t>(num_work);
    a.out = out;
    a.lse = lse;
    a.g = lowbit ? lowbit_geom(f) : bf16_geom(f);
    a.cu_nodes = cu_nodes;
    a.mask = tree_mask;
    a.num_nodes = num_nodes;
    if (split_tokens != 0) {
        const int64_t part_rows = num_splits * rows;
        a.part_o = static_cast<uint16_t*>(workspace);
        a.part_m = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + part_rows * kDc * 2);
        a.part_s = a.part_m + part_rows;
    }
    const bool paper = f->meta == MLA_META_PAPER;
    const mla::CacheKind kind = !lowbit ? mla::KIND_BF16
                                : f->c_bits == 4 ? (paper ? mla::KIND_C4R4P : mla::KIND_C4R4)
                                                 : (paper ? mla::KIND_C2R4P : mla::KIND_C2R4);
    const int launched = hip_status(mla::launch_tree_attn(kind, a, stream));
    if (launched != MLA_OK || split_tokens == 0) return launched;
    mla::TreeCombineArgs c{};
    c.part_m = a.part_m;
    c.part_s = a.part_s;
    c.part_o = a.part_o;
    c.split_indptr = split_indptr;
    c.B = B;
    c.s_q = max_nodes;
    c.H = H;
    c.out = out;
    c.lse = lse;
    c.cu_nodes = cu_nodes;
    c.num_nodes = num_nodes;
    c.num_splits = num_splits;
    return hip_status(mla::launch_tree_combine(c, stream));
}

int commit(const mla_cache_format* f, bool lowbit, void* const* caches, int32_t num_layers, int64_t num_pages,
           const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens, const int32_t* path,
           const int32_t* keep, int32_t max_nodes, int32_t B, int32_t* new_lens, hipStream_t stream) {
    const int st = lowbit ? check_lowbit_format(f) : check_shape(f);
    if (st != MLA_OK) return st;
    if (B < 0 || num_layers < 0 || num_pages < 0 || max_pages_per_seq <= 0 || max_nodes < 1) return MLA_EINVAL;
    if (max_nodes > mla::kMaxNodes || B > kMaxGridAxis) return MLA_ENOTSUP;
    if (static_cast<int64_t>(max_pages_per_seq) * f->page_size > kMaxTokens) return MLA_ENOTSUP;
    if (B == 0 || (num_layers == 0 && new_lens == nullptr)) return MLA_OK;
    if (ctx_lens == nullptr || path == nullptr || keep == nullptr) return MLA_EINVAL;
    if (num_layers > 0 && (caches == nullptr || block_table == nullptr || num_pages == 0)) return MLA_EINVAL;
    if (!blocks_fit(static_cast<int64_t>(B) * std::max(num_layers, 1), 256)) return MLA_ENOTSUP;
    // (a workgroup writes them while others still read the lengths and counts)
    if (new_lens != nullptr && (overlap(new_lens, ctx_lens, B) || overlap(new_lens, keep, B))) return MLA_EINVAL;
    mla::CommitArgs a{};
    a.caches = reinterpret_cast<uint8_t* const*>(caches);
    a.num_layers = num_layers;
    a.num_pages = num_pages;
    a.block_table = block_table;
    a.max_pages = max_pages_per_seq;
    a.ctx_lens = ctx_lens;
    a.path = path;
    a.keep = keep;
    a.max_nodes = max_nodes;
    a.B = B;
    a.new_lens = new_lens;
    a.g = lowbit ? lowbit_geom(f) : bf16_geom(f);
    return hip_status(mla::launch_commit(a, lowbit, stream));
}

}  // namespace

extern "C" {

int32_t mla_tree_split_tokens(const int32_t* seq_lens, int32_t B, int32_t max_nodes, int32_t H) {
    return checked_split_size(seq_lens, nullptr, B, max_nodes, H);
}

int32_t mla_tree_split_tokens_for(const int32_t* seq_lens, const int32_t* nodes, int32_t B, int32_t max_nodes, int32_t H) {
    if (B > 0 && nodes == nullptr) return -MLA_EINVAL;
    return checked_split_size(seq_lens, nodes, B, max_nodes, H);
}

int64_t mla_tree_workspace_bytes(int32_t num_splits, int32_t max_nodes, int32_t H) {
    if (num_splits < 0 || !sizes_ok(max_nodes, H)) return -1;
    return static_cast<int64_t>(num_splits) * max_nodes * H * kPartialBytes;
}

int mla_lowbit_tree_attn(const mla_cache_format* f, const uint16_t* q_lat, const uint16_t* q_rope, const void* cache,
                         int64_t num_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                         const int32_t* ctx_lens, const int32_t* cu_nodes, const uint64_t* tree_mask,
                         int32_t num_nodes, int32_t max_nodes, int32_t B, int32_t H, float softmax_scale,
                         int32_t split_tokens, const int32_t* split_indptr, int32_t num_splits, uint16_t* out,
                         float* lse, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
    return tree_attn(f, true, q_lat, q_rope, cache, num_pages, block_table, max_pages_per_seq, ctx_lens, cu_nodes,
                     tree_mask, num_nodes, max_nodes, B, H, softmax_scale, split_tokens, split_indptr, num_splits, out,
                     lse, workspace, workspace_bytes, stream);
}

int mla_bf16_tree_attn(const mla_cache_format* f, const uint16_t* q_lat, const uint16_t* q_rope, const void* cache,
                       int64_t num_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                       const int32_t* ctx_lens, const int32_t* cu_nodes, const uint64_t* tree_mask, int32_t num_nodes,
                       int32_t max_nodes, int32_t B, int32_t H, float softmax_scale, int32_t split_tokens,
                       const int32_t* split_indptr, int32_t num_splits, uint16_t* out, float* lse, void* workspace,
                       int64_t workspace_bytes, hipStream_t stream) {
    return tree_attn(f, false, q_lat, q_rope, cache, num_pages, block_table, max_pages_per_seq, ctx_lens, cu_nodes,
                     tree_mask, num_nodes, max_nodes, B, H, softmax_scale, split_tokens, split_indptr, num_splits, out,
                     lse, workspace, workspace_bytes, stream);
}

int64_t mla_verify_workspace_bytes(int32_t num_nodes, int32_t B, int32_t vocab) {
    if (num_nodes < 0 || B < 0 || vocab < 1 || vocab > mla::kMaxVocab) return -1;
    // statistics of every chunk, sums of a shared pass, and its counters
    return mla::logit_chunks(vocab) * (num_nodes * int64_t{sizeof(mla::ChunkStat)} + B * int64_t{8}) + B * int64_t{4};
}

int mla_verify_tree(const void* logits, int32_t logits_type, int64_t logits_stride, int32_t vocab,
                    const float* draft_probs, int64_t draft_stride, const int32_t* tokens, const int32_t* parents,
                    const int32_t* cu_nodes, int32_t num_nodes, int32_t max_nodes, int32_t B,
                    const float* temperature, const float* u_accept, const float* u_draw, int32_t* path,
                    int32_t* out_tokens, float* logprobs, int32_t* keep, void* workspace, int64_t workspace_bytes,
                    hipStream_t stream) {
    if (logits_type != MLA_LOGITS_BF16 && logits_type != MLA_LOGITS_FP32) return MLA_EINVAL;
    if (vocab < 1 || B < 0 || num_nodes < 0 || max_nodes < 1 || logits_stride < vocab) return MLA_EINVAL;
    if (draft_probs != nullptr && draft_stride < vocab) return MLA_EINVAL;
    if (vocab > mla::kMaxVocab || max_nodes > mla::kMaxNodes || B > kMaxGridAxis) return MLA_ENOTSUP;
    if (B == 0) return MLA_OK;
    if (cu_nodes == nullptr || path == nullptr || out_tokens == nullptr || keep == nullptr) return MLA_EINVAL;
    if (num_nodes > 0 && (logits == nullptr || tokens == nullptr || parents == nullptr || u_accept == nullptr ||
                          u_draw == nullptr))
        return MLA_EINVAL;
    if (!aligned(logits, logits_type == MLA_LOGITS_FP32 ? 4 : 2) || !aligned(draft_probs, 4)) return MLA_ENOTSUP;
    const int64_t need = mla_verify_workspace_bytes(num_nodes, B, vocab);
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return MLA_EINVAL;
    if (!aligned(workspace, 16)) return MLA_ENOTSUP;
    const int64_t chunk_groups = (mla::logit_chunks(vocab) + 3) / 4;
    if (!blocks_fit(chunk_groups * max_nodes * B, 256)) return MLA_ENOTSUP;
    mla::VerifyArgs a{};
    a.logits = logits;
    a.logits_stride = logits_stride;
    a.fp32 = logits_type == MLA_LOGITS_FP32;
    a.vocab = vocab;
    a.draft_probs = draft_probs;
    a.draft_stride = draft_stride;
    a.tokens = tokens;
    a.parents = parents;
    a.cu_nodes = cu_nodes;
    a.num_nodes = num_nodes;
    a.max_nodes = max_nodes;
    a.B = B;
    a.temperature = temperature;
    a.u_accept = u_accept;
    a.u_draw = u_draw;
    a.path = path;
    a.out_tokens = out_tokens;
    a.logprobs = logprobs;
    a.keep = keep;
    const int64_t chunks = mla::logit_chunks(vocab);
    a.stats = static_cast<mla::ChunkStat*>(workspace);
    a.sums = reinterpret_cast<double*>(a.stats + num_nodes * chunks);
    a.arrived = reinterpret_cast<int32_t*>(a.sums + B * chunks);
    return hip_status(mla::launch_verify(a, stream));
}

int mla_lowbit_commit(const mla_cache_format* f, void* const* caches, int32_t num_layers, int64_t num_pages,
                      const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                      const int32_t* path, const int32_t* keep, int32_t max_nodes, int32_t B, int32_t* new_lens,
                      hipStream_t stream) {
    return commit(f, true, caches, num_layers, num_pages, block_table, max_pages_per_seq, ctx_lens, path, keep,
                  max_nodes, B, new_lens, stream);
}

int mla_bf16_commit(const mla_cache_format* f, void* const* caches, int32_t num_layers, int64_t num_pages,
                    const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                    const int32_t* path, const int32_t* keep, int32_t max_nodes, int32_t B, int32_t* new_lens,
                    hipStream_t stream) {
    return commit(f, false, caches, num_layers, num_pages, block_table, max_pages_per_seq, ctx_lens, path, keep,
                  max_nodes, B, new_lens, stream);
}

}  // extern "C"
