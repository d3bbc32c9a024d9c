// Host side of the C ABI declared in include/mla_prefill.h: argument
// validation, the planner of the expanded attention and kernel dispatch.
//
// Plain C++, as mla_abi.cpp: every check runs before any HIP call, and nothing
// here throws.
#include "mla_prefill.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <new>

#include "abi_checks.h"
#include "prefill_internal.h"

namespace {

using namespace mla::abi;

int check_rotation(const mla_rotation* r, mla::Rotation* out) {
    if (r == nullptr || r->table == nullptr || r->num_positions <= 0) return MLA_EINVAL;
    if (r->layout != MLA_ROPE_PAIRS && r->layout != MLA_ROPE_HALVES) return MLA_EINVAL;
    if (!aligned(r->table, 16)) return MLA_ENOTSUP;
    *out = {r->table, r->num_positions, r->layout == MLA_ROPE_HALVES};
    return MLA_OK;
}

// Dense bf16 rows of `width` channels read or written 16 bytes at a time.
int check_rows(const uint16_t* p, int64_t stride, int32_t width) {
    if (stride < width) return MLA_EINVAL;
    if (stride % 8 != 0 || !aligned(p, 16)) return MLA_ENOTSUP;
    return MLA_OK;
}

int norm_rope_append(const mla_cache_format* f, bool lowbit, const mla_rms_norm* norm, const mla_rotation* rot,
                     const uint16_t* c_kv, int64_t c_kv_stride, const uint16_t* k_rope, int64_t k_rope_stride,
                     const int32_t* positions, const int64_t* slot_mapping, int32_t n, void* cache,
                     int64_t num_pages, uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out,
                     int64_t k_out_stride, hipStream_t stream, mla::NormRopeArgs a = {}) {
    int st = lowbit ? check_lowbit_format(f) : check_shape(f);
    if (st != MLA_OK) return st;
    st = check_rotation(rot, &a.rot);
    if (st != MLA_OK) return st;
    if (norm != nullptr) {
        if (!std::isfinite(norm->eps) || !(norm->eps > 0.0f)) return MLA_EINVAL;
        if (norm->weight != nullptr && !aligned(norm->weight, 16)) return MLA_ENOTSUP;
        a.has_norm = 1;
        a.weight = norm->weight;
        a.eps = norm->eps;
    }
    st = check_append(c_kv, c_kv_stride, k_rope, k_rope_stride, slot_mapping, n, cache, num_pages);
    if (st != MLA_OK || n == 0) return st;
    if (positions == nullptr) return MLA_EINVAL;
    if (c_out != nullptr) {
        st = check_rows(c_out, c_out_stride, kDc);
        if (st != MLA_OK) return st;
        if (c_out == c_kv && c_out_stride != c_kv_stride) return MLA_EINVAL;
    }
    if (k_out != nullptr) {
        st = check_rows(k_out, k_out_stride, kDr);
        if (st != MLA_OK) return st;
        if (k_out == k_rope && k_out_stride != k_rope_stride) return MLA_EINVAL;
    }
    mla::AppendArgs& p = a.append;
    p.c_kv = c_kv;
    p.c_kv_stride = c_kv_stride;
    p.k_rope = k_rope;
    p.k_rope_stride = k_rope_stride;
    p.slot_mapping = slot_mapping;
    p.positions = positions;
    p.n = n;
    p.cache = static_cast<uint8_t*>(cache);
    p.num_slots = num_pages * f->page_size;
    p.g = lowbit ? lowbit_geom(f) : bf16_geom(f);
    a.c_out = c_out;
    a.c_out_stride = c_out_stride;
    a.k_out = k_out;
    a.k_out_stride = k_out_stride;
    return hip_status(mla::launch_norm_rope_append(a, lowbit, stream));
}

int gather(const mla_cache_format* f, bool lowbit, const void* cache, int64_t num_pages, const int32_t* block_table,
           int32_t max_pages_per_seq, const int32_t* first, const int32_t* cu_rows, int32_t B, int32_t n,
           uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out, int64_t k_out_stride, hipStream_t stream,
           mla::GatherArgs a = {}) {
    int st = lowbit ? check_lowbit_format(f) : check_shape(f);
    if (st != MLA_OK) return st;
    if (B < 0 || n < 0 || num_pages < 0 || max_pages_per_seq <= 0) return MLA_EINVAL;
    if (n > mla::kMaxAppendTokens) return MLA_ENOTSUP;
    if (n == 0 || B == 0) return MLA_OK;
    if (cache == nullptr || block_table == nullptr || cu_rows == nullptr || c_out == nullptr || k_out == nullptr)
        return MLA_EINVAL;
    if (num_pages == 0 || !aligned(cache, 256)) return MLA_EINVAL;
    st = check_rows(c_out, c_out_stride, kDc);
    if (st != MLA_OK) return st;
    st = check_rows(k_out, k_out_stride, kDr);
    if (st != MLA_OK) return st;
    a.cache = static_cast<const uint8_t*>(cache);
    a.num_pages = num_pages;
    a.block_table = block_table;
    a.max_pages = max_pages_per_seq;
    a.first = first;
    a.cu_rows = cu_rows;
    a.B = B;
    a.n = n;
    a.g = lowbit ? lowbit_geom(f) : bf16_geom(f);
    a.c_out = c_out;
    a.c_out_stride = c_out_stride;
    a.k_out = k_out;
    a.k_out_stride = k_out_stride;
    return hip_status(mla::launch_gather(a, lowbit, stream));
}

// ---------------------------------------------------------------------------
// Plan of the expanded attention.

constexpr int32_t kMaxLen = 1 << 30;        // rows of a sequence, and of a tensor
constexpr int32_t kKeyTile = 64;            // keys that the cost below is counted in

struct Lengths {
    const int32_t* q;
    const int32_t* kv;
    const int32_t* q_start;
    const int32_t* kv_start;
    int32_t B, causal;
};

// Calls f(b, q_row, rows, kv_row, key1, seen0) for every block of `rows` query rows.
template <typename F>
void each_block(const Lengths& n, int32_t rows, F f) {
    int64_t q_at = 0, kv_at = 0;
    for (int32_t b = 0; b < n.B; ++b) {
        const int32_t q = n.q[b], kv = n.kv[b];
        const int32_t q_row = n.q_start != nullptr ? n.q_start[b] : static_cast<int32_t>(q_at);
        const int32_t kv_row = n.kv_start != nullptr ? n.kv_start[b] : static_cast<int32_t>(kv_at);
        for (int32_t i = 0; i < q; i += rows) {
            const int32_t r = std::min(rows, q - i);
            const int32_t key1 = n.causal ? std::clamp(kv - q + i + r, 0, kv) : kv;
            const int32_t seen0 = n.causal ? kv - q + i + 1 : mla::kPrefillUnmasked;
            f(b, q_row + i, r, kv_row, key1, seen0);
        }
        q_at += q;
        kv_at += kv;
    }
}

int32_t tiles_of(int32_t keys) { return (keys + kKeyTile - 1) / kKeyTile; }

// Key splits of a block of `tiles` tiles when a split may hold `most`.
int32_t splits_of(int32_t tiles, int64_t most) {
    return tiles <= most + most / 2 ? 1 : static_cast<int32_t>((tiles + most - 1) / most);
}

// Workgroups that run at once, and the fewest tiles that are worth a split (a
// partial block is written and read again, and its merge is another launch).
struct Shape {
    int32_t rows, slots, least_tiles;
};
constexpr Shape kShapes[] = {{128, 512, 4}, {256, 256, 8}};

// Up to 128 rows per sequence the reads of the keys bound the kernel, and two small
// workgroups per CU overlap each other's beginnings and ends; beyond, a workgroup of
// 256 rows reads the keys half as often.  Measured, 64 heads, 128 rows / 256 rows: 256
// prompts of 64 243 / 453 us; 128 of 128 235 / 326; 96 of 192 353 / 323; 64 of 256 301 /
// 293; 16 of 1024 660 / 493; 128 rows on 16 x 4096 keys 490 / 519, 129 rows 855 / 518.
// The longest sequence decides for the whole call: one prompt of 1024 beside 255 of 64
// takes 480 us (two calls, one for each kind, 62 + 241), 512 rows beside 63 single tokens
// on 2K keys, 32 heads, 481 (49 + 376).
Shape choose_rows(const Lengths& n) {
    int32_t most = 0;
    for (int32_t b = 0; b < n.B; ++b) most = std::max(most, n.q[b]);
    return most <= kShapes[0].rows ? kShapes[0] : kShapes[1];
}

int check_lengths(const Lengths& n, int64_t* total_q, int64_t* total_kv) {
    int64_t q_at = 0, kv_at = 0, q_end = 0, kv_end = 0;
    for (int32_t b = 0; b < n.B; ++b) {
        if (n.q[b] < 0 || n.kv[b] < 0) return MLA_EINVAL;
        if (n.q_start != nullptr && n.q_start[b] < 0) return MLA_EINVAL;
        if (n.kv_start != nullptr && n.kv_start[b] < 0) return MLA_EINVAL;
        q_at = n.q_start != nullptr ? n.q_start[b] : q_at;
        kv_at = n.kv_start != nullptr ? n.kv_start[b] : kv_at;
        q_at += n.q[b];
        kv_at += n.kv[b];
        if (q_at > kMaxLen || kv_at > kMaxLen) return MLA_ENOTSUP;
        if (n.q[b] > 0) q_end = std::max(q_end, q_at);
        if (n.kv[b] > 0) kv_end = std::max(kv_end, kv_at);
    }
    *total_q = q_end;
    *total_kv = kv_end;
    if (n.q_start == nullptr) return MLA_OK;
    // query ranges given by the caller may not overlap (two blocks would write one row)
    int32_t* order = new (std::nothrow) int32_t[n.B > 0 ? n.B : 1];
    if (order == nullptr) return MLA_ENOTSUP;
    int32_t m = 0;
    for (int32_t b = 0; b < n.B; ++b)
        if (n.q[b] > 0) order[m++] = b;
    std::sort(order, order + m, [&](int32_t x, int32_t y) { return n.q_start[x] < n.q_start[y]; });
    int st = MLA_OK;
    for (int32_t i = 1; i < m; ++i)
        if (n.q_start[order[i - 1]] + n.q[order[i - 1]] > n.q_start[order[i]]) st = MLA_EINVAL;
    delete[] order;
    return st;
}

int64_t plan_ints(const mla_prefill_plan& p) {
    const mla::PrefillLists l = mla::prefill_lists(p.num_items, p.H, p.rows);
    return (static_cast<int64_t>(p.num_items) + p.num_merges) * mla::kPrefillRecordInts + (l.lists > 0 ? l.lists + 1 + l.entries : 0);
}

// Deals (item, head) out to the lists as workgroups would take them, each when it
// is done with the one before: sequence by sequence, a sequence's heads one after
// the other, so that the blocks of a head's rows run at the same time and read its
// keys through one L2; the last rounds by length, so that the short ones fill the
// end.  Blocks that begin together go through their keys from the first on; where
// the lists are spread out, the longest block begins first and all end together,
// so they go from the last key down: either way they read the same keys at the
// same time (8K keys, 128 heads: 2271 us against 2311 all upwards; where a head's keys
// fit the L2 it costs, 4 of 4K, 64 heads: 1305 against 1276).  `items` in the order of
// the plan.
constexpr int32_t kItemTiles = 5;       // an item's fixed cost, in tiles
constexpr int32_t kLastRounds = 2;
constexpr int32_t kL2Tiles = 96;        // tiles of a head that fill an XCD's L2 (40 KiB each)
void fill_lists(const mla::PrefillItem* items, const mla_prefill_plan& p, int32_t* out) {
    const mla::PrefillLists l = mla::prefill_lists(p.num_items, p.H, p.rows);
    const auto tiles = [&](int32_t i) { return tiles_of(items[i].key1 - items[i].key0); };
    struct Load {
        int64_t tiles;
        int32_t list;
    };
    constexpr int32_t kMostLists = 256;
    Load heap[kMostLists];
    int32_t filled[kMostLists], last[kLastRounds * kMostLists];
    const auto later = [](const Load& x, const Load& y) { return x.tiles != y.tiles ? x.tiles > y.tiles : x.list > y.list; };
    const int64_t sorted_from = std::max<int64_t>(0, l.entries - kLastRounds * l.lists);
    // gives f(list, entry) for all entries
    const auto deal = [&](auto f) {
        for (int32_t i = 0; i < l.lists; ++i) heap[i] = {0, i};         // (equal: a heap)
        const auto give = [&](int32_t entry, bool down) {
            std::pop_heap(heap, heap + l.lists, later);
            Load& to = heap[l.lists - 1];
            f(to.list, down ? ~entry : entry);
            to.tiles += kItemTiles + tiles(entry / l.heads);
            std::push_heap(heap, heap + l.lists, later);
        };
        int64_t at = 0;
        int32_t n = 0;
        for (int32_t from = 0, to; from < p.num_items; from = to) {
            for (to = from + 1; to < p.num_items && items[to].seq == items[from].seq;) ++to;
            for (int32_t h = 0; h < l.heads; ++h)
                for (int32_t i = from; i < to;) {
                    const int32_t round_end = std::min(i + l.lists, to);
                    const Load& latest = *std::min_element(heap, heap + l.lists, later);
                    const bool down = tiles(i) >= kL2Tiles && 2 * (latest.tiles - heap[0].tiles) > tiles(i) - tiles(round_end - 1);
                    for (; i < round_end; ++i, ++at) {
                        if (at < sorted_from) give(i * l.heads + h, down);
                        else last[n++] = i * l.heads + h;
                    }
                }
        }
        std::sort(last, last + n, [&](int32_t x, int32_t y) {
            const int32_t tx = tiles(x / l.heads), ty = tiles(y / l.heads);
            return tx != ty ? tx > ty : x < y;
        });
        for (int32_t i = 0; i < n; ++i) give(last[i], false);
    };
    int32_t* const first = out;
    int32_t* const entries = out + l.lists + 1;
    std::fill(first, first + l.lists + 1, 0);
    deal([&](int32_t list, int32_t) { ++first[list + 1]; });
    for (int32_t i = 0; i < l.lists; ++i) {
        first[i + 1] += first[i];
        filled[i] = first[i];
    }
    deal([&](int32_t list, int32_t entry) { entries[filled[list]++] = entry; });
}

int check_head_rows(const mla_head_rows* r, bool heads, mla::HeadRows* out) {
    if (r == nullptr || r->data == nullptr) return MLA_EINVAL;
    const int64_t h = heads ? r->stride_h : 0;
    if (r->stride_t < 0 || h < 0) return MLA_EINVAL;
    if (r->stride_t % 8 != 0 || h % 8 != 0 || !aligned(r->data, 16)) return MLA_ENOTSUP;
    if (r->stride_t >= mla::kMaxHeadStride || h >= mla::kMaxHeadStride) return MLA_ENOTSUP;
    *out = {r->data, r->stride_t, h};
    return MLA_OK;
}

// Whether rows (t, h) of `width` channels are apart: heads within tokens, or tokens within heads.
bool rows_apart(int64_t stride_t, int64_t stride_h, int64_t T, int64_t H, int64_t width) {
    if (T <= 1) return H <= 1 || stride_h >= width;
    if (H <= 1) return stride_t >= width;
    return (stride_h >= width && stride_t >= (H - 1) * stride_h + width) ||
           (stride_t >= width && stride_h >= (T - 1) * stride_t + width);
}

}  // namespace

extern "C" {

int mla_lowbit_norm_rope_append(const mla_cache_format* f, const mla_rms_norm* norm, const mla_rotation* rot,
                                const uint16_t* c_kv, int64_t c_kv_stride, const uint16_t* k_rope,
                                int64_t k_rope_stride, const int32_t* positions, const int64_t* slot_mapping,
                                int32_t n, void* cache, int64_t num_pages, uint16_t* c_out, int64_t c_out_stride,
                                uint16_t* k_out, int64_t k_out_stride, hipStream_t stream) {
    return norm_rope_append(f, true, norm, rot, c_kv, c_kv_stride, k_rope, k_rope_stride, positions, slot_mapping, n,
                            cache, num_pages, c_out, c_out_stride, k_out, k_out_stride, stream);
}

int mla_bf16_norm_rope_append(const mla_cache_format* f, const mla_rms_norm* norm, const mla_rotation* rot,
                              const uint16_t* c_kv, int64_t c_kv_stride, const uint16_t* k_rope,
                              int64_t k_rope_stride, const int32_t* positions, const int64_t* slot_mapping,
                              int32_t n, void* cache, int64_t num_pages, uint16_t* c_out, int64_t c_out_stride,
                              uint16_t* k_out, int64_t k_out_stride, hipStream_t stream) {
    return norm_rope_append(f, false, norm, rot, c_kv, c_kv_stride, k_rope, k_rope_stride, positions, slot_mapping, n,
                            cache, num_pages, c_out, c_out_stride, k_out, k_out_stride, stream);
}

int mla_lowbit_norm_rope_append_protected(const mla_cache_format* f, const mla_protect_policy* p,
                                          const mla_rms_norm* norm, const mla_rotation* rot, const uint16_t* c_kv,
                                          int64_t c_kv_stride, const uint16_t* k_rope, int64_t k_rope_stride,
                                          const int32_t* positions, const int64_t* slot_mapping, int32_t n,
                                          void* cache, int64_t num_pages, const int32_t* token_seq,
                                          const int32_t* seq_lens, const int32_t* prot_slot, int32_t B, void* prot,
                                          int64_t num_prot, uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out,
                                          int64_t k_out_stride, hipStream_t stream) {
    const int st = check_policy(p);
    if (st != MLA_OK) return st;
    if (B < 0 || num_prot < 0) return MLA_EINVAL;
    if (n > 0) {
        if (token_seq == nullptr || seq_lens == nullptr || prot_slot == nullptr || prot == nullptr || B == 0 ||
            num_prot == 0)
            return MLA_EINVAL;
        if (!aligned(prot, 16)) return MLA_ENOTSUP;
    }
    mla::NormRopeArgs a{};
    a.append.prot = static_cast<uint8_t*>(prot);
    a.append.num_prot = num_prot;
    a.append.token_seq = token_seq;
    a.append.seq_lens = seq_lens;
    a.append.prot_slot = prot_slot;
    a.append.B = B;
    a.append.sink = p->sink;
    a.append.recent = p->recent;
    return norm_rope_append(f, true, norm, rot, c_kv, c_kv_stride, k_rope, k_rope_stride, positions, slot_mapping, n,
                            cache, num_pages, c_out, c_out_stride, k_out, k_out_stride, stream, a);
}

int mla_rope_queries(const mla_rotation* rot, const uint16_t* q, int64_t q_stride_t, int64_t q_stride_h,
                     const int32_t* positions, int32_t n, int32_t H, uint16_t* out, int64_t out_stride_t,
                     int64_t out_stride_h, hipStream_t stream) {
    mla::RopeArgs a{};
    const int st = check_rotation(rot, &a.rot);
    if (st != MLA_OK) return st;
    if (n < 0 || H <= 0) return MLA_EINVAL;
    if (n == 0) return MLA_OK;
    if (q == nullptr || positions == nullptr || out == nullptr) return MLA_EINVAL;
    if (q_stride_t < 0 || q_stride_h < 0 || out_stride_t < 0 || out_stride_h < 0) return MLA_EINVAL;
    if (q_stride_t % 8 != 0 || q_stride_h % 8 != 0 || out_stride_t % 8 != 0 || out_stride_h % 8 != 0 ||
        !aligned(q, 16) || !aligned(out, 16))
        return MLA_ENOTSUP;
    if (!rows_apart(out_stride_t, out_stride_h, n, H, kDr)) return MLA_EINVAL;
    if (out == q && (q_stride_t != out_stride_t || q_stride_h != out_stride_h)) return MLA_EINVAL;
    // 8 threads per row, in whole workgroups
    if (static_cast<int64_t>(n) * H > mla::kMaxDispatchItems / 8 - 256) return MLA_ENOTSUP;
    a.q = q;
    a.q_stride_t = q_stride_t;
    a.q_stride_h = q_stride_h;
    a.positions = positions;
    a.n = n;
    a.H = H;
    a.out = out;
    a.out_stride_t = out_stride_t;
    a.out_stride_h = out_stride_h;
    return hip_status(mla::launch_rope_queries(a, stream));
}

int mla_lowbit_gather(const mla_cache_format* f, const void* cache, int64_t num_pages, const int32_t* block_table,
                      int32_t max_pages_per_seq, const int32_t* first, const int32_t* cu_rows, int32_t B, int32_t n,
                      uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out, int64_t k_out_stride,
                      hipStream_t stream) {
    return gather(f, true, cache, num_pages, block_table, max_pages_per_seq, first, cu_rows, B, n, c_out,
                  c_out_stride, k_out, k_out_stride, stream);
}

int mla_bf16_gather(const mla_cache_format* f, const void* cache, int64_t num_pages, const int32_t* block_table,
                    int32_t max_pages_per_seq, const int32_t* first, const int32_t* cu_rows, int32_t B, int32_t n,
                    uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out, int64_t k_out_stride,
                    hipStream_t stream) {
    return gather(f, false, cache, num_pages, block_table, max_pages_per_seq, first, cu_rows, B, n, c_out,
                  c_out_stride, k_out, k_out_stride, stream);
}

int mla_lowbit_gather_protected(const mla_cache_format* f, const mla_protect_policy* p, const void* cache,
                                int64_t num_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                const int32_t* first, const int32_t* cu_rows, int32_t B, int32_t n,
                                const int32_t* seq_lens, const void* prot, int64_t num_prot,
                                const int32_t* prot_slot, uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out,
                                int64_t k_out_stride, hipStream_t stream) {
    const int st = check_policy(p);
    if (st != MLA_OK) return st;
    if (B < 0 || num_prot < 0) return MLA_EINVAL;
    if (n > 0 && B > 0) {
        if (seq_lens == nullptr || prot == nullptr || prot_slot == nullptr || num_prot == 0) return MLA_EINVAL;
        if (!aligned(prot, 16)) return MLA_ENOTSUP;
    }
    mla::GatherArgs a{};
    a.seq_lens = seq_lens;
    a.prot = static_cast<const uint8_t*>(prot);
    a.num_prot = num_prot;
    a.prot_slot = prot_slot;
    a.sink = p->sink;
    a.recent = p->recent;
    return gather(f, true, cache, num_pages, block_table, max_pages_per_seq, first, cu_rows, B, n, c_out,
                  c_out_stride, k_out, k_out_stride, stream, a);
}

int mla_plan_prefill(const int32_t* q_lens, const int32_t* kv_lens, const int32_t* q_starts,
                     const int32_t* kv_starts, int32_t B, int32_t H, int32_t causal, int32_t* plan,
                     int64_t plan_capacity, mla_prefill_plan* info) {
    if (info == nullptr || B < 0 || H <= 0 || (causal != 0 && causal != 1)) return MLA_EINVAL;
    if (B > 0 && (q_lens == nullptr || kv_lens == nullptr)) return MLA_EINVAL;
    const Lengths n{q_lens, kv_lens, q_starts, kv_starts, B, causal};
    mla_prefill_plan p{};
    const int st = check_lengths(n, &p.total_q, &p.total_kv);
    if (st != MLA_OK) return st;

    // A split holds at least a slot's share of the tiles, so keys are split only
    // where whole blocks would leave slots empty or one slot far behind.
    const Shape shape = choose_rows(n);
    int64_t tiles = 0;
    each_block(n, shape.rows, [&](int32_t, int32_t, int32_t, int32_t, int32_t key1, int32_t) { tiles += tiles_of(key1); });
    // (tiles <= 2^30 blocks x 2^24 tiles, and H < 2^31: in double, its rounding is of no matter here)
    const int64_t most = std::max<int64_t>(
        shape.least_tiles, static_cast<int64_t>(std::ceil(static_cast<double>(tiles) * H / shape.slots)));
    int64_t items = 0, merges = 0, parts = 0;
    int32_t part_rows = 0;
    each_block(n, shape.rows, [&](int32_t, int32_t, int32_t rows, int32_t, int32_t key1, int32_t) {
        const int32_t s = splits_of(tiles_of(key1), most);
        items += s;
        if (s > 1) {
            ++merges;
            parts += s;
            part_rows = std::max(part_rows, rows);
        }
    });
    // launches of one dispatch: 2 threads per row of an item, one wave per merged row
    if (items > INT32_MAX / 16 || items * H > mla::kMaxDispatchItems / (2 * shape.rows) - 8 ||
        merges * H > mla::kMaxDispatchItems / 64 / shape.rows)
        return MLA_ENOTSUP;
    p.B = B;
    p.H = H;
    p.causal = causal;
    p.rows = shape.rows;
    p.num_items = static_cast<int32_t>(items);
    p.num_merges = static_cast<int32_t>(merges);
    p.num_parts = static_cast<int32_t>(parts);
    p.plan_ints = plan_ints(p);
    p.part_rows = part_rows;
    p.workspace_bytes = parts * H * part_rows * mla::kPartRowBytes;
    *info = p;
    if (plan == nullptr) return MLA_OK;
    if (plan_capacity < p.plan_ints) return MLA_EINVAL;

    auto* item = reinterpret_cast<mla::PrefillItem*>(plan);
    auto* merge = reinterpret_cast<mla::PrefillMerge*>(item + items);
    mla::PrefillItem* const first_item = item;
    int32_t part = 0;
    each_block(n, shape.rows, [&](int32_t b, int32_t q_row, int32_t rows, int32_t kv_row, int32_t key1, int32_t seen0) {
        const int32_t t = tiles_of(key1), s = splits_of(t, most);
        const int32_t per = (t + s - 1) / s * kKeyTile;
        if (s > 1) *merge++ = {q_row, rows, part, s, seen0, kv_lens[b], {0, 0}};
        for (int32_t k = 0; k < s; ++k) {
            const int64_t from = static_cast<int64_t>(k) * per;
            *item++ = {q_row, rows, kv_row, static_cast<int32_t>(std::min<int64_t>(from, key1)),
                       static_cast<int32_t>(std::min<int64_t>(from + per, key1)), seen0, s > 1 ? part++ : -1, b};
        }
    });
    const auto len = [](const mla::PrefillItem& x) { return tiles_of(x.key1 - x.key0); };
    const auto in_order = [](const mla::PrefillItem& x, const mla::PrefillItem& y) {
        return x.q_row != y.q_row ? x.q_row < y.q_row : x.key0 < y.key0;
    };
    if (shape.rows != mla::kListedRows) {
        // the longest first, so that the short ones fill the launch's end
        std::sort(first_item, item, [&](const mla::PrefillItem& x, const mla::PrefillItem& y) {
            return len(x) != len(y) ? len(x) > len(y) : in_order(x, y);
        });
        return MLA_OK;
    }
    // sequence by sequence, the longest first, and so within a sequence
    std::sort(first_item, item, [&](const mla::PrefillItem& x, const mla::PrefillItem& y) {
        if (x.seq != y.seq) {
            const int32_t kx = kv_lens[x.seq], ky = kv_lens[y.seq];
            return kx != ky ? kx > ky : x.seq < y.seq;
        }
        return len(x) != len(y) ? len(x) > len(y) : in_order(x, y);
    });
    fill_lists(first_item, p, plan + (items + merges) * mla::kPrefillRecordInts);
    return MLA_OK;
}

int mla_prefill_attn(const mla_prefill_plan* info, const int32_t* plan, const mla_head_rows* q_nope,
                     const mla_head_rows* q_rope, const mla_head_rows* k_nope, const mla_head_rows* k_rope,
                     const mla_head_rows* v, float softmax_scale, uint16_t* out, int64_t out_stride_t,
                     int64_t out_stride_h, float* lse, void* workspace, int64_t workspace_bytes,
                     hipStream_t stream) {
    if (info == nullptr || info->B < 0 || info->H <= 0) return MLA_EINVAL;
    if (!std::isfinite(softmax_scale) || !(softmax_scale > 0.0f)) return MLA_EINVAL;
    // what the planner fills: nothing else is launched
    // (no more merges or partials than items, so that the products below stay within 64 bits)
    if (info->num_items < 0 || info->num_merges < 0 || info->num_parts < 0 || info->total_q < 0 ||
        info->num_merges > info->num_items || info->num_parts > info->num_items ||
        info->total_kv < 0 || info->total_q > kMaxLen || info->total_kv > kMaxLen)
        return MLA_EINVAL;
    if (info->plan_ints != plan_ints(*info)) return MLA_EINVAL;
    if (info->num_items == 0) return MLA_OK;
    bool known = false;
    for (const Shape& s : kShapes) known = known || s.rows == info->rows;
    if (!known || info->total_q == 0) return MLA_EINVAL;
    if (static_cast<int64_t>(info->num_items) * info->H > mla::kMaxDispatchItems / (2 * info->rows) - 8 ||
        static_cast<int64_t>(info->num_merges) * info->H > mla::kMaxDispatchItems / 64 / info->rows)
        return MLA_ENOTSUP;
    if (info->part_rows < 0 || info->part_rows > info->rows || (info->num_merges > 0 && info->part_rows == 0)) return MLA_EINVAL;
    const int64_t part_rows = static_cast<int64_t>(info->num_parts) * info->H * info->part_rows;
    if (info->workspace_bytes != part_rows * mla::kPartRowBytes) return MLA_EINVAL;
    if (plan == nullptr || out == nullptr) return MLA_EINVAL;
    if (!aligned(plan, 16) || !aligned(out, 16)) return MLA_ENOTSUP;
    mla::PrefillArgs a{};
    const struct {
        const mla_head_rows* from;
        bool heads;
        mla::HeadRows* to;
    } inputs[] = {{q_nope, true, &a.q_nope}, {q_rope, true, &a.q_rope}, {k_nope, true, &a.k_nope},
                  {k_rope, false, &a.k_rope}, {v, true, &a.v}};
    for (const auto& x : inputs) {
        // (no key at all: nothing of the keys and values is read)
        if (info->total_kv == 0 && x.to != &a.q_nope && x.to != &a.q_rope) continue;
        const int st = check_head_rows(x.from, x.heads, x.to);
        if (st != MLA_OK) return st;
    }
    if (out_stride_t < 0 || out_stride_h < 0) return MLA_EINVAL;
    if (out_stride_t % 8 != 0 || out_stride_h % 8 != 0) return MLA_ENOTSUP;
    if (!rows_apart(out_stride_t, out_stride_h, info->total_q, info->H, mla::kValue)) return MLA_EINVAL;
    if (info->workspace_bytes > 0) {
        if (workspace == nullptr || workspace_bytes < info->workspace_bytes) return MLA_EINVAL;
        if (!aligned(workspace, 256)) return MLA_ENOTSUP;
    }
    a.items = reinterpret_cast<const mla::PrefillItem*>(plan);
    a.merges = reinterpret_cast<const mla::PrefillMerge*>(a.items + info->num_items);
    if (info->rows == mla::kListedRows) a.first = reinterpret_cast<const int32_t*>(a.merges + info->num_merges);
    a.num_items = info->num_items;
    a.num_merges = info->num_merges;
    a.num_parts = info->num_parts;
    a.H = info->H;
    a.rows = info->rows;
    a.part_rows = info->part_rows;
    a.total_q = static_cast<int32_t>(info->total_q);
    a.total_kv = static_cast<int32_t>(info->total_kv);
    a.scale_log2 = softmax_scale * 1.4426950408889634f;
    a.out = out;
    a.out_stride_t = out_stride_t;
    a.out_stride_h = out_stride_h;
    a.lse = lse;
    a.part_o = static_cast<float*>(workspace);
    a.part_m = a.part_o + part_rows * mla::kValue;
    a.part_l = a.part_m + part_rows;
    return hip_status(mla::launch_prefill(a, stream));
}

}  // extern "C"
