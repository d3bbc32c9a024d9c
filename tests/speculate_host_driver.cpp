// Host-only driver of the speculative step's C ABI (csrc/mla_speculate_abi.cpp),
// built with AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_speculate_abi_sanitized.py.  The kernel launchers are replaced by
// stubs that keep their arguments.  Exits non-zero on the first failed check; the
// sanitizers abort on any memory error or undefined behaviour.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <limits>
#include <memory>
#include <vector>

#include "abi_checks.h"
#include "mla_speculate.h"
#include "speculate_internal.h"

namespace {
int g_failures = 0, g_attn = 0, g_merge = 0, g_verify = 0, g_commit = 0;
mla::TreeArgs g_tree{};
mla::TreeCombineArgs g_combine{};
mla::VerifyArgs g_walk{};
mla::CommitArgs g_move{};

#define CHECK(cond)                                                              \
    do {                                                                         \
        if (!(cond)) {                                                           \
            std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
            ++g_failures;                                                        \
        }                                                                        \
    } while (0)

uint64_t g_state = 88172645463325252ull;
uint32_t draw(uint32_t n) {
    g_state ^= g_state << 13;
    g_state ^= g_state >> 7;
    g_state ^= g_state << 17;
    return static_cast<uint32_t>((g_state >> 11) % n);
}
}  // namespace

namespace mla {
hipError_t launch_tree_attn(CacheKind, const TreeArgs& a, hipStream_t) { ++g_attn; g_tree = a; return hipSuccess; }
hipError_t launch_tree_combine(const TreeCombineArgs& a, hipStream_t) { ++g_merge; g_combine = a; return hipSuccess; }
hipError_t launch_verify(const VerifyArgs& a, hipStream_t) { ++g_verify; g_walk = a; return hipSuccess; }
hipError_t launch_commit(const CommitArgs& a, bool, hipStream_t) { ++g_commit; g_move = a; return hipSuccess; }
namespace abi {
int hip_status(hipError_t e) { return e == hipSuccess ? MLA_OK : MLA_EHIP; }
}  // namespace abi
}  // namespace mla

namespace {

template <class T> T* at(uintptr_t p) { return reinterpret_cast<T*>(p); }

mla_cache_format format(int32_t c_bits, int32_t page_size, int32_t meta) { return {512, 64, 64, c_bits, 4, page_size, meta}; }

void split_sizes() {
    for (int n = 0; n < 400; ++n) {
        const int32_t B = static_cast<int32_t>(draw(n % 10 == 0 ? 300 : 40));
        std::unique_ptr<int32_t[]> lens(new int32_t[B > 0 ? B : 1]);
        int32_t longest = 0;
        for (int32_t b = 0; b < B; ++b) {
            lens[b] = static_cast<int32_t>(1 + draw(draw(4) == 0 ? 200000 : 3000));
            if (draw(50) == 0) lens[b] = INT_MAX;
            longest = lens[b] > longest ? lens[b] : longest;
        }
        const int32_t nodes = static_cast<int32_t>(1 + draw(64)), H = static_cast<int32_t>(1 + draw(130));
        const int32_t s = mla_tree_split_tokens(lens.get(), B, nodes, H);
        CHECK(s >= 0 && s % 32 == 0);
        CHECK(s == 0 || s < longest);
    }
    const int32_t huge[3] = {INT_MAX, INT_MAX, INT_MAX};
    CHECK(mla_tree_split_tokens(huge, 3, 64, 16384) >= 0);
    CHECK(mla_tree_split_tokens(huge, 3, 64, 16385) == -MLA_ENOTSUP);
    CHECK(mla_tree_split_tokens(huge, 3, INT_MAX, INT_MAX) == -MLA_ENOTSUP);
    CHECK(mla_tree_split_tokens(nullptr, 0, 1, 1) == 0);
}

int attn(const mla_cache_format& f, bool low, int32_t num_nodes, int32_t max_nodes, int32_t B, int32_t H, int32_t split, int32_t splits,
         int64_t bytes, int32_t max_pages = 4) {
    const auto call = low ? mla_lowbit_tree_attn : mla_bf16_tree_attn;
    return call(&f, at<uint16_t>(4096), at<uint16_t>(8192), at<void>(1 << 20), 9, at<int32_t>(64), max_pages, at<int32_t>(128),
                at<int32_t>(192), at<uint64_t>(256), num_nodes, max_nodes, B, H, 0.07f, split, at<int32_t>(320), splits,
                at<uint16_t>(1 << 16), at<float>(1 << 17), at<void>(1 << 18), bytes, nullptr);
}

void attention() {
    const mla_cache_format f = format(4, 64, MLA_META_FP16);
    for (int n = 0; n < 2000; ++n) {
        const int32_t nodes = static_cast<int32_t>(1 + draw(64)), H = static_cast<int32_t>(1 + draw(256)), splits = static_cast<int32_t>(draw(500));
        const int64_t bytes = mla_tree_workspace_bytes(splits, nodes, H);
        const int before = g_attn;
        CHECK(attn(f, draw(2) == 0, 70, nodes, 3, H, 64, splits, bytes) == MLA_OK);
        CHECK(g_attn == before + 1 && g_tree.num_work == splits && g_tree.s_q == nodes);
        // partials lie inside the workspace, one after the other
        const int64_t rows = int64_t{splits} * nodes * H;
        CHECK(reinterpret_cast<uintptr_t>(g_tree.part_m) == (1 << 18) + static_cast<uintptr_t>(rows) * 1024);
        CHECK(reinterpret_cast<uintptr_t>(g_tree.part_s + rows) == (1 << 18) + static_cast<uintptr_t>(bytes));
        CHECK(g_combine.part_s == g_tree.part_s && g_combine.num_splits == splits);
        CHECK(g_tree.shape.rows == (nodes * H <= 64 ? 64 : 128) && g_tree.shape.waves == 4);
        if (bytes > 0) CHECK(attn(f, true, 70, nodes, 3, H, 64, splits, bytes - 1) == MLA_EINVAL);
        const int merges = g_merge;
        CHECK(attn(f, true, 70, nodes, 3, H, 0, 0, 0) == MLA_OK && g_merge == merges && g_tree.num_work == 3);
    }
    const int launches = g_attn;
    CHECK(attn(f, true, 1, 64, INT_MAX, 16384, 0, 0, 0) == MLA_ENOTSUP);
    CHECK(attn(f, true, INT_MAX, 64, INT_MAX, 1, 64, INT_MAX, LLONG_MAX) == MLA_ENOTSUP);
    CHECK(attn(f, true, 1, 1, 1, 1, 0, 0, 0, INT_MAX) == MLA_ENOTSUP);
    CHECK(attn(f, true, 1, 1, 1, 1, INT_MAX - 31, 1, LLONG_MAX) == MLA_ENOTSUP);
    CHECK(g_attn == launches);
    // launch sizes: whole rounds of runs over the 8 XCDs, every work item's row blocks among them
    for (int64_t work = 0; work < 300; work += 7)
        for (int64_t rows = 1; rows < 9000; rows += 61) {
            const int64_t blocks = (rows + 127) / 128, groups = mla::tree_workgroups(work, rows, 128), run = mla::tree_run(static_cast<int>(blocks));
            CHECK(groups % (8 * run) == 0 && groups >= work * blocks && groups < work * blocks + 8 * run && run >= 1 && run <= 8);
            // block -> position is one to one
            std::vector<char> seen(static_cast<size_t>(groups), 0);
            for (int64_t i = 0; i < groups; ++i) {
                const int64_t p = run * ((i >> 3) / run * 8 + (i & 7)) + (i >> 3) % run;
                CHECK(p >= 0 && p < groups && !seen[static_cast<size_t>(p)]);
                if (p >= 0 && p < groups) seen[static_cast<size_t>(p)] = 1;
            }
        }
    // node ranges stay in the arrays for any values
    const int32_t values[] = {INT_MIN, -1, 0, 1, 5, 9, 10, 11, 1000, INT_MAX};
    for (int32_t c0 : values)
        for (int32_t c1 : values)
            for (int32_t total : {0, 1, 10}) {
                const int32_t cu[2] = {c0, c1};
                const mla::NodeRange r = mla::node_range(cu, 0, total, 6);
                CHECK(r.first >= 0 && r.count >= 0 && r.count <= 6 && r.first + r.count <= total);
            }
}

void verification() {
    for (int n = 0; n < 2000; ++n) {
        const int32_t nodes = static_cast<int32_t>(draw(300)), B = static_cast<int32_t>(1 + draw(70)), V = static_cast<int32_t>(1 + draw(200000));
        const int64_t bytes = mla_verify_workspace_bytes(nodes, B, V);
        auto call = [&](int64_t have) {
            return mla_verify_tree(at<void>(64), MLA_LOGITS_FP32, V + 3, V, draw(2) ? at<float>(128) : nullptr, V, at<int32_t>(192),
                                   at<int32_t>(256), at<int32_t>(320), nodes, 1 + static_cast<int32_t>(draw(64)), B, nullptr, at<float>(384),
                                   at<float>(448), at<int32_t>(512), at<int32_t>(576), nullptr, at<int32_t>(640), at<void>(1 << 20), have, nullptr);
        };
        CHECK(call(bytes) == MLA_OK);
        const int64_t chunks = mla::logit_chunks(V);
        CHECK(reinterpret_cast<uintptr_t>(g_walk.sums) == (1 << 20) + static_cast<uintptr_t>(nodes * chunks * 16));
        CHECK(reinterpret_cast<uintptr_t>(g_walk.arrived + B) == (1 << 20) + static_cast<uintptr_t>(bytes));
        CHECK(call(bytes - 1) == MLA_EINVAL);
    }
    CHECK(mla_verify_workspace_bytes(INT_MAX, INT_MAX, 1 << 21) > 0);
    CHECK(mla_verify_workspace_bytes(INT_MAX, INT_MAX, INT_MAX) == -1);
}

void commits() {
    for (int32_t meta : {MLA_META_FP16, MLA_META_PAPER})
        for (int32_t bits : {2, 4})
            for (int32_t page : {32, 64, 1 << 20}) {
                const mla_cache_format f = format(bits, page, meta);
                CHECK(mla_lowbit_commit(&f, at<void* const>(64), 3, 5, at<int32_t>(128), 7, at<int32_t>(192), at<int32_t>(256),
                                        at<int32_t>(320), 64, 9, at<int32_t>(384), nullptr) == MLA_OK);
                CHECK(g_move.g.page_size == page && g_move.g.page_bytes == mla::abi::lowbit_geom(&f).page_bytes);
                // the kernel's page of a position: the multiplication gives the quotient or one less
                for (uint32_t t : {0u, 1u, static_cast<uint32_t>(page) - 1, static_cast<uint32_t>(page), 123456789u, (1u << 30) - 1}) {
                    const uint32_t q = static_cast<uint32_t>((uint64_t{t} * g_move.g.page_magic) >> 32);
                    CHECK(q == t / page || q + 1 == t / page);
                }
            }
    const mla_cache_format f = format(4, 64, 0);
    const int before = g_commit;
    CHECK(mla_bf16_commit(&f, nullptr, 0, 0, nullptr, 1, at<int32_t>(64), at<int32_t>(128), at<int32_t>(192), 1, 4, at<int32_t>(256), nullptr) == MLA_OK);
    CHECK(g_commit == before + 1);
    CHECK(mla_bf16_commit(&f, at<void* const>(64), INT_MAX, 5, at<int32_t>(128), 7, at<int32_t>(192), at<int32_t>(256), at<int32_t>(320), 64,
                          65535, nullptr, nullptr) == MLA_ENOTSUP);
    CHECK(g_commit == before + 1);
}

}  // namespace

int main() {
    split_sizes();
    attention();
    verification();
    commits();
    if (g_failures == 0) std::printf("all checks passed\n");
    return g_failures == 0 ? 0 : 1;
}
