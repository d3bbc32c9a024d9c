// Host-only driver of the prompt side's C ABI (csrc/mla_prefill_abi.cpp), built
// with AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_prefill_abi_sanitized.py.  The kernel launchers are replaced by
// stubs that keep their arguments.  Plans are made into buffers of exactly
// plan_ints values, from heap copies of the lengths, and checked to cover every
// visible (row, key) pair once.  Exits non-zero on the first failed check; the
// sanitizers abort on any memory error or undefined behaviour.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstdio>
#include <limits>
#include <memory>
#include <vector>

#include "abi_checks.h"
#include "mla_prefill.h"
#include "prefill_internal.h"

namespace {
int g_failures = 0, g_launches = 0;
mla::PrefillArgs g_prefill{};
mla::NormRopeArgs g_append{};
mla::GatherArgs g_gather{};
mla::RopeArgs g_rope{};

#define CHECK(cond)                                                              \
    do {                                                                         \
        if (!(cond)) {                                                           \
            std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
            ++g_failures;                                                        \
        }                                                                        \
    } while (0)
}  // namespace

namespace mla {
hipError_t launch_norm_rope_append(const NormRopeArgs& a, bool, hipStream_t) { ++g_launches; g_append = a; return hipSuccess; }
hipError_t launch_rope_queries(const RopeArgs& a, hipStream_t) { ++g_launches; g_rope = a; return hipSuccess; }
hipError_t launch_gather(const GatherArgs& a, bool, hipStream_t) { ++g_launches; g_gather = a; return hipSuccess; }
hipError_t launch_prefill(const PrefillArgs& a, hipStream_t) { ++g_launches; g_prefill = a; return hipSuccess; }
namespace abi {
int hip_status(hipError_t e) { return e == hipSuccess ? MLA_OK : MLA_EHIP; }
}  // namespace abi
}  // namespace mla

namespace {

uint64_t g_state = 88172645463325252ull;
uint32_t draw(uint32_t n) {         // 0 .. n - 1
    g_state ^= g_state << 13;
    g_state ^= g_state >> 7;
    g_state ^= g_state << 17;
    return static_cast<uint32_t>((g_state >> 11) % n);
}
int32_t spread(uint32_t most) {     // spread over the logarithm, zeros among them
    if (draw(12) == 0) return 0;
    uint32_t top = 1;
    while (top < most && draw(5) != 0) top *= 3;
    return static_cast<int32_t>(draw(std::min(top, most)) + 1);
}

struct Batch {
    std::vector<int32_t> q, kv, qs, ks;
    int32_t H, causal;
    bool q_starts, kv_starts;
};

// A plan in a buffer of exactly its size (nullptr: refused with `status`).
std::unique_ptr<int32_t[]> plan_of(const Batch& b, mla_prefill_plan* info, int* status) {
    const int32_t B = static_cast<int32_t>(b.q.size());
    const int32_t* qs = b.q_starts ? b.qs.data() : nullptr;
    const int32_t* ks = b.kv_starts ? b.ks.data() : nullptr;
    *status = mla_plan_prefill(b.q.data(), b.kv.data(), qs, ks, B, b.H, b.causal, nullptr, 0, info);
    if (*status != MLA_OK) return nullptr;
    std::unique_ptr<int32_t[]> plan(new int32_t[info->plan_ints]);
    mla_prefill_plan again{};
    CHECK(mla_plan_prefill(b.q.data(), b.kv.data(), qs, ks, B, b.H, b.causal, plan.get(), info->plan_ints, &again) == MLA_OK);
    CHECK(again.plan_ints == info->plan_ints && again.num_items == info->num_items && again.workspace_bytes == info->workspace_bytes);
    if (info->plan_ints > 0)
        CHECK(mla_plan_prefill(b.q.data(), b.kv.data(), qs, ks, B, b.H, b.causal, plan.get(), info->plan_ints - 1, &again) == MLA_EINVAL);
    return plan;
}

void check_plan(const Batch& b, const mla_prefill_plan& info, const int32_t* plan) {
    const auto* items = reinterpret_cast<const mla::PrefillItem*>(plan);
    const auto* merges = reinterpret_cast<const mla::PrefillMerge*>(items + info.num_items);
    int64_t want = 0, got = 0;
    for (size_t s = 0; s < b.q.size(); ++s)
        for (int32_t i = 0; i < b.q[s]; ++i) {
            const int64_t sees = b.causal ? std::clamp<int64_t>(static_cast<int64_t>(b.kv[s]) - b.q[s] + i + 1, 0, b.kv[s]) : b.kv[s];
            want += sees;
        }
    std::vector<int> parts(info.num_parts, 0);
    for (int32_t i = 0; i < info.num_items; ++i) {
        const mla::PrefillItem& x = items[i];
        CHECK(x.q_row >= 0 && x.q_rows >= 1 && x.q_rows <= info.rows && x.q_row + x.q_rows <= info.total_q);
        CHECK(x.key0 >= 0 && x.key0 <= x.key1 && x.key1 - x.key0 <= b.kv[x.seq] && x.kv_row >= 0);
        CHECK(x.key1 == 0 || x.kv_row + x.key1 <= info.total_kv);
        CHECK(x.part >= -1 && x.part < info.num_parts);
        if (x.part >= 0) ++parts[x.part];
        for (int32_t r = 0; r < x.q_rows; ++r)
            got += std::max<int64_t>(0, std::min<int64_t>(x.key1, static_cast<int64_t>(x.seen0) + r) - x.key0);
    }
    CHECK(want == got);
    for (int32_t i = 0; i < info.num_merges; ++i) {
        CHECK(merges[i].num_parts > 1 && merges[i].q_rows <= info.part_rows);
        for (int32_t k = 0; k < merges[i].num_parts; ++k) ++parts[merges[i].part0 + k];
    }
    for (const int n : parts) CHECK(n == 2);
    const mla::PrefillLists l = mla::prefill_lists(info.num_items, info.H, info.rows);
    const int32_t* first = reinterpret_cast<const int32_t*>(merges + info.num_merges);
    if (l.lists > 0) {
        CHECK(first[0] == 0 && first[l.lists] == l.entries);
        std::vector<bool> there(l.entries, false);
        for (int64_t i = 0; i < l.entries; ++i) {
            const int32_t e = first[l.lists + 1 + i], x = e < 0 ? ~e : e;
            CHECK(x >= 0 && x < l.entries && !there[x]);
            there[x] = true;
        }
        for (int32_t i = 0; i < l.lists; ++i) CHECK(first[i] < first[i + 1]);
    }
}

alignas(256) uint16_t g_rows[1 << 12];

int attend(const mla_prefill_plan& info, const int32_t* plan) {
    const mla_head_rows r{g_rows, 256, 128};
    return mla_prefill_attn(&info, plan, &r, &r, &r, &r, &r, 0.07f, g_rows, static_cast<int64_t>(info.H) * 128, 128, nullptr,
                            g_rows, std::numeric_limits<int64_t>::max(), nullptr);
}

void random_plans() {
    for (int n = 0; n < 3000; ++n) {
        Batch b;
        const int32_t B = n % 50 == 0 ? static_cast<int32_t>(draw(300)) : spread(12);
        b.H = n % 3 == 0 ? 8 * (1 + static_cast<int32_t>(draw(16))) : 1 + static_cast<int32_t>(draw(128));
        b.causal = draw(3) != 0;
        b.q_starts = draw(4) == 0;
        b.kv_starts = draw(4) == 0;
        int32_t at = 0;
        for (int32_t s = 0; s < B; ++s) {
            b.q.push_back(spread(draw(3) == 0 ? 3000 : 300));
            b.kv.push_back(spread(draw(4) == 0 ? 60000 : 3000));
            b.qs.push_back(at += static_cast<int32_t>(draw(40)));
            at += b.q.back();
            b.ks.push_back(static_cast<int32_t>(draw(1000)));
        }
        mla_prefill_plan info{};
        int status = 0;
        const auto plan = plan_of(b, &info, &status);
        CHECK(status == MLA_OK);
        if (plan == nullptr) continue;
        check_plan(b, info, plan.get());
        const int before = g_launches;
        // (the plan's address stands for the device copy's: 16-byte aligned)
        std::vector<int32_t> copy(info.plan_ints + 4);
        int32_t* aligned = copy.data() + (16 - reinterpret_cast<uintptr_t>(copy.data()) % 16) % 16 / 4;
        CHECK(attend(info, aligned) == MLA_OK);
        CHECK(g_launches == before + (info.num_items > 0));
        if (info.num_items > 0)
            CHECK(g_prefill.num_items == info.num_items && g_prefill.num_parts == info.num_parts && g_prefill.H == info.H &&
                  g_prefill.part_m == g_prefill.part_o + static_cast<int64_t>(info.num_parts) * info.H * info.part_rows * 128);
    }
}

void limits() {
    mla_prefill_plan info{};
    const int32_t big = 1 << 30;
    const auto status = [&](std::vector<int32_t> q, std::vector<int32_t> kv, int32_t H, std::vector<int32_t> qs = {},
                            std::vector<int32_t> ks = {}) {
        return mla_plan_prefill(q.data(), kv.data(), qs.empty() ? nullptr : qs.data(), ks.empty() ? nullptr : ks.data(),
                                static_cast<int32_t>(q.size()), H, 1, nullptr, 0, &info);
    };
    CHECK(status({1}, {big}, 1) == MLA_OK && info.total_kv == big);
    CHECK(status({1}, {big}, 128) == MLA_OK);
    CHECK(status({1}, {INT_MAX}, 1) == MLA_ENOTSUP && status({INT_MAX}, {1}, 1) == MLA_ENOTSUP);
    CHECK(status({big, 1}, {1, 1}, 1) == MLA_ENOTSUP && status({1, 1}, {big, big}, 1) == MLA_ENOTSUP);
    CHECK(status({1}, {1}, 1, {INT_MAX}) == MLA_ENOTSUP && status({1}, {1}, 1, {}, {INT_MAX}) == MLA_ENOTSUP);
    CHECK(status({1, 1}, {1, 1}, 1, {big - 1, 0}, {0, big - 1}) == MLA_OK && info.total_q == big && info.total_kv == big);
    CHECK(status({1}, {1}, INT_MAX) == MLA_ENOTSUP && status({big}, {big}, INT_MAX) == MLA_ENOTSUP);
    CHECK(status({INT_MIN}, {1}, 1) == MLA_EINVAL && status({1}, {INT_MIN}, 1) == MLA_EINVAL && status({1}, {1}, INT_MIN) == MLA_EINVAL);
    CHECK(status({big}, {0}, 1) == MLA_OK && status({300}, {big}, 1) == MLA_OK);
    CHECK(mla_plan_prefill(nullptr, nullptr, nullptr, nullptr, 0, 1, 1, nullptr, 0, &info) == MLA_OK && info.plan_ints == 0);
}

// What a caller may hand in as `info`: every refusal without overflow.
void infos() {
    Batch b{{40, 3}, {5000, 70}, {}, {}, 2, 1, false, false};
    mla_prefill_plan good{};
    int status = 0;
    plan_of(b, &good, &status);
    alignas(16) static int32_t plan[1 << 12];
    CHECK(attend(good, plan) == MLA_OK);
    const int32_t values[] = {INT_MIN, -1, 0, 1, 2, 128, 256, 1 << 24, 1 << 30, INT_MAX};
    int32_t mla_prefill_plan::*const fields[] = {&mla_prefill_plan::B, &mla_prefill_plan::H, &mla_prefill_plan::rows,
                                                 &mla_prefill_plan::num_items, &mla_prefill_plan::num_merges,
                                                 &mla_prefill_plan::num_parts, &mla_prefill_plan::part_rows};
    for (const auto f : fields)
        for (const auto g : fields)
            for (const int32_t v : values)
                for (const int32_t w : values) {
                    mla_prefill_plan p = good;
                    p.*f = v;
                    p.*g = w;
                    attend(p, plan);
                    // with sizes that fit the counts, so that the later checks are reached
                    const mla::PrefillLists l = p.H > 0 && p.num_items >= 0 ? mla::prefill_lists(p.num_items, p.H, p.rows) : mla::PrefillLists{};
                    p.plan_ints = (static_cast<int64_t>(p.num_items) + p.num_merges) * mla::kPrefillRecordInts +
                                  (l.lists > 0 ? l.lists + 1 + l.entries : 0);
                    attend(p, plan);
                }
    for (const int64_t v : {INT64_MIN, int64_t{-1}, int64_t{0}, INT64_MAX}) {
        mla_prefill_plan p = good;
        p.total_q = v;
        CHECK(attend(p, plan) == MLA_EINVAL);
        p = good;
        p.workspace_bytes = v;
        CHECK(attend(p, plan) == MLA_EINVAL);
        p = good;
        p.plan_ints = v;
        CHECK(attend(p, plan) == MLA_EINVAL);
    }
    // more partials than items is no planner's
    mla_prefill_plan p = good;
    p.num_parts = p.num_items + 1;
    p.workspace_bytes = static_cast<int64_t>(p.num_parts) * p.H * p.part_rows * mla::kPartRowBytes;
    CHECK(attend(p, plan) == MLA_EINVAL);
}

void others() {
    const mla_cache_format f{512, 64, 64, 4, 4, 64, MLA_META_FP16};
    const mla_protect_policy policy{4, 128};
    alignas(16) static float table[64];
    const mla_rotation rot{table, 1, MLA_ROPE_PAIRS};
    const mla_rms_norm norm{nullptr, 1e-6f};
    int32_t ints[4] = {};
    int64_t slots[4] = {};
    CHECK(mla_lowbit_norm_rope_append(&f, &norm, &rot, g_rows, 512, g_rows, 64, ints, slots, 4, g_rows, 1 << 20, g_rows, 512, nullptr, 0, nullptr) == MLA_OK);
    CHECK(g_append.append.num_slots == int64_t{64} << 20 && g_append.has_norm == 1 && g_append.append.prot == nullptr);
    CHECK(mla_lowbit_norm_rope_append_protected(&f, &policy, nullptr, &rot, g_rows, 512, g_rows, 64, ints, slots, 4, g_rows, 9, ints, ints,
                                                ints, 1, g_rows, 1, nullptr, 0, nullptr, 0, nullptr) == MLA_OK);
    CHECK(g_append.append.sink == 4 && g_append.append.recent == 128 && g_append.has_norm == 0);
    CHECK(mla_bf16_norm_rope_append(&f, &norm, &rot, g_rows, INT64_MAX - 7, g_rows, 64, ints, slots, 1, g_rows, INT64_MAX / 64, nullptr, 0, nullptr, 0, nullptr) == MLA_OK);
    CHECK(mla_lowbit_gather(&f, g_rows, INT64_MAX, ints, INT_MAX, nullptr, ints, INT_MAX, 1 << 25, g_rows, 512, g_rows, 64, nullptr) == MLA_OK);
    CHECK(mla_lowbit_gather_protected(&f, &policy, g_rows, 1, ints, 1, ints, ints, 1, 1, ints, g_rows, INT64_MAX, ints, g_rows, 512, g_rows, 64, nullptr) == MLA_OK);
    CHECK(mla_bf16_gather(&f, g_rows, 1, ints, 1, nullptr, ints, 1, INT_MAX, g_rows, 512, g_rows, 64, nullptr) == MLA_ENOTSUP);
    CHECK(mla_rope_queries(&rot, g_rows, 0, 0, ints, INT_MAX, INT_MAX, g_rows, 64, 0, nullptr) == MLA_EINVAL);
    CHECK(mla_rope_queries(&rot, g_rows, 0, 0, ints, INT_MAX, INT_MAX, g_rows + 512, int64_t{64} * INT_MAX, 64, nullptr) == MLA_ENOTSUP);
    CHECK(mla_rope_queries(&rot, g_rows, 128, 64, ints, 4, 2, g_rows, 128, 64, nullptr) == MLA_OK);
}

}  // namespace

int main() {
    random_plans();
    limits();
    infos();
    others();
    if (g_failures != 0) return 1;
    std::puts("all checks passed");
    return 0;
}
