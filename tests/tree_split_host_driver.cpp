// Host-only driver of the split choice of tree calls whose node counts are given
// (csrc/mla_speculate_abi.cpp), built with AddressSanitizer and
// UndefinedBehaviorSanitizer by tests/test_tree_split_sanitized.py.  The arrays are
// exactly as long as the call may read; the launchers are never reached.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <memory>

#include "abi_checks.h"
#include "mla_speculate.h"
#include "speculate_internal.h"

namespace mla {
hipError_t launch_tree_attn(CacheKind, const TreeArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_tree_combine(const TreeCombineArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_verify(const VerifyArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_commit(const CommitArgs&, bool, hipStream_t) { return hipErrorUnknown; }
namespace abi {
int hip_status(hipError_t e) { return e == hipSuccess ? MLA_OK : MLA_EHIP; }
}  // namespace abi
}  // namespace mla

namespace {
uint64_t g_state = 88172645463325252ull;
uint32_t draw(uint32_t n) {
    g_state ^= g_state << 13;
    g_state ^= g_state >> 7;
    g_state ^= g_state << 17;
    return static_cast<uint32_t>((g_state >> 11) % n);
}
}  // namespace

int main() {
    for (int n = 0; n < 600; ++n) {
        const int32_t B = static_cast<int32_t>(draw(n % 10 == 0 ? 300 : 90)), most = static_cast<int32_t>(1 + draw(64));
        const int32_t H = n % 50 == 0 ? (1 << 20) / most : static_cast<int32_t>(1 + draw(130));
        std::unique_ptr<int32_t[]> lens(new int32_t[B > 0 ? B : 1]), nodes(new int32_t[B > 0 ? B : 1]);
        int32_t longest = 0;
        for (int32_t b = 0; b < B; ++b) {
            lens[b] = draw(50) == 0 ? INT_MAX : static_cast<int32_t>(1 + draw(draw(4) == 0 ? 200000 : 3000));
            nodes[b] = static_cast<int32_t>(draw(static_cast<uint32_t>(n % 7 == 0 ? 1 : most + 1)));
            longest = lens[b] > longest ? lens[b] : longest;
        }
        const int32_t s = mla_tree_split_tokens_for(lens.get(), nodes.get(), B, most, H);
        if (s < 0 || s % 32 != 0 || (s != 0 && s >= longest)) {
            std::fprintf(stderr, "batch %d: size %d\n", n, s);
            return 1;
        }
        if (B > 0) {
            nodes[B - 1] = most + 1;
            if (mla_tree_split_tokens_for(lens.get(), nodes.get(), B, most, H) != -MLA_EINVAL) return 1;
            nodes[B - 1] = INT_MIN;
            if (mla_tree_split_tokens_for(lens.get(), nodes.get(), B, most, H) != -MLA_EINVAL) return 1;
        }
    }
    std::printf("all checks passed\n");
    return 0;
}
