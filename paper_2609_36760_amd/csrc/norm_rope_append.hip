// Writers with norm and rotation on the way (mla_*_norm_rope_append): the
// content latent's RMS norm and the RoPE key's rotation, then the library's
// quantizer and slot-mapped insertion (writer_common.h) of the bf16 results,
// which also go out as dense rows.
//
// A wave takes the 512 content channels of kTok tokens (64 lanes x 8 channels,
// 16 bytes a lane), or the RoPE keys of 8 tokens (8 lanes each).  The content
// waves come first; the RoPE waves run beside them.
//
// Memory bounds it where there are many tokens: 1152 bytes read, as many written dense
// and 324 (4 bits) packed.  64K tokens, dense rows too, caches cold: 42 us with 4 bits (38
// at a copy's rate), 54 protected (39), 43 into the BF16 cache (49).
//
// The norm: squares of bf16 values are exact in fp64, and the sum of 512 of
// them is rounded so far below bf16 that the order of the reduction does not
// show; x w is exact there too, and its product with 1 / sqrt(mean + eps) is
// rounded to fp32 and then to bf16.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "prefill_internal.h"
#include "rotation.h"
#include "writer_common.h"

namespace mla {
namespace {

constexpr int kThreads = 256;
constexpr int kRopeTokens = 8;      // of a RoPE wave
constexpr int kManyTokens = 16384;

__device__ __forceinline__ double lane_value(double v, int lane) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(u), lane), hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(u >> 32), lane);
    return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}

// Where a token goes: its slot (-1: skipped), and its row of the protection
// buffers (-1: not protected).
struct Place {
    int64_t slot, prot_row;
};
template <bool kProt>
__device__ __forceinline__ Place place_of(const AppendArgs& a, int64_t token) {
    const int64_t slot = a.slot_mapping[token];
    Place at{slot >= 0 && slot < a.num_slots ? slot : -1, -1};
    if constexpr (kProt) {
        const int b = a.token_seq[token], p = a.positions[token];
        const int bs = min(max(b, 0), a.B - 1);        // B >= 1
        const int L = a.seq_lens[bs];
        const int64_t ps = a.prot_slot[bs];
        // p >= L - recent with p < L implies recent >= 1
        if (at.slot >= 0 && b >= 0 && b < a.B && p >= 0 && p < L && (p < a.sink || p >= L - a.recent) && ps >= 0 &&
            ps < a.num_prot)
            at.prot_row = ps * (a.sink + a.recent) + (p < a.sink ? p : a.sink + (p - a.sink) % a.recent);
    }
    return at;
}

// The lane's 8 finished channels into the cache (and the protection buffer).
template <int CBITS, bool kProt, bool kPaper>
__device__ __forceinline__ void store(const AppendArgs& a, const Place& at, const uint4 x, bool rope, int g, int lig) {
    if (at.slot < 0) return;
    const int column = rope ? 1024 + lig * 16 : g * 128 + lig * 16;     // byte of a bf16 row
    if constexpr (kProt) {
        if (at.prot_row >= 0) *reinterpret_cast<uint4*>(a.prot + at.prot_row * 1152 + column) = x;
    }
    const wc::SlotPos s = wc::split_slot(at.slot, a.num_slots, a.g);
    uint8_t* page = a.cache + s.page * a.g.page_bytes;
    if constexpr (CBITS == 16)
        *reinterpret_cast<uint4*>(page + s.off * 1152 + column) = x;
    else
        wc::quantize_store<CBITS, kPaper>(x, rope, g, lig, page, s.off, a.g);
}

// CBITS 16: the BF16 cache.
template <int CBITS, bool kProt, bool kPaper, int kTok>
__global__ __launch_bounds__(kThreads) void norm_rope_append_kernel(NormRopeArgs a) {
    const AppendArgs& p = a.append;
    const int lane = static_cast<int>(threadIdx.x & 63), g = lane >> 3, lig = lane & 7;
    const uint32_t wave = __builtin_amdgcn_readfirstlane((blockIdx.x * kThreads + threadIdx.x) >> 6);
    const uint32_t content_waves = (static_cast<uint32_t>(p.n) + kTok - 1) / kTok;
    if (wave < content_waves) {
        const int64_t first = static_cast<int64_t>(wave) * kTok;
        uint4 raw[kTok];
        Place at[kTok];
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
            const int64_t token = min(first + i, static_cast<int64_t>(p.n) - 1);
            raw[i] = *reinterpret_cast<const uint4*>(p.c_kv + token * p.c_kv_stride + lane * 8);
            at[i] = place_of<kProt>(p, token);
        }
        if (a.has_norm) {
            float w[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
            if (a.weight != nullptr) wc::widen_bf16x8(*reinterpret_cast<const uint4*>(a.weight + lane * 8), w);
            double ss[kTok];
#pragma unroll
            for (int i = 0; i < kTok; ++i) {
                float x[8];
                wc::widen_bf16x8(raw[i], x);
                ss[i] = 0.0;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss[i] = fma(static_cast<double>(x[j]), static_cast<double>(x[j]), ss[i]);
            }
            // Sums over the wave of all tokens at once: each step halves the tokens that a
            // lane holds, so a lane ends with one token's sum and 1 / sqrt is taken once.
            int m = 32;
#pragma unroll
            for (int k = kTok / 2; k >= 1; k >>= 1, m >>= 1)
#pragma unroll
                for (int i = 0; i < k; ++i) {
                    const bool upper = (lane & m) != 0;
                    const double mine = upper ? ss[i + k] : ss[i], other = upper ? ss[i] : ss[i + k];
                    ss[i] = mine + __shfl_xor(other, m);
                }
#pragma unroll
            for (; m >= 1; m >>= 1) ss[0] += __shfl_xor(ss[0], m);
            const double inv = 1.0 / sqrt(ss[0] / 512.0 + a.eps);
#pragma unroll
            for (int i = 0; i < kTok; ++i) {
                const double r = lane_value(inv, i * (64 / kTok));
                float x[8];
                wc::widen_bf16x8(raw[i], x);
                uint32_t y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    y[j] = rt::bf16x2_of(static_cast<double>(x[2 * j]) * w[2 * j] * r, static_cast<double>(x[2 * j + 1]) * w[2 * j + 1] * r);
                raw[i] = make_uint4(y[0], y[1], y[2], y[3]);
            }
        }
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
            if (first + i >= p.n) break;
            if (a.c_out != nullptr) *reinterpret_cast<uint4*>(a.c_out + (first + i) * a.c_out_stride + lane * 8) = raw[i];
            store<CBITS, kProt, kPaper>(p, at[i], raw[i], false, g, lig);
        }
        return;
    }
    const int64_t token = static_cast<int64_t>(wave - content_waves) * kRopeTokens + g;
    if (token >= p.n) return;       // (whole groups of 8 lanes)
    uint4 x = *reinterpret_cast<const uint4*>(p.k_rope + token * p.k_rope_stride + lig * 8);
    const Place at = place_of<kProt>(p, token);
    const bool halves = a.rot.halves != 0;
    x = rt::rotate(x, rt::load_angles(rt::table_row(a.rot, p.positions[token]), halves, lig), halves, lig);
    if (a.k_out != nullptr) *reinterpret_cast<uint4*>(a.k_out + token * a.k_out_stride + lig * 8) = x;
    store<CBITS, kProt, kPaper>(p, at, x, true, 8, lig);
}

template <int CBITS, bool kProt, bool kPaper, int kTok>
hipError_t launch_rows(const NormRopeArgs& a, hipStream_t stream) {
    const int64_t n = a.append.n;
    const int64_t waves = (n + kTok - 1) / kTok + (n + kRopeTokens - 1) / kRopeTokens;
    static_assert((kMaxAppendTokens + kMaxAppendTokens / kRopeTokens + 1) * 64 + kThreads <= kMaxDispatchItems, "launch size");
    const int64_t groups = (waves * 64 + kThreads - 1) / kThreads;
    hipLaunchKernelGGL((norm_rope_append_kernel<CBITS, kProt, kPaper, kTok>), dim3(static_cast<unsigned>(groups)),
                       dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}
template <int CBITS, bool kProt, bool kPaper>
hipError_t launch_as(const NormRopeArgs& a, hipStream_t stream) {
    // Two tokens per wave share the root and overlap their loads, where there are waves
    // enough for the card all the same (64K tokens, 4 bits, protected: 53 us against
    // 60; 32K: 29 against 32; 16K: 18.6 against 18.3, unprotected 13.5 against 14.5; below no
    // difference).
    if (a.append.n >= kManyTokens) return launch_rows<CBITS, kProt, kPaper, 2>(a, stream);
    return launch_rows<CBITS, kProt, kPaper, 1>(a, stream);
}

}  // namespace

hipError_t launch_norm_rope_append(const NormRopeArgs& a, bool lowbit, hipStream_t stream) {
    if (!lowbit) return launch_as<16, false, false>(a, stream);
    const bool prot = a.append.prot != nullptr, paper = a.append.g.paper_meta != 0;
    if (a.append.g.c_bits == 4) {
        if (prot) return paper ? launch_as<4, true, true>(a, stream) : launch_as<4, true, false>(a, stream);
        return paper ? launch_as<4, false, true>(a, stream) : launch_as<4, false, false>(a, stream);
    }
    if (prot) return paper ? launch_as<2, true, true>(a, stream) : launch_as<2, true, false>(a, stream);
    return paper ? launch_as<2, false, true>(a, stream) : launch_as<2, false, false>(a, stream);
}

}  // namespace mla
