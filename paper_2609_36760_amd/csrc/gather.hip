// Cached tokens read back as dense bf16 rows (mla_*_gather): the packed codes of
// a token become bf16(scale * (q - zero)), the product rounded to fp32 first;
// BF16 rows (the BF16 cache, protected tokens) are copied bit for bit.
//
// A wave takes the 512 content channels of an output row (64 lanes x 8 channels:
// one 4-bit code word in, 16 bytes out) or the RoPE keys of 8 rows, or, of many rows,
// both of 8.
// The bytes written are three times the bytes read, so the work split follows
// the output: every store instruction writes whole rows.
//
// Memory bounds it.  128K rows, 4 bits, over 2.6 GB of inputs and outputs in turn: 42 us,
// 4.6 TB/s (a copy's rate 4.9); one row per wave, its RoPE key left to another, 80.  64K
// rows, 0.7 GB in turn: 18.0 us with 4 bits, 24.6 protected, 30.7 from the BF16 cache.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "kernel_common.h"
#include "prefill_internal.h"

namespace mla {
namespace {

constexpr int kThreads = 256;
constexpr int kRopeRows = 8;        // of a RoPE wave
constexpr int kManyRows = 16384;

// Sequences of the output rows first .. first + N - 1 (uniform in the wave): how
// many of cu_rows[1 .. B] are at or below each (B at the rows behind the last
// sequence).
template <int N>
__device__ __forceinline__ void sequences_of(const GatherArgs& a, int first, int lane, int (&b)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) b[k] = 0;
    for (int i = 0; i < a.B; i += 64) {
        const int c = i + lane < a.B ? a.cu_rows[1 + i + lane] : INT32_MAX;
#pragma unroll
        for (int k = 0; k < N; ++k) b[k] += __popcll(__ballot(c <= first + k));
    }
}

// Where a token is: a BF16 row, or offset `off` of a packed page.
struct Source {
    const uint8_t* row;     // null: packed
    const uint8_t* page;
    int off;
};
template <bool kBf16, bool kProt>
__device__ __forceinline__ Source source_of(const GatherArgs& a, int b, int r) {
    const int64_t pos = max(static_cast<int64_t>(a.first != nullptr ? a.first[b] : 0) + r - a.cu_rows[b], int64_t{0});
    if constexpr (kProt) {
        const int64_t L = a.seq_lens[b];
        if (pos < L && (pos < a.sink || pos >= L - a.recent)) {      // (the second implies recent >= 1)
            const int64_t ps = min(max(static_cast<int64_t>(a.prot_slot[b]), int64_t{0}), a.num_prot - 1);
            const int64_t row = pos < a.sink ? pos : a.sink + (pos - a.sink) % a.recent;
            return {a.prot + (ps * (a.sink + a.recent) + row) * 1152, nullptr, 0};
        }
    }
    const int32_t p = static_cast<int32_t>(min(pos, static_cast<int64_t>(INT32_MAX)));
    const int column = page_column(p, a.g.page_size, a.max_pages);
    const int64_t id = min(max(static_cast<int64_t>(a.block_table[static_cast<int64_t>(b) * a.max_pages + column]), int64_t{0}),
                           a.num_pages - 1);
    const uint8_t* page = a.cache + id * a.g.page_bytes;
    const int off = p % a.g.page_size;
    if constexpr (kBf16) return {page + static_cast<int64_t>(off) * 1152, nullptr, 0};
    return {nullptr, page, off};
}

// Eight channels of one group: codes of 4 bits (channel 2i of the word at bits
// 4i, channel 2i + 1 in the upper half), or of 2 bits at `shift`.
template <int BITS>
__device__ __forceinline__ uint4 values(uint32_t word, int shift, float scale, float zero) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = (word >> (shift + BITS * i)) & ((1u << BITS) - 1), hi = (word >> (16 + shift + BITS * i)) & ((1u << BITS) - 1);
        o[i] = kc::pack_bf16x2(scale * (static_cast<float>(lo) - zero), scale * (static_cast<float>(hi) - zero));
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

__device__ __forceinline__ void fp16_meta(uint32_t w, float& scale, float& zero) {
    scale = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(w & 0xFFFFu)));
    zero = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(w >> 16)));
}

// Channels 8 lane .. of the content, or with `rope` channels 8 lig .. of the key.
template <int CBITS, bool kPaper>
__device__ __forceinline__ uint4 read(const GatherArgs& a, const Source& s, bool rope, int lane) {
    const int column = rope ? 1024 + (lane & 7) * 16 : lane * 16;
    if (CBITS == 16 || s.row != nullptr) return *reinterpret_cast<const uint4*>(s.row + column);
    float scale, zero;
    const uint8_t* rec = s.page + a.g.off_mc + static_cast<int64_t>(s.off) * 32;
    if (rope) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(s.page + a.g.off_cr + s.off * 32 + (lane & 7) * 4);
        if constexpr (kPaper) {
            scale = *reinterpret_cast<const float*>(rec + 24);
            zero = static_cast<float>(rec[28]);
        } else {
            fp16_meta(*reinterpret_cast<const uint32_t*>(s.page + a.g.off_mr + s.off * 4), scale, zero);
        }
        return values<4>(w, 0, scale, zero);
    }
    const int g = lane >> 3;
    if constexpr (kPaper) {
        scale = __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(rec + 2 * g)) << 16);
        zero = static_cast<float>(rec[16 + g]);
    } else {
        fp16_meta(*reinterpret_cast<const uint32_t*>(rec + 4 * g), scale, zero);
    }
    if constexpr (CBITS == 4)
        return values<4>(*reinterpret_cast<const uint32_t*>(s.page + s.off * 256 + lane * 4), 0, scale, zero);
    else
        return values<2>(*reinterpret_cast<const uint32_t*>(s.page + s.off * 128 + (lane >> 1) * 4), 8 * (lane & 1), scale, zero);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// kStream: past the caches, as rows that a product reads later, many at a time.
template <bool kStream>
__device__ __forceinline__ void put(uint16_t* to, const uint4& x) {
    if constexpr (kStream) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), reinterpret_cast<u32x4*>(to));
    else *reinterpret_cast<uint4*>(to) = x;
}

// kRows consecutive rows of a wave; a single row's RoPE keys are left to waves of
// their own, behind the others.  CBITS 16: the BF16 cache.
template <int CBITS, bool kProt, bool kPaper, int kRows>
__global__ __launch_bounds__(kThreads) void gather_kernel(GatherArgs a) {
    static_assert(kRows == 1 || kRows == kRopeRows, "8 lanes per RoPE key");
    constexpr bool kStream = kRows > 1;
    const int lane = static_cast<int>(threadIdx.x & 63);
    const uint32_t wave = __builtin_amdgcn_readfirstlane((blockIdx.x * kThreads + threadIdx.x) >> 6);
    const uint32_t content_waves = (static_cast<uint32_t>(a.n) + kRows - 1) / kRows;
    const bool content = wave < content_waves;
    if (content) {
        const int first = static_cast<int>(wave) * kRows;
        int b[kRows];
        sequences_of(a, first, lane, b);
        // (rows behind the last sequence read as if they were the last one's, and are not
        // written)
        Source s[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) s[i] = source_of<CBITS == 16, kProt>(a, min(b[i], a.B - 1), first + i);
        uint4 x[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) x[i] = read<CBITS, kPaper>(a, s[i], false, lane);
        if constexpr (kRows > 1) {
            const int mine = lane >> 3;
            Source t = s[0];
            bool there = b[0] < a.B;
#pragma unroll
            for (int i = 1; i < kRows; ++i) {
                t.row = mine == i ? s[i].row : t.row;
                t.page = mine == i ? s[i].page : t.page;
                t.off = mine == i ? s[i].off : t.off;
                there = mine == i ? b[i] < a.B : there;
            }
            const uint4 k = read<CBITS, kPaper>(a, t, true, lane);
            if (first + mine < a.n && there) put<kStream>(a.k_out + static_cast<int64_t>(first + mine) * a.k_out_stride + (lane & 7) * 8, k);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (first + i < a.n && b[i] < a.B) put<kStream>(a.c_out + static_cast<int64_t>(first + i) * a.c_out_stride + lane * 8, x[i]);
    }
    if constexpr (kRows == 1) {
        if (content) return;
        const int first = static_cast<int>(wave - content_waves) * kRopeRows;
        const int r = first + (lane >> 3);
        int all[kRopeRows], b = a.B;
        sequences_of(a, first, lane, all);
#pragma unroll
        for (int i = 0; i < kRopeRows; ++i) b = (lane >> 3) == i ? all[i] : b;
        if (r >= a.n || b >= a.B) return;
        put<kStream>(a.k_out + static_cast<int64_t>(r) * a.k_out_stride + (lane & 7) * 8,
                     read<CBITS, kPaper>(a, source_of<CBITS == 16, kProt>(a, b, r), true, lane));
    }
}

template <int CBITS, bool kProt, bool kPaper, int kRows>
hipError_t launch_rows(const GatherArgs& a, hipStream_t stream) {
    const int64_t n = a.n;
    const int64_t waves = (n + kRows - 1) / kRows + (kRows == 1 ? (n + kRopeRows - 1) / kRopeRows : 0);
    static_assert((kMaxAppendTokens + kMaxAppendTokens / kRopeRows + 1) * 64 + kThreads <= kMaxDispatchItems, "launch size");
    const int64_t groups = (waves * 64 + kThreads - 1) / kThreads;
    hipLaunchKernelGGL((gather_kernel<CBITS, kProt, kPaper, kRows>), dim3(static_cast<unsigned>(groups)), dim3(kThreads), 0,
                       stream, a);
    return hipGetLastError();
}
template <int CBITS, bool kProt, bool kPaper>
hipError_t launch_as(const GatherArgs& a, hipStream_t stream) {
    // Eight rows per wave overlap their chains of loads (row -> page -> codes) and share
    // the search and the RoPE keys' wave, where there are waves enough for the card all
    // the same (32K rows, 4 bits, caches cold: 12.2 us against 16.6, protected 17.4 against
    // 18.2; 16K: 9.3 against 12.0, but protected 16.5 against 13.1).
    if (a.n >= kManyRows) return launch_rows<CBITS, kProt, kPaper, kRopeRows>(a, stream);
    return launch_rows<CBITS, kProt, kPaper, 1>(a, stream);
}

}  // namespace

hipError_t launch_gather(const GatherArgs& a, bool lowbit, hipStream_t stream) {
    if (!lowbit) return launch_as<16, false, false>(a, stream);
    const bool prot = a.prot != nullptr, paper = a.g.paper_meta != 0;
    if (a.g.c_bits == 4) {
        if (prot) return paper ? launch_as<4, true, true>(a, stream) : launch_as<4, true, false>(a, stream);
        return paper ? launch_as<4, false, true>(a, stream) : launch_as<4, false, false>(a, stream);
    }
    if (prot) return paper ? launch_as<2, true, true>(a, stream) : launch_as<2, true, false>(a, stream);
    return paper ? launch_as<2, false, true>(a, stream) : launch_as<2, false, false>(a, stream);
}

}  // namespace mla
