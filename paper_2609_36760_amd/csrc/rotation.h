// Device helper of the kernels that rotate RoPE channels (norm_rope_append.hip,
// rope_queries.hip).  Internal; not part of the public C ABI.
//
// A row of 64 bf16 channels is held by 8 consecutive lanes, 8 channels each.
// Products and sums run in fp64 (a bf16 channel times an fp32 table entry is
// exact there), rounded to fp32 and then to bf16: codes that are made of the
// result step at borders, so it must not depend on how a sum was fused.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "prefill_internal.h"
#include "writer_common.h"

namespace mla {
namespace rt {

// Two values rounded to fp32, then to bf16.  (Kept apart by the empty asm: as one
// conversion from fp64 to bf16 the compiler makes eight instructions of it.)
__device__ __forceinline__ uint32_t bf16x2_of(double lo, double hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    float a = static_cast<float>(lo), b = static_cast<float>(hi);
    asm("" : "+v"(a), "+v"(b));
    const bf16x2 v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, v);
}

// Row of `table` for a device-resident position, kept inside it.
__device__ __forceinline__ const float* table_row(const Rotation& r, int32_t position) {
    const int64_t p = min(max(static_cast<int64_t>(position), int64_t{0}), r.num_positions - 1);
    return r.table + p * 64;
}

// cos and sin of the lane's pairs: 4 pairs (lig 4 .. + 3), or with `halves` the
// 8 pairs of its 8 channels.
struct Angles {
    float c[8], s[8];
};
__device__ __forceinline__ Angles load_angles(const float* row, bool halves, int lig) {
    Angles a;
    const float* p = row + (halves ? (lig & 3) * 8 : lig * 4);
    const float4 c0 = *reinterpret_cast<const float4*>(p), s0 = *reinterpret_cast<const float4*>(p + 32);
    float4 c1 = c0, s1 = s0;
    if (halves) {
        c1 = *reinterpret_cast<const float4*>(p + 4);
        s1 = *reinterpret_cast<const float4*>(p + 36);
    }
    const float c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        a.c[i] = c[i];
        a.s[i] = s[i];
    }
    return a;
}

// The lane's 8 channels rotated (all 8 lanes of the row active).
__device__ __forceinline__ uint4 rotate(const uint4 raw, const Angles& a, bool halves, int lig) {
    float x[8];
    wc::widen_bf16x8(raw, x);
    uint32_t w[4];
    if (halves) {
        uint4 other;        // the same channels of the other half: 4 lanes on
        other.x = __shfl_xor(raw.x, 4);
        other.y = __shfl_xor(raw.y, 4);
        other.z = __shfl_xor(raw.z, 4);
        other.w = __shfl_xor(raw.w, 4);
        float y[8];
        wc::widen_bf16x8(other, y);
        const double sign = lig < 4 ? -1.0 : 1.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double lo = static_cast<double>(x[2 * i]) * a.c[2 * i] + sign * y[2 * i] * a.s[2 * i];
            const double hi = static_cast<double>(x[2 * i + 1]) * a.c[2 * i + 1] + sign * y[2 * i + 1] * a.s[2 * i + 1];
            w[i] = bf16x2_of(lo, hi);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double p = x[2 * i], q = x[2 * i + 1], c = a.c[i], s = a.s[i];
            w[i] = bf16x2_of(p * c - q * s, p * s + q * c);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace rt
}  // namespace mla
