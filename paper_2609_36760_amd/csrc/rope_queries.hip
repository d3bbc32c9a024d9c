// Rotation of the queries' RoPE channels (mla_rope_queries): pair (a, b) at angle t
// becomes (a cos t - b sin t, a sin t + b cos t), in fp64 and rounded once to bf16.
//
// 8 lanes per (token, head) row, 16 bytes each: memory bounds it (a row's 128
// bytes read and written; the angles stay in the caches over a token's heads), and
// fp64, at half the rate of fp32, hides behind that.  8192 tokens, 128 heads: 56 us,
// 4.8 TB/s, a copy's rate; small calls take the launch.
#include <hip/hip_runtime.h>

#include "prefill_internal.h"
#include "rotation.h"

namespace mla {
namespace {

constexpr int kThreads = 256;

__global__ __launch_bounds__(kThreads) void rope_queries_kernel(RopeArgs a) {
    const uint32_t tid = blockIdx.x * kThreads + threadIdx.x;   // the launch fits 32 bits (the host refuses more)
    const int lig = static_cast<int>(threadIdx.x & 7);
    const uint32_t row = tid >> 3;
    if (row >= static_cast<uint32_t>(a.n) * static_cast<uint32_t>(a.H)) return;
    const uint32_t t = row / static_cast<uint32_t>(a.H), h = row - t * static_cast<uint32_t>(a.H);
    const uint4 raw = *reinterpret_cast<const uint4*>(a.q + t * a.q_stride_t + h * a.q_stride_h + lig * 8);
    const rt::Angles g = rt::load_angles(rt::table_row(a.rot, a.positions[t]), a.rot.halves != 0, lig);
    *reinterpret_cast<uint4*>(a.out + t * a.out_stride_t + h * a.out_stride_h + lig * 8) =
        rt::rotate(raw, g, a.rot.halves != 0, lig);
}

}  // namespace

hipError_t launch_rope_queries(const RopeArgs& a, hipStream_t stream) {
    const int64_t threads = static_cast<int64_t>(a.n) * a.H * 8;
    hipLaunchKernelGGL(rope_queries_kernel, dim3(static_cast<unsigned>((threads + kThreads - 1) / kThreads)),
                       dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace mla
