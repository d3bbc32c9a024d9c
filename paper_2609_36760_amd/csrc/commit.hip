// Commit of accepted drafted tokens: cached rows move up behind the context, in
// all layers' caches.
//
// A workgroup takes one sequence in one layer.  Rows may move onto places that
// other rows of the sequence still have to leave, so every piece (16 bytes, or
// the 4 bytes of fp16 RoPE metadata) is loaded into a register before any is
// stored.  Bound by its launch: a batch of 48 sequences moves 50 KB a layer.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "speculate_internal.h"

namespace mla {
namespace {

constexpr int kThreads = 256;

// Pieces of a cached row: 72 of a BF16 row; content codes, 2 of RoPE codes, 2 of
// metadata and (fp16 metadata) one of RoPE metadata.
template <bool kLowbit>
__global__ __launch_bounds__(kThreads) void commit_kernel(CommitArgs a) {
    const int layer = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int ctx = max(a.ctx_lens[b], 0), keep = min(max(a.keep[b], 0), a.max_nodes);
    if (layer == 0 && tid == 0 && a.new_lens != nullptr) a.new_lens[b] = ctx + keep;
    if (a.num_layers == 0) return;
    uint8_t* cache = a.caches[layer];
    const int P = a.g.page_size;
    const int code_pieces = a.g.cc_bytes / 16;
    const int pieces = !kLowbit ? 72 : code_pieces + 4 + (a.g.paper_meta ? 0 : 1);
    constexpr int kMost = kLowbit ? (kMaxNodes * 21 + kThreads - 1) / kThreads : kMaxNodes * 72 / kThreads;

    // byte offset of piece r of the row at position t, -1 outside the cache
    auto place = [&](int64_t t, int r) -> int64_t {
        const int64_t page = t / P;
        if (page >= a.max_pages) return -1;
        const int id = a.block_table[static_cast<int64_t>(b) * a.max_pages + page];
        if (id < 0 || id >= a.num_pages) return -1;
        const int64_t base = id * a.g.page_bytes, off = t % P;
        if (!kLowbit) return base + off * 1152 + 16 * r;
        if (r < code_pieces) return base + off * a.g.cc_bytes + 16 * r;
        r -= code_pieces;
        if (r < 2) return base + a.g.off_cr + off * 32 + 16 * r;
        if (r < 4) return base + a.g.off_mc + off * 32 + 16 * (r - 2);
        return base + a.g.off_mr + off * 4;
    };
    uint4 v[kMost];
    int64_t to[kMost];
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        const int i = j * kThreads + tid, k = i / pieces, r = i % pieces;
        to[j] = -1;
        if (k >= keep) continue;
        const int node = a.path[static_cast<int64_t>(b) * a.max_nodes + k];
        if (node < 0 || node >= a.max_nodes || node == k) continue;
        const int64_t from = place(static_cast<int64_t>(ctx) + node, r);
        to[j] = from < 0 ? -1 : place(static_cast<int64_t>(ctx) + k, r);
        if (to[j] < 0) continue;
        if (kLowbit && r == code_pieces + 4) v[j].x = *reinterpret_cast<const uint32_t*>(cache + from);
        else v[j] = *reinterpret_cast<const uint4*>(cache + from);
    }
    // every load has returned before the first store
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        if (to[j] < 0) continue;
        if (kLowbit && (j * kThreads + tid) % pieces == code_pieces + 4) *reinterpret_cast<uint32_t*>(cache + to[j]) = v[j].x;
        else *reinterpret_cast<uint4*>(cache + to[j]) = v[j];
    }
}

}  // namespace

hipError_t launch_commit(const CommitArgs& a, bool lowbit, hipStream_t stream) {
    if (a.B == 0 || (a.num_layers == 0 && a.new_lens == nullptr)) return hipSuccess;
    const dim3 grid(static_cast<unsigned>(a.num_layers > 0 ? a.num_layers : 1), static_cast<unsigned>(a.B));
    if (lowbit) hipLaunchKernelGGL(commit_kernel<true>, grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL(commit_kernel<false>, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace mla
