// Commit of accepted drafted tokens: cached rows move up behind the context, in
// all layers' caches.
//
// A workgroup takes one sequence in some layers, whose places are the same: one
// thread per token finds them, then the layer's rows go through LDS in pieces of
// 16 bytes (4 of fp16 RoPE metadata).  Rows may move onto places that other rows
// of the sequence still have to leave, so a layer's pieces are all loaded before
// any is stored.  Bound by latency: lengths and path, page ids, rows, one after the
// other, for the 50 KB that a layer of 48 sequences moves.  The loops are short
// code on purpose: held in registers, a row's pieces took 8 KB of unrolled code,
// and 16-18 us in place of 5.4 at 48 sequences and 32 layers.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "speculate_internal.h"

namespace mla {
namespace {

constexpr int kThreads = 256;

// A cached row in pieces: kCodes of content codes (BF16: all 72 of the row), then
// 2 of RoPE codes, 2 of metadata and, with fp16 metadata, one of RoPE metadata.
template <bool kLowbit, int kCodes, bool kPaper>
__global__ __launch_bounds__(kThreads) void commit_kernel(CommitArgs a) {
    constexpr int kPieces = !kLowbit ? kCodes : kCodes + 4 + (kPaper ? 0 : 1);
    __shared__ uint4 piece[kMaxNodes * kPieces];
    __shared__ int64_t from_page[kMaxNodes], to_page[kMaxNodes];    // byte offsets
    __shared__ uint32_t from_off[kMaxNodes], to_off[kMaxNodes];     // tokens in the page
    __shared__ int moves;
    const int layer0 = blockIdx.x * a.layers_each, b = blockIdx.y, tid = threadIdx.x;
    const int ctx = max(a.ctx_lens[b], 0), keep = min(max(a.keep[b], 0), a.max_nodes);
    if (blockIdx.x == 0 && tid == 0 && a.new_lens != nullptr) a.new_lens[b] = ctx + keep;
    const int layers = min(a.layers_each, a.num_layers - layer0);
    if (layers <= 0) return;
    const uint32_t P = a.g.page_size, most = static_cast<uint32_t>(a.max_pages) * P;    // (fits: checked on the host)

    // the page id (-1: none) and the offset in the page of position t
    auto find = [&](uint32_t t, uint32_t& off) {
        if (t >= most) return -1;
        uint32_t page = __umulhi(t, a.g.page_magic);        // the quotient or one less, as in split_slot
        off = t - page * P;
        if (off >= P) {
            ++page;
            off -= P;
        }
        const int id = a.block_table[static_cast<int64_t>(b) * a.max_pages + page];
        return id < a.num_pages ? id : -1;
    };
    if (tid < 64) {
        // one wave: the tokens that move, side by side
        const int node = tid < a.max_nodes ? a.path[static_cast<int64_t>(b) * a.max_nodes + tid] : -1;
        bool move = tid < keep && node >= 0 && node < a.max_nodes && node != tid;
        uint32_t off = 0, dst_off = 0;
        int id = -1, dst = -1;
        if (move) {
            id = find(static_cast<uint32_t>(ctx) + node, off);
            dst = find(static_cast<uint32_t>(ctx) + tid, dst_off);
        }
        move = move && id >= 0 && dst >= 0;
        const uint64_t all = __builtin_amdgcn_ballot_w64(move);
        const int at = __builtin_popcountll(all & ((uint64_t{1} << tid) - 1));
        if (move) {
            from_page[at] = id * a.g.page_bytes;
            to_page[at] = dst * a.g.page_bytes;
            from_off[at] = off;
            to_off[at] = dst_off;
        }
        if (tid == 0) moves = __builtin_popcountll(all);
    }
    __syncthreads();
    const int n = moves * kPieces;
    // byte offset of piece r of the row at `off` in a page
    auto place = [&](uint32_t off, int r) -> uint32_t {
        if (!kLowbit || r < kCodes) return off * (16u * kCodes) + 16 * r;
        r -= kCodes;
        if (r < 2) return a.g.off_cr + off * 32u + 16 * r;
        if (r < 4) return a.g.off_mc + off * 32u + 16 * (r - 2);
        return a.g.off_mr + off * 4u;
    };
    for (int layer = 0; layer < layers; ++layer) {
        uint8_t* cache = a.caches[layer0 + layer];
        for (int i = tid; i < n; i += kThreads) {
            const int k = i / kPieces, r = i % kPieces;
            const uint8_t* src = cache + from_page[k] + place(from_off[k], r);
            if (kLowbit && r == kCodes + 4) piece[i].x = *reinterpret_cast<const uint32_t*>(src);
            else piece[i] = *reinterpret_cast<const uint4*>(src);
        }
        __syncthreads();
        // (a thread stores the pieces that it loaded: the next layer needs no barrier before it)
        for (int i = tid; i < n; i += kThreads) {
            const int k = i / kPieces, r = i % kPieces;
            uint8_t* dst = cache + to_page[k] + place(to_off[k], r);
            if (kLowbit && r == kCodes + 4) *reinterpret_cast<uint32_t*>(dst) = piece[i].x;
            else *reinterpret_cast<uint4*>(dst) = piece[i];
        }
    }
}

}  // namespace

hipError_t launch_commit(const CommitArgs& a, bool lowbit, hipStream_t stream) {
    if (a.B == 0 || (a.num_layers == 0 && a.new_lens == nullptr)) return hipSuccess;
    CommitArgs args = a;
    const int64_t all = static_cast<int64_t>(a.num_layers) * a.B;
    args.layers_each = static_cast<int32_t>((all + 2 * kCus - 1) / (2 * kCus));
    if (args.layers_each < 1) args.layers_each = 1;
    const dim3 grid(static_cast<unsigned>(a.num_layers > 0 ? (a.num_layers + args.layers_each - 1) / args.layers_each : 1),
                    static_cast<unsigned>(a.B)), block(kThreads);
    if (!lowbit) hipLaunchKernelGGL((commit_kernel<false, 72, true>), grid, block, 0, stream, args);
    else if (a.g.c_bits == 4 && a.g.paper_meta) hipLaunchKernelGGL((commit_kernel<true, 16, true>), grid, block, 0, stream, args);
    else if (a.g.c_bits == 4) hipLaunchKernelGGL((commit_kernel<true, 16, false>), grid, block, 0, stream, args);
    else if (a.g.paper_meta) hipLaunchKernelGGL((commit_kernel<true, 8, true>), grid, block, 0, stream, args);
    else hipLaunchKernelGGL((commit_kernel<true, 8, false>), grid, block, 0, stream, args);
    return hipGetLastError();
}

}  // namespace mla
