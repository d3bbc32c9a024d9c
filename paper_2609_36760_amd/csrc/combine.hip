// Split-KV combine: global softmax normalisation of per-split partials
// (Appendix C.5, "Global attention normalization"):
//   m = max_j m_j,  s = sum_j e^{m_j - m} s_j,  O = (sum_j e^{m_j - m} o_j) / s,
//   lse = m + ln s,
// skipping splits with m_j = -inf (no visible key).  A split's aggregation is
// stored normalized, u_j = o_j / s_j in fp16, so o_j = s_j u_j.
//
// Workgroups of four waves; each lane owns 8 of the 512 latent channels of an
// output row (sequence, query token, head), so a
// split's partial row is one coalesced 1 KiB read (16 bytes per lane).  The
// kernel is bound by the reads of the partials and their latency: a wave
// issues every load of a batch of splits (maximum, sum, latent row) before
// using any and keeps a running maximum across batches.  With few splits per
// sequence each wave combines one row alone; with many (kShare or more on
// average) a workgroup takes one row and its four waves share the row's splits
// (wave w takes j0 + w, j0 + w + 4, ..) and merge their (maximum, sum,
// weighted row) through LDS, so a row of S splits costs ceil(S / 32)
// dependent rounds of loads.  An empty split holds
// zeros and weighs e^{-inf} s = 0.
//
// Trees of drafted tokens (kTree): rows are (node, head) of a ragged batch, a
// split holds s_q * H of them, s_q the most nodes of a sequence; rows past a
// sequence's own are skipped, and no row before or behind them is written.  A
// row's sum that is NaN gives NaN, and a sum of nothing 0 and -inf.  Sequences of
// one split have none to merge.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "internal.h"
#include "speculate_internal.h"

namespace mla {
namespace {

constexpr int kDc = 512;
constexpr int kWaves = 4;         // waves (and rows) per workgroup
static_assert(64 * kWaves == kCombineThreads, "launch shape the host checks");
constexpr int kShare = 16;        // splits per sequence from which the waves share a row
// kBatch: splits whose loads are in flight together (4 when sequences have
// at most 4 splits on average, so that no load re-reads a split, else 8)
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
    return __builtin_bit_cast(uint32_t, v);
}

// One wave's combine state for one row over the splits j0 + first + step k.
struct RowState {
    float mx, s, o[8];
};

template <int kBatch>
__device__ __forceinline__ RowState combine_splits(const CombineArgs& a, int r, int rows_per_seq, int j0, int j1,
                                                   int first, int step, int lane) {
    RowState st{-INFINITY, 0.0f, {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
    for (int jb = j0 + first; jb < j1; jb += step * kBatch) {
        uint4 u[kBatch];
        float mk[kBatch], sk[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int jk = jb + step * k;
            const int j = min(jk, j1 - 1);
            const int64_t pr = static_cast<int64_t>(j) * rows_per_seq + r;
            u[k] = *reinterpret_cast<const uint4*>(a.part_o + pr * kDc + lane * 8);
            mk[k] = jk < j1 ? a.part_m[pr] : -INFINITY;
            sk[k] = a.part_s[pr];
        }
        float bm = mk[0];
#pragma unroll
        for (int k = 1; k < kBatch; ++k) bm = fmaxf(bm, mk[k]);
        const float nm = fmaxf(st.mx, bm);
        if (nm == -INFINITY) continue;          // no visible key so far
        const float c = expf(st.mx - nm);       // 0 while mx = -inf
        st.s *= c;
#pragma unroll
        for (int q = 0; q < 8; ++q) st.o[q] *= c;
        st.mx = nm;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const float ws = expf(mk[k] - st.mx) * sk[k];     // an empty split weighs 0
            st.s += ws;
            const uint32_t w4[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f16x2 h2 = __builtin_bit_cast(f16x2, w4[q]);
                st.o[2 * q] += ws * static_cast<float>(h2[0]);
                st.o[2 * q + 1] += ws * static_cast<float>(h2[1]);
            }
        }
    }
    return st;
}

template <bool kTree>
__device__ __forceinline__ void store_row(const CombineArgs& a, int64_t row, const float O[8], float M, float S,
                                          int lane) {
    const float inv = S > 0.0f ? 1.0f / S : 0.0f;
    *reinterpret_cast<uint4*>(a.out + row * kDc + lane * 8) =
        make_uint4(pack_bf16x2(O[0] * inv, O[1] * inv), pack_bf16x2(O[2] * inv, O[3] * inv),
                   pack_bf16x2(O[4] * inv, O[5] * inv), pack_bf16x2(O[6] * inv, O[7] * inv));
    if (a.lse != nullptr && lane == 0) a.lse[row] = (kTree ? S != 0.0f : S > 0.0f) ? M + logf(S) : -INFINITY;
}

// kShared: one row per workgroup, its splits shared by the four waves (many
// splits per sequence); else four rows per workgroup, one per wave.
template <bool kShared, int kBatch, bool kTree = false>
__global__ __launch_bounds__(64 * kWaves) void combine_kernel(std::conditional_t<kTree, TreeCombineArgs, CombineArgs> a) {
    // rows (b * s_q + i) * H + h in 8 contiguous ranges of blocks, range x on
    // XCD x (block id mod 8), the XCD whose decode workgroups wrote most of them
    constexpr int kRows = kShared ? 1 : kWaves;
    const int64_t rows_all = static_cast<int64_t>(a.B) * a.s_q * a.H;
    const int64_t blocks_all = (rows_all + kRows - 1) / kRows;
    const int64_t per_xcd = (blocks_all + 7) / 8;
    const int64_t blk = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (blk >= blocks_all) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rows_per_seq = a.s_q * a.H;
    int64_t row = blk * kRows + (kShared ? 0 : wave);
    if (!kShared && row >= rows_all) return;
    const int b = static_cast<int>(row / rows_per_seq);
    const int r = static_cast<int>(row % rows_per_seq);
    if constexpr (kTree) {
        const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.s_q);
        if (r >= nodes.count * a.H) return;
        row = static_cast<int64_t>(nodes.first) * a.H + r;
    }
    int j0 = a.split_indptr[b];
    int j1 = a.split_indptr[b + 1];
    if constexpr (kTree) {
        if (j1 - j0 == 1) return;       // the attention wrote the rows itself
        j0 = max(j0, 0);
        j1 = min(j1, a.num_splits);
    }

    if constexpr (!kShared) {
        const RowState st = combine_splits<kBatch>(a, r, rows_per_seq, j0, j1, 0, 1, lane);
        store_row<kTree>(a, row, st.o, st.mx, st.s, lane);
    } else {
        __shared__ float sh_o[kWaves][8][64];
        __shared__ float sh_ms[kWaves][2];
        const RowState st = combine_splits<kBatch>(a, r, rows_per_seq, j0, j1, wave, kWaves, lane);
#pragma unroll
        for (int q = 0; q < 8; ++q) sh_o[wave][q][lane] = st.o[q];
        if (lane == 0) {
            sh_ms[wave][0] = st.mx;
            sh_ms[wave][1] = st.s;
        }
        __syncthreads();
        if (wave != 0) return;
        float M = sh_ms[0][0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sh_ms[w][0]);
        float S = 0.0f;
        float O[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (M != -INFINITY) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float c = expf(sh_ms[w][0] - M);      // 0 for a wave with no visible key
                S += c * sh_ms[w][1];
#pragma unroll
                for (int q = 0; q < 8; ++q) O[q] += c * sh_o[w][q][lane];
            }
        }
        store_row<kTree>(a, row, O, M, S, lane);
    }
}

// Rows of a tree launch.  Where a batch is ragged most rows that the sizes allow do
// not exist, or need no merge; as many waves as the card holds go through those that
// do, found by the lanes' sequences (up to 64 of them; larger batches go through
// all rows).  24 sequences of up to 32 nodes at 128 heads, all of them merged: 19 us, 35
// with a wave for every row that may exist (bound by being started), 35 with one for
// every eight; 11.6 where those of one split write their rows themselves, as now.
template <int kBatch>
__global__ __launch_bounds__(64 * kWaves) void tree_rows_kernel(TreeCombineArgs a) {
    const int rows_per_seq = a.s_q * a.H;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t from = static_cast<int64_t>(blockIdx.x) * kWaves + wave, step = static_cast<int64_t>(gridDim.x) * kWaves;
    auto merge = [&](int first, int r, int j0, int j1) {
        const RowState st = combine_splits<kBatch>(a, r, rows_per_seq, max(j0, 0), min(j1, a.num_splits), 0, 1, lane);
        store_row<true>(a, static_cast<int64_t>(first) * a.H + r, st.o, st.mx, st.s, lane);
    };
    if (a.B > 64) {
        for (int64_t row = from; row < static_cast<int64_t>(a.B) * rows_per_seq; row += step) {
            const int b = static_cast<int>(row / rows_per_seq), r = static_cast<int>(row % rows_per_seq);
            const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.s_q);
            const int j0 = a.split_indptr[b], j1 = a.split_indptr[b + 1];
            // (of one split, the attention wrote the rows itself)
            if (r < nodes.count * a.H && j1 - j0 != 1) merge(nodes.first, r, j0, j1);
        }
        return;
    }
    const int b = min(lane, a.B - 1);
    const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.s_q);
    const int j0 = a.split_indptr[b], j1 = a.split_indptr[b + 1];
    const int rows = lane < a.B && j1 - j0 != 1 ? nodes.count * a.H : 0;
    int to = rows;                      // rows up to this lane's last
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(to, d);
        to += lane >= d ? o : 0;
    }
    const int all = __builtin_amdgcn_readlane(to, 63);
    for (int64_t i = from; i < all; i += step) {
        const int at = static_cast<int>(i);
        const int pick = __builtin_popcountll(__builtin_amdgcn_ballot_w64(to <= at));
        merge(__builtin_amdgcn_readlane(nodes.first, pick), at - __builtin_amdgcn_readlane(to - rows, pick),
              __builtin_amdgcn_readlane(j0, pick), __builtin_amdgcn_readlane(j1, pick));
    }
}

}  // namespace

hipError_t launch_combine(const CombineArgs& a, int32_t num_splits, hipStream_t stream) {
    const int64_t rows = static_cast<int64_t>(a.B) * a.s_q * a.H;
    if (rows == 0) return hipSuccess;
    if (num_splits >= static_cast<int64_t>(kShare) * a.B) {
        hipLaunchKernelGGL((combine_kernel<true, 8>), dim3(static_cast<unsigned>((rows + 7) / 8 * 8)),
                           dim3(64 * kWaves), 0, stream, a);
    } else {
        const int64_t blocks = (rows + kWaves - 1) / kWaves;
        const dim3 grid(static_cast<unsigned>((blocks + 7) / 8 * 8)), block(64 * kWaves);
        if (num_splits <= 4 * static_cast<int64_t>(a.B))
            hipLaunchKernelGGL((combine_kernel<false, 4>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((combine_kernel<false, 8>), grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

hipError_t launch_tree_combine(const TreeCombineArgs& a, hipStream_t stream) {
    const int32_t num_splits = a.num_splits;
    const int64_t rows = static_cast<int64_t>(a.B) * a.s_q * a.H;
    if (rows == 0) return hipSuccess;
    if (num_splits >= static_cast<int64_t>(kShare) * a.B) {
        hipLaunchKernelGGL((combine_kernel<true, 8, true>), dim3(static_cast<unsigned>((rows + 7) / 8 * 8)),
                           dim3(64 * kWaves), 0, stream, a);
    } else {
        const int64_t blocks = (rows + kWaves - 1) / kWaves;
        const dim3 grid(static_cast<unsigned>(blocks < 8 * kCus ? blocks : 8 * kCus)), block(64 * kWaves);
        if (num_splits <= 4 * static_cast<int64_t>(a.B))
            hipLaunchKernelGGL((tree_rows_kernel<4>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((tree_rows_kernel<8>), grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace mla
