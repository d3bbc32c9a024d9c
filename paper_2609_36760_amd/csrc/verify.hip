// Verification of drafted tokens against the target's logits and given random
// numbers (the rules stand in mla_speculate.h).
//
// Two launches.  The first (stats_kernel) takes every row of logits once, a wave
// per chunk of 2 048, and keeps of each chunk its maximum m and the sum of its
// weights w = e^((l - m) / T); at temperature 0 the first place of the maximum.
// The second (walk_kernel) walks the trees with what the chunks give: a node's
// chances need single logits only, and the token that is drawn at the end one
// chunk, found by the chunks' sums.
//
// Drawn drafts.  After k rejections at a node what is left of p is
//   r_k = max(p - c_k q, 0) / F(c_k),  F(c) = sum_x max(p(x) - c q(x), 0),
// with c_0 = 0 and c_{k+1} = c_k + F(c_k): (max(p - c q, 0) / F - q, 0) is, where
// it is above 0, (p - (c + F) q) / F.  So one rejection costs one pass over the
// row and its q, and no pass needs what the ones before left of single tokens.
// The walk works with weights instead of p: w - (c Z) q, Z the row's sum.  The
// first pass of a sequence is shared by several workgroups, each of which has
// walked so far by itself; the last one to be done goes on (further passes, at
// trees that try several drawn drafts at a node, are its own).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "speculate_internal.h"

namespace mla {
namespace {

constexpr int kSteps = kLogitChunk / 512;       // pieces of 8 consecutive logits per lane and chunk
constexpr int kWalk = 512;                      // threads of a walk
constexpr int kMaxChunks = logit_chunks(kMaxVocab);
constexpr double kLog2e = 1.4426950408889634074;

// 2^y for y in [-2000, 0]: y = k + f with f in [-1/2, 1/2], 2^f by a polynomial of
// degree 9 through the Chebyshev points of that interval (relative error below
// 2e-14; 1 at f = 0).
__device__ __forceinline__ double pow2(double y) {
    const double k = __builtin_rint(y);
    const double f = y - k;
    double p = 0x1.b6571de2f2351p-24;
    p = __builtin_fma(p, f, 0x1.63ef969a64d3cp-20);
    p = __builtin_fma(p, f, 0x1.ffcb76789860fp-17);
    p = __builtin_fma(p, f, 0x1.43088e257f341p-13);
    p = __builtin_fma(p, f, 0x1.5d87fe908f88ap-10);
    p = __builtin_fma(p, f, 0x1.3b2ab72b175eep-7);
    p = __builtin_fma(p, f, 0x1.c6b08d7044119p-5);
    p = __builtin_fma(p, f, 0x1.ebfbdff8149f2p-3);
    p = __builtin_fma(p, f, 0x1.62e42fefa39f7p-1);
    p = __builtin_fma(p, f, 1.0);
    return __builtin_ldexp(p, static_cast<int>(k));
}

// Weight of logit l <= m beside a finite maximum m; scale = log2(e) / T.  A logit
// of -inf, and anything below 2^-1074, weighs 0.
__device__ __forceinline__ double weight(float l, float m, double scale) {
    return pow2(fmax((static_cast<double>(l) - static_cast<double>(m)) * scale, -2000.0));
}

// Eight consecutive logits as they lie in memory (rows need no alignment beyond
// their type's).
template <bool kF32>
struct Piece {
    uint32_t w[kF32 ? 8 : 4];
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (kF32) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    }
};
template <bool kF32>
__device__ __forceinline__ Piece<kF32> load_piece(const VerifyArgs& a, int64_t row, int x) {
    using T = std::conditional_t<kF32, uint32_t, uint16_t>;
    Piece<kF32> p;
    __builtin_memcpy(p.w, static_cast<const T*>(a.logits) + row * a.logits_stride + x, sizeof(p.w));
    return p;
}
// The same where the row may end: -inf behind its end.
template <bool kF32>
__device__ __forceinline__ Piece<kF32> load_end(const VerifyArgs& a, int64_t row, int x) {
    using T = std::conditional_t<kF32, uint32_t, uint16_t>;
    if (x + 8 <= a.vocab) return load_piece<kF32>(a, row, x);
    const T* from = static_cast<const T*>(a.logits) + row * a.logits_stride + x;
    Piece<kF32> p;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t l = x + i < a.vocab ? from[i] : kF32 ? 0xFF800000u : 0xFF80u;
        if constexpr (kF32) p.w[i] = l;
        else p.w[i >> 1] = i & 1 ? p.w[i >> 1] | l << 16 : l;
    }
    return p;
}
// A lane's pieces of a chunk.  They go round in their registers, so that loops over
// them need not be unrolled: the code runs once or twice per wave, and fetching
// it counts.
template <class P>
struct Round {
    P at[kSteps];
    __device__ __forceinline__ void next() {
        const P p = at[0];
#pragma unroll
        for (int j = 0; j + 1 < kSteps; ++j) at[j] = at[j + 1];
        at[kSteps - 1] = p;
    }
};
template <bool kF32>
__device__ __forceinline__ Round<Piece<kF32>> load_chunk(const VerifyArgs& a, int64_t row, int chunk, int x0) {
    Round<Piece<kF32>> l;
    if ((chunk + 1) * kLogitChunk <= a.vocab) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) l.at[j] = load_piece<kF32>(a, row, x0 + 512 * j);
    } else {
#pragma unroll 1
        for (int j = 0; j < kSteps; ++j) {
            l.at[0] = load_end<kF32>(a, row, x0 + 512 * j);
            l.next();
        }
    }
    return l;
}
template <bool kF32>
__device__ __forceinline__ float load1(const VerifyArgs& a, int64_t row, int x) {
    const int64_t at = row * a.logits_stride + x;
    if constexpr (kF32) return static_cast<const float*>(a.logits)[at];
    else return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.logits)[at]) << 16);
}

// A value of each lane's partner at distance 1, 2, (mirrored) 4 and 8, 16 and 32: six
// exchanges without LDS that bring a symmetric operation to all lanes.
template <int kStep>
__device__ __forceinline__ uint32_t partner(uint32_t v) {
    if constexpr (kStep == 0) return __builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xB1, 0xF, 0xF, true);        // quad_perm 1, 0, 3, 2
    else if constexpr (kStep == 1) return __builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4E, 0xF, 0xF, true);   // quad_perm 2, 3, 0, 1
    else if constexpr (kStep == 2) return __builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x141, 0xF, 0xF, true);  // row_half_mirror
    else if constexpr (kStep == 3) return __builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x140, 0xF, 0xF, true);  // row_mirror
    else if constexpr (kStep == 4) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return (threadIdx.x & 16) != 0 ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return (threadIdx.x & 32) != 0 ? r[0] : r[1];
    }
}
template <int kStep>
__device__ __forceinline__ double partner(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = partner<kStep>(static_cast<uint32_t>(u)), hi = partner<kStep>(static_cast<uint32_t>(u >> 32));
    return __builtin_bit_cast(double, hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) {
    v += partner<0>(v);
    v += partner<1>(v);
    v += partner<2>(v);
    v += partner<3>(v);
    v += partner<4>(v);
    v += partner<5>(v);
    return v;
}
// The largest of a wave's values, NaN if one is.
template <int kStep>
__device__ __forceinline__ float larger(float v) {
    return __builtin_elementwise_maximum(v, __uint_as_float(partner<kStep>(__float_as_uint(v))));
}
__device__ __forceinline__ float wave_max(float v) {
    return larger<5>(larger<4>(larger<3>(larger<2>(larger<1>(larger<0>(v))))));
}
template <int kStep>
__device__ __forceinline__ int smaller(int v) { return min(v, static_cast<int>(partner<kStep>(static_cast<uint32_t>(v)))); }
__device__ __forceinline__ int wave_min(int v) {
    return smaller<5>(smaller<4>(smaller<3>(smaller<2>(smaller<1>(smaller<0>(v))))));
}
__device__ __forceinline__ double lane_value(double v, int lane) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(u), lane);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(u >> 32), lane);
    return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

__device__ __forceinline__ float temperature_of(const VerifyArgs& a, int b) {
    const float t = a.temperature == nullptr ? 1.0f : a.temperature[b];
    return t > 0.0f ? fminf(t, 1e30f) : 0.0f;
}
// log2(e) / t, within 2^-51: a division in fp64 would take as long as the weights
// of two logits per lane.
__device__ __forceinline__ double scale_of(float t) {
    const double d = t;
    double r = __builtin_amdgcn_rcp(d);
    r = __builtin_fma(r, __builtin_fma(-d, r, 1.0), r);
    r = __builtin_fma(r, __builtin_fma(-d, r, 1.0), r);
    return kLog2e * r;
}

// ---------------------------------------------------------------------------
// A wave holds its chunk's 2 048 logits in registers.  Bound by its instructions, 9 in
// fp64 and 5 others a logit and 150 a wave: 432 rows of 131 072 bf16 logits take 31 us
// in steady state (3.6 TB/s; 19 us without the weights).  A polynomial of degree 9
// without the table, 14 and 3 instructions: 39 us; weights by their definition, 18 and
// 3: a tenth more than that.  Tried: a wave that goes through many chunks with the next
// one's loads on their way (a fifth slower: fewer waves fit), exchanges through LDS and
// a division in fp64 (a third slower).
template <bool kF32>
__global__ __launch_bounds__(256, kF32 ? 5 : 8) void stats_kernel(VerifyArgs a) {
    const int lane = threadIdx.x & 63;
    const int chunk = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int node = blockIdx.y, b = blockIdx.z;
    if (blockIdx.x == 0 && node == 0 && threadIdx.x == 0) a.arrived[b] = 0;
    const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.max_nodes);
    const int chunks = logit_chunks(a.vocab);
    if (node >= nodes.count) return;
    const int64_t row = nodes.first + node;
    const float t = temperature_of(a, b);
    const int x0 = chunk * kLogitChunk + 8 * lane;
    Round<Piece<kF32>> l{};
    if (chunk < chunks) l = load_chunk<kF32>(a, row, chunk, x0);
    // 2^(j / 32), less j in the place where 32 k + j is added to its exponent (32 entries
    // of 8 bytes: as many banks, so lanes with different ones don't meet)
    __shared__ uint2 exponents[32];
    if (threadIdx.x < 32) {
        const uint64_t e = __builtin_bit_cast(uint64_t, pow2(lane * (1.0 / 32)));
        exponents[lane] = make_uint2(static_cast<uint32_t>(e), static_cast<uint32_t>(e >> 32) - (static_cast<uint32_t>(lane) << 15));
    }
    __syncthreads();
    if (chunk >= chunks) return;
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) m = __builtin_elementwise_maximum(m, l.at[j][i]);
    m = wave_max(m);
    double s = 0.0;
    if (!(m < INFINITY)) {
        m = NAN;            // a NaN or +inf: the row cannot be used
    } else if (t == 0.0f) {
        int first = a.vocab;
#pragma unroll 1
        for (int j = 0; j < kSteps; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) first = l.at[0][i] == m ? min(first, x0 + 512 * j + i) : first;
            l.next();
        }
        s = wave_min(first);
    } else if (m != -INFINITY) {
        const double scale = scale_of(t), top = m * scale;
        if (fabs(top) <= 0x1p20) {
            // beside 2^K, K the whole number next to the maximum's exponent, in 32nds:
            // l scale + (1.5 2^52 - 32 K) has a logit's number of 32nds in its low bits, 32 k
            // + j, and the rest f in [-1/2, 1/2] is one exact product and difference away.
            // 2^(f / 32) by a polynomial of degree 4 through the Chebyshev points (relative
            // error below 2e-13, 1 at f = 0), times 2^(j / 32 + k) in the step that adds it.
            // Logits below the maximum by 140 T or more weigh e^-140 (2^-190 of the sum for all).
            const double whole = __builtin_rint(top), magic = 0x1.8p52 - 32.0 * whole, scale32 = 32.0 * scale;
            const float lowest = static_cast<float>(static_cast<double>(m) - 140.0 * static_cast<double>(t));
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double x = __builtin_elementwise_maximum(l.at[j][i], lowest);
                    const double at = __builtin_fma(x, scale32, magic);
                    const double f = __builtin_fma(x, scale32, magic - at);
                    const uint32_t n = static_cast<uint32_t>(__builtin_bit_cast(uint64_t, at));
                    const uint2 e = exponents[n % 32];
                    double p = 0x1.3b2b07bdf358dp-27;
                    p = __builtin_fma(p, f, 0x1.c6b13c3465457p-20);
                    p = __builtin_fma(p, f, 0x1.ebfbdff82240ap-13);
                    p = __builtin_fma(p, f, 0x1.62e42fef8dc67p-6);
                    p = __builtin_fma(p, f, 1.0);
                    s = __builtin_fma(p, __builtin_bit_cast(double, static_cast<uint64_t>((n << 15) + e.y) << 32 | e.x), s);
                }
            s = wave_sum(s) * pow2(__builtin_fma(-static_cast<double>(m), scale, whole));
        } else {
#pragma unroll 1
            for (int j = 0; j < kSteps; ++j) {
#pragma unroll
                for (int i = 0; i < 8; ++i) s += weight(l.at[0][i], m, scale);
                l.next();
            }
            s = wave_sum(s);
        }
    }
    if (lane == 0) a.stats[row * chunks + chunk] = ChunkStat{s, m, 0.0f};
}

// ---------------------------------------------------------------------------
template <int kThreads>
struct WalkShared {
    double total[kMaxNodes];            // sum of a row's weights beside its maximum
    float row_max[kMaxNodes];           // NaN: a row that cannot be used
    int best[kMaxNodes];                // temperature 0: the largest logit's place
    double weight_of[kMaxNodes];        // of a node's token in its parent's row
    double sum[kMaxChunks];             // of the row's chunks, as they are left
    double wave[kThreads / 64];
    int first[kThreads / 64], final[kThreads / 64];
    double below;
    float logit;
    int last;
};

// The smallest `first` and the largest `final` of the workgroup's threads, each
// growing with the thread where it is set (kNone and -1 where not).
constexpr int kNone = 0x7FFFFFFF;
template <int kThreads>
__device__ __forceinline__ void block_ends(WalkShared<kThreads>& sh, int& first, int& final) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t some = __builtin_amdgcn_ballot_w64(first != kNone), any = __builtin_amdgcn_ballot_w64(final >= 0);
    // (read before the branch: the values of lanes outside it need not be there)
    const int lowest = __builtin_amdgcn_readlane(first, some != 0 ? __builtin_ctzll(some) : 0);
    const int highest = __builtin_amdgcn_readlane(final, any != 0 ? 63 - __builtin_clzll(any) : 0);
    if (lane == 0) {
        sh.first[wave] = lowest;
        sh.final[wave] = highest;
    }
    __syncthreads();
    first = wave_min(lane < kThreads / 64 ? sh.first[lane] : kNone);
    final = -wave_min(lane < kThreads / 64 ? -sh.final[lane] : 1);
    __syncthreads();
}

// Inclusive sum over the workgroup's threads, and the whole sum.
template <int kThreads>
__device__ __forceinline__ double block_scan(WalkShared<kThreads>& sh, double v, double& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    __syncthreads();        // (the last use of sh.wave is over)
    if (lane == 63) sh.wave[wave] = v;
    __syncthreads();
    double before = 0.0;
    all = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        const double x = sh.wave[w];
        before += w < wave ? x : 0.0;
        all += x;
    }
    return before + v;
}

// A workgroup a sequence; under drawn drafts gridDim.x of them, which share the
// first pass over a row.  Each lane of every wave holds one node, and every
// wave walks by itself.  Bound by one load after the other (nodes, tokens, their logits;
// chunks' statistics; the last chunk: 1.2, 1.0 and 3.9 us of 7.4 for 8 nodes of 131 072
// fixed), and under drawn drafts by the passes: 9 us the shared one for 48 x 9 nodes
// (4.5 TB/s), 10 each later one over 50 257 fp32 logits.  Tried for these: 1 024 threads
// (36 us for 31 of 16 ragged trees), weights as in stats_kernel (the same time).
template <bool kF32, bool kSampled>
__global__ __launch_bounds__(kWalk, 4) void walk_kernel(VerifyArgs a) {
    constexpr int kThreads = kWalk, kWaves = kThreads / 64;
    __shared__ WalkShared<kThreads> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.y;
    const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.max_nodes);
    const int n = nodes.count, V = a.vocab, chunks = logit_chunks(V);
    const float t = temperature_of(a, b);
    const bool greedy = t == 0.0f;
    const double scale = greedy ? 0.0 : scale_of(t);

    // this lane's node: its parent, its token and what decides about it
    int parent = -1, token = -1;
    float u = 1.0f, prob = 0.0f, logit = 0.0f;
    if (lane > 0 && lane < n) {
        const int64_t at = nodes.first + lane;
        const int p = a.parents[at], x = a.tokens[at];
        if (p >= 0 && p < lane) {
            parent = p;
            u = a.u_accept[at];
            if (x >= 0 && x < V) {
                token = x;
                if (wave == 0 && !greedy) logit = load1<kF32>(a, nodes.first + p, x);
                if constexpr (kSampled) prob = a.draft_probs[(nodes.first + p) * a.draft_stride + x];
            }
        }
    }
    // every row's maximum and sum of weights (the first wave last: it waits for the logits)
    for (int i = kWaves - 1 - wave; i < n; i += kWaves) {
        const ChunkStat* st = a.stats + static_cast<int64_t>(nodes.first + i) * chunks;
        float m = -INFINITY;
        for (int c = lane; c < chunks; c += 64) m = __builtin_elementwise_maximum(m, st[c].max);
        m = wave_max(m);
        const bool usable = m > -INFINITY;          // (a NaN is not)
        double s = 0.0;
        int first = V;
        for (int c = lane; c < chunks && usable; c += 64) {
            const ChunkStat x = st[c];
            if (greedy) first = x.max == m ? min(first, static_cast<int>(x.sum)) : first;
            else s += x.sum * weight(x.max, m, scale);
        }
        if (greedy) first = wave_min(first);
        else s = wave_sum(s);
        if (lane == 0) {
            sh.row_max[i] = usable ? m : NAN;
            sh.total[i] = s;
            sh.best[i] = first;
        }
    }
    __syncthreads();
    if (wave == 0) sh.weight_of[lane] = token >= 0 && !greedy ? weight(logit, sh.row_max[parent], scale) : 0.0;
    __syncthreads();
    const double my_weight = sh.weight_of[lane];
    const double my_total = sh.total[lane];         // (lanes from n on: nothing)
    const float my_max = sh.row_max[lane];
    const int my_best = sh.best[lane];

    // what lane k of the outputs gets: node k of the path, token k, p of the token as my_w / my_z
    int my_path = -1, my_out = -1;
    double my_w = 1.0, my_z = 1.0;

    int v = 0, keep = 0;                // node, nodes that stay
    bool usable = false;
    uint64_t rejected = 0;              // fixed drafts: nodes that were not taken
    double cut = 0.0, left = 0.0;       // drawn drafts: c Z, and the sum of max(w - cut q, 0)
    bool passed = false;                // this sequence's shared pass is over
    bool summed = false;                // sh.sum holds the row's chunks as they are left

    // weights of a chunk as they are left, summed by a wave
    auto chunk_sum = [&](int c, int64_t row, float m) {
        double s = 0.0;
        const int x0 = c * kLogitChunk + 8 * lane;
        Round<Piece<kF32>> l = load_chunk<kF32>(a, row, c, x0);
        Round<Piece<true>> q;               // the drafting model's probabilities (0 past the row's end)
        if constexpr (kSampled) {
            const float* from = a.draft_probs + row * a.draft_stride;
            if ((c + 1) * kLogitChunk <= V) {
#pragma unroll
                for (int j = 0; j < kSteps; ++j) __builtin_memcpy(q.at[j].w, from + x0 + 512 * j, sizeof(q.at[j].w));
            } else {
#pragma unroll 1
                for (int j = 0; j < kSteps; ++j) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        q.at[0].w[i] = x0 + 512 * j + i < V ? __float_as_uint(from[x0 + 512 * j + i]) : 0u;
                    q.next();
                }
            }
        }
#pragma unroll 1
        for (int j = 0; j < kSteps; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                double w = weight(l.at[0][i], m, scale);
                if constexpr (kSampled) {
                    w = fmax(__builtin_fma(-cut, static_cast<double>(q.at[0][i]), w), 0.0);
                } else {
                    for (uint64_t r = rejected; r != 0; r &= r - 1)
                        w = lane_value(token, __builtin_ctzll(r)) == x0 + 512 * j + i ? 0.0 : w;
                }
                s += w;
            }
            l.next();
            if constexpr (kSampled) q.next();
        }
        return wave_sum(s);
    };

    double* const shared_sums = a.sums + static_cast<int64_t>(b) * chunks;
    while (n > 0) {
        my_path = lane == keep ? v : my_path;
        ++keep;
        const float m = lane_value(my_max, v);
        const double total = lane_value(my_total, v);
        const int64_t row = nodes.first + v;
        usable = m == m;
        if (!usable) break;
        rejected = 0;
        cut = 0.0;
        left = total;
        summed = false;
        int taken = -1;
        for (uint64_t children = __builtin_amdgcn_ballot_w64(parent == v); children != 0; children &= children - 1) {
            const int i = __builtin_ctzll(children);
            const int x = lane_value(token, i);
            const double chance = lane_value(u, i);
            bool yes;
            if (greedy) {
                yes = x == lane_value(my_best, v);
            } else if constexpr (!kSampled) {
                // (a token that an earlier sibling had has no weight left)
                const bool again = (__builtin_amdgcn_ballot_w64(token == x) & rejected) != 0;
                const double w = x < 0 || again ? 0.0 : lane_value(my_weight, i);
                yes = chance * left < w;
                if (!yes && w > 0.0) {
                    left -= w;
                    rejected |= uint64_t{1} << i;
                }
            } else {
                const double q = lane_value(prob, i);
                const double w = fmax(__builtin_fma(-cut, q, lane_value(my_weight, i)), 0.0);
                yes = x >= 0 && chance * q * left < w;
                if (!yes) {
                    const double cut_before = cut, left_before = left;
                    cut += left;
                    const int shares = passed ? 1 : gridDim.x, share = passed ? 0 : blockIdx.x;
                    __syncthreads();
                    for (int c = share * kWaves + wave; c < chunks; c += shares * kWaves) {
                        const double s = chunk_sum(c, row, m);
                        if (lane == 0 && shares > 1) __hip_atomic_store(&shared_sums[c], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        if (lane == 0 && shares <= 1) sh.sum[c] = s;
                    }
                    if (shares > 1) {
                        // (stores and loads that pass the caches between the XCDs; a fence of
                        // the whole card by every wave costs 100 us here)
                        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                        __syncthreads();
                        if (tid == 0)
                            sh.last = __hip_atomic_fetch_add(&a.arrived[b], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == shares - 1;
                        __syncthreads();
                        if (sh.last == 0) return;
                        for (int c = tid; c < chunks; c += kThreads)
                            sh.sum[c] = __hip_atomic_load(&shared_sums[c], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
                    passed = true;
                    __syncthreads();
                    double s = 0.0, all;
                    for (int c = tid; c < chunks; c += kThreads) s += sh.sum[c];
                    block_scan(sh, s, all);
                    left = all;
                    summed = left > 0.0;
                    if (!summed) {
                        cut = cut_before;
                        left = left_before;
                    }
                }
            }
            if (yes) {
                taken = i;
                break;
            }
        }
        if (taken < 0) break;
        const int x = lane_value(token, taken);
        const double w = lane_value(my_weight, taken);
        if (lane == keep - 1) {
            my_out = x;
            my_w = greedy ? 1.0 : w;
            my_z = greedy ? 1.0 : total;
        }
        v = taken;
    }
    // the other workgroups of a sequence without a shared pass
    if (!passed && blockIdx.x > 0) return;

    // the next token
    if (n > 0 && usable) {
        const float m = lane_value(my_max, v);
        const double total = lane_value(my_total, v);
        const int64_t row = nodes.first + v;
        int x = lane_value(my_best, v);
        double w = 1.0;
        if (!greedy) {
            // what is left of every chunk (twice where rounding leaves nothing: then of p)
            constexpr int kEach = (kMaxChunks + kThreads - 1) / kThreads;       // chunks per thread
            double mine[kEach], sum, up, all;
            for (;;) {
                const ChunkStat* st = a.stats + row * chunks;
                __syncthreads();
                if (kSampled && cut > 0.0) {
                    for (int c = wave; c < chunks && !summed; c += kWaves) {
                        const double s = chunk_sum(c, row, m);
                        if (lane == 0) sh.sum[c] = s;
                    }
                } else {
                    for (int c = tid; c < chunks; c += kThreads) sh.sum[c] = st[c].sum * weight(st[c].max, m, scale);
                    __syncthreads();
                    // chunks with tokens that were not taken: less their weights, or, where
                    // that would leave too few digits, summed again without them
                    int j = 0;
                    for (uint64_t r = rejected; r != 0; r &= r - 1, ++j) {
                        if (j % kWaves != wave) continue;
                        const int c = lane_value(token, __builtin_ctzll(r)) / kLogitChunk;
                        const bool here = ((rejected >> lane) & 1) != 0 && token / kLogitChunk == c;
                        const double before = st[c].sum * weight(st[c].max, m, scale);
                        double s = before - wave_sum(here ? my_weight : 0.0);
                        if (!(s > 0x1p-14 * before)) s = chunk_sum(c, row, m);
                        if (lane == 0) sh.sum[c] = s;       // (several tokens of a chunk: the same)
                    }
                }
                __syncthreads();
                sum = 0.0;
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    mine[i] = tid * kEach + i < chunks ? sh.sum[tid * kEach + i] : 0.0;
                    sum += mine[i];
                }
                up = block_scan(sh, sum, all);
                if (all > 0.0 || (rejected == 0 && cut == 0.0)) break;
                rejected = 0;
                cut = 0.0;
            }
            const double target = fmax(static_cast<double>(a.u_draw[b]), 0.0) * all;
            // the first chunk that passes the target (for a number of 1 the last with weight, for NaN as for 0)
            double at = up - sum;
            int first = kNone, final = -1;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                at += mine[i];
                if (mine[i] > 0.0) final = tid * kEach + i;
                if (mine[i] > 0.0 && at > target && first == kNone) first = tid * kEach + i;
            }
            block_ends(sh, first, final);
            const int c = first != kNone ? first : max(final, 0);
            at = up - sum;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (tid * kEach + i == c) sh.below = at;
                at += mine[i];
            }
            // its tokens, consecutive ones per thread
            constexpr int kTokens = kLogitChunk / kThreads;
            double ws[kTokens];
            float ls[kTokens];
            const int y0 = c * kLogitChunk + tid * kTokens;
            sum = 0.0;
#pragma unroll
            for (int i = 0; i < kTokens; ++i) {
                const int y = y0 + i;
                ls[i] = y < V ? load1<kF32>(a, row, y) : -INFINITY;
                ws[i] = weight(ls[i], m, scale);
                if constexpr (kSampled) {
                    if (cut > 0.0 && y < V)
                        ws[i] = fmax(__builtin_fma(-cut, static_cast<double>(a.draft_probs[row * a.draft_stride + y]), ws[i]), 0.0);
                } else {
                    for (uint64_t r = rejected; r != 0; r &= r - 1)
                        ws[i] = lane_value(token, __builtin_ctzll(r)) == y ? 0.0 : ws[i];
                }
                sum += ws[i];
            }
            up = block_scan(sh, sum, all);
            at = sh.below + up - sum;
            first = kNone;
            final = -1;
#pragma unroll
            for (int i = 0; i < kTokens; ++i) {
                at += ws[i];
                if (ws[i] > 0.0) final = y0 + i;
                if (ws[i] > 0.0 && at > target && first == kNone) first = y0 + i;
            }
            block_ends(sh, first, final);
            // (the target may lie behind the tokens' own sum, by its rounding)
            x = first != kNone ? first : final;
#pragma unroll
            for (int i = 0; i < kTokens; ++i)
                if (y0 + i == x) sh.logit = ls[i];
            __syncthreads();
            w = x >= 0 ? weight(sh.logit, m, scale) : 1.0;
        }
        if (lane == keep - 1) {
            my_out = x;
            my_w = w;
            my_z = greedy || x < 0 ? 1.0 : total;
        }
    }
    if (tid < a.max_nodes) {
        const int64_t at = static_cast<int64_t>(b) * a.max_nodes + tid;
        a.path[at] = my_path;
        a.out_tokens[at] = my_out;
        if (a.logprobs != nullptr) a.logprobs[at] = my_out < 0 ? 0.0f : static_cast<float>(log(my_w / my_z));
    }
    if (tid == 0) a.keep[b] = keep;
}

template <bool kF32>
void launch(const VerifyArgs& a, hipStream_t stream) {
    const int chunks = logit_chunks(a.vocab);
    if (a.num_nodes > 0) {
        const dim3 grid(static_cast<unsigned>((chunks + 3) / 4), static_cast<unsigned>(a.max_nodes), static_cast<unsigned>(a.B));
        hipLaunchKernelGGL((stats_kernel<kF32>), grid, dim3(256), 0, stream, a);
    }
    if (a.draft_probs != nullptr) {
        // workgroups that share a pass: no more than fill the card once, nor than there are chunks for their waves
        const int most = (chunks + kWalk / 64 - 1) / (kWalk / 64), share = 2 * kCus / a.B;
        const int g = a.num_nodes == 0 ? 1 : share < 1 ? 1 : share < most ? share : most;
        hipLaunchKernelGGL((walk_kernel<kF32, true>), dim3(g, a.B), dim3(kWalk), 0, stream, a);
    } else {
        hipLaunchKernelGGL((walk_kernel<kF32, false>), dim3(1, a.B), dim3(kWalk), 0, stream, a);
    }
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
    if (a.B == 0) return hipSuccess;
    if (a.fp32) launch<true>(a, stream);
    else launch<false>(a, stream);
    return hipGetLastError();
}

}  // namespace mla
