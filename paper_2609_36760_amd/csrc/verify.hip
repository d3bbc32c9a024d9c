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

#include "speculate_internal.h"

namespace mla {
namespace {

constexpr int kSteps = kLogitChunk / 512;       // pieces of 8 consecutive logits per lane and chunk
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

// Logits x .. x + 7 of a row, -inf past its end (rows need no alignment beyond
// their type's).
template <bool kF32>
__device__ __forceinline__ void load8(const VerifyArgs& a, int64_t row, int x, float l[8]) {
    if constexpr (kF32) {
        const float* p = static_cast<const float*>(a.logits) + row * a.logits_stride + x;
        if (x + 8 <= a.vocab) {
            __builtin_memcpy(l, p, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) l[i] = x + i < a.vocab ? p[i] : -INFINITY;
        }
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(a.logits) + row * a.logits_stride + x;
        if (x + 8 <= a.vocab) {
            uint32_t w[4];
            __builtin_memcpy(w, p, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                l[2 * i] = __uint_as_float(w[i] << 16);
                l[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) l[i] = x + i < a.vocab ? __uint_as_float(static_cast<uint32_t>(p[i]) << 16) : -INFINITY;
        }
    }
}
template <bool kF32>
__device__ __forceinline__ float load1(const VerifyArgs& a, int64_t row, int x) {
    const int64_t at = row * a.logits_stride + x;
    if constexpr (kF32) return static_cast<const float*>(a.logits)[at];
    else return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.logits)[at]) << 16);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// The largest of a wave's values, NaN if one is.
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = __builtin_elementwise_maximum(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = min(v, __shfl_xor(v, d));
    return v;
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
    return t > 0.0f ? t : 0.0f;
}

// ---------------------------------------------------------------------------
// A wave holds its chunk's 2 048 logits in registers.  Bound by the reads, with
// the weights close behind: about 20 fp64 instructions a logit.
template <bool kF32>
__global__ __launch_bounds__(256) void stats_kernel(VerifyArgs a) {
    const int lane = threadIdx.x & 63;
    const int chunk = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int node = blockIdx.y, b = blockIdx.z;
    if (blockIdx.x == 0 && node == 0 && threadIdx.x == 0) a.arrived[b] = 0;
    const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.max_nodes);
    const int chunks = logit_chunks(a.vocab);
    if (node >= nodes.count || chunk >= chunks) return;
    const int64_t row = nodes.first + node;
    const float t = temperature_of(a, b);
    float l[kSteps][8];
    const int x0 = chunk * kLogitChunk + 8 * lane;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) load8<kF32>(a, row, x0 + 512 * j, l[j]);
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) m = __builtin_elementwise_maximum(m, l[j][i]);
    m = wave_max(m);
    double s = 0.0;
    if (!(m < INFINITY)) {
        m = NAN;            // a NaN or +inf: the row cannot be used
    } else if (t == 0.0f) {
        int first = a.vocab;
#pragma unroll
        for (int j = kSteps - 1; j >= 0; --j)
#pragma unroll
            for (int i = 7; i >= 0; --i) first = l[j][i] == m ? x0 + 512 * j + i : first;
        s = wave_min(first);
    } else if (m != -INFINITY) {
        const double scale = kLog2e / static_cast<double>(t);
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += weight(l[j][i], m, scale);
        s = wave_sum(s);
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
    double below;
    int found, last;
};

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
// wave walks by itself.
template <bool kF32, bool kSampled>
__global__ __launch_bounds__(kSampled ? 1024 : 512) void walk_kernel(VerifyArgs a) {
    constexpr int kThreads = kSampled ? 1024 : 512, kWaves = kThreads / 64;
    __shared__ WalkShared<kThreads> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.y;
    const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.max_nodes);
    const int n = nodes.count, V = a.vocab, chunks = logit_chunks(V);
    const float t = temperature_of(a, b);
    const bool greedy = t == 0.0f;
    const double scale = greedy ? 0.0 : kLog2e / static_cast<double>(t);

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
        float l[kSteps][8];
        double s = 0.0;
        const int x0 = c * kLogitChunk + 8 * lane;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) load8<kF32>(a, row, x0 + 512 * j, l[j]);
        if constexpr (kSampled) {
            const float* q = a.draft_probs + row * a.draft_stride;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const int x = x0 + 512 * j;
                float d[8];
                if (x + 8 <= V) {
                    __builtin_memcpy(d, q + x, 32);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = x + i < V ? q[x + i] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    s += fmax(__builtin_fma(-cut, static_cast<double>(d[i]), weight(l[j][i], m, scale)), 0.0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int x = x0 + 512 * j + i;
                    bool out = false;
                    for (uint64_t r = rejected; r != 0; r &= r - 1) out |= lane_value(token, __builtin_ctzll(r)) == x;
                    s += out ? 0.0 : weight(l[j][i], m, scale);
                }
        }
        return wave_sum(s);
    };

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
                        if (lane == 0) (shares > 1 ? a.sums + static_cast<int64_t>(b) * chunks : sh.sum)[c] = s;
                    }
                    if (shares > 1) {
                        __threadfence();
                        __syncthreads();
                        if (tid == 0) sh.last = atomicAdd(&a.arrived[b], 1) == shares - 1;
                        __syncthreads();
                        if (sh.last == 0) return;
                        __threadfence();
                        for (int c = tid; c < chunks; c += kThreads) sh.sum[c] = a.sums[static_cast<int64_t>(b) * chunks + c];
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
                    int j = 0;
                    for (uint64_t r = rejected; r != 0; r &= r - 1, ++j) {
                        if (j % kWaves != wave) continue;
                        const int c = lane_value(token, __builtin_ctzll(r)) / kLogitChunk;
                        const double s = chunk_sum(c, row, m);
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
            if (tid == 0) {
                sh.found = kMaxChunks;
                sh.last = 0;
            }
            __syncthreads();
            // the first chunk that passes the target (for a number of 1, or NaN, the last with weight)
            double at = up - sum;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                at += mine[i];
                if (mine[i] > 0.0) atomicMax(&sh.last, tid * kEach + i);
                if (mine[i] > 0.0 && at > target) atomicMin(&sh.found, tid * kEach + i);
            }
            __syncthreads();
            const int c = sh.found < kMaxChunks ? sh.found : sh.last;
            at = up - sum;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (tid * kEach + i == c) sh.below = at;
                at += mine[i];
            }
            __syncthreads();
            // its tokens, consecutive ones per thread
            constexpr int kTokens = kLogitChunk / kThreads;
            double ws[kTokens];
            const int y0 = c * kLogitChunk + tid * kTokens;
            sum = 0.0;
#pragma unroll
            for (int i = 0; i < kTokens; ++i) {
                const int y = y0 + i;
                ws[i] = 0.0;
                if (y < V) {
                    ws[i] = weight(load1<kF32>(a, row, y), m, scale);
                    if constexpr (kSampled) {
                        if (cut > 0.0)
                            ws[i] = fmax(__builtin_fma(-cut, static_cast<double>(a.draft_probs[row * a.draft_stride + y]), ws[i]), 0.0);
                    } else {
                        for (uint64_t r = rejected; r != 0; r &= r - 1)
                            if (lane_value(token, __builtin_ctzll(r)) == y) ws[i] = 0.0;
                    }
                }
                sum += ws[i];
            }
            at = sh.below;
            up = block_scan(sh, sum, all);
            if (tid == 0) {
                sh.found = V;
                sh.last = -1;
            }
            __syncthreads();
            at += up - sum;
#pragma unroll
            for (int i = 0; i < kTokens; ++i) {
                at += ws[i];
                if (ws[i] > 0.0) atomicMax(&sh.last, y0 + i);
                if (ws[i] > 0.0 && at > target) atomicMin(&sh.found, y0 + i);
            }
            __syncthreads();
            // (the target may lie behind the tokens' own sum, by its rounding)
            x = sh.found < V ? sh.found : sh.last;
            w = x >= 0 ? weight(load1<kF32>(a, row, x), m, scale) : 1.0;
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
        const int most = (chunks + 15) / 16, share = kCus / a.B;
        const int g = a.num_nodes == 0 ? 1 : share < 1 ? 1 : share < most ? share : most;
        hipLaunchKernelGGL((walk_kernel<kF32, true>), dim3(g, a.B), dim3(1024), 0, stream, a);
    } else {
        hipLaunchKernelGGL((walk_kernel<kF32, false>), dim3(1, a.B), dim3(512), 0, stream, a);
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
