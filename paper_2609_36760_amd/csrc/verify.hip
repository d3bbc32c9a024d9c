// Verification of drafted tokens against the target's logits and given random
// numbers (the rules stand in mla_speculate.h).
//
// Two launches.  The first takes every row of logits once, a wave per chunk of
// 2 048, and keeps of each chunk its maximum and the sum of its weights
// w = e^((l - max) / T); at temperature 0 the first place of the maximum.  The
// second walks the trees, a workgroup a sequence.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "speculate_internal.h"

namespace mla {
namespace {

constexpr int kPer = kLogitChunk / 64;          // logits per lane and chunk
constexpr int kWalk = 512;                      // threads of a walk
constexpr int kMaxChunks = logit_chunks(kMaxVocab);

// 2^y for y <= 0 (anything below -1100 gives 0): y = k + f with f in [-1/2, 1/2],
// 2^f by a polynomial of degree 9 through the Chebyshev points of that interval
// (relative error below 2e-14; 1 at f = 0).
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

// Weight of logit l beside a maximum of m; scale = log2(e) / T.  -inf has no
// weight (its difference would be NaN), a NaN gives NaN.
__device__ __forceinline__ double weight(float l, float m, double scale) {
    const double d = static_cast<double>(l) - static_cast<double>(m);
    return l == -INFINITY ? 0.0 : pow2(fmax(d * scale, -2000.0));
}

__device__ __forceinline__ float load_logit(const VerifyArgs& a, int64_t row, int x) {
    const int64_t at = row * a.logits_stride + x;
    if (a.fp32) return static_cast<const float*>(a.logits)[at];
    return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.logits)[at]) << 16);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

__device__ __forceinline__ float temperature_of(const VerifyArgs& a, int b) {
    const float t = a.temperature == nullptr ? 1.0f : a.temperature[b];
    return t > 0.0f ? t : 0.0f;
}
constexpr double kLog2e = 1.4426950408889634074;

// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void stats_kernel(VerifyArgs a) {
    const int lane = threadIdx.x & 63;
    const int chunk = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int node = blockIdx.y, b = blockIdx.z;
    const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.max_nodes);
    const int chunks = logit_chunks(a.vocab);
    if (node >= nodes.count || chunk >= chunks) return;
    const int64_t row = nodes.first + node;
    const float t = temperature_of(a, b);
    float l[kPer];
    float m = -INFINITY;
    bool bad = false;
    const int x0 = chunk * kLogitChunk + lane;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        l[i] = x0 + 64 * i < a.vocab ? load_logit(a, row, x0 + 64 * i) : -INFINITY;
        bad |= l[i] != l[i] || l[i] == INFINITY;
        m = fmaxf(m, l[i]);
    }
    m = wave_max(m);
    double s = 0.0;
    if (t == 0.0f) {
        int first = a.vocab;
#pragma unroll
        for (int i = kPer - 1; i >= 0; --i) first = l[i] == m ? x0 + 64 * i : first;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) first = min(first, __shfl_xor(first, d));
        s = first;
    } else if (m != -INFINITY) {
        const double scale = kLog2e / static_cast<double>(t);
#pragma unroll
        for (int i = 0; i < kPer; ++i) s += weight(l[i], m, scale);
        s = wave_sum(s);
    }
    if (__any(bad)) m = NAN;
    if (lane == 0) a.stats[row * chunks + chunk] = ChunkStat{s, m, 0.0f};
}

// ---------------------------------------------------------------------------
struct WalkShared {
    double total[kMaxNodes];            // sum of a row's weights beside its maximum
    double weight_of[kMaxNodes];        // of a node's token in its parent's row
    double prefix[kMaxChunks];
    double scan[kWalk];
    float row_max[kMaxNodes];           // NaN: a row that cannot be used
    float prob_of[kMaxNodes];           // of a node's token in the drafting model
    int best[kMaxNodes];                // temperature 0: the largest logit's place
    int parent[kMaxNodes], token[kMaxNodes];
    float u[kMaxNodes];
    double inverse[kMaxNodes];          // of the sums that the residuals were divided by
    int rejected[kMaxNodes];            // fixed drafts: the tokens that were not taken
    int path[kMaxNodes], emitted[kMaxNodes];
    float logprob[kMaxNodes];
    double wave[kWalk / 64];
    int found;
};

// What is left of the row's probability p at x after `k` rejections.
struct Residual {
    const float* probs;                 // the drafting model's row
    const double* inverse;
    int k;
    __device__ __forceinline__ double operator()(double p, int x) const {
        if (k == 0) return p;
        const double q = probs[x];
        for (int i = 0; i < k; ++i) {
            const double d = p - q;
            p = d > 0.0 ? d : 0.0;
            if (i + 1 < k) p *= inverse[i];
        }
        return p;
    }
};

template <bool kSampled>
__global__ __launch_bounds__(kWalk) void walk_kernel(VerifyArgs a) {
    __shared__ WalkShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kWaves = kWalk / 64;
    const int b = blockIdx.x;
    const NodeRange nodes = node_range(a.cu_nodes, b, a.num_nodes, a.max_nodes);
    const int n = nodes.count, V = a.vocab, chunks = logit_chunks(V);
    const float t = temperature_of(a, b);
    const bool greedy = t == 0.0f;
    const double scale = greedy ? 0.0 : kLog2e / static_cast<double>(t);

    // every row's maximum and sum of weights
    for (int i = wave; i < n; i += kWaves) {
        const ChunkStat* st = a.stats + static_cast<int64_t>(nodes.first + i) * chunks;
        float m = -INFINITY;
        bool bad = false;
        for (int c = lane; c < chunks; c += 64) {
            const float x = st[c].max;
            bad |= x != x;
            m = fmaxf(m, x);
        }
        m = wave_max(m);
        bad = __any(bad) || m == -INFINITY;
        double s = 0.0;
        int first = V;
        for (int c = lane; c < chunks && !bad; c += 64) {
            const ChunkStat x = st[c];
            if (greedy) first = x.max == m ? min(first, static_cast<int>(x.sum)) : first;
            else s += x.sum * weight(x.max, m, scale);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) first = min(first, __shfl_xor(first, d));
        s = wave_sum(s);
        if (lane == 0) {
            sh.row_max[i] = bad ? NAN : m;
            sh.total[i] = s;
            sh.best[i] = first;
        }
    }
    __syncthreads();
    // every node's token in its parent's row
    if (tid < n) {
        const int64_t at = nodes.first + tid;
        const int p = a.parents[at], x = a.tokens[at];
        const bool ok = tid > 0 && p >= 0 && p < tid;
        const bool real = ok && x >= 0 && x < V;
        sh.parent[tid] = ok ? p : -1;
        sh.token[tid] = real ? x : -1;
        sh.u[tid] = ok ? a.u_accept[at] : 1.0f;
        sh.weight_of[tid] = real && !greedy ? weight(load_logit(a, nodes.first + p, x), sh.row_max[p], scale) : 0.0;
        sh.prob_of[tid] = kSampled && real ? a.draft_probs[(nodes.first + p) * a.draft_stride + x] : 0.0f;
    }
    if (tid < a.max_nodes) {
        sh.path[tid] = -1;
        sh.emitted[tid] = -1;
        sh.logprob[tid] = 0.0f;
    }
    __syncthreads();

    // The walk: every thread the same, from what stands in LDS.  Wave-wide votes
    // give a node's children.
    const int my_parent = lane < n ? sh.parent[lane] : -1;
    int v = 0, keep = 0, k = 0;         // node, nodes that stay, rejections at it
    bool usable = false;
    const float* probs = nullptr;
    // the row's weights of one chunk as they are left, summed (a wave)
    auto chunk_sum = [&](int c, auto left) {
        double s = 0.0;
        for (int i = 0; i < kPer; ++i) {
            const int x = c * kLogitChunk + 64 * i + lane;
            if (x < V) s += left(x);
        }
        return wave_sum(s);
    };
    while (n > 0) {
        if (tid == 0) sh.path[keep] = v;
        ++keep;
        k = 0;
        usable = sh.row_max[v] == sh.row_max[v];
        if (!usable) break;
        const float m = sh.row_max[v];
        const double total = sh.total[v];
        const int64_t row = nodes.first + v;
        if constexpr (kSampled) probs = a.draft_probs + row * a.draft_stride;
        double mass = total;            // fixed drafts: what is left of the row
        int taken = -1;
        for (uint64_t children = __ballot(my_parent == v); children != 0 && taken < 0; children &= children - 1) {
            const int i = __builtin_ctzll(children);
            const int x = sh.token[i];
            bool yes;
            if (greedy) {
                yes = x == sh.best[v];
            } else if constexpr (!kSampled) {
                double w = x >= 0 ? sh.weight_of[i] : 0.0;
                for (int j = 0; j < k; ++j) w = sh.rejected[j] == x ? 0.0 : w;
                yes = static_cast<double>(sh.u[i]) * mass < w;
                if (!yes && w > 0.0) {
                    mass -= w;
                    __syncthreads();
                    if (tid == 0) sh.rejected[k] = x;
                    ++k;
                    __syncthreads();
                }
            } else {
                const Residual left{probs, sh.inverse, k};
                // (the last division is left to the reader)
                const double r = x >= 0 ? left(sh.weight_of[i] / total, x) * (k > 0 ? sh.inverse[k - 1] : 1.0) : 0.0;
                yes = x >= 0 && static_cast<double>(sh.u[i]) * static_cast<double>(sh.prob_of[i]) < r;
                if (!yes) {
                    const Residual next{probs, sh.inverse, k + 1};
                    __syncthreads();
                    double mine = 0.0;
                    for (int c = wave; c < chunks; c += kWaves) {
                        const double s = chunk_sum(c, [&](int y) {
                            return next(weight(load_logit(a, row, y), m, scale) / total, y);
                        });
                        mine += s;
                    }
                    if (lane == 0) sh.wave[wave] = mine;
                    __syncthreads();
                    double s = 0.0;
                    for (int w = 0; w < kWaves; ++w) s += sh.wave[w];
                    if (s > 0.0) {
                        if (tid == 0) sh.inverse[k] = 1.0 / s;
                        ++k;
                    }
                    __syncthreads();
                }
            }
            if (yes) taken = i;
        }
        if (taken < 0) break;
        if (tid == 0) {
            sh.emitted[keep - 1] = sh.token[taken];
            sh.logprob[keep - 1] = greedy ? 0.0f : static_cast<float>(log(sh.weight_of[taken] / total));
        }
        v = taken;
    }

    // the next token
    if (n > 0 && usable) {
        const int64_t row = nodes.first + v;
        const float m = sh.row_max[v];
        const double total = sh.total[v];
        auto left = [&](int x) {
            double w = weight(load_logit(a, row, x), m, scale);
            if constexpr (kSampled) {
                if (k > 0) w = Residual{probs, sh.inverse, k}(w / total, x);
            } else {
                for (int j = 0; j < k; ++j) w = sh.rejected[j] == x ? 0.0 : w;
            }
            return w;
        };
        int x = sh.best[v];
        if (!greedy) {
            const ChunkStat* st = a.stats + row * chunks;
            // (twice where rounding leaves nothing of r: then from p)
            for (;;) {
                for (int c = wave; c < chunks; c += kWaves) {
                    bool touched = kSampled && k > 0;
                    if constexpr (!kSampled)
                        for (int j = 0; j < k; ++j) touched |= sh.rejected[j] / kLogitChunk == c;
                    double s;
                    if (touched) s = chunk_sum(c, left);
                    else s = st[c].sum * weight(st[c].max, m, scale);
                    if (lane == 0) sh.prefix[c] = s;
                }
                __syncthreads();
                bool some = false;
                for (int c = lane; c < chunks; c += 64) some |= sh.prefix[c] > 0.0;
                if (__any(some) || k == 0) break;
                k = 0;
                __syncthreads();
            }
            if (tid == 0) {
                double up = 0.0;
                for (int c = 0; c < chunks; ++c) up = sh.prefix[c] += up;
                const double target = fmax(static_cast<double>(a.u_draw[b]), 0.0) * up;
                int c = 0;
                while (c < chunks && !(sh.prefix[c] > target)) ++c;
                // (a random number of 1 or NaN: the last chunk with weight)
                if (c == chunks)
                    for (--c; c > 0 && !(sh.prefix[c] > sh.prefix[c - 1]); --c) {}
                sh.found = c;
                sh.scan[0] = target;
            }
            __syncthreads();
            const int c = sh.found;
            const double target = sh.scan[0], below = c > 0 ? sh.prefix[c - 1] : 0.0;
            __syncthreads();
            // consecutive tokens of the chunk per thread
            constexpr int kEach = kLogitChunk / kWalk;
            double w[kEach], mine = 0.0;
            for (int i = 0; i < kEach; ++i) {
                const int y = c * kLogitChunk + tid * kEach + i;
                w[i] = y < V ? left(y) : 0.0;
                mine += w[i];
            }
            double up = mine;
            for (int d = 1; d < 64; d <<= 1) {
                const double o = __shfl_up(up, d);
                if (lane >= d) up += o;
            }
            if (lane == 63) sh.wave[wave] = up;
            if (tid == 0) sh.found = V;
            __syncthreads();
            double at = below;
            for (int q = 0; q < wave; ++q) at += sh.wave[q];
            at += up - mine;
            int hit = V, last = -1;
            for (int i = 0; i < kEach; ++i) {
                at += w[i];
                const int y = c * kLogitChunk + tid * kEach + i;
                if (hit == V && w[i] > 0.0 && at > target) hit = y;
                if (w[i] > 0.0) last = y;
            }
            if (hit < V) atomicMin(&sh.found, hit);
            __syncthreads();
            if (sh.found == V) {        // the border lies behind the chunk's own sum, by its rounding
                __syncthreads();
                if (tid == 0) sh.found = -1;
                __syncthreads();
                if (last >= 0) atomicMax(&sh.found, last);
                __syncthreads();
            }
            x = sh.found;
        }
        if (tid == 0) {
            sh.emitted[keep - 1] = x;
            sh.logprob[keep - 1] = greedy || x < 0 ? 0.0f : static_cast<float>(log(weight(load_logit(a, row, x), m, scale) / total));
        }
    }
    __syncthreads();
    if (tid < a.max_nodes) {
        const int64_t at = static_cast<int64_t>(b) * a.max_nodes + tid;
        a.path[at] = sh.path[tid];
        a.out_tokens[at] = sh.emitted[tid];
        if (a.logprobs != nullptr) a.logprobs[at] = sh.logprob[tid];
    }
    if (tid == 0) a.keep[b] = keep;
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
    if (a.B == 0) return hipSuccess;
    if (a.num_nodes > 0) {
        const dim3 grid(static_cast<unsigned>((logit_chunks(a.vocab) + 3) / 4), static_cast<unsigned>(a.max_nodes),
                        static_cast<unsigned>(a.B));
        hipLaunchKernelGGL(stats_kernel, grid, dim3(256), 0, stream, a);
    }
    if (a.draft_probs != nullptr) hipLaunchKernelGGL((walk_kernel<true>), dim3(static_cast<unsigned>(a.B)), dim3(kWalk), 0, stream, a);
    else hipLaunchKernelGGL((walk_kernel<false>), dim3(static_cast<unsigned>(a.B)), dim3(kWalk), 0, stream, a);
    return hipGetLastError();
}

}  // namespace mla
