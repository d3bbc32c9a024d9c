// Expanded latent attention (mla_prefill_attn): softmax(tau (q_nope . k_nope +
// q_rope . k_rope)) v over 192 score channels (64 of them one key row for all
// heads) and 128 value channels, for blocks of query rows.
//
// One workgroup takes a plan's work item for one head: 32 query rows per wave,
// all waves over the same key tiles.  Per tile of KT keys (KT / 32 key blocks):
//   1. the tile's rows go from memory straight into LDS, one tile ahead, 16
//      bytes a lane; LDS places are linear in the lane, so the bank swizzle is
//      applied to which 16 bytes of a row a lane fetches;
//   2. S^T[key][row] = K . Q^T, v_mfma_f32_32x32x16_bf16 (M = 32 keys, N = the
//      wave's 32 rows, K = 192 channels in 12 steps), Q^T in registers
//      throughout: a lane ends up with one row's scores for half of the keys,
//      its partner lane ^ 32 with the other half;
//   3. one pass over the scores: weights 2^(s - reference) in fp32 on the row's
//      running reference, rounded to bf16, their sums;
//   4. O^T[channel][row] += V^T . P^T (M = 128 channels in 4 blocks, K = KT
//      keys): P^T comes straight from the score registers, because the
//      transposing LDS reads fetch V's keys in the order in which the score
//      product left them.
//
// Roundings: the weights are bf16 operands of the second product (at most 2^-8
// of a weight, as the bf16 output's own rounding).  The output is normalized by
// the sum of the rounded weights, so that a row that one key dominates is not
// scaled by that key's rounding; lse takes the sum of the fp32 weights.
// Scores, reference, sums and accumulators are fp32.
//
// The reference.  bf16 has the range of fp32, so a row's weights may be taken on
// any reference that keeps them far from overflow: a row's is its maximum over
// its first tile, and it stays until a tile's weights add up to kMost or more
// (or to no number); then it moves to that tile's maximum, the accumulators
// follow, and the tile is weighed again.  So the maximum is only looked for in
// such tiles.  The reference starts at the lowest finite value: hidden scores
// (-inf) weigh 0 on it, every other overflows and moves it.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "internal.h"
#include "kernel_common.h"
#include "prefill_internal.h"

namespace mla {
namespace {

using kc::bf16x8;
using kc::f32x16;
using kc::i16x4;
using kc::lds_i16x4;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kMost = 0x1p30f;
constexpr float kUnset = -FLT_MAX;

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Maximum / sum of a value and its copy in lane ^ 32.
__device__ __forceinline__ float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ void tile_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

// LDS of one tile: KT rows of 128 nope channels (16 chunks of 16 bytes), KT of
// 64 RoPE channels (8 chunks), KT of 128 value channels (16 chunks).  Chunk c
// of row r stands at place c ^ x(r): the score reads (one chunk of 32 rows) and
// the transposing reads (4 chunks of 8 rows) then touch every bank equally.
constexpr int kNopeRow = 256, kRopeRow = 128, kValueRow = 256;
__device__ __forceinline__ int nope_xor(int r) { return r & 15; }
__device__ __forceinline__ int rope_xor(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int value_xor(int r) { return ((r & 3) << 2) | (((r >> 2) & 1) << 1); }

template <int NW, int KT>
struct Shape {
    static constexpr int kb = KT / 32;                      // key blocks of a tile
    static constexpr int rope_at = KT * kNopeRow;
    static constexpr int value_at = rope_at + KT * kRopeRow;
    static constexpr int tile = value_at + KT * kValueRow;
    // loads of 1 KiB per wave and region
    static constexpr int nope_loads = KT * kNopeRow / 1024 / NW;
    static constexpr int rope_loads = KT * kRopeRow / 1024 / NW;
    static constexpr int value_loads = KT * kValueRow / 1024 / NW;
    static_assert(rope_loads * 1024 * NW == KT * kRopeRow, "whole loads per wave");
};

template <int NW, int KT>
__global__ __launch_bounds__(64 * NW, 2) void prefill_kernel(PrefillArgs a) {
    using S = Shape<NW, KT>;
    constexpr int KB = S::kb;
    __shared__ __align__(1024) uint8_t smem[2 * S::tile];

    const int lane = static_cast<int>(threadIdx.x) & 63;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const int half = lane >> 5, col = lane & 31;

    // Workgroup -> (head, item).  Workgroup i runs on XCD i mod 8: where the heads
    // divide by 8 an XCD takes whole heads, one after the other, so that the
    // blocks of a head's rows read its keys through one L2.
    const int wg = static_cast<int>(blockIdx.x);
    int head, item_id;
    if ((a.H & 7) == 0) {
        const int k = wg >> 3;
        const int h = k / a.num_items;
        head = (wg & 7) * (a.H >> 3) + h;
        item_id = k - h * a.num_items;
    } else {
        item_id = wg / a.H;
        head = wg - item_id * a.H;
    }
    const PrefillItem* ip = a.items + item_id;
    // indices from the plan, kept inside the tensors whatever it holds
    const int q_row = min(max(ip->q_row, 0), a.total_q - 1);
    const int q_rows = min(min(max(ip->q_rows, 1), NW * kRowsPerWave), a.total_q - q_row);
    const int kv_row = min(max(ip->kv_row, 0), a.total_kv);
    const int key1 = min(max(ip->key1, 0), a.total_kv - kv_row);
    const int key0 = min(max(ip->key0, 0), key1);
    const int seen0 = ip->seen0;
    const int part = min(ip->part, a.num_parts - 1);

    const int r = wave * kRowsPerWave + col;        // the lane's row of the block
    const int seen = static_cast<int>(min(static_cast<int64_t>(key1), static_cast<int64_t>(seen0) + r));
    const int see_first = static_cast<int>(min(static_cast<int64_t>(key1), static_cast<int64_t>(seen0)));   // of row 0
    // the most keys that a row of this wave sees (rows that exist)
    const int r_first = wave * kRowsPerWave, r_last = min(r_first + kRowsPerWave, q_rows) - 1;
    const int see_max = r_last < r_first ? key0
                                         : static_cast<int>(min(static_cast<int64_t>(key1), static_cast<int64_t>(seen0) + r_last));

    // ---- staging ----------------------------------------------------------
    const uint32_t kn_b = static_cast<uint32_t>(a.k_nope.stride_t * 2), kr_b = static_cast<uint32_t>(a.k_rope.stride_t * 2),
                   vv_b = static_cast<uint32_t>(a.v.stride_t * 2);
    const uint8_t* const kn = reinterpret_cast<const uint8_t*>(a.k_nope.data + static_cast<int64_t>(head) * a.k_nope.stride_h) +
                              static_cast<int64_t>(kv_row) * kn_b;
    const uint8_t* const kr = reinterpret_cast<const uint8_t*>(a.k_rope.data) + static_cast<int64_t>(kv_row) * kr_b;
    const uint8_t* const vv = reinterpret_cast<const uint8_t*>(a.v.data + static_cast<int64_t>(head) * a.v.stride_h) +
                              static_cast<int64_t>(kv_row) * vv_b;
    const uint32_t lds0 = kc::lds_addr(smem);
    // A lane's places of the first load of each region; the following loads are
    // 4 NW (8 NW) rows on, where the swizzle repeats.
    const int n0 = wave * 64 + lane;
    const int nrow = n0 >> 4, rrow = n0 >> 3;
    const uint32_t nc = ((n0 & 15) ^ nope_xor(nrow)) * 16, rc = ((n0 & 7) ^ rope_xor(rrow)) * 16,
                   vc = ((n0 & 15) ^ value_xor(nrow)) * 16;
    static_assert((4 * NW) % 16 == 0 || S::nope_loads * 4 * NW <= 16 || NW < 4, "swizzle period");
    // tile from `key`; rows past the range's end re-read its last key
    auto stage = [&](int key, int buf) __attribute__((always_inline)) {
        const int last = key1 - 1 - key;
        const uint32_t at = lds0 + buf * S::tile + wave * 1024;
        const uint8_t* const n_base = kn + static_cast<int64_t>(key) * kn_b;
        const uint8_t* const r_base = kr + static_cast<int64_t>(key) * kr_b;
        const uint8_t* const v_base = vv + static_cast<int64_t>(key) * vv_b;
        if (last >= KT - 1 && NW >= 4) {
            const uint32_t vn = nrow * kn_b + nc, vr = rrow * kr_b + rc, vv_ = nrow * vv_b + vc;
#pragma unroll
            for (int i = 0; i < S::nope_loads; ++i)
                kc::dma16_m0(n_base + static_cast<uint64_t>(i * 4 * NW) * kn_b, vn, at + i * NW * 1024);
#pragma unroll
            for (int i = 0; i < S::rope_loads; ++i)
                kc::dma16_m0(r_base + static_cast<uint64_t>(i * 8 * NW) * kr_b, vr, at + S::rope_at + i * NW * 1024);
#pragma unroll
            for (int i = 0; i < S::value_loads; ++i)
                kc::dma16_m0(v_base + static_cast<uint64_t>(i * 4 * NW) * vv_b, vv_, at + S::value_at + i * NW * 1024);
            return;
        }
#pragma unroll
        for (int i = 0; i < S::nope_loads; ++i) {
            const int row = nrow + i * 4 * NW, c = (n0 & 15) ^ nope_xor(row);
            kc::dma16_m0(n_base, static_cast<uint32_t>(min(row, last)) * kn_b + c * 16, at + i * NW * 1024);
        }
#pragma unroll
        for (int i = 0; i < S::rope_loads; ++i) {
            const int row = rrow + i * 8 * NW, c = (n0 & 7) ^ rope_xor(row);
            kc::dma16_m0(r_base, static_cast<uint32_t>(min(row, last)) * kr_b + c * 16, at + S::rope_at + i * NW * 1024);
        }
#pragma unroll
        for (int i = 0; i < S::value_loads; ++i) {
            const int row = nrow + i * 4 * NW, c = (n0 & 15) ^ value_xor(row);
            kc::dma16_m0(v_base, static_cast<uint32_t>(min(row, last)) * vv_b + c * 16, at + S::value_at + i * NW * 1024);
        }
    };
    if (key0 < key1) stage(key0, 0);

    // ---- queries: operand B of step ks holds channels 16 ks + 8 half .. + 7 of row `col`
    const int64_t qr = q_row + min(r, q_rows - 1);
    const uint16_t* const qn_p = a.q_nope.data + qr * a.q_nope.stride_t + static_cast<int64_t>(head) * a.q_nope.stride_h + 8 * half;
    const uint16_t* const qr_p = a.q_rope.data + qr * a.q_rope.stride_t + static_cast<int64_t>(head) * a.q_rope.stride_h + 8 * half;
    bf16x8 q[12];
#pragma unroll
    for (int ks = 0; ks < 12; ++ks)
        q[ks] = *reinterpret_cast<const bf16x8*>(ks < 8 ? qn_p + 16 * ks : qr_p + 16 * (ks - 8));

    // ---- LDS read addresses of the lane, one per swizzled chunk; blocks, steps
    // and the buffer are immediate offsets
    const uint8_t* ka[12];
    const uint8_t* va[4];
    const int tr_row = 4 * half + ((lane & 15) >> 2);
#pragma unroll
    for (int ks = 0; ks < 12; ++ks) {
        int x = ks < 8 ? col * kNopeRow + (((2 * ks + half) ^ nope_xor(col)) << 4)
                       : S::rope_at + col * kRopeRow + (((2 * (ks - 8) + half) ^ rope_xor(col)) << 4);
        asm volatile("" : "+v"(x));
        ka[ks] = smem + x;
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        int x = S::value_at + tr_row * kValueRow +
                (((4 * m + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ value_xor(tr_row)) << 4) + (lane & 1) * 8;
        asm volatile("" : "+v"(x));
        va[m] = smem + x;
    }
    auto value_operand = [&](int off, int ks, int m) __attribute__((always_inline)) {
        const uint8_t* at = va[m] + off + ks * 16 * kValueRow;
        const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at);
        const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + 8 * kValueRow));
        return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    f32x16 acc[4];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[m][i] = 0.0f;
    float ref = kUnset, sum = 0.0f, rounded = 0.0f;      // sums of the weights, and of the rounded ones
    const float c2 = a.scale_log2;

    // register i of block b is key `key + 32 b + (i & 3) + 8 (i >> 2) + 4 half`
    auto scores = [&](int off, f32x16 (&s)[KB]) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < 12; ++ks)
#pragma unroll
            for (int b = 0; b < KB; ++b)
                s[b] = mfma(*reinterpret_cast<const bf16x8*>(ka[ks] + off + b * 32 * (ks < 8 ? kNopeRow : kRopeRow)), q[ks], s[b]);
    };
    // weights of a tile on the present reference; false if a row's weights went past
    // what the reference is for
    auto weigh = [&](const f32x16 (&s)[KB], bf16x8 (&p)[2 * KB], float& tile, float& tile_rounded) __attribute__((always_inline)) {
        tile = 0.0f;
        tile_rounded = 0.0f;
        uint32_t w[8 * KB];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float e0 = __builtin_amdgcn_exp2f(fmaf(s[b][i], c2, -ref));
                const float e1 = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], c2, -ref));
                const uint32_t pair = kc::pack_bf16x2(e0, e1);
                w[8 * b + (i >> 1)] = pair;
                tile += e0;
                tile += e1;
                tile_rounded = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u),
                                                               tile_rounded, false);
            }
#pragma unroll
        for (int k = 0; k < 2 * KB; ++k) {
            const u32x4 x = {w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]};
            p[k] = __builtin_bit_cast(bf16x8, x);
        }
        return __ballot(!(tile < kMost)) == 0;
    };
    // the reference of every row up to its maximum in this tile
    auto move_reference = [&](const f32x16 (&s)[KB]) __attribute__((always_inline)) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = max_halves(top) * c2;
        const float next = fminf(fmaxf(ref, top), FLT_MAX);     // (a score of +inf: weight, sum and lse +inf)
        const float f = exp2f(ref - next);
        ref = next;
        sum *= f;
        rounded *= f;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][i] *= f;
    };
    auto values = [&](int off, const bf16x8 (&p)[2 * KB]) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < 2 * KB; ++ks)
#pragma unroll
            for (int m = 0; m < 4; ++m) acc[m] = mfma(__builtin_bit_cast(bf16x8, value_operand(off, ks, m)), p[ks], acc[m]);
    };

    // ---- tiles that every row sees whole
    int key = key0;
    const int whole = max(key0, min(see_first, key1));      // (see_first: keys that the block's first row sees)
    auto step = [&](int off, int buf) __attribute__((always_inline)) {
        tile_barrier();         // this tile is in LDS; every wave is done with the other buffer
        if (key + KT < key1) stage(key + KT, buf ^ 1);
        f32x16 s[KB];
        bf16x8 p[2 * KB];
        float t, tr;
        scores(off, s);
        if (!weigh(s, p, t, tr)) {
            move_reference(s);
            weigh(s, p, t, tr);
        }
        sum += t;
        rounded += tr;
        values(off, p);
        key += KT;
    };
    int buf = 0;
    while (key + KT <= whole) {
        step(0, 0);
        buf = 1;
        if (key + KT > whole) break;
        step(S::tile, 1);
        buf = 0;
    }

    // ---- the others: the causal limit, the range's end
    for (; key < key1; key += KT, buf ^= 1) {
        tile_barrier();
        if (key + KT < key1) stage(key + KT, buf ^ 1);
        if (key >= see_max) continue;       // no row of this wave sees any of it
        const int off = buf * S::tile;
        f32x16 s[KB];
        bf16x8 p[2 * KB];
        float t, tr;
        scores(off, s);
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (key + 32 * b + (i & 3) + 8 * (i >> 2) + 4 * half >= seen) s[b][i] = -INFINITY;
        if (!weigh(s, p, t, tr)) {
            move_reference(s);
            weigh(s, p, t, tr);
        }
        sum += t;
        rounded += tr;

        // a key that some row does not see must not reach that row through 0 * inf
        // or 0 * NaN: values that are not finite are left out of the product, and
        // added to the rows that see them (to which they give what they are)
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < KT * kValueRow / 1024; ++i) {
            const uint4 x = *reinterpret_cast<const uint4*>(smem + off + S::value_at + i * 1024 + lane * 16);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) found |= ((w[j] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;  // an exponent of all ones carries
        }
        if (__ballot(found != 0) == 0) {
            values(off, p);
            continue;
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
#pragma unroll
            for (int ks = 0; ks < 2 * KB; ++ks) {
                auto v8 = value_operand(off, ks, m);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if ((v8[j] & 0x7F80) == 0x7F80) v8[j] = 0;
                acc[m] = mfma(__builtin_bit_cast(bf16x8, v8), p[ks], acc[m]);
            }
#pragma unroll 1
            for (int j = 0; j < KT; ++j) {
                const uint8_t* row = smem + off + S::value_at + j * kValueRow;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int ch = 32 * m + (i & 3) + 8 * (i >> 2) + 4 * half;
                    const uint32_t bits = *reinterpret_cast<const uint16_t*>(row + (((ch >> 3) ^ value_xor(j)) << 4) + (ch & 7) * 2);
                    if ((bits & 0x7F80u) == 0x7F80u && key + j < seen) acc[m][i] += __uint_as_float(bits << 16);
                }
            }
        }
    }

    // ---- results: register i of block m is channel 32 m + (i & 3) + 8 (i >> 2) + 4 half
    sum = sum_halves(sum);
    rounded = sum_halves(rounded);
    if (r >= q_rows) return;
    // weights that all vanish leave 0 here; whether that is a row without keys is
    // decided below, by what the row sees
    const float inv = rounded == 0.0f ? 0.0f : 1.0f / rounded;
    if (part >= 0) {
        const int64_t row = (static_cast<int64_t>(part) * a.H + head) * (NW * kRowsPerWave) + r;
        float* o = a.part_o + row * kValue + 4 * half;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4*>(o + 32 * m + 2 * i) = make_float4(acc[m][i] * inv, acc[m][i + 1] * inv, acc[m][i + 2] * inv, acc[m][i + 3] * inv);
        if (half == 0) {
            a.part_m[row] = ref;
            a.part_l[row] = sum;
        }
        return;
    }
    // a row that sees no key is 0 (lse -inf); one whose keys all weigh nothing is not a number
    const bool none = seen <= key0;
    const float scale = none || sum != 0.0f ? inv : NAN;
    uint16_t* o = a.out + (static_cast<int64_t>(q_row) + r) * a.out_stride_t + static_cast<int64_t>(head) * a.out_stride_h + 4 * half;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<uint2*>(o + 32 * m + 2 * i) = make_uint2(kc::pack_bf16x2(acc[m][i] * scale, acc[m][i + 1] * scale),
                                                                       kc::pack_bf16x2(acc[m][i + 2] * scale, acc[m][i + 3] * scale));
    if (a.lse != nullptr && half == 0)
        a.lse[(static_cast<int64_t>(q_row) + r) * a.H + head] = none ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
}

// Joins a block's partials: one wave per (block, head, row), two channels a lane.
__global__ __launch_bounds__(256) void prefill_merge_kernel(PrefillArgs a) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    const uint32_t w = blockIdx.x * 4 + (threadIdx.x >> 6);
    const uint32_t per_block = static_cast<uint32_t>(a.H) * a.rows;
    const uint32_t id = w / per_block, rest = w - id * per_block;
    if (id >= static_cast<uint32_t>(a.num_merges)) return;
    const int head = static_cast<int>(rest / a.rows), r = static_cast<int>(rest % a.rows);
    const PrefillMerge g = a.merges[id];
    if (r >= g.q_rows || g.q_row < 0 || g.q_row + r >= a.total_q) return;
    const int part0 = max(g.part0, 0), parts = min(g.num_parts, a.num_parts - part0);
    const int64_t step = static_cast<int64_t>(a.H) * a.rows;
    const int64_t row = part0 * step + static_cast<int64_t>(head) * a.rows + r;
    float top = kUnset;
    for (int j = 0; j < parts; ++j) top = fmaxf(top, a.part_m[row + j * step]);
    float sum = 0.0f;
    float2 o = make_float2(0.0f, 0.0f);
    for (int j = 0; j < parts; ++j) {
        const int64_t at = row + j * step;
        const float f = exp2f(a.part_m[at] - top) * a.part_l[at];
        const float2 x = *reinterpret_cast<const float2*>(a.part_o + at * kValue + 2 * lane);
        sum += f;
        o.x = fmaf(f, x.x, o.x);
        o.y = fmaf(f, x.y, o.y);
    }
    const bool none = min(static_cast<int64_t>(g.kv_len), static_cast<int64_t>(g.seen0) + r) <= 0;
    const float inv = none ? 0.0f : 1.0f / sum;
    const int64_t q = static_cast<int64_t>(g.q_row) + r;
    *reinterpret_cast<uint32_t*>(a.out + q * a.out_stride_t + static_cast<int64_t>(head) * a.out_stride_h + 2 * lane) =
        kc::pack_bf16x2(o.x * inv, o.y * inv);
    if (a.lse != nullptr && lane == 0)
        a.lse[q * a.H + head] = none ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace

hipError_t launch_prefill(const PrefillArgs& a, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(a.num_items) * static_cast<unsigned>(a.H));
    if (a.rows == 32)
        hipLaunchKernelGGL((prefill_kernel<1, 32>), grid, dim3(64), 0, stream, a);
    else if (a.rows == 128)
        hipLaunchKernelGGL((prefill_kernel<4, 64>), grid, dim3(256), 0, stream, a);
    else
        return hipErrorInvalidValue;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.num_merges == 0) return e;
    const int64_t waves = static_cast<int64_t>(a.num_merges) * a.H * a.rows;
    hipLaunchKernelGGL(prefill_merge_kernel, dim3(static_cast<unsigned>((waves + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace mla
