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
// its first tile, and it stays until a block's weights add up to kMost or more
// (or to no number); then it moves to that block's maximum, the accumulators
// follow, and the block is weighed again.  So whole tiles are not searched for
// maxima.  The reference starts at the lowest finite value, on which hidden
// scores (-inf) weigh 0.
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
typedef short i16x8 __attribute__((ext_vector_type(8)));
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

// LDS of one tile: five planes of 64 channels (128-byte rows) of all KT keys --
// nope 0-63, nope 64-127, RoPE, values 0-63, values 64-127.  16 bytes c of row r
// of a plane stand at place c ^ x(r): a read of the same 16 bytes of 32 rows, and
// a transposing read of 64 bytes of 8 rows, then touch every bank equally.  With
// planes, a lane's addresses differ by immediate offsets only, but for the
// swizzled places (4 registers for the scores, 2 for the values).
constexpr int kRow = 128;
__device__ __forceinline__ int score_xor(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int value_xor(int r) { return ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1; }

template <int NW, int KT>
struct Shape {
    static constexpr int kb = KT / 32;                      // key blocks of a tile
    static constexpr int plane = KT * kRow;
    static constexpr int value_at = 3 * plane, tile = 5 * plane;
    static constexpr int blocks = KT / 8;                   // loads of 1 KiB (8 rows) per plane
    static constexpr int loads = 5 * blocks / NW;           // per wave
    static_assert(blocks % NW == 0, "a wave's load belongs to one plane");
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
    // Load i of a wave's part of a tile into LDS byte `to`, from the tile's first
    // rows n, r, v; row(x) is the row to fetch for the tile's row x.
    auto load = [&](int lane, int i, uint32_t to, const uint8_t* n, const uint8_t* r, const uint8_t* v, auto row) __attribute__((always_inline)) {
        const int plane = i * NW / S::blocks, block = i * NW % S::blocks + wave;
        const int x = block * 8 + (lane >> 3);
        const uint32_t c = static_cast<uint32_t>((lane & 7) ^ (plane < 3 ? score_xor(x) : value_xor(x))) * 16;
        const uint32_t at = lds0 + to + plane * S::plane + block * 1024;
        if (plane < 2) kc::dma16_m0(n + plane * kRow, row(x) * kn_b + c, at);
        else if (plane == 2) kc::dma16_m0(r, row(x) * kr_b + c, at);
        else kc::dma16_m0(v + (plane - 3) * kRow, row(x) * vv_b + c, at);
    };
    // tile from `key`; rows past the range's end re-read its last key
    auto stage = [&](int key, int to) __attribute__((always_inline)) {
        const int last = key1 - 1 - key;
        int l = lane;
        asm volatile("" : "+v"(l));         // (what follows from it is not worth registers across the loops)
#pragma unroll
        for (int i = 0; i < S::loads; ++i)
            load(l, i, to, kn + static_cast<int64_t>(key) * kn_b, kr + static_cast<int64_t>(key) * kr_b,
                 vv + static_cast<int64_t>(key) * vv_b, [&](int x) { return static_cast<uint32_t>(min(x, last)); });
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

    // (waited for here: the wait that the compiler would put into the loop, for
    // its first pass, would hold every pass up until the next tile is staged)
#pragma unroll
    for (int ks = 0; ks < 12; ++ks) asm volatile("" : "+v"(q[ks]));

    // ---- LDS read addresses of the lane; planes, blocks and steps are immediate
    // offsets
    int ka[4], va[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) ka[j] = col * kRow + (((2 * j + half) ^ score_xor(col)) << 4);
    // the transposing read: 16 lanes fetch 4 rows x 16 channels, 8 bytes each
    const int tr_row = 4 * half + ((lane & 15) >> 2);
#pragma unroll
    for (int j = 0; j < 2; ++j)
        va[j] = S::value_at + tr_row * kRow + (((4 * j + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ value_xor(tr_row)) << 4) +
                (lane & 1) * 8;
    // (the base of an LDS access is a register that the tile's place is added to once)
    auto at_tile = [&](int x, int off) __attribute__((always_inline)) {
        x += off;
        asm volatile("" : "+v"(x));
        return x;
    };
    auto value_operand = [&](const int (&base)[2], int ks, int m) __attribute__((always_inline)) {
        const uint8_t* at = smem + base[m & 1] + (m >> 1) * S::plane + ks * 16 * kRow;
        const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at);
        const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + 8 * kRow));
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
    f32x16 s[KB];
    uint32_t w[8 * KB];         // weights, bf16 pairs
    float tile, tile_rounded;   // sums of a block's weights
    auto key_operand = [&](const int (&base)[4], int st) __attribute__((always_inline)) {
        const int b = st / 12, ks = st % 12;
        return *reinterpret_cast<const bf16x8*>(smem + base[ks & 3] + (ks >> 2) * S::plane + b * 32 * kRow);
    };
    auto score = [&](int st, bf16x8 k) __attribute__((always_inline)) {
        const int b = st / 12, ks = st % 12;
        const f32x16 zero = {};
        s[b] = mfma(k, q[ks], ks == 0 ? zero : s[b]);
    };
    // weights of registers 2j, 2j + 1 of block b on the present reference
    auto weigh = [&](int b, int j) __attribute__((always_inline)) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[b][2 * j], c2, -ref));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[b][2 * j + 1], c2, -ref));
        const uint32_t pair = kc::pack_bf16x2(e0, e1);
        w[8 * b + j] = pair;
        tile = j == 0 ? e0 : tile + e0;
        tile += e1;
        tile_rounded = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u),
                                                       j == 0 ? 0.0f : tile_rounded, false);
        // (computed here: the compiler would sink it behind the next branch)
        asm volatile("" : "+v"(w[8 * b + j]), "+v"(tile), "+v"(tile_rounded));
    };
    auto weights = [&](int ks) __attribute__((always_inline)) {
        const u32x4 x = {w[4 * ks], w[4 * ks + 1], w[4 * ks + 2], w[4 * ks + 3]};
        return __builtin_bit_cast(bf16x8, x);
    };
    auto too_large = [&]() __attribute__((always_inline)) { return __ballot(!(tile < kMost)) != 0; };

    // Any tile (its operands at kt, vt), from block `from` on: the causal limit, the
    // range's end, references that move.
    auto any_tile = [&](int key, int off, int from) __attribute__((always_inline)) {
        const int kt[4] = {at_tile(ka[0], off), at_tile(ka[1], off), at_tile(ka[2], off), at_tile(ka[3], off)};
        const int vt[2] = {at_tile(va[0], off), at_tile(va[1], off)};
        const int seen_here = seen - key - 4 * half;
        // a key that some row does not see must not reach that row through 0 * inf
        // or 0 * NaN: values that are not finite are left out of the product, and
        // added to the rows that see them (to which they give what they are)
        uint32_t found = 0;
        if (key + KT > see_first) {
#pragma unroll
            for (int i = 0; i < 2 * S::plane / 1024; ++i) {
                const uint4 x = *reinterpret_cast<const uint4*>(smem + off + S::value_at + i * 1024 + lane * 16);
                const uint32_t w4[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) found |= ((w4[j] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;  // an exponent of all ones carries
            }
        }
        const bool odd = __ballot(found != 0) != 0;
        auto block = [&](int b) __attribute__((always_inline)) {
#pragma unroll
            for (int ks = 0; ks < 12; ++ks) score(12 * b + ks, key_operand(kt, 12 * b + ks));
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (32 * b + (i & 3) + 8 * (i >> 2) >= seen_here) s[b][i] = -INFINITY;
            float top = s[b][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, s[b][i]);
            top = max_halves(top) * c2;
            if (__ballot(top > ref) != 0) {
                const float next = fminf(fmaxf(ref, top), FLT_MAX);     // (a score of +inf: weight, sum and lse +inf)
                const float f = __builtin_amdgcn_exp2f(ref - next);
                ref = next;
                sum *= f;
                rounded *= f;
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[m][i] *= f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) weigh(b, j);
            sum += tile;
            rounded += tile_rounded;
#pragma unroll
            for (int st = 8 * b; st < 8 * b + 8; ++st) {
                auto v8 = value_operand(vt, st >> 2, st & 3);
                if (odd) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if ((v8[j] & 0x7F80) == 0x7F80) v8[j] = 0;
                }
                acc[st & 3] = mfma(__builtin_bit_cast(bf16x8, v8), weights(st >> 2), acc[st & 3]);
            }
        };
        if (from == 0) block(0);
        if constexpr (KB == 2) block(1);
        if (!odd) return;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll 1
            for (int j = 32 * from; j < KT; ++j) {
                const uint8_t* row = smem + off + S::value_at + (m >> 1) * S::plane + j * kRow;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int c = 4 * (m & 1) + (i >> 2);       // 16 bytes of the row: channels 8c .. 8c + 7 of the plane
                    const uint32_t bits = *reinterpret_cast<const uint16_t*>(row + ((c ^ value_xor(j)) << 4) + 8 * half + 2 * (i & 3));
                    if ((bits & 0x7F80u) == 0x7F80u && key + j < seen) acc[m][i] += __uint_as_float(bits << 16);
                }
            }
    };

    // The loads of a whole tile: a wave's are a swizzle period (16 rows) apart, or
    // half of one, so a lane has two offsets per kind of row, and the rest is scalar.
    const int x0 = wave * 8 + (lane >> 3);
    const uint32_t c0 = ((lane & 7) ^ score_xor(x0)) * 16;
    const uint32_t at_n[2] = {x0 * kn_b + c0, x0 * kn_b + (c0 ^ 64)}, at_r[2] = {x0 * kr_b + c0, x0 * kr_b + (c0 ^ 64)};
    const uint32_t at_v = x0 * vv_b + ((lane & 7) ^ value_xor(x0)) * 16;
    auto load_whole = [&](int i, uint32_t to, const uint8_t* n, const uint8_t* r, const uint8_t* v) __attribute__((always_inline)) {
        const int plane = i * NW / S::blocks, first = i * NW % S::blocks;
        const uint32_t at = lds0 + to + plane * S::plane + (first + wave) * 1024;
        if (plane < 2) kc::dma16_m0(n + plane * kRow + static_cast<uint64_t>(first * 8) * kn_b, at_n[first & 1], at);
        else if (plane == 2) kc::dma16_m0(r + static_cast<uint64_t>(first * 8) * kr_b, at_r[first & 1], at);
        else kc::dma16_m0(v + (plane - 3) * kRow + static_cast<uint64_t>(first * 8) * vv_b, at_v, at);
    };

    // One tile by any_tile, then as many as there are that every row sees whole, with
    // another whole tile behind them, until one's weights are too large for a
    // reference: that one goes to any_tile again, from its block on.
    //
    // A slot is one matrix instruction and what is issued in its shadow: the operand
    // read of a later slot, a load of the next tile, a piece of the softmax.  The
    // scheduling barriers keep that order.  (Moving the reference here would make the
    // compiler copy the accumulators in every tile.)
    const int whole = min(see_first, key1 - KT);        // (see_first: keys that the block's first row sees)
    int key = key0, off = 0, from = 0;
    bool entered = false;
    while (key < key1) {
        if (!entered) {
            tile_barrier();         // this tile is in LDS; every wave is done with the other buffer
            if (key + KT < key1) stage(key + KT, S::tile - off);
        }
        if (key < see_max) any_tile(key, off, from);    // (else no row of this wave sees any of it)
        entered = false;
        from = 0;
        key += KT;
        off = S::tile - off;

        constexpr int kScores = 12 * KB, kValues = 8 * KB, kAhead = 4;
        static_assert(S::loads <= kScores || NW == 1, "loads of the next tile in the score slots");
        while (key + KT <= whole) {
            tile_barrier();
            const uint32_t to = S::tile - off;
            const uint8_t* const next_n = kn + static_cast<int64_t>(key + KT) * kn_b;
            const uint8_t* const next_r = kr + static_cast<int64_t>(key + KT) * kr_b;
            const uint8_t* const next_v = vv + static_cast<int64_t>(key + KT) * vv_b;
            const int kt[4] = {at_tile(ka[0], off), at_tile(ka[1], off), at_tile(ka[2], off), at_tile(ka[3], off)};
            const int vt[2] = {at_tile(va[0], off), at_tile(va[1], off)};
            bf16x8 k[kAhead];
            i16x8 v[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) k[j] = key_operand(kt, j);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int st = 0; st < kScores; ++st) {
                score(st, k[st % kAhead]);
                if (st + kAhead < kScores) k[st % kAhead] = key_operand(kt, st + kAhead);
                else v[st + kAhead - kScores] = value_operand(vt, 0, st + kAhead - kScores);
#pragma unroll
                for (int i = st; i < S::loads; i += kScores) load_whole(i, to, next_n, next_r, next_v);
                if (KB == 2 && st >= 14 && st < 22) weigh(0, st - 14);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (KB == 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) weigh(0, j);
            }
            entered = too_large();
            if (entered) break;
            sum += tile;
            rounded += tile_rounded;
            __builtin_amdgcn_sched_barrier(0);
            auto values = [&](int b) __attribute__((always_inline)) {
#pragma unroll
                for (int st = 8 * b; st < 8 * b + 8; ++st) {
                    const int m = st & 3;
                    acc[m] = mfma(__builtin_bit_cast(bf16x8, v[st % kAhead]), weights(st >> 2), acc[m]);
                    if (st + kAhead < kValues) v[st % kAhead] = value_operand(vt, (st + kAhead) >> 2, m);
                    if (b + 1 < KB && st > 0) weigh(b + 1, st - 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            values(0);
            if constexpr (KB == 2) {
                weigh(1, 7);
                if (too_large()) {
                    entered = true;
                    from = 1;
                    break;
                }
                sum += tile;
                rounded += tile_rounded;
                __builtin_amdgcn_sched_barrier(0);
                values(1);
            }
            key += KT;
            off = S::tile - off;
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
