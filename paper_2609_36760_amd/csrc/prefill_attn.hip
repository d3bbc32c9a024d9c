// Expanded latent attention (mla_prefill_attn): softmax(tau (q_nope . k_nope +
// q_rope . k_rope)) v over 192 score channels (64 of them one key row for all
// heads) and 128 value channels, for blocks of query rows.
//
// One workgroup takes a plan's work item for one head: G groups of 32 query rows
// per wave, all waves over the same key tiles.  Per tile of KT keys (KT / 32 key
// blocks):
//   1. the tile's rows go from memory straight into LDS, two tiles ahead, 16
//      bytes a lane; LDS places are linear in the lane, so the bank swizzle is
//      applied to which 16 bytes of a row a lane fetches;
//   2. S^T[key][row] = K . Q^T, v_mfma_f32_32x32x16_bf16 (M = 32 keys, N = 32
//      rows, K = 192 channels in 12 steps), Q^T in registers throughout: a lane
//      ends up with one row's scores for half of the keys, its partner lane ^ 32
//      with the other half;
//   3. one pass over the scores: weights 2^(s - reference) in fp32 on the row's
//      running reference, rounded to bf16, their sums;
//   4. O^T[channel][row] += V^T . P^T (M = 128 channels in 4 blocks, K = KT
//      keys): P^T comes straight from the score registers, because the
//      transposing LDS reads fetch V's keys in the order in which the score
//      product left them.
//
// What bounds it is the matrix unit, and the power that everything around it
// draws (the clock falls from 2.4 to 1.65 GHz under the two-waves-per-SIMD form
// of this kernel).  So a wave has two row groups where there are rows enough:
// every operand read from LDS feeds two products, every tile staged 256 rows.
// Such a wave has a SIMD to itself (acc 128, Q 96, scores 64, weights 32
// registers), and overlaps by its own instruction order: the softmax of one key
// block runs between the products of the next.
//
// Roundings: the weights are bf16 operands of the second product (at most 2^-8
// of a weight, as the bf16 output's own rounding; bf16 values allow no wider
// ones).  Scores, reference, sum and accumulators are fp32, the sum taken of the
// weights before their rounding.  (Normalizing by the sum of the rounded weights
// would spare rows that one key dominates that key's rounding, but bf16 dot
// products take the matrix unit's time, 11 cycles each, and unpacking the weights
// four more vector instructions a pair.)
//
// The reference.  bf16 has the range of fp32, so a row's weights may be taken on
// any reference that keeps them from overflow: a row's is its maximum over its
// first 32 keys, and it stays, and no later tile is searched for maxima, as long
// as a block's weights add up to less than 2^100 -- scores 69 above the first
// ones in natural units.  A workgroup that meets larger sums, sums that are no
// number, or values that are not finite where a row is hidden from them, does its
// rows over in careful_rows, which moves references tile by tile.  (Kept apart, so
// that the accumulators have one place throughout: any other use of them between
// the products made the compiler copy them in every tile.)
#include <hip/hip_runtime.h>

#include <cfloat>
#include <type_traits>

#include "internal.h"
#include "kernel_common.h"
#include "prefill_internal.h"

namespace mla {
namespace {

using kc::bf16x8;
using kc::f32x16;
using kc::i16x4;
using kc::lds_i16x4;

typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kMost = 0x1p100f;
constexpr float kUnset = -FLT_MAX;

// Score products accumulate in vector registers, with the queries in accumulation
// registers beside the output: kept with the output, the compiler would copy every
// score out.  As inline assembly they get no wait states from it: the first
// product of a chain writes without reading, the following ones accumulate back
// to back (no wait between products of one shape), and scores_ready supplies the
// wait before vector instructions read the result (12 wait states after a
// 32 x 32 x 16 product).
__device__ __forceinline__ void score_mfma(f32x16& c, bf16x8 a, bf16x8 b, bool first) {
    if (first) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "a"(b));
    else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "a"(b));
}
__device__ __forceinline__ void scores_ready(f32x16& c) { asm volatile("s_nop 7\n\ts_nop 7" : "+v"(c)); }
// The same after four more products (each holds the matrix unit for 32 cycles).
__device__ __forceinline__ void scores_past(f32x16& c) { asm volatile("s_nop 4" : "+v"(c)); }

// Maximum / sum of a value and its copy in lane ^ 32.
__device__ __forceinline__ float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
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

// NW waves of G row groups over tiles of KT keys.
template <int NW, int G, int KT>
struct Shape {
    static constexpr int rows = NW * G * kRowsPerWave;
    static constexpr int kb = KT / 32;                      // key blocks of a tile
    static constexpr int plane = KT * kRow;
    static constexpr int value_at = 3 * plane, tile = 5 * plane;
    static constexpr int blocks = KT / 8;                   // loads of 1 KiB (8 rows) per plane
    static constexpr int loads = 5 * blocks / NW;           // per wave
    static_assert(blocks % NW == 0, "a wave's load belongs to one plane");
    static constexpr int buffers = 3;
    static constexpr int lds = buffers * tile + (buffers + 1) * NW * 4;
    static_assert(lds <= 160 * 1024 && NW * G * kRowsPerWave * 256 <= (buffers - 1) * tile, "LDS; results beside the last tile");
};

template <int NW, int G, int KT>
__global__ __launch_bounds__(64 * NW, 1) void prefill_kernel(PrefillArgs a) {
    using S = Shape<NW, G, KT>;
    constexpr int KB = S::kb;
    __shared__ __align__(1024) uint8_t smem[S::buffers * S::tile];
    __shared__ uint32_t flags[(S::buffers + 1) * NW];

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
    const int q_rows = min(min(max(ip->q_rows, 1), S::rows), a.total_q - q_row);
    const int kv_row = min(max(ip->kv_row, 0), a.total_kv);
    const int key1 = min(max(ip->key1, 0), a.total_kv - kv_row);
    const int key0 = min(max(ip->key0, 0), key1);
    const int seen0 = ip->seen0;
    const int part = min(ip->part, a.num_parts - 1);

    // keys that row x of the block sees
    auto sees = [&](int x) { return static_cast<int>(min(static_cast<int64_t>(key1), static_cast<int64_t>(seen0) + x)); };
    const int r0 = wave * G * kRowsPerWave;         // the wave's first row of the block
    const int see_block = sees(0), see_first = sees(r0);
    const int r_last = min(r0 + G * kRowsPerWave, q_rows) - 1;
    const int see_last = r_last < r0 ? key0 : sees(r_last);     // the most keys that a row of this wave sees

    // ---- staging ----------------------------------------------------------
    const uint32_t kn_b = static_cast<uint32_t>(a.k_nope.stride_t * 2), kr_b = static_cast<uint32_t>(a.k_rope.stride_t * 2),
                   vv_b = static_cast<uint32_t>(a.v.stride_t * 2);
    const uint8_t* const kn = reinterpret_cast<const uint8_t*>(a.k_nope.data + static_cast<int64_t>(head) * a.k_nope.stride_h) +
                              static_cast<int64_t>(kv_row) * kn_b;
    const uint8_t* const kr = reinterpret_cast<const uint8_t*>(a.k_rope.data) + static_cast<int64_t>(kv_row) * kr_b;
    const uint8_t* const vv = reinterpret_cast<const uint8_t*>(a.v.data + static_cast<int64_t>(head) * a.v.stride_h) +
                              static_cast<int64_t>(kv_row) * vv_b;
    const uint32_t lds0 = kc::lds_addr(smem);
    // A wave's loads of a tile: i * NW + wave counts the tile's 8-row blocks, plane by
    // plane.  Rows past the range's end re-read its last key.
    auto stage = [&](int key, int to) __attribute__((always_inline)) {
        const int last = key1 - 1 - key;
        int l = lane;
        asm volatile("" : "+v"(l));         // (what follows from it is not worth registers across the loops)
        const uint8_t* const n = kn + static_cast<int64_t>(key) * kn_b;
        const uint8_t* const r = kr + static_cast<int64_t>(key) * kr_b;
        const uint8_t* const v = vv + static_cast<int64_t>(key) * vv_b;
#pragma unroll
        for (int i = 0; i < S::loads; ++i) {
            const int plane = i * NW / S::blocks, block = i * NW % S::blocks + wave;
            const int x = block * 8 + (l >> 3);
            const uint32_t row = static_cast<uint32_t>(min(x, last));
            const uint32_t c = static_cast<uint32_t>((l & 7) ^ (plane < 3 ? score_xor(x) : value_xor(x))) * 16;
            const uint32_t at = lds0 + to + plane * S::plane + block * 1024;
            if (plane < 2) kc::dma16_m0(n + plane * kRow, row * kn_b + c, at);
            else if (plane == 2) kc::dma16_m0(r, row * kr_b + c, at);
            else kc::dma16_m0(v + (plane - 3) * kRow, row * vv_b + c, at);
        }
    };
    // Load i of a tile that is there whole: a wave's loads are a swizzle period (16
    // rows) apart, or half of one, so a lane has two offsets per kind of row, and the
    // rest is scalar.
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
    // A value that some row does not see must not reach that row through 0 * inf or
    // 0 * NaN.  A wave looks through the values that it staged itself, once they are
    // there, of the tiles that some row sees in part; `flags` says whether any wave
    // found one that is not finite (the buffer's NW words).
    auto look = [&](int key, int to) __attribute__((always_inline)) {
        if (key + KT <= see_block) return;
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < S::loads; ++i) {
            const int plane = i * NW / S::blocks, block = i * NW % S::blocks + wave;
            if (plane < 3) continue;
            const uint4 x = *reinterpret_cast<const uint4*>(smem + to + plane * S::plane + block * 1024 + lane * 16);
            const uint32_t w4[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) found |= ((w4[j] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;  // an exponent of all ones carries
        }
        const uint32_t any = __ballot(found != 0) != 0;
        if (lane == 0) flags[to / S::tile * NW + wave] = any;
    };
    auto odd_values = [&](int off) __attribute__((always_inline)) {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) any |= flags[off / S::tile * NW + i];
        return __builtin_amdgcn_readfirstlane(any) != 0;
    };
    // Buffers are used in turn: tile j + 2 goes where tile j - 1 was.
    auto after = [&](int off) __attribute__((always_inline)) { return off == (S::buffers - 1) * S::tile ? 0 : off + S::tile; };
    // Once per tile, anywhere in a wave's work on it: the next tile is there, and no
    // wave reads the one before any more.
    auto meet = [&](int key, int off) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        if (key + KT < key1) look(key + KT, after(off));
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    };
    auto stage_ahead = [&](int key, int off) __attribute__((always_inline)) {
        if (key + 2 * KT < key1) stage(key + 2 * KT, after(after(off)));
    };
    if (key0 < key1) stage(key0, 0);

    // ---- queries: operand B of step ks holds channels 16 ks + 8 half .. + 7 of the
    // lane's row of the group
    bf16x8 q[G][12];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int64_t qr = q_row + min(r0 + 32 * g + col, q_rows - 1);
        const uint16_t* const qn_p = a.q_nope.data + qr * a.q_nope.stride_t + static_cast<int64_t>(head) * a.q_nope.stride_h + 8 * half;
        const uint16_t* const qr_p = a.q_rope.data + qr * a.q_rope.stride_t + static_cast<int64_t>(head) * a.q_rope.stride_h + 8 * half;
#pragma unroll
        for (int ks = 0; ks < 12; ++ks)
            q[g][ks] = *reinterpret_cast<const bf16x8*>(ks < 8 ? qn_p + 16 * ks : qr_p + 16 * (ks - 8));
    }
    // (waited for here: the wait that the compiler would put into the loop, for
    // its first pass, would hold every pass up until the next tile is staged)
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int ks = 0; ks < 12; ++ks) asm volatile("" : "+a"(q[g][ks]));

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
    // operand A: keys of block st / 12, channels of step st % 12
    auto key_operand = [&](const int (&base)[4], int st) __attribute__((always_inline)) {
        const int b = st / 12, ks = st % 12;
        return *reinterpret_cast<const bf16x8*>(smem + base[ks & 3] + (ks >> 2) * S::plane + b * 32 * kRow);
    };
    // operand A: channels of block m = st % 4, the 16 keys of step st / 4
    auto value_operand = [&](const int (&base)[2], int st) __attribute__((always_inline)) {
        const int ks = st >> 2, m = st & 3;
        const uint8_t* at = smem + base[m & 1] + (m >> 1) * S::plane + ks * 16 * kRow;
        const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at);
        const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + 8 * kRow));
        return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    f32x16 acc[G][4];
    float ref[G], sum[G];                   // reference, sum of the weights
#pragma unroll
    for (int g = 0; g < G; ++g) {
        ref[g] = kUnset;
        sum[g] = 0.0f;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[g][m][i] = 0.0f;
    }
    const float c2 = a.scale_log2;
    bool careful = false;                   // whether the rows have to be done over

    // register i of block b is key `key + 32 b + (i & 3) + 8 (i >> 2) + 4 half`
    f32x16 s[KB][G];
    uint32_t w[G][8 * KB];                  // weights, bf16 pairs
    float block_sum[G];
    auto hide = [&](int b, int g, int key) __attribute__((always_inline)) {
        const int here = sees(r0 + 32 * g + col) - key - 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (32 * b + (i & 3) + 8 * (i >> 2) >= here) s[b][g][i] = -INFINITY;
    };
    // the row's largest score of block b, log2 units
    auto top_of = [&](int b, int g) __attribute__((always_inline)) {
        float top = s[b][g][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[b][g][i]);
        return max_halves(top) * c2;
    };
    auto weights = [&](int g, int ks) __attribute__((always_inline)) {
        const u32x4 x = {w[g][4 * ks], w[g][4 * ks + 1], w[g][4 * ks + 2], w[g][4 * ks + 3]};
        return __builtin_bit_cast(bf16x8, x);
    };
    auto take_sums = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < G; ++g) sum[g] += block_sum[g];
    };

    // A tile's products are
    //   A  scores of block 0        B  scores of block 1
    //   C  values of block 0        D  values of block 1
    // and block 0's softmax lies between A and C, block 1's between B and D.  From tile
    // to tile they run in the order  B(j) C(j) A(j+1) D(j): either softmax then has a
    // score and a value phase to spread over.
    //
    // A slot is one matrix instruction and what is issued in its shadow: at most one
    // weight, the operand read of a later slot, a load of the tile after the next.  The
    // scheduling barriers keep that order.
    constexpr int kAhead = 4, kWeights = 16 * G;
    constexpr int kUnits = kWeights + 2, kEarly = G == 2 ? 12 : 8;      // of them in the value phase
    bf16x8 ring[kAhead];                        // operands on their way from LDS
    int kt[4], vt[2];                           // the tile's operand addresses
    auto set_tile = [&](int off) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) kt[j] = at_tile(ka[j], off);
#pragma unroll
        for (int j = 0; j < 2; ++j) vt[j] = at_tile(va[j], off);
    };
    auto nothing = [](int) __attribute__((always_inline)) {};
    // Slots of block b's scores / values; ahead(f) reads operand f from the phase's start
    // that lies behind it; more(slot) goes with the slot.
    auto score_phase = [&](int b, auto ahead, auto more) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < 12; ++f) {
            const bf16x8 op = ring[f % kAhead];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                score_mfma(s[b][g], op, q[g][f], f == 0);
                if (g == 0) ring[f % kAhead] = f + kAhead < 12 ? key_operand(kt, 12 * b + f + kAhead) : ahead(f + kAhead - 12);
                more(f * G + g);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto value_phase = [&](int b, auto ahead, auto more) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < 8; ++f) {
            const bf16x8 op = ring[f % kAhead];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                acc[g][f & 3] = mfma(op, weights(g, 2 * b + (f >> 2)), acc[g][f & 3]);
                if (g == 0)
                    ring[f % kAhead] = f + kAhead < 8 ? __builtin_bit_cast(bf16x8, value_operand(vt, 8 * b + f + kAhead)) : ahead(f + kAhead - 8);
                more(f * G + g);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto keys_of = [&](int b) __attribute__((always_inline)) { return [&, b](int f) __attribute__((always_inline)) { return key_operand(kt, 12 * b + f); }; };
    auto values_of = [&](int b) __attribute__((always_inline)) { return [&, b](int f) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x8, value_operand(vt, 8 * b + f)); }; };
    auto keep = [&](int f) __attribute__((always_inline)) { return ring[f]; };
    // The softmax of block b, in units: the argument of weight u, the exponential of
    // weight u - 1, the sum (and rounding) of weight u - 2, so that no instruction of a
    // unit waits for another (a wave alone on its SIMD would stand still for it).  The
    // early units start in slot 4 of the value phase (4 products after the scores), the
    // late ones, and the test of the sums, fill the score phase.
    float argument, weight, kept;               // in the units' pipeline
    int here[G];                                // keys of the tile that the lane's rows see, less 4 half
    auto set_here = [&](int key) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < G; ++g) here[g] = sees(r0 + 32 * g + col) - key - 4 * half;
    };
    auto unit = [&](int b, int u, bool hide) __attribute__((always_inline)) {
        if (u >= 2 && u - 2 < kWeights) {
            const int g = (u - 2) / 16, i = (u - 2) % 16;
            block_sum[g] = i == 0 ? weight : block_sum[g] + weight;
            if (i & 1) w[g][8 * b + (i >> 1)] = kc::pack_bf16x2(kept, weight);
            else kept = weight;
            asm volatile("" : "+v"(block_sum[g]));      // (computed here, not sunk behind the next branch)
            if (i & 1) asm volatile("" : "+v"(w[g][8 * b + (i >> 1)]));
        }
        if (u >= 1 && u - 1 < kWeights) {
            weight = __builtin_amdgcn_exp2f(argument);
            asm volatile("" : "+v"(weight));
        }
        if (u < kWeights) {
            const int i = u % 16;
            argument = fmaf(s[b][u / 16][i], c2, -ref[u / 16]);
            if (hide) argument = 32 * b + (i & 3) + 8 * (i >> 2) < here[u / 16] ? argument : -INFINITY;
            asm volatile("" : "+v"(argument));
        }
    };
    auto early = [&](int b, int slot, bool hide) __attribute__((always_inline)) {
        if (slot < 4) return;
        if (slot == 4) {
#pragma unroll
            for (int g = 0; g < G; ++g) scores_past(s[b][g]);
        }
        constexpr int per = kEarly / (8 * G - 4);
#pragma unroll
        for (int u = 0; u < per; ++u) unit(b, (slot - 4) * per + u, hide);
    };
    auto late = [&](int b, int slot, bool hide) __attribute__((always_inline)) {
        if (kEarly + slot < kUnits) unit(b, kEarly + slot, hide);
        else if (slot == 12 * G - 1) take_sums();
    };
    static_assert(kUnits - kEarly < 12 * G, "the last slot takes the sums");
    auto weigh_rest = [&](int b, int from, bool hide) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (u >= from) unit(b, u, hide);
        take_sums();
    };
    const uint8_t *next_n, *next_r, *next_v;    // rows of the tile after the next
    // A of a tile by itself, and its early weights; the first tile of all sets the
    // references.  Ends with B's (or C's) operands on their way.
    auto begin_tile = [&](int key, int off) __attribute__((always_inline)) {
        set_tile(off);
        set_here(key);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) ring[j] = key_operand(kt, j);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (KB == 2) score_phase(0, keys_of(1), nothing);
        else score_phase(0, values_of(0), nothing);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            scores_ready(s[0][g]);
            if (key + KT > see_first) hide(0, g, key);
        }
        if (key == key0) {
#pragma unroll
            for (int g = 0; g < G; ++g) ref[g] = fmaxf(kUnset, top_of(0, g));      // (no key: any finite value)
        }
#pragma unroll
        for (int u = 0; u < kEarly; ++u) unit(0, u, false);
    };
    // The rest of a tile after begin_tile; kNext: with the next tile's A and early
    // weights, else by itself.  kPart: some row of the wave may not see all of it (or of
    // the next); otherwise it and the next are whole, and another whole one is behind
    // them.  `careful` is set where the tile is not for this path.
    auto finish_tile = [&](int key, int off, auto with_next, auto in_part) __attribute__((always_inline)) {
        constexpr bool kNext = decltype(with_next)::value, kPart = decltype(in_part)::value;
        const int next = after(off);
        const uint32_t to = after(next);
        meet(key, off);
        if constexpr (kPart) {
            stage_ahead(key, off);
            careful = careful || (key + KT > see_block && odd_values(off));
        }
        // (spread over the 20 G slots of B and C)
        auto load_slot = [&](int slot) __attribute__((always_inline)) {
            if constexpr (!kPart) {
#pragma unroll
                for (int i = 0; i < S::loads; ++i)
                    if (i * 20 * G / S::loads == slot) load_whole(i, to, next_n, next_r, next_v);
            }
        };
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (KB == 1) {
            weigh_rest(0, kEarly, kPart);
            value_phase(0, keep, nothing);
        } else {
            score_phase(1, values_of(0), [&](int slot) __attribute__((always_inline)) {
                late(0, slot, kPart);
                load_slot(slot);
            });
            if constexpr (kNext) {
#pragma unroll
                for (int j = 0; j < 4; ++j) kt[j] = at_tile(ka[j], next);
                value_phase(0, keys_of(0), [&](int slot) __attribute__((always_inline)) {
                    early(1, slot, kPart);
                    load_slot(12 * G + slot);
                });
                score_phase(0, values_of(1), [&](int slot) __attribute__((always_inline)) { late(1, slot, kPart); });
                if constexpr (kPart) {
#pragma unroll
                    for (int g = 0; g < G; ++g) here[g] -= KT;
                }
                value_phase(1, keys_of(1), [&](int slot) __attribute__((always_inline)) {
                    early(0, slot, kPart);
                    if (!kPart && slot == 0) {
                        next_n += static_cast<uint64_t>(KT) * kn_b;
                        next_r += static_cast<uint64_t>(KT) * kr_b;
                        next_v += static_cast<uint64_t>(KT) * vv_b;
                    }
                });
#pragma unroll
                for (int j = 0; j < 2; ++j) vt[j] = at_tile(va[j], next);
            } else {
                value_phase(0, values_of(1), [&](int slot) __attribute__((always_inline)) { early(1, slot, kPart); });
                weigh_rest(1, kEarly, kPart);
                value_phase(1, keep, nothing);
            }
        }
    };

    if (key0 < key1) {
        if (key0 + KT < key1) {
            stage(key0 + KT, S::tile);
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"(S::loads) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        }
        look(key0, 0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    }
    int key = key0, off = 0;
    if (key < see_last) {
        begin_tile(key, off);
        if constexpr (KB == 2) {
            const int last_followed = min(see_first - 2 * KT, key1 - 3 * KT);
            next_n = kn + static_cast<int64_t>(key + 2 * KT) * kn_b;
            next_r = kr + static_cast<int64_t>(key + 2 * KT) * kr_b;
            next_v = vv + static_cast<int64_t>(key + 2 * KT) * vv_b;
            while (key <= last_followed) {
                finish_tile(key, off, std::true_type{}, std::false_type{});
                key += KT;
                off = after(off);
            }
            set_here(key);
            while (key + KT < see_last) {
                finish_tile(key, off, std::true_type{}, std::true_type{});
                key += KT;
                off = after(off);
            }
            finish_tile(key, off, std::false_type{}, std::true_type{});
        } else {
            // (one key block: a tile begins and ends by itself)
            while (true) {
                finish_tile(key, off, std::false_type{}, std::true_type{});
                if (key + KT >= see_last) break;
                key += KT;
                off = after(off);
                begin_tile(key, off);
            }
        }
        key += KT;
        off = after(off);
    }
    // tiles of which no row of the wave sees any
    for (; key < key1; key += KT, off = after(off)) {
        meet(key, off);
        stage_ahead(key, off);
    }

    // ---- results of the 32 rows from row x of the block on; register i of block m is
    // channel 32 m + (i & 3) + 8 (i >> 2) + 4 half.  `own`: 8 KiB of LDS for the wave.
    auto put_rows = [&](int x, f32x16 (&o)[4], float ref, float sum, uint8_t* own) __attribute__((always_inline)) {
        const float total = sum_halves(sum);
        // weights that all vanish leave 0 here; whether that is a row without keys is
        // decided below, by what the row sees
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        const int r = x + col;
        if (part >= 0) {
            if (r >= q_rows) return;
            const int64_t row = (static_cast<int64_t>(part) * a.H + head) * S::rows + r;
            float* to = a.part_o + row * kValue + 4 * half;
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<float4*>(to + 32 * m + 2 * i) = make_float4(o[m][i] * inv, o[m][i + 1] * inv, o[m][i + 2] * inv, o[m][i + 3] * inv);
            if (half == 0) {
                a.part_m[row] = ref;
                a.part_l[row] = total;
            }
            return;
        }
        // a row that sees no key is 0 (lse -inf); one whose keys all weigh nothing is not a number
        const bool none = sees(r) <= key0;
        const float scale = none || total != 0.0f ? inv : NAN;
        if (a.lse != nullptr && half == 0 && r < q_rows)
            a.lse[(static_cast<int64_t>(q_row) + r) * a.H + head] = none ? -INFINITY : (ref + log2f(total)) * 0.6931471805599453f;
        // Through LDS, so that a store instruction writes whole rows: 32 rows of 256
        // bytes, 16 bytes c of row y at place c ^ (y & 15).
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int c = 4 * m + (i >> 2);
                *reinterpret_cast<uint2*>(own + col * 256 + ((c ^ (col & 15)) << 4) + 8 * half) =
                    make_uint2(kc::pack_bf16x2(o[m][i] * scale, o[m][i + 1] * scale), kc::pack_bf16x2(o[m][i + 2] * scale, o[m][i + 3] * scale));
            }
        // (a wave reads back only what it wrote: LDS accesses of a wave are in order)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int y = 4 * i + (lane >> 4), c = lane & 15;
            const uint4 z = *reinterpret_cast<const uint4*>(own + y * 256 + ((c ^ (y & 15)) << 4));
            if (x + y < q_rows)
                *reinterpret_cast<uint4*>(a.out + (static_cast<int64_t>(q_row) + x + y) * a.out_stride_t +
                                          static_cast<int64_t>(head) * a.out_stride_h + 8 * c) = z;
        }
    };

    // Whether any wave wants the rows done over (a finite sum below kMost, of weights
    // >= 0, had no block at or over it).
#pragma unroll
    for (int g = 0; g < G; ++g) careful = careful || __ballot(!(sum[g] < kMost)) != 0;
    if (lane == 0) flags[S::buffers * NW + wave] = careful;
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) any |= flags[S::buffers * NW + i];
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(any) == 0, 1)) {
        // in the place of the tiles, which no wave reads any more
#pragma unroll
        for (int g = 0; g < G; ++g) {
            put_rows(r0 + 32 * g, acc[g], ref[g], sum[g], smem + (wave * G + g) * 32 * 256);
        }
        return;
    }

    // careful_rows: 32 rows of a wave at a time, a tile at a time.
#pragma unroll 1
    for (int g = 0; g < G; ++g) {
        const int x = r0 + 32 * g;
        const int limit = sees(x + col);
        const int64_t qr = q_row + min(x + col, q_rows - 1);
        const uint16_t* const qn_p = a.q_nope.data + qr * a.q_nope.stride_t + static_cast<int64_t>(head) * a.q_nope.stride_h + 8 * half;
        const uint16_t* const qr_p = a.q_rope.data + qr * a.q_rope.stride_t + static_cast<int64_t>(head) * a.q_rope.stride_h + 8 * half;
        bf16x8 qc[12];
#pragma unroll
        for (int ks = 0; ks < 12; ++ks) qc[ks] = *reinterpret_cast<const bf16x8*>(ks < 8 ? qn_p + 16 * ks : qr_p + 16 * (ks - 8));
        f32x16 o[4] = {};
        float rc = kUnset, sc = 0.0f;
#pragma unroll 1
        for (int kc0 = key0; kc0 < key1; kc0 += KT) {
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");       // no wave reads the tile before
            stage(kc0, 0);
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" : : : "memory");
            uint32_t found = 0;
#pragma unroll 1
            for (int i = lane * 16; i < 2 * S::plane; i += 1024) {
                const uint4 y = *reinterpret_cast<const uint4*>(smem + S::value_at + i);
                const uint32_t w4[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) found |= ((w4[j] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
            }
            const bool odd = __ballot(found != 0) != 0;
#pragma unroll 1
            for (int b = 0; b < KB; ++b) {
                f32x16 z = {};
#pragma unroll
                for (int ks = 0; ks < 12; ++ks)
                    z = mfma(*reinterpret_cast<const bf16x8*>(smem + ka[ks & 3] + (ks >> 2) * S::plane + b * 32 * kRow), qc[ks], z);
                const int seen_here = limit - kc0 - 32 * b - 4 * half;
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    z[i] = (i & 3) + 8 * (i >> 2) < seen_here ? z[i] : -INFINITY;
                    top = fmaxf(top, z[i]);
                }
                const float to = fminf(fmaxf(rc, max_halves(top) * c2), FLT_MAX);   // (a score of +inf: weight, sum and lse +inf)
                const float f = __builtin_amdgcn_exp2f(rc - to);
                rc = to;
                sc *= f;
                uint32_t pairs[8];
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(z[i], c2, -rc)), e1 = __builtin_amdgcn_exp2f(fmaf(z[i + 1], c2, -rc));
                    sc += e0;
                    sc += e1;
                    pairs[i >> 1] = kc::pack_bf16x2(e0, e1);
                }
#pragma unroll
                for (int m = 0; m < 4; ++m) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[m][i] *= f;
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks) {
                        const uint8_t* at = smem + va[m & 1] + (m >> 1) * S::plane + (2 * b + ks) * 16 * kRow;
                        const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at);
                        const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + 8 * kRow));
                        i16x8 v = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
                        // values that are not finite are left out of the product ...
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = (v[j] & 0x7F80) == 0x7F80 ? 0 : v[j];
                        const u32x4 p4 = {pairs[4 * ks], pairs[4 * ks + 1], pairs[4 * ks + 2], pairs[4 * ks + 3]};
                        o[m] = mfma(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p4), o[m]);
                    }
                }
            }
            // ... and added to the rows that see them, to which they give what they are
            if (odd) {
#pragma unroll 1
                for (int j = 0; j < KT; ++j) {
#pragma unroll
                    for (int m = 0; m < 4; ++m)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int c = 4 * (m & 1) + (i >> 2);       // 16 bytes of the row: channels 8c .. 8c + 7 of the plane
                            const uint32_t bits = *reinterpret_cast<const uint16_t*>(
                                smem + S::value_at + (m >> 1) * S::plane + j * kRow + ((c ^ value_xor(j)) << 4) + 8 * half + 2 * (i & 3));
                            o[m][i] += (bits & 0x7F80u) == 0x7F80u && kc0 + j < limit ? __uint_as_float(bits << 16) : 0.0f;
                        }
                }
            }
        }
        put_rows(x, o, rc, sc, smem + S::tile + wave * 32 * 256);
    }
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
        hipLaunchKernelGGL((prefill_kernel<1, 1, 32>), grid, dim3(64), 0, stream, a);
    else if (a.rows == 128)
        hipLaunchKernelGGL((prefill_kernel<4, 1, 64>), grid, dim3(256), 0, stream, a);
    else if (a.rows == 256)
        hipLaunchKernelGGL((prefill_kernel<4, 2, 64>), grid, dim3(256), 0, stream, a);
    else
        return hipErrorInvalidValue;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.num_merges == 0) return e;
    const int64_t waves = static_cast<int64_t>(a.num_merges) * a.H * a.rows;
    hipLaunchKernelGGL(prefill_merge_kernel, dim3(static_cast<unsigned>((waves + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace mla
