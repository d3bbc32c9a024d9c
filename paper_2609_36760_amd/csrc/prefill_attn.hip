// Expanded latent attention (mla_prefill_attn): softmax(tau (q_nope . k_nope +
// q_rope . k_rope)) v over 192 score channels (64 of them one key row for all
// heads) and 128 value channels, for blocks of query rows.
//
// One workgroup takes blocks of query rows of one head: G groups of 32 rows per
// wave, all waves over the same key tiles.  Per tile of KT keys (KT / 32 key blocks):
//   1. the tile's rows go from memory straight into LDS, two tiles ahead, 16
//      bytes a lane; LDS places are linear in the lane, so the bank swizzle is
//      applied to which 16 bytes of a row a lane fetches;
//   2. S^T[key][row] = K . Q^T, v_mfma_f32_32x32x16_bf16 (M = 32 keys, N = 32
//      rows, K = 192 channels in 12 steps), Q^T in registers throughout: a lane
//      ends up with one row's scores for half of the keys, its partner lane ^ 32
//      with the other half;
//   3. one pass over the scores: weights 2^(s - reference) in fp32 on the row's
//      reference, rounded to bf16, their sums;
//   4. O^T[channel][row] += V^T . P^T (M = 128 channels in 4 blocks, K = KT
//      keys): P^T comes straight from the score registers, because the
//      transposing LDS reads fetch V's keys in the order in which the score
//      product left them.
//
// Two shapes (which one: choose_rows in mla_prefill_abi.cpp):
//   256 rows, 64 keys: a wave has two row groups and a SIMD to itself (acc 128,
//     Q 96, scores 64, weights 32 registers): every operand read from LDS feeds two
//     products, every tile staged 256 rows, and the softmax of one key block runs
//     between the products of the next, by the order of the instructions.  (The form
//     with two 32-row waves per SIMD reads twice as much LDS and memory per product;
//     the power that it drew brought the clock from 2.4 to 1.65 GHz, 8K keys, 128
//     heads, causal: 3.16 ms.)  A workgroup has a CU to itself, so nothing would hide a
//     block's beginning and end: it goes through a list of blocks; the first two tiles
//     of the next come in while the last ones are worked on, its queries while the
//     results go out (loaded earlier, they kept other waves waiting: 12 ragged prompts,
//     128 heads 842 us against 819, then 769 against 750).
//   128 rows, 32 keys: two workgroups per CU overlap each other; for up to 128 rows
//     per sequence, where the reads of keys and values are the bound.
//
// Measured (MI355X), 256 rows: 8K keys, causal, 128 heads 2.2-2.3 ms, 1200-1250 TFLOP/s of
// the visible keys' products; 8K x 8K, 64 heads 2.11 ms, 1300 (at 1.80 GHz; all-zero
// inputs, in the same cycles at 2.40 GHz, 1.53 ms: what is left is the power limit).  A
// tile takes 3.5K cycles for 2.56K of products, a block about 12K beside its tiles.  128
// rows: one token on 24 x 2K keys, 32 heads 169 us, 165 at a copy's rate; 256 prompts
// of 64, 64 heads 243 us (245).
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
// any reference near their scores: a row's is its largest score of the first 32
// keys that its wave meets, seen by the row or not, and it stays; no later tile is
// searched for maxima.  A row whose weights add up to less than 2^-60 or more than
// 2^60 (scores 41 off in natural units), or to no number, whose results are not
// finite (values above 2^67 may leave fp32's range under sums that large, those
// near 2^127 under any), or that is hidden from values that are not finite, sends its
// workgroup through careful_rows, which does the block over, moves references tile by
// tile and takes the second product's weights times 2^-32 (2^30 keys of equal weight
// then add up to 2^-2).  Weights under 2^-66 of a row's sum, and products with a value
// under 2^-66, may leave fp32's range below.  (Kept apart, so that the accumulators
// have one place throughout: any other use of them between the products made the
// compiler copy them in every tile.  References 40 log2 units above the scores would
// spare the look at the results, which takes 0.1-0.7 % of a call, but differences that
// large round 6 times coarser in lse.)
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

constexpr float kLeast = 0x1p-60f, kMost = 0x1p60f;     // sums that stand
constexpr float kLowered = 0x1p-32f;                    // of the weights of rows that are done over
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

// Sixteen bytes a lane from base + voff straight into LDS, 1 KiB from `lds` on.  The
// base goes through a scalar instruction here: if the compiler brings it back by
// v_readlane, a memory instruction may not read it for five wait states, and it does
// not see that one does.  (It is the wait state after the write of M0 as well; five
// of s_nop in its place took 1 % more of a prompt's time.)  kOnce: rows that one block
// reads, past the caches; those that several blocks read stay (12 ragged prompts, 128
// heads: 774 us against 839; 4 of 4K, 64 heads: 1272 against 1414).
template <bool kOnce>
__device__ __forceinline__ void dma16(const uint8_t* base, uint32_t voff, uint32_t lds) {
    uint64_t from;
    if constexpr (kOnce)
        asm volatile("s_mov_b64 %0, %2\n\tglobal_load_lds_dwordx4 %1, %0 nt" : "=&s"(from) : "v"(voff), "s"(base), "{m0}"(lds) : "memory");
    else
        asm volatile("s_mov_b64 %0, %2\n\tglobal_load_lds_dwordx4 %1, %0" : "=&s"(from) : "v"(voff), "s"(base), "{m0}"(lds) : "memory");
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
    static constexpr bool listed = rows == kListedRows;     // goes through a list of blocks
    static constexpr int lds = buffers * tile + (buffers + 1) * NW * 4;
    static_assert(lds <= 160 * 1024 && NW * kRowsPerWave * 256 <= (listed ? 1 : buffers - 1) * tile, "LDS; results in the place of tiles");
};

template <int NW, int G, int KT>
__global__ __launch_bounds__(64 * NW, G == 2 ? 1 : 2) void prefill_kernel(PrefillArgs a) {
    using S = Shape<NW, G, KT>;
    constexpr int KB = S::kb;
    __shared__ __align__(1024) uint8_t smem[S::buffers * S::tile];
    __shared__ uint32_t flags[(S::buffers + 1) * NW];

    const int lane = static_cast<int>(threadIdx.x) & 63;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const int half = lane >> 5, col = lane & 31;

    // Workgroup -> (item, head).  Workgroup i runs on XCD i mod 8: where the heads
    // divide by 8 an XCD takes whole heads, so that the blocks of a head's rows read
    // its keys through one L2.
    struct Block {
        int head, q_row, q_rows, kv_row, key0, key1, seen0, part;
        int tiles;
        bool down;          // the tiles from the last to the first
    };
    const int wg = static_cast<int>(blockIdx.x);
    const bool by_xcd = (a.H & 7) == 0;
    const int heads = by_xcd ? a.H >> 3 : a.H, head0 = by_xcd ? (wg & 7) * heads : 0;
    const int list = by_xcd ? wg >> 3 : wg;
    auto block_of = [&](int entry) __attribute__((always_inline)) {
        // indices from the plan, kept inside the tensors whatever it holds
        const bool down = S::listed && entry < 0;
        const uint32_t e = static_cast<uint32_t>(down ? ~entry : entry), item = e / static_cast<uint32_t>(heads);
        const PrefillItem* const ip = a.items + min(item, static_cast<uint32_t>(a.num_items - 1));
        Block x;
        x.head = head0 + static_cast<int>(e - item * static_cast<uint32_t>(heads));
        x.q_row = min(max(ip->q_row, 0), a.total_q - 1);
        x.q_rows = min(min(max(ip->q_rows, 1), S::rows), a.total_q - x.q_row);
        x.kv_row = min(max(ip->kv_row, 0), a.total_kv);
        x.key1 = min(max(ip->key1, 0), a.total_kv - x.kv_row);
        x.key0 = min(max(ip->key0, 0), x.key1);
        x.seen0 = max(ip->seen0, -S::rows);      // (no row sees a key: differences from it stay within 32 bits)
        x.part = min(ip->part, a.num_parts - 1);
        x.tiles = (x.key1 - x.key0 + KT - 1) / KT;
        x.down = down;
        return x;
    };
    // a list's entries, for a workgroup of 256 rows (the launch has one per list)
    int at = 0, end = 1;
    const int32_t* entries = nullptr;
    if constexpr (S::listed) {
        const int lists = by_xcd ? static_cast<int>(gridDim.x >> 3) : static_cast<int>(gridDim.x);
        const int most = a.num_items * heads;
        entries = a.first + lists + 1;
        at = min(max(a.first[list], 0), most);
        end = min(a.first[list + 1], most);
        if (at >= end) return;
    }
    Block cur = block_of(S::listed ? entries[at] : list);

    const int r0 = wave * G * kRowsPerWave;         // the wave's first row of a block
    // a block's tile t, in the order in which they are gone through
    auto key_of = [&](const Block& b, int t) __attribute__((always_inline)) { return b.key0 + KT * (b.down ? b.tiles - 1 - t : t); };
    // keys that row x of a block sees
    auto sees_of = [&](const Block& b, int x) { return static_cast<int>(min(static_cast<int64_t>(b.key1), static_cast<int64_t>(b.seen0) + x)); };

    // ---- staging ----------------------------------------------------------
    const uint32_t kn_b = static_cast<uint32_t>(a.k_nope.stride_t * 2), kr_b = static_cast<uint32_t>(a.k_rope.stride_t * 2),
                   vv_b = static_cast<uint32_t>(a.v.stride_t * 2);
    // rows of key `key` of a block
    auto nope_at = [&](const Block& b, int key) __attribute__((always_inline)) {
        return reinterpret_cast<const uint8_t*>(a.k_nope.data + static_cast<int64_t>(b.head) * a.k_nope.stride_h) + (static_cast<int64_t>(b.kv_row) + key) * kn_b;
    };
    auto rope_at = [&](const Block& b, int key) __attribute__((always_inline)) {
        return reinterpret_cast<const uint8_t*>(a.k_rope.data) + (static_cast<int64_t>(b.kv_row) + key) * kr_b;
    };
    auto value_at = [&](const Block& b, int key) __attribute__((always_inline)) {
        return reinterpret_cast<const uint8_t*>(a.v.data + static_cast<int64_t>(b.head) * a.v.stride_h) + (static_cast<int64_t>(b.kv_row) + key) * vv_b;
    };
    const uint32_t lds0 = kc::lds_addr(smem);
    // The lane, for what is used once per block: what follows from it is not worth
    // registers across the loops.
    auto fresh_lane = [&]() __attribute__((always_inline)) {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };
    // A wave's loads of a tile: i * NW + wave counts the tile's 8-row blocks, plane by
    // plane.  Rows past the range's end re-read its last key.
    auto stage = [&](const Block& b, int key, int to) __attribute__((always_inline)) {
        const int last = b.key1 - 1 - key;
        const int l = fresh_lane();
        const uint8_t *const n = nope_at(b, key), *const r = rope_at(b, key), *const v = value_at(b, key);
#pragma unroll
        for (int i = 0; i < S::loads; ++i) {
            const int plane = i * NW / S::blocks, block = i * NW % S::blocks + wave;
            const int x = block * 8 + (l >> 3);
            const uint32_t row = static_cast<uint32_t>(min(x, last));
            const uint32_t c = static_cast<uint32_t>((l & 7) ^ (plane < 3 ? score_xor(x) : value_xor(x))) * 16;
            const uint32_t at = lds0 + to + plane * S::plane + block * 1024;
            if (plane < 2) dma16<!S::listed>(n + plane * kRow, row * kn_b + c, at);
            else if (plane == 2) dma16<!S::listed>(r, row * kr_b + c, at);
            else dma16<!S::listed>(v + (plane - 3) * kRow, row * vv_b + c, at);
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
        if (plane < 2) dma16<!S::listed>(n + plane * kRow + static_cast<uint64_t>(first * 8) * kn_b, at_n[first & 1], at);
        else if (plane == 2) dma16<!S::listed>(r + static_cast<uint64_t>(first * 8) * kr_b, at_r[first & 1], at);
        else dma16<!S::listed>(v + (plane - 3) * kRow + static_cast<uint64_t>(first * 8) * vv_b, at_v, at);
    };
    // A value that some row does not see must not reach that row through 0 * inf or
    // 0 * NaN.  A wave looks through the values that it staged itself, once they are
    // there, of the tiles that some row sees in part; `flags` says whether any wave
    // found one that is not finite (the buffer's NW words).
    auto look = [&](int key, int to) __attribute__((always_inline)) {
        if (key + KT <= sees_of(cur, 0)) return;
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
    auto meet = [&](int t, int off) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        if (t + 1 < cur.tiles) look(key_of(cur, t + 1), after(off));
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    };
    // The tile after the next, past the block's end one of the first two of the next
    // block (of `following`, if there is one).
    Block following = cur;
    bool more = false;
    auto stage_ahead = [&](int t, int off) __attribute__((always_inline)) {
        const int left = cur.tiles - t;
        if (left > 2) return stage(cur, key_of(cur, t + 2), after(after(off)));
        if constexpr (S::listed) {
            if (!more) return;
            if (following.tiles > 0 && (left == 2 || t == 0))
                stage(following, key_of(following, 0), left == 2 ? after(after(off)) : after(off));
            if (following.tiles > 1 && left == 1) stage(following, key_of(following, 1), after(after(off)));
        }
    };

    // ---- queries: operand B of step ks holds channels 16 ks + 8 half .. + 7 of the
    // lane's row of the group
    bf16x8 q[G][12];
    auto load_queries = [&](const Block& b) __attribute__((always_inline)) {
        const int l = fresh_lane(), col = l & 31, half = l >> 5;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int64_t qr = b.q_row + min(r0 + 32 * g + col, b.q_rows - 1);
            const uint16_t* const qn_p = a.q_nope.data + qr * a.q_nope.stride_t + static_cast<int64_t>(b.head) * a.q_nope.stride_h + 8 * half;
            const uint16_t* const qr_p = a.q_rope.data + qr * a.q_rope.stride_t + static_cast<int64_t>(b.head) * a.q_rope.stride_h + 8 * half;
#pragma unroll
            for (int ks = 0; ks < 12; ++ks)
                q[g][ks] = *reinterpret_cast<const bf16x8*>(ks < 8 ? qn_p + 16 * ks : qr_p + 16 * (ks - 8));
        }
    };
    // A block's first two tiles, where no block before it had tiles to stage them from.
    auto stage_first = [&](const Block& b, int off) __attribute__((always_inline)) {
        if (b.tiles > 0) stage(b, key_of(b, 0), off);
        if (b.tiles > 1) stage(b, key_of(b, 1), after(off));
    };
    // (waited for here: the wait that the compiler would put into the loop over the
    // tiles, for its first pass, would hold every pass up until the next tile is staged)
    auto settle = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int ks = 0; ks < 12; ++ks) asm volatile("" : "+a"(q[g][ks]));
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    };
    int off = 0;
    stage_first(cur, off);
    load_queries(cur);
    settle();

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
    const float c2 = a.scale_log2;
    bool careful;                           // whether the rows have to be done over
    int see_block;                          // keys that the block's first row sees

    // register i of block b is key `key + 32 b + (i & 3) + 8 (i >> 2) + 4 half`
    f32x16 s[KB][G];
    uint32_t w[G][8 * KB];                  // weights, bf16 pairs
    float block_sum[G];
    // the row's largest score of the tile's first key block, log2 units
    auto top_of = [&](int g) __attribute__((always_inline)) {
        float top = s[0][g][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[0][g][i]);
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
        for (int g = 0; g < G; ++g) here[g] = sees_of(cur, r0 + 32 * g + col) - key - 4 * half;
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
    int64_t step_n, step_r, step_v;             // from a tile's rows to the next tile's
    // A of a tile by itself, and its early weights; the wave's first tile sets the
    // references.  Ends with B's (or C's) operands on their way.
    auto begin_tile = [&](int t, int off, bool first) __attribute__((always_inline)) {
        set_tile(off);
        set_here(key_of(cur, t));
#pragma unroll
        for (int j = 0; j < kAhead; ++j) ring[j] = key_operand(kt, j);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (KB == 2) score_phase(0, keys_of(1), nothing);
        else score_phase(0, values_of(0), nothing);
#pragma unroll
        for (int g = 0; g < G; ++g) scores_ready(s[0][g]);
        if (first) {
#pragma unroll
            for (int g = 0; g < G; ++g) ref[g] = fmaxf(kUnset, top_of(g));
        }
#pragma unroll
        for (int u = 0; u < kEarly; ++u) unit(0, u, true);
    };
    // The rest of tile t after begin_tile; kNext: with the next tile's A and early
    // weights, else by itself.  kPart: some row of the wave may not see all of it (or of
    // the next); otherwise it and the next are whole, and another whole one is behind
    // them.  `careful` is set where the tile is not for this path.
    auto finish_tile = [&](int t, int off, auto with_next, auto in_part) __attribute__((always_inline)) {
        constexpr bool kNext = decltype(with_next)::value, kPart = decltype(in_part)::value;
        const int next = after(off);
        const uint32_t to = after(next);
        meet(t, off);
        if constexpr (kPart) {
            stage_ahead(t, off);
            const int key = key_of(cur, t);
            careful = careful || (key + KT > see_block && odd_values(off));
            set_here(key);
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
                    for (int g = 0; g < G; ++g) here[g] += cur.down ? KT : -KT;
                }
                value_phase(1, keys_of(1), [&](int slot) __attribute__((always_inline)) {
                    early(0, slot, kPart);
                    if (!kPart && slot == 0) {
                        next_n += step_n;
                        next_r += step_r;
                        next_v += step_v;
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

    // ---- results of the 32 rows from row x of the block on; register i of block m is
    // channel 32 m + (i & 3) + 8 (i >> 2) + 4 half, times `lowered` to the sum's weights.
    // `own`: 8 KiB of LDS for the wave.
    auto put_rows = [&](int x, f32x16 (&o)[4], float ref, float sum, float lowered, uint8_t* own) __attribute__((always_inline)) {
        const int l = fresh_lane(), col = l & 31, half = l >> 5;
        const float total = sum_halves(sum);
        // weights that all vanish leave 0 here; whether that is a row without keys is
        // decided below, by what the row sees
        const float inv = total == 0.0f ? 0.0f : 1.0f / (total * lowered);
        const int r = x + col;
        if (cur.part >= 0) {
            if (r >= min(cur.q_rows, a.part_rows)) return;
            const int64_t row = (static_cast<int64_t>(cur.part) * a.H + cur.head) * a.part_rows + r;
            float* to = a.part_o + row * kValue + 4 * half;
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<float4*>(to + 32 * m + 2 * i) = make_float4(o[m][i] * inv, o[m][i + 1] * inv, o[m][i + 2] * inv, o[m][i + 3] * inv);
            if (half == 0) {
                // a partial that weighs nothing has no reference: a row that sees no key of
                // the split may have taken its own from keys that it does not see
                a.part_m[row] = total == 0.0f ? kUnset : ref;
                a.part_l[row] = total;
            }
            return;
        }
        if (x >= cur.q_rows) return;
        // a row that sees no key is 0 (lse -inf); one whose keys all weigh nothing is not a number
        const bool none = sees_of(cur, r) <= cur.key0;
        const float scale = none || total != 0.0f ? inv : NAN;
        if (a.lse != nullptr && half == 0 && r < cur.q_rows)
            a.lse[(static_cast<int64_t>(cur.q_row) + r) * a.H + cur.head] = none ? -INFINITY : (ref + log2f(total)) * 0.6931471805599453f;
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
        // (a wave reads back only what it wrote: LDS accesses of a wave are in order; lanes
        // past the block's last row write that row once more)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int y = min(4 * i + (l >> 4), cur.q_rows - 1 - x), c = l & 15;
            const uint4 z = *reinterpret_cast<const uint4*>(own + y * 256 + ((c ^ (y & 15)) << 4));
            *reinterpret_cast<uint4*>(a.out + (static_cast<int64_t>(cur.q_row) + x + y) * a.out_stride_t +
                                      static_cast<int64_t>(cur.head) * a.out_stride_h + 8 * c) = z;
        }
    };

    while (true) {
        see_block = sees_of(cur, 0);
        // In key order: the first `whole` tiles are seen by all rows of the wave, the
        // first `some` by any.
        const int see_first = sees_of(cur, r0), r_last = min(r0 + G * kRowsPerWave, cur.q_rows) - 1;
        const int whole = max(see_first - cur.key0, 0) / KT;
        const int some = r_last < r0 ? 0 : (max(sees_of(cur, r_last) - cur.key0, 0) + KT - 1) / KT;
        const int t_begin = cur.down ? cur.tiles - some : 0, t_end = cur.down ? cur.tiles : some;
        if constexpr (S::listed) {
            more = at + 1 < end;
            if (more) following = block_of(entries[at + 1]);
        }
        careful = false;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            ref[g] = kUnset;
            sum[g] = 0.0f;
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[g][m][i] = 0.0f;
        }
        if (cur.tiles > 0) look(key_of(cur, 0), off);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
        int t = 0;
        // (tiles of which no row of the wave sees any, here and at the end)
        for (; t < t_begin && t < cur.tiles; ++t, off = after(off)) {
            meet(t, off);
            stage_ahead(t, off);
        }
        if (some > 0) {
            begin_tile(t, off, true);
            if constexpr (KB == 2) {
                // tiles that are whole, as is the next, and the one to be staged
                const int first = cur.down ? cur.tiles - whole : 0;
                const int last = cur.down ? cur.tiles - 3 : min(whole - 2, (cur.key1 - cur.key0) / KT - 3);
                while (t < first && t + 1 < t_end) {
                    finish_tile(t, off, std::true_type{}, std::true_type{});
                    ++t;
                    off = after(off);
                }
                next_n = nope_at(cur, key_of(cur, t + 2));
                next_r = rope_at(cur, key_of(cur, t + 2));
                next_v = value_at(cur, key_of(cur, t + 2));
                const int64_t step = cur.down ? -KT : KT;
                step_n = step * kn_b;
                step_r = step * kr_b;
                step_v = step * vv_b;
                while (t <= last) {
                    finish_tile(t, off, std::true_type{}, std::false_type{});
                    ++t;
                    off = after(off);
                }
                while (t + 1 < t_end) {
                    finish_tile(t, off, std::true_type{}, std::true_type{});
                    ++t;
                    off = after(off);
                }
                finish_tile(t, off, std::false_type{}, std::true_type{});
            } else {
                // (one key block: a tile begins and ends by itself)
                while (true) {
                    finish_tile(t, off, std::false_type{}, std::true_type{});
                    if (t + 1 >= t_end) break;
                    ++t;
                    off = after(off);
                    begin_tile(t, off, false);
                }
            }
            ++t;
            off = after(off);
        }
        for (; t < cur.tiles; ++t, off = after(off)) {
            meet(t, off);
            stage_ahead(t, off);
        }
        // (after the last tile's meeting, where no other wave waits for them)
        if (more) load_queries(following);
        // Whether any wave wants the rows done over.
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float total = sum_halves(sum[g]);
            const int row = r0 + 32 * g + col;
            // results that are not finite leave a sum of their products that is not
            float odd[2] = {0.0f, 0.0f};
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 16; i += 2) odd[(i >> 1) & 1] = fmaf(acc[g][m][i], acc[g][m][i + 1], odd[(i >> 1) & 1]);
            const bool stands = total < kMost && total > kLeast && fabsf(odd[0] + odd[1]) < INFINITY;
            careful = careful || __ballot(!stands && row < cur.q_rows && sees_of(cur, row) > cur.key0) != 0;
        }
        if (lane == 0) flags[S::buffers * NW + wave] = careful;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) any |= flags[S::buffers * NW + i];
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(any) == 0, 1)) {
            // in the place of the last tile, which no wave reads any more (the other two
            // are the next block's)
#pragma unroll
            for (int g = 0; g < G; ++g) put_rows(r0 + 32 * g, acc[g], ref[g], sum[g], 1.0f, smem + (S::listed ? after(after(off)) : 0) + wave * 32 * 256);
            if (more && cur.tiles == 0) stage_first(following, off);
        } else {
            // careful_rows: 32 rows of a wave at a time, a tile at a time.
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");     // (of the next block's tiles)
#pragma unroll 1
            for (int g = 0; g < G; ++g) {
                const int x = r0 + 32 * g;
                const int limit = sees_of(cur, x + col);
                const int64_t qr = cur.q_row + min(x + col, cur.q_rows - 1);
                const uint16_t* const qn_p = a.q_nope.data + qr * a.q_nope.stride_t + static_cast<int64_t>(cur.head) * a.q_nope.stride_h + 8 * half;
                const uint16_t* const qr_p = a.q_rope.data + qr * a.q_rope.stride_t + static_cast<int64_t>(cur.head) * a.q_rope.stride_h + 8 * half;
                bf16x8 qc[12];
#pragma unroll
                for (int ks = 0; ks < 12; ++ks) qc[ks] = *reinterpret_cast<const bf16x8*>(ks < 8 ? qn_p + 16 * ks : qr_p + 16 * (ks - 8));
                f32x16 o[4] = {};
                float rc = kUnset, sc = 0.0f;
#pragma unroll 1
                for (int kc0 = cur.key0; kc0 < cur.key1; kc0 += KT) {
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");       // no wave reads the tile before
                    stage(cur, kc0, 0);
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
                            pairs[i >> 1] = kc::pack_bf16x2(e0 * kLowered, e1 * kLowered);
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
                put_rows(x, o, rc, sc, kLowered, smem + S::tile + wave * 32 * 256);
            }
            if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");       // no wave reads the last tile
                off = 0;
                stage_first(following, off);
            }
        }
        if (!more) return;
        settle();
        cur = following;
        ++at;
    }
}

// Joins a block's partials: one wave per (block, head, row), two channels a lane.
__global__ __launch_bounds__(256) void prefill_merge_kernel(PrefillArgs a) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    const uint32_t w = blockIdx.x * 4 + (threadIdx.x >> 6);
    const uint32_t per_block = static_cast<uint32_t>(a.H) * a.part_rows;
    const uint32_t id = w / per_block, rest = w - id * per_block;
    if (id >= static_cast<uint32_t>(a.num_merges)) return;
    const int head = static_cast<int>(rest / a.part_rows), r = static_cast<int>(rest % a.part_rows);
    const PrefillMerge g = a.merges[id];
    if (r >= g.q_rows || g.q_row < 0 || g.q_row >= a.total_q - r) return;
    const int part0 = max(g.part0, 0), parts = min(g.num_parts, a.num_parts - part0);
    const int64_t step = static_cast<int64_t>(a.H) * a.part_rows;
    const int64_t row = part0 * step + static_cast<int64_t>(head) * a.part_rows + r;
    // The row's reference and sum first, then its partials by their share of the sum, so
    // that finite rows give a finite one (a token on 64K keys, 16 heads, 32 splits: 108 us
    // a call against 107 in one pass).  The loads of eight partials before any is used (3
    // us of that call).
    const auto load = [&](int j0, float (&m)[8], float (&l)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t at = row + min(j0 + i, parts - 1) * step;
            m[i] = a.part_m[at];
            l[i] = a.part_l[at];
        }
    };
    const auto load_rows = [&](int j0, float2 (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = *reinterpret_cast<const float2*>(a.part_o + (row + min(j0 + i, parts - 1) * step) * kValue + 2 * lane);
    };
    float top = kUnset, sum = 0.0f;
    float2 o = make_float2(0.0f, 0.0f);
    float m0[8], l0[8];
    float2 x0[8];
    if (parts > 0) {
        load(0, m0, l0);
        load_rows(0, x0);
    }
    for (int j0 = 0; j0 < parts; j0 += 8) {
        float m[8], l[8];
        if (j0 > 0) load(j0, m, l);
        const float before = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = j0 > 0 ? m[i] : m0[i];
            l[i] = j0 > 0 ? l[i] : l0[i];
            top = fmaxf(top, m[i]);
        }
        sum *= exp2f(before - top);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (j0 + i < parts) sum += exp2f(m[i] - top) * l[i];
    }
    const bool none = min(static_cast<int64_t>(g.kv_len), static_cast<int64_t>(g.seen0) + r) <= 0;
    const float inv = none ? 0.0f : 1.0f / sum;
    for (int j0 = 0; j0 < parts; j0 += 8) {
        float m[8], l[8];
        float2 x[8];
        if (j0 > 0) {
            load(j0, m, l);
            load_rows(j0, x);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (j0 + i >= parts) break;
            const float share = exp2f((j0 > 0 ? m[i] : m0[i]) - top) * (j0 > 0 ? l[i] : l0[i]) * inv;
            o.x = fmaf(share, j0 > 0 ? x[i].x : x0[i].x, o.x);
            o.y = fmaf(share, j0 > 0 ? x[i].y : x0[i].y, o.y);
        }
    }
    const int64_t q = static_cast<int64_t>(g.q_row) + r;
    *reinterpret_cast<uint32_t*>(a.out + q * a.out_stride_t + static_cast<int64_t>(head) * a.out_stride_h + 2 * lane) =
        kc::pack_bf16x2(o.x, o.y);
    if (a.lse != nullptr && lane == 0)
        a.lse[q * a.H + head] = none ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace

hipError_t launch_prefill(const PrefillArgs& a, hipStream_t stream) {
    const PrefillLists l = prefill_lists(a.num_items, a.H, a.rows);
    const dim3 grid(l.lists > 0 ? static_cast<unsigned>(l.lists) * (a.H % 8 == 0 ? 8u : 1u)
                                : static_cast<unsigned>(a.num_items) * static_cast<unsigned>(a.H));
    if (a.rows == 128)
        hipLaunchKernelGGL((prefill_kernel<4, 1, 32>), grid, dim3(256), 0, stream, a);
    else if (a.rows == 256)
        hipLaunchKernelGGL((prefill_kernel<4, 2, 64>), grid, dim3(256), 0, stream, a);
    else
        return hipErrorInvalidValue;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.num_merges == 0) return e;
    const int64_t waves = static_cast<int64_t>(a.num_merges) * a.H * a.part_rows;
    hipLaunchKernelGGL(prefill_merge_kernel, dim3(static_cast<unsigned>((waves + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace mla
