/*
 * mla_prefill.h -- C ABI of the prompt side of the low-bit MLA library for
 * AMD MI355X (gfx950): what runs before and beside the decode calls of
 * mla_lowbit.h.
 *
 *   - writers that normalize the content latent and rotate the RoPE key on the
 *     way into the paged cache, and hand the same values on as dense rows;
 *   - readers that turn cached tokens back into dense bf16 rows;
 *   - the rotation of the queries' RoPE channels;
 *   - attention in its expanded form (Sec. 2.1: per-head keys and values
 *     expanded from the latents by the caller's products), for prompts,
 *     prompt chunks over a cached prefix, and single tokens.
 *
 * The conventions of mla_lowbit.h hold for every entry point: device buffers
 * of the current HIP device, owned by the caller; bf16 as uint16_t; work
 * enqueued on `stream`, no call synchronizes or allocates; arguments checked
 * on the host before any HIP call; its return codes.  A launch that would not
 * fit one dispatch is refused with MLA_ENOTSUP.  Device-resident values
 * (positions, slots, page ids, lengths, plans) are preconditions; the kernels
 * clamp every index that comes from them into its buffer.
 */
#ifndef MLA_PREFILL_H
#define MLA_PREFILL_H

#include "mla_lowbit.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Position rotation of the d_r = 64 RoPE channels.  `table` (device, fp32
 * [num_positions][64], 16-byte aligned) holds for every position the cosines
 * of the 32 pair angles, then their sines, with whatever frequency scaling the
 * model uses.  Pair i of a row x is
 *   MLA_ROPE_PAIRS   channels (2i, 2i+1), the cache's own convention
 *   MLA_ROPE_HALVES  channels (i, i+32)
 * and becomes (x cos - y sin, x sin + y cos), computed in fp64 from the bf16
 * channels and the fp32 table, rounded to fp32 and then to bf16.
 * Positions (device, int32) must lie in [0, num_positions).
 */
enum { MLA_ROPE_PAIRS = 0, MLA_ROPE_HALVES = 1 };
typedef struct mla_rotation {
    const float* table;
    int64_t num_positions;
    int32_t layout;
} mla_rotation;

/*
 * RMS norm of the d_c = 512 content channels (Sec. 3.3: weightless in the
 * fused coordinates, Appendix C; a weight is for latents that are not fused):
 *   y = x w / sqrt(mean(x^2) + eps)
 * in fp64, rounded to fp32 and then to bf16.  The values that are quantized,
 * protected or stored are these bf16 values, so neither codes nor rows depend
 * on an order of summation.
 *   weight  device, bf16 [512], 16-byte aligned, or NULL (all ones)
 *   eps     finite and > 0
 */
typedef struct mla_rms_norm {
    const uint16_t* weight;
    float eps;
} mla_rms_norm;

/*
 * Append with norm and rotation: exactly mla_lowbit_quant_append (or
 * mla_bf16_append, mla_lowbit_quant_append_protected) of the normalized
 * latents and rotated keys, in one pass.
 *   norm       NULL: c_kv holds normalized latents already
 *   rot        the rotation (not NULL)
 *   c_kv, k_rope, strides, slot_mapping, n, cache, num_pages: as there;
 *              k_rope is the key before its rotation
 *   positions  device, int32 [n]: position of each token (a skipped token's
 *              may be anything); the protected writer also places the token by
 *              it in its sequence
 *   c_out      device, bf16 [n][c_out_stride]: the normalized latents, or NULL
 *   k_out      device, bf16 [n][k_out_stride]: the rotated keys, or NULL
 * The dense rows are written for all n tokens, skipped ones too (16-byte
 * aligned, strides multiples of 8, at least 512 and 64).  c_out may be c_kv and
 * k_out may be k_rope, with the same stride; other overlaps are not allowed.
 * n = 0 is a no-op.
 */
int mla_lowbit_norm_rope_append(const mla_cache_format* f, const mla_rms_norm* norm, const mla_rotation* rot,
                                const uint16_t* c_kv, int64_t c_kv_stride,
                                const uint16_t* k_rope, int64_t k_rope_stride,
                                const int32_t* positions, const int64_t* slot_mapping, int32_t n,
                                void* cache, int64_t num_pages,
                                uint16_t* c_out, int64_t c_out_stride,
                                uint16_t* k_out, int64_t k_out_stride, hipStream_t stream);
int mla_bf16_norm_rope_append(const mla_cache_format* f, const mla_rms_norm* norm, const mla_rotation* rot,
                              const uint16_t* c_kv, int64_t c_kv_stride,
                              const uint16_t* k_rope, int64_t k_rope_stride,
                              const int32_t* positions, const int64_t* slot_mapping, int32_t n,
                              void* cache, int64_t num_pages,
                              uint16_t* c_out, int64_t c_out_stride,
                              uint16_t* k_out, int64_t k_out_stride, hipStream_t stream);
int mla_lowbit_norm_rope_append_protected(const mla_cache_format* f, const mla_protect_policy* p,
                                          const mla_rms_norm* norm, const mla_rotation* rot,
                                          const uint16_t* c_kv, int64_t c_kv_stride,
                                          const uint16_t* k_rope, int64_t k_rope_stride,
                                          const int32_t* positions, const int64_t* slot_mapping, int32_t n,
                                          void* cache, int64_t num_pages,
                                          const int32_t* token_seq, const int32_t* seq_lens,
                                          const int32_t* prot_slot, int32_t B, void* prot, int64_t num_prot,
                                          uint16_t* c_out, int64_t c_out_stride,
                                          uint16_t* k_out, int64_t k_out_stride, hipStream_t stream);

/*
 * Rotate the RoPE channels of n x H query rows:
 *   q    device, bf16, row (t, h) at q + t * q_stride_t + h * q_stride_h, 64 channels
 *   out  the same shape with its own strides; may be q with the same strides
 *        (other overlaps are not allowed)
 *   positions  device, int32 [n]: token t's position, for all its heads
 * Rows are 16-byte aligned (pointers, and strides multiples of 8; strides may
 * not be negative, and the output's rows may not overlap).  n = 0 is a no-op.
 */
int mla_rope_queries(const mla_rotation* rot, const uint16_t* q, int64_t q_stride_t, int64_t q_stride_h,
                     const int32_t* positions, int32_t n, int32_t H,
                     uint16_t* out, int64_t out_stride_t, int64_t out_stride_h, hipStream_t stream);

/*
 * Read cached tokens back as dense rows (the latents and RoPE keys that a
 * prompt chunk's expansion takes of its prefix): output row r with
 * cu_rows[b] <= r < cu_rows[b+1] is the token of sequence b at position
 * first[b] + r - cu_rows[b].
 *   block_table  device, int32 [B][max_pages_per_seq], as for the decode
 *   first        device, int32 [B]: first position of each range, or NULL: 0
 *   cu_rows      device, int32 [B+1], ascending from 0; rows from cu_rows[B] on
 *                are left as they are
 *   n            rows of the output (host; cu_rows[B] <= n)
 *   c_out, k_out device, bf16 [n][stride], 512 and 64 channels (16-byte
 *                aligned, strides multiples of 8)
 * Low-bit caches give bf16(scale * (q - zero)), the product rounded to fp32
 * first; BF16 caches their rows bit for bit.  The protected reader takes the
 * positions of P_L (L = seq_lens[b], device int32 [B]) from the sequence's
 * protection buffer bit for bit, as the protected decode does.  n = 0 and
 * B = 0 are no-ops.
 */
int mla_lowbit_gather(const mla_cache_format* f, const void* cache, int64_t num_pages,
                      const int32_t* block_table, int32_t max_pages_per_seq,
                      const int32_t* first, const int32_t* cu_rows, int32_t B, int32_t n,
                      uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out, int64_t k_out_stride,
                      hipStream_t stream);
int mla_bf16_gather(const mla_cache_format* f, const void* cache, int64_t num_pages,
                    const int32_t* block_table, int32_t max_pages_per_seq,
                    const int32_t* first, const int32_t* cu_rows, int32_t B, int32_t n,
                    uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out, int64_t k_out_stride,
                    hipStream_t stream);
int mla_lowbit_gather_protected(const mla_cache_format* f, const mla_protect_policy* p,
                                const void* cache, int64_t num_pages,
                                const int32_t* block_table, int32_t max_pages_per_seq,
                                const int32_t* first, const int32_t* cu_rows, int32_t B, int32_t n,
                                const int32_t* seq_lens, const void* prot, int64_t num_prot,
                                const int32_t* prot_slot,
                                uint16_t* c_out, int64_t c_out_stride, uint16_t* k_out, int64_t k_out_stride,
                                hipStream_t stream);

/*
 * Expanded attention.  For query row i of sequence b (i < q_lens[b]), head h
 * and the keys j < kv_lens[b] of the sequence:
 *   z_j = softmax_scale (q_nope[i,h,:] . k_nope[j,h,:] + q_rope[i,h,:] . k_rope[j,:])
 *   out[i,h,:] = sum_j softmax(z)_j v[j,h,:],   lse[i,h] = ln sum_j e^{z_j}
 * with 128 "nope" channels, 64 RoPE channels shared by all heads, 128 value
 * channels.  Causal: row i sees j <= kv_lens[b] - q_lens[b] + i (the ends are
 * aligned, so a chunk's rows see the whole prefix).  A row that sees no key
 * gives out = 0 and lse = -inf.  Keys that a row does not see have no part in
 * it, whatever they hold (NaN and infinities included).
 *
 * The plan is made on the host from the lengths and copied to the device by
 * the caller; it serves every layer and every call with these lengths and H.
 *   q_lens, kv_lens    host, int32 [B], each >= 0
 *   q_starts, kv_starts host, int32 [B] or NULL: first row of each sequence in
 *                      the query / key tensors (NULL: one after the other).
 *                      Query ranges may not overlap; key ranges may.
 *   plan               host, int32 [plan_ints], or NULL: only *info is filled
 *   info               host: what the call needs to know (plain sizes; callers
 *                      read plan_ints, workspace_bytes, total_q, total_kv)
 * Returns MLA_OK, MLA_EINVAL (lengths, overlap, plan_capacity < plan_ints) or
 * MLA_ENOTSUP.
 */
typedef struct mla_prefill_plan {
    int64_t plan_ints;          /* int32 values of the plan                     */
    int64_t workspace_bytes;    /* device workspace of a call (0: none)         */
    int64_t total_q, total_kv;  /* rows the query / key tensors must have       */
    int32_t B, H, causal;
    int32_t rows;               /* query rows of a workgroup                    */
    int32_t num_items;          /* work items per head                          */
    int32_t num_merges;         /* row blocks whose keys are split              */
    int32_t num_parts;          /* partial row blocks per head                  */
    int32_t part_rows;          /* rows of a partial block                      */
} mla_prefill_plan;
int mla_plan_prefill(const int32_t* q_lens, const int32_t* kv_lens, const int32_t* q_starts,
                     const int32_t* kv_starts, int32_t B, int32_t H, int32_t causal,
                     int32_t* plan, int64_t plan_capacity, mla_prefill_plan* info);

/* A bf16 tensor of rows (t, h) at data + t * stride_t + h * stride_h (device,
 * 16-byte aligned; strides multiples of 8, not negative, below 2^24). */
typedef struct mla_head_rows {
    const uint16_t* data;
    int64_t stride_t, stride_h;
} mla_head_rows;

/*
 * The call, on a plan's device copy.  k_rope is one row of 64 channels per key
 * (its stride_h is not read).  out rows may not overlap; rows that belong to no
 * sequence are left as they are.
 *   info       host: as filled by mla_plan_prefill
 *   plan       device, int32 [info->plan_ints], 16-byte aligned
 *   out        device, bf16 rows (t, h), strides as for the inputs
 *   lse        device, fp32 [total_q][H], or NULL
 *   workspace  device, 256-byte aligned, workspace_bytes (at least
 *              info->workspace_bytes); calls that may overlap need one each
 * Products run in bf16 with fp32 accumulation, the softmax in fp32, its
 * weights rounded to bf16 for the second product; the output is rounded once.
 * Finite inputs whose scores are finite and whose values are at most 2^126 in size
 * give finite outputs; weights under 2^-66 of a row's sum, and products of weight
 * and value under 2^-66, may be taken as 0.  A row that sees a value that is not
 * finite is not finite in that channel (NaN in an infinity's place, where its
 * weight is taken as 0).
 * Two calls on the same plan and inputs give the same bits.
 */
int mla_prefill_attn(const mla_prefill_plan* info, const int32_t* plan,
                     const mla_head_rows* q_nope, const mla_head_rows* q_rope,
                     const mla_head_rows* k_nope, const mla_head_rows* k_rope, const mla_head_rows* v,
                     float softmax_scale, uint16_t* out, int64_t out_stride_t, int64_t out_stride_h, float* lse,
                     void* workspace, int64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MLA_PREFILL_H */
