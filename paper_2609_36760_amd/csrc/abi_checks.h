// Host-side argument checks and page geometry, shared by the translation units
// of the C ABI (mla_abi.cpp, mla_prefill_abi.cpp).  Not part of the public C ABI.
#pragma once

#include "mla_lowbit.h"

#include <cstdint>

#include "internal.h"

namespace mla {
namespace abi {

constexpr int32_t kDc = 512;
constexpr int32_t kDr = 64;
constexpr int32_t kGroup = 64;
constexpr int32_t kTile = 32;

constexpr int32_t kMaxPageSize = 1 << 20;
constexpr int32_t kMaxProtRows = 65536;
constexpr int32_t kPaperMetaBytes = 32;
constexpr int64_t kReverseMapBytes = 8;     // per physical page, eq. physical_cache_storage
constexpr int64_t kProtRowBytes = (kDc + kDr) * 2;

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }

inline int check_policy(const mla_protect_policy* p) {
    if (p == nullptr) return MLA_EINVAL;
    if (p->sink < 0 || p->recent < 0) return MLA_EINVAL;
    const int64_t rows = static_cast<int64_t>(p->sink) + p->recent;
    if (rows < 1 || rows > kMaxProtRows) return MLA_EINVAL;
    return MLA_OK;
}

// Structural checks shared by both cache kinds.
inline int check_shape(const mla_cache_format* f) {
    if (f == nullptr) return MLA_EINVAL;
    if (f->d_c <= 0 || f->d_r <= 0 || f->page_size <= 0) return MLA_EINVAL;
    if (f->page_size % 16 != 0) return MLA_EINVAL;
    if (f->d_c != kDc || f->d_r != kDr) return MLA_ENOTSUP;
    if (f->page_size % kTile != 0) return MLA_ENOTSUP;
    if (f->page_size > kMaxPageSize) return MLA_ENOTSUP;      // a page's bytes fit 31 bits
    return MLA_OK;
}

inline int check_lowbit_format(const mla_cache_format* f) {
    const int st = check_shape(f);
    if (st != MLA_OK) return st;
    if (f->group <= 0 || f->d_c % f->group != 0 || f->d_r % f->group != 0) return MLA_EINVAL;
    if (f->c_bits != 4 && f->c_bits != 2) return MLA_EINVAL;
    if (f->r_bits != 4) return MLA_EINVAL;
    if (f->meta != MLA_META_FP16 && f->meta != MLA_META_PAPER) return MLA_EINVAL;
    if (f->group != kGroup) return MLA_ENOTSUP;
    return MLA_OK;
}

// page_size >= 32, so the quotient fits 32 bits
inline uint32_t page_magic(int32_t page_size) {
    return static_cast<uint32_t>((uint64_t{1} << 32) / static_cast<uint32_t>(page_size));
}

inline mla::PageGeom lowbit_geom(const mla_cache_format* f) {
    mla::PageGeom g{};
    const int32_t P = f->page_size;
    g.page_size = P;
    g.page_magic = page_magic(P);
    g.c_bits = f->c_bits;
    g.cc_bytes = f->d_c * f->c_bits / 8;
    g.cr_bytes = f->d_r * f->r_bits / 8;
    g.off_cr = P * g.cc_bytes;
    g.off_mc = g.off_cr + P * g.cr_bytes;
    int64_t end;
    if (f->meta == MLA_META_PAPER) {
        // one 32-byte record per token: bf16 scales, byte zeros, fp32 RoPE scale, byte RoPE zero
        g.paper_meta = 1;
        g.off_mr = g.off_mc;
        end = g.off_mc + static_cast<int64_t>(P) * kPaperMetaBytes;
    } else {
        g.off_mr = g.off_mc + P * (f->d_c / f->group) * 4;
        end = g.off_mr + static_cast<int64_t>(P) * (f->d_r / f->group) * 4;
    }
    g.page_bytes = (end + 255) / 256 * 256;
    return g;
}

inline mla::PageGeom bf16_geom(const mla_cache_format* f) {
    mla::PageGeom g{};
    g.page_size = f->page_size;
    g.page_magic = page_magic(f->page_size);
    g.page_bytes = static_cast<int64_t>(f->page_size) * (f->d_c + f->d_r) * 2;
    return g;
}

inline int check_append(const uint16_t* c_kv, int64_t c_kv_stride, const uint16_t* k_rope, int64_t k_rope_stride,
                        const int64_t* slot_mapping, int32_t n, const void* cache, int64_t num_pages) {
    if (n < 0 || num_pages < 0) return MLA_EINVAL;
    if (n == 0) return MLA_OK;
    if (n > mla::kMaxAppendTokens) return MLA_ENOTSUP;   // the launch would not fit one dispatch
    if (c_kv == nullptr || k_rope == nullptr || slot_mapping == nullptr || cache == nullptr) return MLA_EINVAL;
    if (num_pages == 0) return MLA_EINVAL;
    if (c_kv_stride < kDc || k_rope_stride < kDr) return MLA_EINVAL;
    if (!aligned(cache, 256)) return MLA_EINVAL;
    // 16-byte vector loads of 8 channels
    if (c_kv_stride % 8 != 0 || k_rope_stride % 8 != 0 || !aligned(c_kv, 16) || !aligned(k_rope, 16))
        return MLA_ENOTSUP;
    return MLA_OK;
}

// MLA_OK, or MLA_EHIP with the error kept for mla_last_hip_error (mla_abi.cpp).
int hip_status(hipError_t e);

}  // namespace abi
}  // namespace mla
