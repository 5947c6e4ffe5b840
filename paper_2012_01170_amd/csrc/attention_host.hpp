// Host side of the linear attention's entry points: checks and the split of the
// token axis.
#pragma once

#include <initializer_list>

#include "attention.hpp"

namespace sbc {

inline sbc_status check_attention(const sbc_attention *a) {
    if (!a) return fail(SBC_ERR_INVALID_ARG, "attention is null");
    if (a->n < 0 || a->n_batch < 0) return fail(SBC_ERR_INVALID_ARG, "n and n_batch must be >= 0");
    if (a->heads <= 0 || a->dk <= 0 || a->dv <= 0)
        return fail(SBC_ERR_INVALID_ARG, "heads, dk and dv must be > 0");
    if (!known_dtype(a->dtype)) return fail(SBC_ERR_INVALID_ARG, "unknown dtype");
    if (a->dk > 128 || a->dv > 128)
        return fail(SBC_ERR_UNSUPPORTED, "dk and dv must be <= 128");
    if (a->heads > 65535) return fail(SBC_ERR_UNSUPPORTED, "heads must be <= 65535");
    if (a->n > 0 && !a->rates) return fail(SBC_ERR_INVALID_ARG, "rates is null");
    return SBC_OK;
}

// Sequences of a whole-sequence call.
inline sbc_status check_sequences(const sbc_attention *a) {
    SBC_TRY(check_attention(a));
    if (!a->splits && a->n_batch != 1)
        return fail(SBC_ERR_INVALID_ARG, "without splits there is one sequence (n_batch 1)");
    if (a->n > 0 && a->n_batch == 0)
        return fail(SBC_ERR_INVALID_ARG, "tokens without a sequence (n_batch 0)");
    return SBC_OK;
}

inline int attn_tile(int32_t dc) { return dc <= 32 ? 32 : 64; }
inline int32_t attn_tiles(int32_t dc) { return (dc + attn_tile(dc) - 1) / attn_tile(dc); }

// Whether rows are read in whole 16-byte pieces at 32-bit offsets within a chunk.
inline bool whole_rows(const sbc_attention *a, std::initializer_list<const sbc_heads *> arrays) {
    const int v = a->dtype == SBC_F32 ? 4 : 8;
    if (a->dk % v || a->dv % v) return false;
    for (const sbc_heads *x : arrays)
        if (x->token_stride >= 1 << 22) return false;
    return true;
}

// Segments of the token axis: as many as give every CU `per_cu` workgroups, of no
// fewer than kLeastSeg tokens.
// (Gradients in bf16, 11003 tokens of 3 heads of 64 channels: 74 us at 64, 51 at 128, 55 at
// 256.  The wider the state, the rather 256: 16384 tokens of 2 heads of 128: 132, 132, 124.)
constexpr int32_t kLeastSeg = 128;
inline void attn_segments(int32_t n, int64_t blocks_a_segment, int per_cu, int32_t *seg_len,
                          int32_t *n_seg) {
    const int64_t want = ((int64_t)per_cu * device_cus() + blocks_a_segment - 1) / blocks_a_segment;
    int64_t len = ((int64_t)n + want - 1) / want;
    if (len < kLeastSeg) len = kLeastSeg;
    len = (len + kChunk - 1) / kChunk * kChunk;
    const int64_t segs = ((int64_t)n + len - 1) / len;
    *seg_len = (int32_t)(len > INT32_MAX ? INT32_MAX : len);
    *n_seg = (int32_t)(segs < 1 ? 1 : segs);
}

inline int64_t state_stride(int32_t dk, int32_t dv) { return ((int64_t)dk * dv + 3) / 4 * 4; }

}  // namespace sbc
