// Host side of softmax attention's entry points: checks, and how rows and keys are divided.
#pragma once

#include <cmath>

#include "softmax.hpp"

namespace sbc {

inline sbc_status check_softmax(const sbc_softmax_attention *a) {
    if (!a) return fail(SBC_ERR_INVALID_ARG, "attention is null");
    if (a->n < 0 || a->m < 0 || a->n_batch < 0)
        return fail(SBC_ERR_INVALID_ARG, "n, m and n_batch must be >= 0");
    if (a->heads <= 0 || a->kv_heads <= 0 || a->dk <= 0 || a->dv <= 0)
        return fail(SBC_ERR_INVALID_ARG, "heads, kv_heads, dk and dv must be > 0");
    if (a->heads % a->kv_heads)
        return fail(SBC_ERR_INVALID_ARG, "heads must be a multiple of kv_heads");
    if (!known_dtype(a->dtype)) return fail(SBC_ERR_INVALID_ARG, "unknown dtype");
    if (!(a->scale > 0.f) || !(a->scale < 2e38f))  // (times log2 e it is finite)
        return fail(SBC_ERR_INVALID_ARG, "scale must be > 0 and below 2e38");
    if (a->dk > 128 || a->dv > 128)
        return fail(SBC_ERR_UNSUPPORTED, "dk and dv must be <= 128");
    if (a->heads > 65535) return fail(SBC_ERR_UNSUPPORTED, "heads must be <= 65535");
    if ((int64_t)a->n * a->heads > kMostRows || (int64_t)a->m * a->kv_heads > kMostRows)
        return fail(SBC_ERR_UNSUPPORTED, "n * heads and m * kv_heads must be <= 2^31 - 1024");
    return SBC_OK;
}
// Sequences of keys that lie in one array
inline sbc_status check_softmax_sequences(const sbc_softmax_attention *a) {
    SBC_TRY(check_softmax(a));
    if (!a->splits && a->n_batch != 1)
        return fail(SBC_ERR_INVALID_ARG, "without splits there is one sequence (n_batch 1)");
    if (a->n > 0 && a->n_batch == 0)
        return fail(SBC_ERR_INVALID_ARG, "tokens without a sequence (n_batch 0)");
    if (!a->k_splits && a->splits && a->m != a->n)
        return fail(SBC_ERR_INVALID_ARG, "without k_splits there are as many keys as queries");
    return SBC_OK;
}

inline int64_t softmax_places(const sbc_softmax_attention *a, int32_t rows) {
    return (int64_t)a->n * (a->heads / a->kv_heads) / rows + a->n_batch;
}

// Whole 16-byte pieces of rows, at 32-bit offsets within a tile
inline bool softmax_whole(const sbc_softmax_attention *a,
                          std::initializer_list<const sbc_heads *> arrays) {
    const int v = a->dtype == SBC_F32 ? 4 : 8;
    if (a->dk % v || a->dv % v) return false;
    for (const sbc_heads *x : arrays)
        if (x->token_stride >= 1 << 22) return false;
    return true;
}

// Rows that DirectTile can load: these loads are taken at addresses of whole pieces alone
inline bool softmax_direct(const sbc_softmax_attention *a,
                           std::initializer_list<const sbc_heads *> arrays) {
    if (a->dtype != SBC_BF16 || a->dk != a->dv) return false;
    for (const sbc_heads *x : arrays)
        if ((uintptr_t)x->data % 16 || x->token_stride % 8 || x->head_stride % 8) return false;
    return true;
}

// The kernels' arguments that every call has
inline SoftmaxArgs softmax_args(const sbc_softmax_attention *a) {
    SoftmaxArgs p{};
    p.n = a->n;
    p.m = a->m;
    p.n_batch = a->n_batch;
    p.heads = a->heads;
    p.kv_heads = a->kv_heads;
    p.dk = a->dk;
    p.dv = a->dv;
    p.causal = a->causal != 0;
    p.group = divisor(a->heads / a->kv_heads);
    p.scale = a->scale;
    p.scale2 = (float)((double)a->scale * 1.4426950408889634);
    p.splits = a->splits;
    p.k_splits = a->k_splits ? a->k_splits : a->splits;
    p.parts = 1;
    return p;
}

// The forward pass takes rows 128 to a workgroup, or few rows 32 to one, whose waves share
// their keys out.  Either has the keys in parts where there are not workgroups enough for every CU
// (12 chunks of some 300 tokens over 5000 kept, 4 heads of 64 bf16 channels: 150 us of 128 rows
// in one part, 68 of 32 rows, 57 of 128 rows in 4 parts).  Few are 64 rows a sequence on average, which
// a workgroup of 128 would leave half empty, and problems too small for it to fill the CUs even in
// parts; there a second launch pays past 512 keys (256 points, float32: 11 us in one part, 15 in two).
// The lengths of packed sequences lie on the GPU, so that their plan takes all keys as one
// sequence's: a batch of many short ones may get parts that are empty, and a join.
struct SoftmaxPlan {
    bool few;
    int32_t parts;
    int64_t blocks;
};
// most_keys: that one sequence can have
inline SoftmaxPlan softmax_plan(const sbc_softmax_attention *a, int64_t most_keys) {
    const int64_t rows = (int64_t)a->n * (a->heads / a->kv_heads);
    const int cus = device_cus();
    auto plan = [&](bool few, int64_t blocks_a_cu, int64_t least_keys) {
        const int64_t tiles = softmax_places(a, few ? 32 : 128) * a->kv_heads;
        int64_t parts = tiles > 0 ? blocks_a_cu * cus / tiles : 1;
        const int64_t most = (most_keys + least_keys - 1) / least_keys;
        if (parts > most) parts = most;
        if (parts > 64) parts = 64;
        if (parts < 1) parts = 1;
        return SoftmaxPlan{few, (int32_t)parts, tiles * parts};
    };
    const SoftmaxPlan many = plan(false, 3, 256);
    SoftmaxPlan s = many;
    if (rows <= (int64_t)64 * a->n_batch || many.blocks < cus) s = plan(true, 4, most_keys > 512 ? 128 : 512);
    // (a workgroup of the join for each row)
    if (s.parts > 1 && (int64_t)a->n * a->heads >= (int64_t)1 << 24) {
        s.blocks /= s.parts;
        s.parts = 1;
    }
    return s;
}
inline size_t softmax_workspace(const sbc_softmax_attention *a, const SoftmaxPlan &s) {
    if (s.parts <= 1) return 0;
    Carver c(nullptr);
    c.take<float>((size_t)s.parts * a->n * a->heads * a->dv);
    c.take<float>((size_t)s.parts * a->n * a->heads);
    return c.used;
}

}  // namespace sbc
