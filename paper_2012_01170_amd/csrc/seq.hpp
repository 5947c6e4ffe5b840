// What the sequence operators (layer norm, rotary positions, linear attention)
// share: element types, vectors of 16 bytes, sums over groups of lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>
#include <initializer_list>

#include "common.hpp"

namespace sbc {

// Element types: float, and bf16 as its bits.
typedef uint16_t bf16_t;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return __uint_as_float((uint32_t)x << 16); }

// float32 -> element, to nearest even (outputs are rounded here, once)
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float x) {
    return __builtin_bit_cast(bf16_t, (__bf16)x);
}

template <typename T> constexpr int kVec = 16 / sizeof(T);  // elements of 16 bytes

typedef uint32_t raw16 __attribute__((ext_vector_type(4)));  // 16 bytes as they lie

// kVec<T> elements at p, of which the first `have` exist (the others read as 0 and
// are not touched).  p needs an element's alignment only: global memory takes
// 16-byte accesses at any address, and one that is not aligned costs a second cache
// line at most, less than accesses by elements.
template <typename T> __device__ __forceinline__ raw16 load_raw16(const T *p, int have) {
    raw16 r;
    if (have >= kVec<T>) {
        __builtin_memcpy(&r, p, 16);
    } else {
        T e[kVec<T>];
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) e[i] = i < have ? p[i] : T(0);
        __builtin_memcpy(&r, e, 16);
    }
    return r;
}
template <typename T> __device__ __forceinline__ void unpack(const raw16 &r, float (&out)[kVec<T>]) {
    T e[kVec<T>];
    __builtin_memcpy(e, &r, 16);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) out[i] = to_f32(e[i]);
}
// the same as float32
template <typename T>
__device__ __forceinline__ void load_vec(const T *p, int have, float (&out)[kVec<T>]) {
    unpack<T>(load_raw16<T>(p, have), out);
}

template <typename T>
__device__ __forceinline__ void store_vec(T *p, int have, const float (&in)[kVec<T>]) {
    T raw[kVec<T>];
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) raw[i] = from_f32<T>(in[i]);
    if (have >= kVec<T>) {
        __builtin_memcpy(p, raw, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i)
            if (i < have) p[i] = raw[i];
    }
}

template <int N>
__device__ __forceinline__ void load_f32(const float *p, int have, float (&out)[N]) {
    if (have >= N) {
        __builtin_memcpy(out, p, N * 4);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = i < have ? p[i] : 0.f;
    }
}

// Sum over groups of G consecutive lanes (G a power of two up to 64), in every
// lane.  Up to 16 lanes by moves within the vector ALU.
template <int G> __device__ __forceinline__ float group_sum(float x) {
#define SBC_STEP(ctrl) \
    x += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), ctrl, 0xf, 0xf, true))
    if constexpr (G > 1) SBC_STEP(0xB1);    // quad_perm [1, 0, 3, 2]
    if constexpr (G > 2) SBC_STEP(0x4E);    // quad_perm [2, 3, 0, 1]
    if constexpr (G > 4) SBC_STEP(0x141);   // row_half_mirror
    if constexpr (G > 8) SBC_STEP(0x140);   // row_mirror
#undef SBC_STEP
    if constexpr (G > 16) x += __shfl_xor(x, 16);
    if constexpr (G > 32) x += __shfl_xor(x, 32);
    return x;
}

inline bool known_dtype(sbc_dtype d) { return d == SBC_F32 || d == SBC_BF16; }
inline size_t dtype_bytes(sbc_dtype d) { return d == SBC_F32 ? 4 : 2; }

// ---------------------------------------------------------------- overlaps
// Where an argument lies: `blocks` blocks of `span` bytes, `stride` bytes apart.
struct Region {
    const void *data;
    int64_t span, stride, blocks;
    int64_t extent() const { return data && blocks > 0 ? stride * (blocks - 1) + span : 0; }
};
inline Region region(const void *data, int64_t count, int64_t element) {
    return {data, count * element, 0, 1};
}
inline Region region_rows(const void *data, int64_t n, int64_t width, int64_t stride, sbc_dtype dt) {
    const int64_t e = (int64_t)dtype_bytes(dt);
    return {data, width * e, stride * e, n};
}
inline Region region_heads(const sbc_heads *x, int64_t heads, int64_t n, int64_t d, sbc_dtype dt) {
    if (!x || heads <= 0 || n <= 0) return {nullptr, 0, 0, 0};
    const int64_t e = (int64_t)dtype_bytes(dt), ts = x->token_stride * e, hs = x->head_stride * e;
    if (heads == 1 || (n > 1 && ts >= hs))
        return {x->data, (heads - 1) * hs + d * e, ts, ts == 0 ? 1 : n};
    return {x->data, (n - 1) * ts + d * e, hs, heads};
}

// Whether two of them share memory.  Rows of the same stride may lie in each other's gaps
// (parts of one projection), and so may a block in those of rows.
inline bool meet(const Region &a, const Region &b) {
    const int64_t na = a.extent(), nb = b.extent();
    const int64_t off = (int64_t)((uintptr_t)b.data - (uintptr_t)a.data);
    if (na <= 0 || nb <= 0 || off >= na || -off >= nb) return false;
    if (a.blocks == 1 && b.blocks > 1) return meet(b, a);
    if (a.blocks == 1 || a.stride < a.span) return true;
    if (b.blocks > 1 ? a.stride != b.stride : off < 0) return true;
    const int64_t at = ((off % a.stride) + a.stride) % a.stride;
    return !(at >= a.span && at + b.span <= a.stride);
}

// Outputs share memory with no input and with no other output.
inline sbc_status check_apart(std::initializer_list<Region> outputs,
                              std::initializer_list<Region> inputs) {
    for (const Region *o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Region &i : inputs)
            if (meet(*o, i)) return fail(SBC_ERR_INVALID_ARG, "an output overlaps an input");
        for (const Region *p = outputs.begin(); p != o; ++p)
            if (meet(*o, *p)) return fail(SBC_ERR_INVALID_ARG, "two outputs overlap");
    }
    return SBC_OK;
}

// ---------------------------------------------------------------- sbc_heads
// An input: any strides that do not go backwards (0: the same for all).
inline sbc_status check_heads(const sbc_heads *x, int32_t heads, int32_t n, int32_t d,
                              sbc_dtype dt, const char *name) {
    if (heads == 0 || n == 0) return SBC_OK;
    if (!x || !x->data) return fail(SBC_ERR_INVALID_ARG, std::string(name) + " is null");
    if (x->token_stride < 0 || x->head_stride < 0)
        return fail(SBC_ERR_INVALID_ARG, std::string(name) + " has a negative stride");
    if (((uintptr_t)x->data) % dtype_bytes(dt))
        return fail(SBC_ERR_INVALID_ARG, std::string(name) + " is not aligned to its elements");
    return SBC_OK;
}

// An output: besides, no two of its elements in one place.
inline sbc_status check_out_heads(const sbc_heads *x, int32_t heads, int32_t n, int32_t d,
                                  sbc_dtype dt, const char *name) {
    SBC_TRY(check_heads(x, heads, n, d, dt, name));
    if (heads == 0 || n == 0) return SBC_OK;
    const int64_t ts = x->token_stride, hs = x->head_stride;
    const bool tokens_outside = (heads == 1 || hs >= d) && (n == 1 || ts >= (heads - 1) * hs + d);
    const bool heads_outside = (n == 1 || ts >= d) && (heads == 1 || hs >= (n - 1) * ts + d);
    if (!tokens_outside && !heads_outside)
        return fail(SBC_ERR_INVALID_ARG, std::string(name) + "'s elements overlap");
    return SBC_OK;
}

}  // namespace sbc
