// Linear attention with decays: what the forward and the backward pass share.
//
// One pass (attn_pass_kernel) computes, for tokens i in the pass' order (along a
// sequence, or back along it with kRev),
//     y_i = scale * sum over j up to i of D_ij (a_i . b_j) c_j,
//     D_ij = exp(-rate |t_i - t_j|),
// which is the forward (a, b, c = q, k, v) and each gradient: dq has dO, v, k
// along the sequence, dk has v, dO, q and dv has k, q, dO back along it.
//
// A sequence is taken in chunks of 64 tokens.  Pairs in a chunk are products of
// 16 x 16 tiles, masked and decayed in registers; what came before is a state
// S = sum D b c^T [da, dc] at the time of the last token, so that
//     y_i = scale (sum over the chunk + D(i, last) a_i S).
// The work is split along the token axis into segments of seg_len tokens, cut
// anywhere in the sequences: attn_state_kernel sums each segment's part of the
// state that it hands on, attn_scan_kernel joins them, and the pass starts each
// segment from what came in.  (One segment: the pass alone.)
//
// Decays of the state over many chunks (step_factor): while they are weak, S += S
// expm1(-rate dt) rather than a product with exp(-rate dt), whose rounding is the
// same in every chunk of equal length and adds up over those that S lasts.
#pragma once

#include <hip/hip_runtime.h>

#include "common.hpp"
#include "seq.hpp"
#include "split.hpp"

namespace sbc {

constexpr int kChunk = 64;     // tokens of a chunk
constexpr int kWaves = 4;
constexpr int kAttnThreads = 64 * kWaves;
constexpr float kFresh = 1.f;  // a state's factor where nothing of it is left

struct AttnPass {
    int32_t n, n_batch, heads;
    int32_t da, dc;               // channels of a and b, and of c and y
    int32_t seg_len, n_seg;
    int32_t tiles;                // column tiles of c that blocks take
    float scale;
    const float *rates;
    const int32_t *splits, *t;
    sbc_heads a, b, c, y;
    // the states that segments start from: element (i, j) of segment g, head h at
    // carry[(g * heads + h) * state_stride + i * carry_i + j * carry_j]
    float *carry;
    int64_t state_stride;
    int32_t carry_i, carry_j;
    float *factor;                // [n_seg, heads]: step_factor() of what passes through
    const float *state_in;        // [n_batch, heads, da, dc]
    const int32_t *state_time;
    float *state_out;
    int32_t *time_out;
    // x . y of every token, if wanted: x [n, heads, dc], dots [tiles, heads, n]
    sbc_heads x;
    float *dots;
};

__device__ __forceinline__ int32_t split_at(const AttnPass &p, int32_t b) {
    return p.splits ? p.splits[b] : (b == 0 ? 0 : p.n);
}
__device__ __forceinline__ int32_t time_at(const AttnPass &p, int32_t i) {
    return p.t ? p.t[i] : i;
}
// the first b in [0, n_batch] with splits[b] >= at (n_batch if none)
__device__ __forceinline__ int32_t first_from(const AttnPass &p, int32_t at) {
    int32_t lo = 0, hi = p.n_batch;
    while (lo < hi) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (split_at(p, mid) >= at)
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}
// elapsed time from the earlier of two tokens in the pass' order to the later
template <bool kRev> __device__ __forceinline__ float elapsed(int32_t later, int32_t earlier) {
    return (float)(kRev ? (uint32_t)earlier - (uint32_t)later : (uint32_t)later - (uint32_t)earlier);
}
constexpr float kLog2E = 1.44269504088896340736f;
// exp(-rate dt) with rate2 = rate log2 e.  (The product's rounding moves the
// result by 2^-24 rate dt exp(-rate dt), under 2^-25 of 1.)
__device__ __forceinline__ float decay(float rate2, float dt) {
    return __builtin_amdgcn_exp2f(-rate2 * dt);
}

// A state's decay over dt as one number: expm1(-x) <= 0 for x = rate dt below 1/2,
// exp(-x) > 0 from there on, kFresh where that is 0.
__device__ __forceinline__ float step_factor(float rate, float dt) {
    const float x = rate * dt;
    if (x < 0.5f) return expm1f(-x);
    const float e = __builtin_amdgcn_exp2f(-x * kLog2E);
    return e > 0.f ? e : kFresh;
}
__device__ __forceinline__ float apply_factor(float f, float s) {
    return f <= 0.f ? fmaf(s, f, s) : f == kFresh ? 0.f : s * f;
}
// the factor of f, then g
__device__ __forceinline__ float join_factors(float f, float g) {
    if (f == kFresh || g == kFresh) return kFresh;
    if (f <= 0.f && g <= 0.f) {
        const float r = fmaf(f, g, f + g);
        return r > -0.5f ? r : 1.f + r;
    }
    const float e = (f > 0.f ? f : 1.f + f) * (g > 0.f ? g : 1.f + g);
    return e > 0.f ? e : kFresh;
}

// ---------------------------------------------------------------- fragments
// An operand's parts: 1 of a bf16 input, 3 of a float32 one.
template <typename T> constexpr int kParts = sizeof(T) == 4 ? 3 : 1;

// acc += a b, all products of parts that reach above the smallest part's own
// rounding, smallest first
template <int NA, int NB>
__device__ __forceinline__ void mma(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], floatx4 &acc) {
    constexpr int kMost = NA > NB ? NA : NB;
#pragma unroll
    for (int s = kMost - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[s - i], acc, 0, 0, 0);
}

// 8 values -> N parts: their first 8, 16 or 24 bits
template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&out)[N]) {
    u32x4v h, m, l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        if constexpr (N == 3) {
            uint32_t u, v, w;
            split2(a, b, u, v, w);
            h[i] = u;
            m[i] = v;
            l[i] = w;
        } else {
            h[i] = pack_bf16(a, b);
            if constexpr (N == 2)
                m[i] = pack_bf16(a - __uint_as_float(h[i] << 16),
                                 b - __uint_as_float(h[i] & 0xFFFF0000u));
        }
    }
    out[0] = __builtin_bit_cast(bf16x8, h);
    if constexpr (N > 1) out[1] = __builtin_bit_cast(bf16x8, m);
    if constexpr (N > 2) out[2] = __builtin_bit_cast(bf16x8, l);
}

// the sum of the parts of 8 values
template <int N> __device__ __forceinline__ void join8(const bf16x8 (&in)[N], float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float s = (float)in[N - 1][e];
#pragma unroll
        for (int i = N - 2; i >= 0; --i) s += (float)in[i][e];
        x[e] = s;
    }
}

// A tile of D columns in LDS, row after row, one plane a part.  The 16-byte
// pieces of a row are permuted by its number, so that the same piece of rows in
// turn lies in other banks.
template <int D> __device__ __forceinline__ int tile_at(int row, int col) {
    constexpr int kMask = D / 8 - 1;
    return row * D + ((((col >> 3) ^ row) & kMask) << 3) + (col & 7);
}
// 8 columns of a row
template <int D, int N>
__device__ __forceinline__ void frag_row(const bf16_t *tile, int plane, int row, int col,
                                         bf16x8 (&out)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        out[i] = *reinterpret_cast<const bf16x8 *>(tile + i * plane + tile_at<D>(row, col));
}
// For every lane 8 rows of one column: with l = lane & 15 and g = lane >> 4,
// rows row0 + 4 g .. + 3 and row0 + 16 + 4 g .. + 3 of column col0 + l: the order
// in which a product of two 16-row tiles leaves its rows in a lane's registers.
// (The transposing read gives lane l of 16 the l-th column of the 4 x 16 block
// whose rows' quarters the 16 lanes address.)
template <int D, int N>
__device__ __forceinline__ void frag_col(const bf16_t *tile, int plane, int row0, int col0,
                                         bf16x8 (&out)[N]) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef short s8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s4 *lds_s4;
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
    const int row = row0 + 4 * g + (l >> 2), col = col0 + 4 * (l & 3);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        bf16_t *base = const_cast<bf16_t *>(tile) + i * plane;
        const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(base + tile_at<D>(row, col)));
        const s4 hi =
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(base + tile_at<D>(row + 16, col)));
        out[i] = __builtin_bit_cast(bf16x8, s8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
}

// ---------------------------------------------------------------- loads
// The tokens of a chunk in the pass' order: the first is `first`, `count` exist.
template <bool kRev> __device__ __forceinline__ int64_t token_of(int32_t first, int l) {
    return kRev ? (int64_t)first - l : (int64_t)first + l;
}

// 16 bytes of a row at column col, zero past `d` and without a token
template <typename T>
__device__ __forceinline__ u32x4v load_raw(const T *row, int col, int d, bool there) {
    u32x4v r{0, 0, 0, 0};
    if (!there) return r;
    if (col + kVec<T> <= d) {
        __builtin_memcpy(&r, row + col, 16);
    } else {
        T raw[kVec<T>];
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) raw[i] = col + i < d ? row[col + i] : T(0);
        __builtin_memcpy(&r, raw, 16);
    }
    return r;
}

// A chunk of 64 rows x D columns on its way to LDS, kSteps 16-byte pieces a lane
template <typename T, int D> struct Staged {
    static constexpr int kPerRow = D / kVec<T>;
    static constexpr int kRows = kAttnThreads / kPerRow;
    static constexpr int kSteps = kChunk / kRows;
    u32x4v raw[kSteps];

    template <bool kRev>
    __device__ __forceinline__ void load(const sbc_heads &x, int32_t head, int32_t first,
                                         int count, int col0, int d) {
        const T *base = static_cast<const T *>(x.data) + (int64_t)head * x.head_stride + col0;
        const int col = (threadIdx.x % kPerRow) * kVec<T>;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int l = s * kRows + threadIdx.x / kPerRow;
            raw[s] = load_raw<T>(base + token_of<kRev>(first, l) * x.token_stride, col, d - col0,
                                 l < count);
        }
    }
    __device__ __forceinline__ void store(bf16_t *tile) const {
        const int col = (threadIdx.x % kPerRow) * kVec<T>;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = tile_at<D>(s * kRows + threadIdx.x / kPerRow, col);
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<u32x4v *>(tile + at) = raw[s];
            } else {
                uint32_t h[2], m[2], l[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    split2(__uint_as_float(raw[s][2 * i]), __uint_as_float(raw[s][2 * i + 1]), h[i],
                           m[i], l[i]);
                constexpr int kPlane = kChunk * D;
                *reinterpret_cast<uint2 *>(tile + at) = uint2{h[0], h[1]};
                *reinterpret_cast<uint2 *>(tile + kPlane + at) = uint2{m[0], m[1]};
                *reinterpret_cast<uint2 *>(tile + 2 * kPlane + at) = uint2{l[0], l[1]};
            }
        }
    }
};

// 8 columns of a row in global memory as an operand's parts
template <typename T>
__device__ __forceinline__ void frag_global(const T *row, int col, int d, bool there,
                                            bf16x8 (&out)[kParts<T>]) {
    if constexpr (sizeof(T) == 2) {
        out[0] = __builtin_bit_cast(bf16x8, load_raw<T>(row, col, d, there));
    } else {
        const u32x4v lo = load_raw<T>(row, col, d, there), hi = load_raw<T>(row, col + 4, d, there);
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(lo[i]);
            x[4 + i] = __uint_as_float(hi[i]);
        }
        split8<3>(x, out);
    }
}

// ---------------------------------------------------------------- state
// The state's tiles [DA x DCT] over the four waves: a wave has 16 columns and
// kTiles tiles of 16 rows.  A lane holds column `col` and rows row(u) .. + 3.
template <int DA, int DCT> struct StateTiles {
    static constexpr int kCols = DCT / 16;              // waves side by side
    static constexpr int kDown = kWaves / kCols;
    static constexpr int kTiles = DA / 16 / kDown;
    static_assert(kCols * kDown == kWaves && kTiles >= 1, "tiles");
    __device__ __forceinline__ static int wave() { return threadIdx.x >> 6; }
    __device__ __forceinline__ static int col0() { return 16 * (wave() % kCols); }
    __device__ __forceinline__ static int col() { return col0() + (threadIdx.x & 15); }
    __device__ __forceinline__ static int row0(int u) { return 16 * ((wave() / kCols) * kTiles + u); }
    __device__ __forceinline__ static int row(int u) { return row0(u) + 4 * ((threadIdx.x & 63) >> 4); }
};

// acc += sum over the chunk's tokens of w_j b_j c_j^T
template <typename T, int DA, int DCT>
__device__ __forceinline__ void add_chunk(const bf16_t *bt, const bf16_t *ct, const float *w,
                                          floatx4 (&acc)[StateTiles<DA, DCT>::kTiles]) {
    using S = StateTiles<DA, DCT>;
    constexpr int NP = kParts<T>;
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < kChunk / 32; ++s) {
        bf16x8 raw[NP], cw[3];
        frag_col<DCT, NP>(ct, kChunk * DCT, 32 * s, S::col0(), raw);
        float x[8];
        join8<NP>(raw, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] *= w[32 * s + 4 * g + e];
            x[4 + e] *= w[32 * s + 16 + 4 * g + e];
        }
        split8<3>(x, cw);
#pragma unroll
        for (int u = 0; u < S::kTiles; ++u) {
            bf16x8 b[NP];
            frag_col<DA, NP>(bt, kChunk * DA, 32 * s, S::row0(u), b);
            mma<NP, 3>(b, cw, acc[u]);
        }
    }
}

}  // namespace sbc
