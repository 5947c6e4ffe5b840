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
// Products whose result is then split are rounded first (no contraction with the
// split's differences), so that variants of a kernel agree in every bit.
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
    // for the rates' gradient (kDots): rows whose products with y are wanted, the states
    // that come into the segments back along the sequence, and the sums, [tiles, n_seg, heads]
    sbc_heads x;
    const float *behind;
    double *slope;
};

__device__ __forceinline__ int32_t split_at(const AttnPass &p, int32_t b) {
    return p.splits ? p.splits[b] : (b == 0 ? 0 : p.n);
}
__device__ __forceinline__ int32_t time_at(const AttnPass &p, int32_t i) {
    return p.t ? p.t[i] : i;
}
// The first b in [0, n_batch] with splits[b] >= at (n_batch if none): the wave's lanes
// take 64 places of the range at once, so that up to 64 sequences are one round of
// loads and 4096 two (one by one, each halving of the range waited for memory).
__device__ __forceinline__ int32_t first_from(const AttnPass &p, int32_t at) {
    int32_t lo = 0, hi = p.n_batch;
    while (lo < hi) {
        const int32_t step = (hi - lo + 63) / 64;
        const int64_t b = lo + (int64_t)(threadIdx.x & 63) * step;
        const bool below = b < hi && split_at(p, (int32_t)b) < at;
        const int32_t n = __popcll(__ballot(below));
        if (n == 0) break;
        const int64_t up = lo + (int64_t)n * step;
        lo += (n - 1) * step + 1;
        hi = up < hi ? (int32_t)up : hi;
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
// rounding, smallest first.  (Of three parts each, m l, l m and l l are left out, up to
// 2^-22 of the product; the sum of all is one float32, where split.hpp's mma_split keeps the largest
// apart, at twice the registers.)
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

// 8 values -> N parts: their first 16 or 24 bits
template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&out)[N]) {
#pragma clang fp contract(off)
    static_assert(N == 2 || N == 3, "parts");
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
            m[i] = pack_bf16(a - __uint_as_float(h[i] << 16),
                             b - __uint_as_float(h[i] & 0xFFFF0000u));
        }
    }
    out[0] = __builtin_bit_cast(bf16x8, h);
    out[1] = __builtin_bit_cast(bf16x8, m);
    if constexpr (N > 2) out[2] = __builtin_bit_cast(bf16x8, l);
}

// value e of an operand's parts
template <int N> __device__ __forceinline__ float part_sum(const bf16x8 (&in)[N], int e) {
    float s = (float)in[N - 1][e];
#pragma unroll
    for (int i = N - 2; i >= 0; --i) s += (float)in[i][e];
    return s;
}
// the sum of the parts of 8 values
template <int N> __device__ __forceinline__ void join8(const bf16x8 (&in)[N], float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = part_sum<N>(in, e);
}

// A tile of D columns in LDS, row after row, one plane a part.  The 16-byte
// pieces of a row are permuted by its number, so that the same piece of rows in
// turn lies in other banks.
template <int D> __device__ __forceinline__ int tile_at(int row, int col) {
    constexpr int kMask = ((D / 8) & -(D / 8)) - 1;  // (as many low bits as stay inside the row)
    return row * D + (((col >> 3) ^ (row & kMask)) << 3) + (col & 7);
}
// x, of which the compiler knows nothing: what is computed from it inside a loop
// stays there.  (Comparisons of lanes with sizes, kept in scalar registers across the
// chunks, took all of those and spilled.)
__device__ __forceinline__ int in_loop(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// A lane's places in such a tile (l = lane & 15, g = lane >> 4), which are the same 16
// rows further on: three, from which the others of the first 16 rows differ in bits of
// the piece's number and the rest lies at constant distances.  (Left to the compiler,
// every fragment's address took a register for the whole loop.)
template <int D> struct LaneAt {
    static constexpr int kMask = ((D / 8) & -(D / 8)) - 1;  // (tile_at)
    int row0, split0, col0;
    __device__ __forceinline__ LaneAt() {
        const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
        row0 = in_loop(tile_at<D>(l, 8 * g));
        split0 = in_loop(tile_at<D>(l, 4 * g));
        col0 = in_loop(tile_at<D>(4 * g + (l >> 2), 4 * (l & 3)));
    }
    // `pieces` further along the row (a multiple of a power of two above the lanes' own)
    __device__ __forceinline__ static int along(int at, int pieces) {
        return (at ^ ((pieces & kMask) << 3)) + ((pieces & ~kMask) << 3);
    }
    // row l, columns 32 k + 8 g .. + 7
    __device__ __forceinline__ int row(int k) const { return along(row0, 4 * k); }
    // row l, columns 32 k + 16 half + 4 g .. + 3
    __device__ __forceinline__ int split(int k, int half) const {
        return along(split0, 4 * k + 2 * half);
    }
    // for frag_col: row 4 g + l / 4, columns 16 t + 4 (l & 3) .. + 3
    __device__ __forceinline__ int col(int t) const { return along(col0, 2 * t); }
};
// 8 columns of row 16 t + l: k-step k of an operand
template <int D, int N>
__device__ __forceinline__ void frag_row(const bf16_t *tile, int plane, int t, int k,
                                         const LaneAt<D> &at, bf16x8 (&out)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        out[i] = *reinterpret_cast<const bf16x8 *>(tile + (i * plane + 16 * t * D) + at.row(k));
}
// The same in the order of frag_col's rows: columns 32 k + 4 g .. + 3 and 32 k + 16 +
// 4 g .. + 3
template <int D, int N>
__device__ __forceinline__ void frag_row_split(const bf16_t *tile, int plane, int t, int k,
                                               const LaneAt<D> &at, bf16x8 (&out)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bf16_t *row = tile + (i * plane + 16 * t * D);
        const uint2 lo = *reinterpret_cast<const uint2 *>(row + at.split(k, 0));
        const uint2 hi = *reinterpret_cast<const uint2 *>(row + at.split(k, 1));
        out[i] = __builtin_bit_cast(bf16x8, u32x4v{lo.x, lo.y, hi.x, hi.y});
    }
}
// For every lane 8 rows of one column: with l = lane & 15 and g = lane >> 4,
// rows 32 s + 4 g .. + 3 and 32 s + 16 + 4 g .. + 3 of column 16 t + l, at = LaneAt::col(t):
// the order in which a product of two 16-row tiles leaves its rows in a lane's
// registers.  (The transposing read gives lane l of 16 the l-th column of the 4 x 16
// block whose rows' quarters the 16 lanes address.)
template <int D, int N>
__device__ __forceinline__ void frag_col(const bf16_t *tile, int plane, int s, int at,
                                         bf16x8 (&out)[N]) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef short s8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s4 *lds_s4;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        bf16_t *base = const_cast<bf16_t *>(tile) + (i * plane + 32 * s * D);
        const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(base + at));
        const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(base + 16 * D + at));
        out[i] = __builtin_bit_cast(bf16x8, s8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
}

// This wave's number, in a scalar register: branches on it are then branches.
__device__ __forceinline__ int wave_of_block() {
    return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

// ---------------------------------------------------------------- loads
// Loads of 16-byte pieces of rows.  Where the channels fill whole pieces (kWhole),
// one that does not exist (past the channels, or of no token) is read from the
// first row's start and zeroed on its way to LDS, so that no branch lies between the
// loads, and a lane keeps its pieces' places in a full chunk; else pieces are read
// by elements.
template <typename T>
__device__ __forceinline__ u32x4v load_elements(const T *row, int col, int d, bool there) {
    T raw[kVec<T>];
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) raw[i] = there && col + i < d ? row[col + i] : T(0);
    u32x4v r;
    __builtin_memcpy(&r, raw, 16);
    return r;
}

// One head's rows of an array, from the lowest token of a chunk on: row l of the
// pass' order is `rows - 1 - l` (kRev) or l tokens above it.
template <typename T> struct Rows {
    const T *base;
    int64_t stride;
    __device__ __forceinline__ Rows(const sbc_heads &x, int32_t head, int32_t col0)
        : base(static_cast<const T *>(x.data) + (int64_t)head * x.head_stride + col0),
          stride(x.token_stride) {}
};

// A chunk of 64 rows x D columns on its way to LDS, kSteps 16-byte pieces a lane
template <typename T, int D, bool kWhole, bool kRev> struct Staged {
    static constexpr int kPerRow = D / kVec<T>;
    static constexpr int kSteps = kChunk * kPerRow / kAttnThreads;
    static_assert(kChunk * kPerRow % kAttnThreads == 0, "pieces");
    u32x4v raw[kSteps];
    uint32_t off[kSteps];  // the pieces' bytes in a full chunk (kWhole: strides below 2^22)

    __device__ __forceinline__ static int row_of(int s, int tid) {
        return (s * kAttnThreads + tid) / kPerRow;
    }
    __device__ __forceinline__ static int col_of(int s, int tid) {
        return (s * kAttnThreads + tid) % kPerRow * kVec<T>;
    }
    __device__ __forceinline__ Staged(const Rows<T> &x, int width) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int l = row_of(s, threadIdx.x), col = col_of(s, threadIdx.x);
            off[s] = ((kRev ? kChunk - 1 - l : l) * (uint32_t)x.stride + (col < width ? col : 0)) *
                     (uint32_t)sizeof(T);
        }
    }
    // the chunk of `count` tokens from token `lowest` on; `width` columns exist
    __device__ __forceinline__ void load(const Rows<T> &x, int32_t lowest, int count, int width) {
        const T *base = x.base + (int64_t)lowest * x.stride;
        if (kWhole && count == kChunk) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
                __builtin_memcpy(&raw[s], reinterpret_cast<const char *>(base) + off[s], 16);
        } else {
            const int tid = in_loop(threadIdx.x);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int l = row_of(s, tid), col = col_of(s, tid);
                const T *row = base + (int64_t)(kRev ? count - 1 - l : l) * x.stride;
                if constexpr (kWhole)
                    __builtin_memcpy(&raw[s], l < count && col < width ? row + col : base, 16);
                else
                    raw[s] = load_elements<T>(row, col, width, l < count);
            }
        }
    }
    // whether any of the lane's values is infinite or NaN (after store())
    __device__ __forceinline__ bool not_finite() const {
        uint32_t found = 0;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = raw[s][i];
                found |= (w & 0x7F800000u) == 0x7F800000u;
                if constexpr (sizeof(T) == 2) found |= (w & 0x7F80u) == 0x7F80u;
            }
        return found != 0;
    }
    __device__ __forceinline__ void store(bf16_t *tile, int count, int width) {
        if (kWhole && (count < kChunk || width < D)) {
            const int tid = in_loop(threadIdx.x);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const bool ok = row_of(s, tid) < count && col_of(s, tid) < width;
#pragma unroll
                for (int i = 0; i < 4; ++i) raw[s][i] = ok ? raw[s][i] : 0u;
            }
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = tile_at<D>(row_of(s, threadIdx.x), col_of(s, threadIdx.x));
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<u32x4v *>(tile + at) = raw[s];
            } else {
                uint32_t h[2], m[2], lo[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    split2(__uint_as_float(raw[s][2 * i]), __uint_as_float(raw[s][2 * i + 1]),
                           h[i], m[i], lo[i]);
                constexpr int kPlane = kChunk * D;
                *reinterpret_cast<uint2 *>(tile + at) = uint2{h[0], h[1]};
                *reinterpret_cast<uint2 *>(tile + kPlane + at) = uint2{m[0], m[1]};
                *reinterpret_cast<uint2 *>(tile + 2 * kPlane + at) = uint2{lo[0], lo[1]};
            }
        }
    }
};

// Each lane's own row (token `mine` of the chunk) as an operand of D columns:
// columns 32 k + 8 g .. + 7 of k-step k, or (kSplit) 32 k + 4 g .. + 3 and 32 k + 16 +
// 4 g .. + 3
template <typename T, int D, bool kWhole, bool kRev, bool kSplit = false> struct RowFrag {
    static constexpr int kRaw = 8 / kVec<T>;
    u32x4v raw[D / 32][kRaw];

    // the columns' start for half of 4 (part) elements
    __device__ __forceinline__ static int col_of(int k, int half) {
        return 32 * k + (kSplit ? 16 * half : 4 * half);
    }
    __device__ __forceinline__ void load(const Rows<T> &x, int32_t lowest, int count, int width,
                                         int mine) {
        const T *base = x.base + (int64_t)lowest * x.stride;
        const int lane0 = (kSplit ? 4 : 8) * ((threadIdx.x & 63) >> 4);
        const bool there = mine < count;
        const int up = kRev ? count - 1 - mine : mine;
        const T *row = kWhole
                           ? base + (uint32_t)((there ? up : 0) * (uint32_t)x.stride + lane0)
                           : base + (int64_t)(there ? up : 0) * x.stride + lane0;
        constexpr int kBytes = sizeof(T) * 4;  // of a half
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            if constexpr (!kSplit && sizeof(T) == 2) {
                if constexpr (kWhole)
                    __builtin_memcpy(&raw[k][0], 32 * k + lane0 < width ? row + 32 * k : base, 16);
                else
                    raw[k][0] = load_elements<T>(row, 32 * k, width - lane0, there);
            } else {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int col = col_of(k, half);
                    char *to = reinterpret_cast<char *>(&raw[k][0]) + half * kBytes;
                    if constexpr (kWhole) {
                        __builtin_memcpy(to, col + lane0 < width ? row + col : base, kBytes);
                    } else {
                        T e[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            e[i] = there && col + lane0 + i < width ? row[col + i] : T(0);
                        __builtin_memcpy(to, e, kBytes);
                    }
                }
            }
        }
    }
    __device__ __forceinline__ void parts(bf16x8 (&out)[D / 32][kParts<T>], int count, int width,
                                          int mine) {
        if (kWhole && (count < kChunk || width < D)) {
            const int lane0 = in_loop((kSplit ? 4 : 8) * ((threadIdx.x & 63) >> 4));
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const bool ok = mine < count && col_of(k, half) + lane0 < width;
                    constexpr int kWords = sizeof(T);  // of a half
#pragma unroll
                    for (int e = 0; e < kWords; ++e) {
                        const int at = half * kWords + e;
                        raw[k][at / 4][at % 4] = ok ? raw[k][at / 4][at % 4] : 0u;
                    }
                }
        }
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            if constexpr (sizeof(T) == 2) {
                out[k][0] = __builtin_bit_cast(bf16x8, raw[k][0]);
            } else {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(raw[k][i / 4][i % 4]);
                split8<3>(x, out[k]);
            }
        }
    }
};

// A lane's channels of its token's row of an output: 16 t + 4 g .. + 3 of tile t
template <typename T, bool kWhole> struct RowOut {
    T *row;
    int width;  // channels from the lane's first on; none without a token
    __device__ __forceinline__ RowOut(const Rows<T> &x, int64_t token, int d, bool there) {
        const int c0 = in_loop(4 * ((threadIdx.x & 63) >> 4));
        row = const_cast<T *>(x.base) + token * x.stride + c0;
        width = there ? d - c0 : 0;
    }
    __device__ __forceinline__ void put(int t, const floatx4 &o) const {
        T raw[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) raw[r] = from_f32<T>(o[r]);
        if constexpr (kWhole) {
            if (16 * t < width) __builtin_memcpy(row + 16 * t, raw, sizeof(raw));
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * t + r < width) row[16 * t + r] = raw[r];
        }
    }
};

// ---------------------------------------------------------------- state
// The state's tiles [DA x DCT] over the four waves: a wave has 16 columns and
// kTiles tiles of 16 rows.  A lane holds column `col` and rows row(u) .. + 3.
template <int DA, int DCT> struct StateTiles {
    static constexpr int kCols = DCT / 16;              // waves side by side
    static constexpr int kDown = kWaves / kCols;
    static constexpr int kTiles = DA / 16 / kDown;
    static_assert(kCols * kDown == kWaves && kTiles >= 1, "tiles");
    __device__ __forceinline__ static int wave() { return wave_of_block(); }
    __device__ __forceinline__ static int col0() { return 16 * (wave() % kCols); }
    __device__ __forceinline__ static int col() { return col0() + (threadIdx.x & 15); }
    __device__ __forceinline__ static int row0(int u) { return 16 * ((wave() / kCols) * kTiles + u); }
    __device__ __forceinline__ static int row(int u) { return row0(u) + 4 * ((threadIdx.x & 63) >> 4); }
};

// acc += sum over the chunk's tokens of w_j b_j c_j^T; at_c: the lane's place in ct for
// its wave's columns
template <typename T, int DA, int DCT>
__device__ __forceinline__ void add_chunk(const bf16_t *bt, const bf16_t *ct,
                                          const LaneAt<DA> &at_b, int at_c, const float *w,
                                          floatx4 (&acc)[StateTiles<DA, DCT>::kTiles]) {
#pragma clang fp contract(off)
    using S = StateTiles<DA, DCT>;
    constexpr int NP = kParts<T>;
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < kChunk / 32; ++s) {
        bf16x8 raw[NP], cw[3];
        frag_col<DCT, NP>(ct, kChunk * DCT, s, at_c, raw);
        float x[8];
        join8<NP>(raw, x);
        const floatx4 lo = *reinterpret_cast<const floatx4 *>(w + 32 * s + 4 * g);
        const floatx4 hi = *reinterpret_cast<const floatx4 *>(w + 32 * s + 16 + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] *= lo[e];
            x[4 + e] *= hi[e];
        }
        split8<3>(x, cw);
#pragma unroll
        for (int u = 0; u < S::kTiles; ++u) {
            bf16x8 b[NP];
            frag_col<DA, NP>(bt, kChunk * DA, s, at_b.col(S::row0(u) / 16), b);
            mma<NP, 3>(b, cw, acc[u]);
        }
    }
}

// acc *= the decay of `f`, which is the same for all lanes
template <int N> __device__ __forceinline__ void decay_state(float f, floatx4 (&acc)[N]) {
    f = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(f)));
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[u][r] = apply_factor(f, acc[u][r]);
}

// The state in LDS as parts, column after column of c, its rows (the channels of a)
// the contraction's axis
template <int DA, int DCT, int NS>
__device__ __forceinline__ void store_state(
    bf16_t *st, const floatx4 (&acc)[StateTiles<DA, DCT>::kTiles]) {
    using S = StateTiles<DA, DCT>;
#pragma unroll
    for (int u = 0; u < S::kTiles; ++u) {
        const int o = tile_at<DA>(S::col(), S::row(u));
        uint32_t w[3][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float x = acc[u][2 * i], z = acc[u][2 * i + 1];
            if constexpr (NS == 3) {
                split2(x, z, w[0][i], w[1][i], w[2][i]);
            } else {
                w[0][i] = pack_bf16(x, z);
                w[1][i] = pack_bf16(x - __uint_as_float(w[0][i] << 16),
                                    z - __uint_as_float(w[0][i] & 0xFFFF0000u));
            }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i)
            *reinterpret_cast<uint2 *>(st + i * DCT * DA + o) = uint2{w[i][0], w[i][1]};
    }
}

}  // namespace sbc
