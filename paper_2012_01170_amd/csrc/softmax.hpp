// Softmax attention: what the forward pass, its form over a paged cache and the
// gradients share.
//
// Head h of the queries reads head h / group of the keys (group = heads / kv_heads).
// The rows of one sequence and key head are its tokens' queries of the whole group,
// row r = token r / group, head r % group of the group: keys are read once for all of
// them, a single token still fills `group` rows, and the gradients of a shared head are
// sums along the rows.
//
// Products are v_mfma_f32_32x32x16_bf16 on operands split into parts (split.hpp, one part
// of a bf16 input, three of a float32 one).  They are taken so that a lane holds one row's
// scores: S^T = K Q^T has row l = lane & 31 in the lanes l and l + 32, and of its 32 keys
// those of 8 (r / 4) + 4 (lane >> 5) + r % 4 in register r.  Maximum and sum are then along
// a lane's registers (one exchange between the halves for the maximum), and the registers are
// the next product's operand as they are, O^T = V^T P^T, if V's rows come in the same
// order, as the transposing reads of LDS give them.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "attention.hpp"
#include "common.hpp"
#include "seq.hpp"
#include "split.hpp"

namespace sbc {

typedef float floatx16 __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------- division
// n / d for n < 2^31 by a multiplication (round-up method): q = (hi(m n) + n) >> s
struct Divisor {
    uint32_t m, d;
    int32_t s;
};
inline Divisor divisor(int32_t d) {
    int32_t s = 0;
    while (((int64_t)1 << s) < d) ++s;
    const uint64_t m = ((((uint64_t)1 << s) - (uint64_t)d) << 32) / (uint64_t)d + 1;
    return {(uint32_t)m, (uint32_t)d, s};
}
__device__ __forceinline__ int32_t divide(int32_t n, const Divisor &by) {
    return (int32_t)((__umulhi((uint32_t)n, by.m) + (uint32_t)n) >> by.s);
}

// ---------------------------------------------------------------- arguments
// Rows and keys are counted in 32 bits, up to a few tiles past the last
constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1024;

struct SoftmaxPages {  // a paged cache, in place of k, v and k_splits
    sbc_pages k, v;
    int32_t n_pages, width;
    Divisor page;
    const int32_t *table, *lengths;
};
struct SoftmaxArgs {
    int32_t n, m, n_batch, heads, kv_heads, dk, dv;
    int32_t causal;
    Divisor group;
    float scale, scale2;  // scale2 = scale log2 e
    const int32_t *splits, *k_splits;
    sbc_heads q, k, v, o;
    float *lse;
    int32_t slots;  // places of tiles (tile_place)
    SoftmaxPages pages;
    // keys of a sequence in parts (softmax_rows_kernel): what each part gives, float32
    int32_t parts;
    float *part_o, *part_lse;
    // gradients
    sbc_heads d_o, dq, dk_out, dv_out;
    const float *lse_in;
    // the rows' deltas, and their sums in units of log 2 (infinite where no key has a weight), a
    // key head's rows behind each other (packed_row)
    float *row_delta, *row_lse;
    float *part_dk, *part_dv;
    int32_t even_rows;  // whether tiles of rows begin with a token's first head, at 32-bit offsets
};

__device__ __forceinline__ int32_t clamp_i(int32_t x, int32_t lo, int32_t hi) {
    return x < lo ? lo : x > hi ? hi : x;
}
// Where row `row` of key head head_k lies among the packed ones
__device__ __forceinline__ int64_t packed_row(const SoftmaxArgs &p, int32_t head_k, int32_t q0,
                                              int32_t row) {
    return ((int64_t)head_k * p.n + q0) * p.group.d + row;
}
// (whatever the splits hold, rows are read and written inside the arrays)
__device__ __forceinline__ int32_t q_split(const SoftmaxArgs &p, int32_t b) {
    return p.splits ? clamp_i(p.splits[b], 0, p.n) : p.pages.table ? b : b == 0 ? 0 : p.n;
}
__device__ __forceinline__ int32_t k_split(const SoftmaxArgs &p, int32_t b) {
    return p.k_splits ? clamp_i(p.k_splits[b], 0, p.m) : b == 0 ? 0 : p.m;
}

// Tiles of kRows rows are laid out by places: those of sequence b begin at place
// (rows before it) / kRows + b, which leaves room for its last, partly filled one, so that
// no sum over the sequences' tiles is needed to launch or to find them.  The last b in
// [0, n_batch) whose places begin at or before x, -1 if none; 64 lanes look at 64 places
// of the range at once.
//
// begins(lo, step, hi): a bit for each b = lo + lane * step below hi that begins at or before x.
// The range goes on behind the last bit of those that hold from the first on, so that the
// result is a b that was seen to begin there, also where splits are not in order.  (By the
// number of bits it could be one that begins behind x, and a tile's rows negative.)
template <typename F> constexpr int32_t last_beginning(int32_t n_batch, F begins) {
    int32_t lo = 0, hi = n_batch;
    while (lo < hi) {
        const int32_t step = (hi - lo + 63) / 64;
        const uint64_t bits = begins(lo, step, hi);
        const int32_t c = bits == ~0ull ? 64 : __builtin_ctzll(~bits);
        if (c == 0) break;
        const int64_t up = lo + (int64_t)c * step;
        lo += (c - 1) * step + 1;
        hi = up < hi ? (int32_t)up : hi;
    }
    return lo - 1;
}
template <typename F>
__device__ __forceinline__ int32_t sequence_of(int32_t n_batch, int32_t x, F begin) {
    return last_beginning(n_batch, [&](int32_t lo, int32_t step, int32_t hi) -> uint64_t {
        const int64_t b = lo + (int64_t)(threadIdx.x & 63) * step;
        return __ballot(b < hi && begin((int32_t)b) <= x);
    });
}

// One sequence's tokens and keys
struct Sequence {
    int32_t b, q0, lq, k0, lk;
    // keys that the token sees: causal, the last token sees the last key
    __device__ __forceinline__ int32_t limit(int32_t token, int32_t causal) const {
        return causal ? clamp_i(token - lq + lk + 1, 0, lk) : lk;
    }
};
template <bool kPaged>
__device__ __forceinline__ Sequence sequence_at(const SoftmaxArgs &p, int32_t b) {
    Sequence s;
    s.b = b;
    s.q0 = q_split(p, b);
    s.lq = q_split(p, b + 1) - s.q0;
    if (s.lq < 0) s.lq = 0;
    if constexpr (kPaged) {
        const int64_t room = (int64_t)p.pages.width * p.pages.page.d;
        s.k0 = 0;
        s.lk = clamp_i(p.pages.lengths[b], 0, room > kMostRows ? (int32_t)kMostRows : (int32_t)room);
    } else {
        s.k0 = k_split(p, b);
        s.lk = k_split(p, b + 1) - s.k0;
        if (s.lk < 0) s.lk = 0;
    }
    return s;
}

// ---------------------------------------------------------------- fragments
template <int NA, int NB>
__device__ __forceinline__ void mma32(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB],
                                      floatx16 &acc) {
    constexpr int kMost = NA > NB ? NA : NB;
#pragma unroll
    for (int s = kMost - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB)
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[s - i], acc, 0, 0, 0);
}
template <int N> __device__ __forceinline__ void clear(floatx16 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[i][r] = 0.f;
}

// A tile of D columns in LDS, row after row, one plane a part, the 16-byte pieces of a row
// permuted by its number so that lanes which LDS serves in one cycle do not meet in one of its 64
// banks (256 bytes): of reads of 16 bytes, 16 rows of different residues by 16; of the transposing
// reads, 4 rows x 64 bytes, which have to fall into different quarters of the banks.  (Permuted
// by the row's number itself, the transposing reads of neighbouring rows met: 43 % of LDS' cycles.)
template <int D> struct TileAt {
    static constexpr int kMask = D % 128 == 0 ? 15 : D % 64 == 0 ? 7 : 3;
    __device__ __forceinline__ static int at(int row, int col) {
        const int by = (row >> 2 & 3) | (kMask == 15 ? (row & 3) << 2 : kMask == 7 ? (row & 2) << 1 : 0);
        return row * D + (((col >> 3) ^ by) << 3) + (col & 7);
    }
};
// A lane's places in such a tile for 32 x 32 products
template <int D> struct LaneAt32 {
    static constexpr int kMask = TileAt<D>::kMask;
    int row0, col0;
    __device__ __forceinline__ LaneAt32() {
        const int lane = threadIdx.x & 63, quarter = lane >> 4, i = lane & 15;
        const int r = 4 * (quarter >> 1) + (i >> 2), c = 16 * (quarter & 1) + 4 * (i & 3);
        row0 = in_loop(TileAt<D>::at(lane & 31, 8 * (lane >> 5)));
        col0 = in_loop(TileAt<D>::at(r, c));
    }
    // The same, of which the compiler knows nothing: the places further along the rows are then
    // made where they are used, not kept in some 20 registers across the loop.
    __device__ __forceinline__ LaneAt32(const LaneAt32 &x)
        : row0(in_loop(x.row0)), col0(in_loop(x.col0)) {}
    __device__ __forceinline__ static int along(int at, int pieces) {
        return (at ^ ((pieces & kMask) << 3)) + ((pieces & ~kMask) << 3);
    }
};
// Row 32 u + l, columns 16 k + 8 g .. + 7 (g = lane >> 5)
template <int D, int N>
__device__ __forceinline__ void frag_row32(const bf16_t *tile, int plane, int u, int k,
                                           const LaneAt32<D> &at, bf16x8 (&out)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        out[i] = *reinterpret_cast<const bf16x8 *>(tile + (i * plane + 32 * u * D) +
                                                   LaneAt32<D>::along(at.row0, 2 * k));
}
// Rows 16 s + 4 g .. + 3 and 16 s + 8 + 4 g .. + 3 of column 32 t + l
template <int D, int N>
__device__ __forceinline__ void frag_col32(const bf16_t *tile, int plane, int s, int t,
                                           const LaneAt32<D> &at, bf16x8 (&out)[N]) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef short s8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s4 *lds_s4;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        bf16_t *base = const_cast<bf16_t *>(tile) + (i * plane + 16 * s * D) +
                       LaneAt32<D>::along(at.col0, 4 * t);
        // (8 rows on: the pieces' permutation differs in its second bit)
        bf16_t *up = const_cast<bf16_t *>(tile) + (i * plane + (16 * s + 8) * D) +
                     LaneAt32<D>::along(at.col0 ^ 16, 4 * t);
        const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)base);
        const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)up);
        out[i] = __builtin_bit_cast(bf16x8, s8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
}
// Registers 8 h .. + 7 of a product as an operand of the next, in N parts: keys 16 h + 4 g .. + 3
// and 16 h + 8 + 4 g .. + 3 of its 32.
template <int N>
__device__ __forceinline__ void frag_regs(const floatx16 &x, int h, bf16x8 (&out)[N]) {
    if constexpr (N == 1) {
        u32x4v w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[8 * h + 2 * i], x[8 * h + 2 * i + 1]);
        out[0] = __builtin_bit_cast(bf16x8, w);
    } else {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[8 * h + i];
        split8<N>(y, out);
    }
}

// 16-byte pieces of rows whose channels fill no whole pieces.  Of bf16, a row's last piece is
// read as the 16 bytes up to the row's end and moved down afterwards, so that no piece is read by
// elements (4096 tokens, 8 heads of 33 and 31 channels: 119 -> 87 us, gradients 293 -> 233);
// narrower rows than a piece are, and float32 ones (whose gradients lack the registers: 573 -> 653).
// Columns c on of `width`; without `ok` some bytes of `any`.
template <typename T> __device__ __forceinline__ bool by_elements(int width) {
    return sizeof(T) == 4 || width < kVec<T>;
}
template <typename T>
__device__ __forceinline__ u32x4v load_odd(const T *row, int c, int width, bool ok, const T *any) {
    if (by_elements<T>(width)) return load_elements<T>(ok ? row : any, c, width, ok);
    const int at = c + kVec<T> <= width ? c : width - kVec<T>;
    u32x4v raw;
    __builtin_memcpy(&raw, ok && c < width ? row + at : any, 16);
    return raw;
}
template <typename T>
__device__ __forceinline__ u32x4v settle_odd(u32x4v w, int c, int width, bool ok) {
    if (by_elements<T>(width)) return w;
    const int over = c + kVec<T> - width;  // elements that the piece was read too early
    const uint32_t bits = (over > 0 ? over : 0) * (uint32_t)sizeof(T) * 8u;
    if (bits & 64u) w = u32x4v{w[2], w[3], 0u, 0u};
    if (bits & 32u) w = u32x4v{w[1], w[2], w[3], 0u};
    const uint32_t by = bits & 16u;
    w = u32x4v{__builtin_amdgcn_alignbit(w[1], w[0], by), __builtin_amdgcn_alignbit(w[2], w[1], by),
               __builtin_amdgcn_alignbit(w[3], w[2], by), w[3] >> by};
    return ok && c < width ? w : u32x4v{0u, 0u, 0u, 0u};
}

// A lane's row of an input as an operand of D columns, 16 k + 8 g .. + 7 of k-step k; `row` may
// be read also without `there`.
template <typename T, int D, bool kWhole>
__device__ __forceinline__ void load_row(const T *row, bool there, int width,
                                         u32x4v (&raw)[D / 16][8 / kVec<T>]) {
    const int c0 = 8 * ((threadIdx.x & 63) >> 5);
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 8 / kVec<T>; ++i) {
            const int c = 16 * k + c0 + i * kVec<T>;
            if constexpr (kWhole)
                __builtin_memcpy(&raw[k][i], row + (c < width ? c : 0), 16);
            else
                raw[k][i] = load_odd<T>(row, c, width, there, row);
        }
}
// What load_row read past the columns, and all of a row that is not there, to zero
template <typename T, int D, bool kWhole>
__device__ __forceinline__ void settle_row(bool there, int width,
                                           u32x4v (&raw)[D / 16][8 / kVec<T>]) {
    if (kWhole && width == D && __all(there)) return;
    const int c0 = in_loop(8 * ((threadIdx.x & 63) >> 5));
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 8 / kVec<T>; ++i) {
            const int c = 16 * k + c0 + i * kVec<T>;
            const bool ok = there && c < width;
            if constexpr (!kWhole) {
                raw[k][i] = settle_odd<T>(raw[k][i], c, width, there);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[k][i][e] = ok ? raw[k][i][e] : 0u;
            }
        }
}
template <typename T>
__device__ __forceinline__ void raw_parts(const u32x4v (&raw)[8 / kVec<T>],
                                          bf16x8 (&out)[kParts<T>]) {
    if constexpr (sizeof(T) == 2) {
        out[0] = __builtin_bit_cast(bf16x8, raw[0]);
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(raw[i / 4][i % 4]);
        split8<3>(x, out);
    }
}
template <typename T, int D, bool kWhole>
__device__ __forceinline__ void row_operand(const T *row, bool there, int width,
                                            bf16x8 (&out)[D / 16][kParts<T>]) {
    u32x4v raw[D / 16][8 / kVec<T>];
    load_row<T, D, kWhole>(row, there, width, raw);
    settle_row<T, D, kWhole>(there, width, raw);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) raw_parts<T>(raw[k], out[k]);
}

__device__ __forceinline__ bool finite_bits(uint32_t w, bool pair) {
    return (w & 0x7F800000u) != 0x7F800000u && !(pair && (w & 0x7F80u) == 0x7F80u);
}

// kRows x D values on their way to LDS by kThreads threads, kSteps 16-byte pieces each
template <typename T, int D, int kRows, int kThreads, bool kWhole> struct TileLoad {
    static constexpr int kPerRow = D / kVec<T>;
    static constexpr int kSteps = kRows * kPerRow / kThreads;
    static_assert(kRows * kPerRow % kThreads == 0, "pieces");
    u32x4v raw[kSteps];
    uint32_t there;  // a bit for each piece that exists (the others are zeroed in settle())
    uint32_t off[kSteps], columns;  // of load_all(): the pieces' bytes, and those that exist
    __device__ __forceinline__ static int tid() { return threadIdx.x % kThreads; }
    __device__ __forceinline__ static int row_of(int s) { return (s * kThreads + tid()) / kPerRow; }
    __device__ __forceinline__ static int col_of(int s) {
        return (s * kThreads + tid()) % kPerRow * kVec<T>;
    }
    // For tiles whose rows all exist, `stride` elements apart (kWhole; below 2^22)
    __device__ __forceinline__ void places(int64_t stride, int width) {
        places([&](int r) { return (uint32_t)r * (uint32_t)stride; }, width);
    }
    // or whose row r is at(r) elements from the first
    template <typename F> __device__ __forceinline__ void places(F at, int width) {
        columns = 0;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const bool ok = col_of(s) < width;
            off[s] = (at(row_of(s)) + (ok ? col_of(s) : 0)) * (uint32_t)sizeof(T);
            columns |= (uint32_t)ok << s;
        }
    }
    __device__ __forceinline__ void load_all(const T *base) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            __builtin_memcpy(&raw[s], reinterpret_cast<const char *>(base) + off[s], 16);
        there = columns;
    }
    // row_at(row): where the tile's row begins, nullptr if it does not exist; `any` is an address
    // that may be read
    template <typename F>
    __device__ __forceinline__ void load(F row_at, const T *any, int width) {
        there = 0;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const T *row = row_at(row_of(s));
            const int c = col_of(s);
            if constexpr (kWhole) {
                const bool ok = row != nullptr && c < width;
                __builtin_memcpy(&raw[s], ok ? row + c : any, 16);
                there |= (uint32_t)ok << s;
            } else {
                raw[s] = load_odd<T>(row, c, width, row != nullptr, any);
                there |= (uint32_t)(row != nullptr) << s;
            }
        }
    }
    // after the loads' wait, before store()
    __device__ __forceinline__ void settle(int width) {
        if constexpr (!kWhole) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
                raw[s] = settle_odd<T>(raw[s], col_of(s), width, there >> s & 1u);
            return;
        }
        if (there == (1u << kSteps) - 1u) return;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[s][i] = there >> s & 1u ? raw[s][i] : 0u;
    }
    // Values that are infinite or NaN to zero, and the first such row of each column, counted from
    // `first` on, to first_bad[column].  Where some rows of a product see a tile only in part, the
    // others' weight 0 times such a value would be NaN; what they are to those that do see them is
    // made up for at the end (FirstBad).
    __device__ __forceinline__ void put_bad_apart(int32_t first, int32_t *first_bad) {
        bool found = false;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) found |= !finite_bits(raw[s][i], sizeof(T) == 2);
        if (!found) return;
        for (int s = 0; s < kSteps; ++s) {
            uint32_t w[4];
            T e[kVec<T>];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = 0;
#pragma unroll
                for (int r = 0; r < kSteps; ++r) w[i] = r == s ? raw[r][i] : w[i];
            }
            __builtin_memcpy(e, w, 16);
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i)
                if ((__float_as_uint(to_f32(e[i])) & 0x7F800000u) == 0x7F800000u) {
                    e[i] = T(0);
                    atomicMin(first_bad + col_of(s) + i, first + row_of(s));
                }
            __builtin_memcpy(w, e, 16);
#pragma unroll
            for (int r = 0; r < kSteps; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) raw[r][i] = r == s ? w[i] : raw[r][i];
        }
    }
    __device__ __forceinline__ void store(bf16_t *tile) const {
        constexpr int kPlane = kRows * D;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = TileAt<D>::at(row_of(s), col_of(s));
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<u32x4v *>(tile + at) = raw[s];
            } else {
                uint32_t h[2], m[2], lo[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    split2(__uint_as_float(raw[s][2 * i]), __uint_as_float(raw[s][2 * i + 1]),
                           h[i], m[i], lo[i]);
                *reinterpret_cast<uint2 *>(tile + at) = uint2{h[0], h[1]};
                *reinterpret_cast<uint2 *>(tile + kPlane + at) = uint2{m[0], m[1]};
                *reinterpret_cast<uint2 *>(tile + 2 * kPlane + at) = uint2{lo[0], lo[1]};
            }
        }
    }
};

// kRows x D bf16 values straight to LDS, 16 bytes a lane: the pieces of a wave land behind each
// other, so that the rows' permutation (TileAt) is in what each lane asks for.  The compiler does
// not count these loads (it would wait for all of them before any LDS read): wait_direct() does.
template <int D, int kRows, int kThreads> struct DirectTile {
    static constexpr int kPerRow = D / 8, kSteps = kRows * kPerRow / kThreads;
    static_assert(kRows * kPerRow % kThreads == 0 && D % 64 == 0, "pieces");
    uint32_t off[kSteps];
    // row r is at(r) elements from the base
    template <typename F> __device__ __forceinline__ void places(F at) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int piece = s * kThreads + threadIdx.x, row = piece / kPerRow;
            const int in_row = piece % kPerRow * 8;
            const int col = TileAt<D>::at(row, in_row) - row * D;  // (the permutation is its own inverse)
            off[s] = (at(row) + (uint32_t)col) * 2u;
        }
    }
    // base, tile: the same in all lanes of a wave
    __device__ __forceinline__ void load(const bf16_t *base, const bf16_t *tile) const {
        typedef __attribute__((address_space(3))) const bf16_t *lds_p;
        const uint32_t to = (uint32_t)(uintptr_t)(lds_p)tile;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const uint32_t m0 = __builtin_amdgcn_readfirstlane(
                to + (uint32_t)(s * kThreads + 64 * wave_of_block()) * 16u);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                         :
                         : "s"(m0), "v"(off[s]), "s"(base)
                         : "memory", "m0");
        }
    }
    // Values of the tile, which has landed, as TileLoad::put_bad_apart has them
    __device__ __forceinline__ static void put_bad_apart(bf16_t *tile, int32_t first,
                                                         int32_t *first_bad) {
        for (int s = 0; s < kSteps; ++s) {
            const int piece = s * kThreads + threadIdx.x, row = piece / kPerRow;
            u32x4v w = *reinterpret_cast<const u32x4v *>(tile + piece * 8);
            if (finite_bits(w[0], true) && finite_bits(w[1], true) && finite_bits(w[2], true) &&
                finite_bits(w[3], true))
                continue;
            const int col = TileAt<D>::at(row, piece % kPerRow * 8) - row * D;
            bf16_t e[8];
            __builtin_memcpy(e, &w, 16);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((e[i] & 0x7F80u) == 0x7F80u) {
                    e[i] = 0;
                    atomicMin(first_bad + col + i, first + row);
                }
            __builtin_memcpy(&w, e, 16);
            *reinterpret_cast<u32x4v *>(tile + piece * 8) = w;
        }
    }
};
// `count` float32 values (64 at most) behind each other to LDS
__device__ __forceinline__ void direct_floats(const float *base, const float *to, int count) {
    typedef __attribute__((address_space(3))) const float *lds_p;
    const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_p)to);
    const int lane = threadIdx.x & 63;
    if (lane < count)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                     :
                     : "s"(m0), "v"((uint32_t)lane * 4u), "s"(base)
                     : "memory", "m0");
}
// until at most kLeft of this wave's loads are on their way
template <int kLeft> __device__ __forceinline__ void wait_direct() {
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kLeft) : "memory");
}

// A row's two halves joined, in both
__device__ __forceinline__ float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Where the keys of a tile lie: lane j looks up key first + j (j below kKeys), with look() well
// before settle().
struct KeyPlaces {
    int32_t page, at;  // -1: no such key
    uint64_t there;    // a bit for each key of the tile
    template <int kKeys>
    __device__ __forceinline__ void look(const SoftmaxArgs &p, const Sequence &s, int32_t first,
                                         int32_t end) {
        const int32_t key = first + (int32_t)(threadIdx.x & (kKeys - 1));
        page = -1;
        at = 0;
        if (key < end) {
            const int32_t i = divide(key, p.pages.page);
            at = key - i * (int32_t)p.pages.page.d;
            page = p.pages.table[(int64_t)s.b * p.pages.width + i];
        }
    }
    template <int kKeys> __device__ __forceinline__ void settle(const SoftmaxArgs &p) {
        if ((uint32_t)page >= (uint32_t)p.pages.n_pages) page = -1;
        there = __ballot(page >= 0);
        if constexpr (kKeys == 32) there &= 0xFFFFFFFFull;
    }
    template <typename T>
    __device__ __forceinline__ const T *row(const sbc_pages &x, int32_t head, int32_t j) const {
        const int32_t g = __shfl(page, j), a = __shfl(at, j);
        return g < 0 ? nullptr
                     : static_cast<const T *>(x.data) + g * x.page_stride + a * x.token_stride +
                           head * x.head_stride;
    }
};

// ---------------------------------------------------------------- softmax
constexpr float kLn2 = 0.69314718055994530942f;

// Rows' running softmax: a lane's row has its maximum m (in units of log 2, scaled), its
// own keys' part of the sum l, and its channels 32 t + 8 (r / 4) + 4 g + r % 4 of the sum of
// products.
template <int D> struct RowSums {
    floatx16 o[D / 32];
    float m, l;
    __device__ __forceinline__ RowSums() : m(-INFINITY), l(0.f) { clear(o); }
};

// The keys that a lane's row sees of 32 (bit 8 (r / 4) + r % 4 of the result is register r)
__device__ __forceinline__ uint32_t seen_bits(uint64_t there, int u, int32_t visible) {
    const int32_t n = clamp_i(visible - 32 * u, 0, 32);
    const uint32_t low = n == 32 ? 0xFFFFFFFFu : (1u << n) - 1u;
    return ((uint32_t)(there >> (32 * u)) & low) >> (4 * ((threadIdx.x & 63) >> 5));
}

// Scores x of kSub x 32 keys -> their weights, in place; the sums follow the maximum.  The
// maximum that weights refer to moves only where a score lies 2^8 above it (a weight then is
// at most 2^8, and rounded as a smaller one is), so that most tiles leave the sums alone.  Sums of
// products with values up to 2^119 / keys stay in range.  (To take larger ones, all weights could lie
// below 1 / keys: exponents that far from zero are rounded by 2^-20, and o and lse of float32
// inputs with them.  Or a workgroup whose sums are not finite could go through its keys again like
// that: 20 to 50 registers more in every instance, a wave a SIMD less of 64 bf16 channels.)
template <int D, int kSub>
__device__ __forceinline__ void softmax_weights(floatx16 (&x)[kSub], float scale2, RowSums<D> &s) {
    float top = fmaxf(x[0][0], x[kSub - 1][15]);
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int r = 0; r < 16; r += 2) top = fmaxf(fmaxf(top, x[u][r]), x[u][r + 1]);
    top = halves_max(top) * scale2;
    if (__any(top > s.m + 8.f)) {
        const float m = fmaxf(s.m, top);
        const float f = m == s.m ? 1.f : __builtin_amdgcn_exp2f(s.m - m);
        s.m = m;
        s.l *= f;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s.o[t][r] *= f;
    }
    const float m = s.m == -INFINITY ? 0.f : s.m;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            x[u][r] = __builtin_amdgcn_exp2f(fmaf(x[u][r], scale2, -m));
            sum[r % 4] += x[u][r];
        }
    s.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// What may move past a point of the schedule: anything but matrix products and LDS reads,
// which are to stay in the order that the loops below give them.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x6 | 0x70); }

// x[j] += the rows that read(k, j) gives of step k times operand j, kJobs products side by side.
// The rows of kAhead steps are on their way from LDS while a step's products run: read where
// they are used, a wave waited out LDS' latency every two products.
template <typename T, int D, int kJobs, int kAhead, typename Read, typename Operand>
__device__ __forceinline__ void row_products(Read read, Operand operand, floatx16 (&x)[kJobs]) {
    constexpr int NP = kParts<T>, kSteps = D / 16;
    bf16x8 f[kAhead][kJobs][NP];
#pragma unroll
    for (int k = 0; k < kAhead && k < kSteps; ++k)
#pragma unroll
        for (int j = 0; j < kJobs; ++j) read(k, j, f[k][j]);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        keep_order();
#pragma unroll
        for (int j = 0; j < kJobs; ++j) mma32<NP, NP>(f[k % kAhead][j], operand(k, j), x[j]);
        if (k + kAhead < kSteps) {
            keep_order();
#pragma unroll
            for (int j = 0; j < kJobs; ++j) read(k + kAhead, j, f[k % kAhead][j]);
        }
    }
    __builtin_amdgcn_s_setprio(0);
}

// acc[t] += columns 32 t .. + 31 of the tile, transposed, times weights by rows: k-step h takes
// rows 16 h .. + 15.  First read(), which may lie well before, then add().
// kBuffers: steps that are in registers at once, 2 or 1.  kWeights: the weights' parts.  A bf16
// call's softmax weights have one (over a cache of few rows two, kFewWeights): each is rounded by
// up to 2^-8, independently of the others, beside the output's own rounding of as much.
template <typename T, int D, int kRows, int kBuffers = 2, int kWeights = kParts<T>>
struct ColumnProducts {
    static constexpr int NP = kParts<T>, kSteps = kRows / 16;
    bf16x8 f[kBuffers][D / 32][NP];
    // step h of the rows that begin `first` (a multiple of 32) into a tile
    __device__ __forceinline__ void fetch(const bf16_t *tile, int plane, int first,
                                          const LaneAt32<D> &at, int h) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t) frag_col32<D, NP>(tile, plane, first / 16 + h, t, at, f[h % kBuffers][t]);
    }
    __device__ __forceinline__ void read(const bf16_t *tile, int plane, int first,
                                         const LaneAt32<D> &at) {
        fetch(tile, plane, first, at, 0);
        keep_order();
    }
    __device__ __forceinline__ void add(const floatx16 (&x)[kRows / 32], const bf16_t *tile,
                                        int plane, int first, const LaneAt32<D> &at,
                                        floatx16 (&acc)[D / 32]) {
#pragma clang fp contract(off)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int h = 0; h < kSteps; ++h) {
            if (kBuffers == 2 && h + 1 < kSteps) fetch(tile, plane, first, at, h + 1);
            bf16x8 w[kWeights];
            frag_regs<kWeights>(x[h / 2], h % 2, w);
            keep_order();
#pragma unroll
            for (int t = 0; t < D / 32; ++t) mma32<NP, kWeights>(f[h % kBuffers][t], w, acc[t]);
            keep_order();
            if (kBuffers == 1 && h + 1 < kSteps) fetch(tile, plane, first, at, h + 1);
        }
        __builtin_amdgcn_s_setprio(0);
    }
};

// Four channels of an output's row: columns c .. + 3 of `width`
template <typename T, bool kWhole>
__device__ __forceinline__ void put4(T *row, int c, int width, const float (&x)[4]) {
    T raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = from_f32<T>(x[i]);
    if constexpr (kWhole) {
        if (c < width) __builtin_memcpy(row + c, raw, sizeof(raw));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < width) row[c + i] = raw[i];
    }
}

// f(D) with D the channels' tile as a constant
template <typename F> void softmax_dispatch(int32_t d, F f) {
    if (d <= 32)
        f(std::integral_constant<int, 32>{});
    else if (d <= 64)
        f(std::integral_constant<int, 64>{});
    else if (d <= 96)
        f(std::integral_constant<int, 96>{});
    else
        f(std::integral_constant<int, 128>{});
}

}  // namespace sbc
