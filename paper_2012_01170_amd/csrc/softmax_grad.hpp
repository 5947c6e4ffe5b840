// The kernels of softmax attention's gradients (softmax.hpp).  With P the weights,
// delta_i = dO_i . o_i and dS = P (dO V^T - delta):
//     dq = scale dS k,   dk = scale dS^T q,   dv = P^T dO.
// One kernel goes along the keys for dq (and leaves delta), one along the rows for dk and
// dv, so that every sum has one owner and one order: seven products of a pair instead of the
// five that one pass with atomic sums for dq would take.
#pragma once

#include "softmax.hpp"

namespace sbc {

constexpr int kGradThreads = 256;

// dS' parts: of a bf16 call two (2^-17).  Its terms cancel in dq and dk, so that with one the
// roundings, 2^-8 of each, were up to 1.5 times what the outputs' own rounding leaves (dq of drawn
// problems: 2.6e-3 from float64 where rounding alone gives 1.8e-3).
template <typename T> constexpr int kGradParts = sizeof(T) == 4 ? 3 : 2;

// dq: a workgroup has 128 rows, 32 a wave, as softmax_tile_kernel.
template <typename T, int D> constexpr int kGradKeys = sizeof(T) == 4 && D > 64 ? 32 : 64;
// Waves a SIMD: the rows' operands and sums of wide heads in float32 fill its registers alone.  At
// two, heads of 64 float32 channels do not fit whole: 40 registers go to scratch in dq, 20 in dk and
// dv, 97 where all are made in one launch (the offsets of a tile's pieces; bf16 heads: none in dq, up to
// 14 in dk and dv, up to 82 in one launch).
template <typename T, int D> constexpr int kGradWaves = sizeof(T) == 4 && D > 64 ? 1 : 2;
template <typename T, int D> constexpr int kKeyGradWaves = sizeof(T) == 4 && D > 64 ? 1 : 2;

template <typename T, int D> struct RowGradShared {
    // (one array, so that both tiles are at constant distances from a lane's places)
    alignas(16) bf16_t tiles[2 * kParts<T> * kGradKeys<T, D> * D];
};
template <typename T, int D, bool kWhole>
__device__ __forceinline__ void row_grads(const SoftmaxArgs &p, int32_t block,
                                          RowGradShared<T, D> &lds) {
#pragma clang fp contract(off)
    constexpr int NP = kParts<T>, KB = kGradKeys<T, D>, kSub = KB / 32, kPlane = KB * D;
    bf16_t *const kt = lds.tiles, *const vt = lds.tiles + NP * kPlane;
    const int32_t head_k = block % p.kv_heads;
    const int32_t x = p.slots - 1 - block / p.kv_heads;
    const int32_t group = p.group.d;
    auto begin = [&](int32_t b) { return (int32_t)((int64_t)q_split(p, b) * group / 128) + b; };
    const int32_t b = sequence_of(p.n_batch, x, begin);
    if (b < 0) return;
    const Sequence s = sequence_at<false>(p, b);
    const int32_t r0 = (x - begin(b)) * 128, rows = s.lq * group;
    if (r0 >= rows) return;
    const int wave = wave_of_block(), lane = threadIdx.x & 63;
    const int32_t wave_row = r0 + 32 * wave, row = wave_row + (lane & 31);
    const bool there = row < rows;
    const int32_t token = divide(there ? row : rows - 1, p.group);
    const int32_t head = head_k * group + (there ? row - token * group : 0);
    const int32_t limit = s.limit(token, p.causal);
    auto limit_of = [&](int32_t r) {
        return s.limit(divide(r < rows ? r : rows - 1, p.group), p.causal);
    };
    const int32_t most = __builtin_amdgcn_readfirstlane(limit_of(r0 + 127));
    const int32_t wave_least = __builtin_amdgcn_readfirstlane(limit_of(wave_row));

    const int64_t place = s.q0 + token;
    bf16x8 q[D / 16][NP], g[D / 16][NP];
    float delta = 0.f;
    {
        u32x4v raw[D / 16][8 / kVec<T>], out[D / 16][8 / kVec<T>];
        row_operand<T, D, kWhole>(static_cast<const T *>(p.q.data) + place * p.q.token_stride +
                                      (int64_t)head * p.q.head_stride,
                                  there, p.dk, q);
        load_row<T, D, kWhole>(static_cast<const T *>(p.d_o.data) + place * p.d_o.token_stride +
                                   (int64_t)head * p.d_o.head_stride,
                               there, p.dv, raw);
        load_row<T, D, kWhole>(static_cast<const T *>(p.o.data) + place * p.o.token_stride +
                                   (int64_t)head * p.o.head_stride,
                               there, p.dv, out);
        settle_row<T, D, kWhole>(there, p.dv, raw);
        settle_row<T, D, kWhole>(there, p.dv, out);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            raw_parts<T>(raw[k], g[k]);
#pragma unroll
            for (int i = 0; i < 8 / kVec<T>; ++i) {
                float a[kVec<T>], c[kVec<T>];
                unpack<T>(__builtin_bit_cast(raw16, raw[k][i]), a);
                unpack<T>(__builtin_bit_cast(raw16, out[k][i]), c);
#pragma unroll
                for (int e = 0; e < kVec<T>; ++e) delta = fmaf(a[e], c[e], delta);
            }
        }
        delta = halves_sum(delta);
    }
    const int64_t flat = place * p.heads + head;
    // (of a row whose scores are all -inf no key has a weight)
    float lse2 = there ? p.lse_in[flat] * kLog2E : 0.f;
    if (lse2 == -INFINITY) lse2 = INFINITY;
    if (p.row_delta && there && lane < 32) {
        p.row_delta[packed_row(p, head_k, s.q0, row)] = delta;
        p.row_lse[packed_row(p, head_k, s.q0, row)] = lse2;
    }

    const T *const kbase =
        static_cast<const T *>(p.k.data) + s.k0 * p.k.token_stride + head_k * p.k.head_stride;
    const T *const vbase =
        static_cast<const T *>(p.v.data) + s.k0 * p.v.token_stride + head_k * p.v.head_stride;
    TileLoad<T, D, KB, kGradThreads, kWhole> sk, sv;
    if (kWhole) {
        sk.places(p.k.token_stride, p.dk);
        sv.places(p.v.token_stride, p.dv);
    }
    auto fetch = [&](int32_t k0) {
        if (kWhole && k0 + KB <= s.lk) {
            sk.load_all(kbase + k0 * p.k.token_stride);
            sv.load_all(vbase + k0 * p.v.token_stride);
            return;
        }
        sk.load([&](int r) { return k0 + r < s.lk ? kbase + (k0 + r) * p.k.token_stride : nullptr; },
                kbase, p.dk);
        sv.load([&](int r) { return k0 + r < s.lk ? vbase + (k0 + r) * p.v.token_stride : nullptr; },
                vbase, p.dv);
    };
    const LaneAt32<D> places;
    floatx16 acc[D / 32];
    clear(acc);
    if (most > 0) fetch(0);
    for (int32_t k0 = 0; k0 < most; k0 += KB) {
        __syncthreads();
        sk.settle(p.dk);
        sv.settle(p.dv);
        sk.store(kt);
        sv.store(vt);
        __syncthreads();
        if (k0 + KB < most) fetch(k0 + KB);
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const LaneAt32<D> at(places);
            floatx16 w[2];  // scores, and dO v
            clear(w);
            row_products<T, D, 2, 2>(
                [&](int k, int j, bf16x8(&f)[NP]) {
                    frag_row32<D, NP>(j ? vt : kt, kPlane, u, k, at, f);
                },
                [&](int k, int j) -> const bf16x8(&)[NP] { return j ? g[k] : q[k]; }, w);
            ColumnProducts<T, D, 32, 2, kGradParts<T>> keys;
            keys.read(kt, kPlane, 32 * u, at);
            const bool masked = k0 + 32 * u + 32 > wave_least;
            const uint32_t seen = masked ? seen_bits(~0ull, 0, limit - k0 - 32 * u) : ~0u;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float e = __builtin_amdgcn_exp2f(fmaf(w[0][r], p.scale2, -lse2));
                const float d = e * (w[1][r] - delta);
                w[0][r] = !masked || (seen >> (8 * (r / 4) + r % 4) & 1u) ? d : 0.f;
            }
            keys.add(reinterpret_cast<const floatx16(&)[1]>(w[0]), kt, kPlane, 32 * u, at, acc);
        }
    }
    if (!there) return;
    T *out = static_cast<T *>(p.dq.data) + place * p.dq.token_stride + (int64_t)head * p.dq.head_stride;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = acc[t][4 * j + i] * p.scale;
            put4<T, kWhole>(out, 32 * t + 8 * j + 4 * (lane >> 5), p.dk, y);
        }
}

template <typename T, int D, bool kWhole>
__global__ __launch_bounds__(kGradThreads, (kGradWaves<T, D>)) void softmax_dq_kernel(SoftmaxArgs p) {
    __shared__ RowGradShared<T, D> lds;
    row_grads<T, D, kWhole>(p, blockIdx.x, lds);
}

// dk and dv: a workgroup has 128 keys of one key head, 32 a wave, and goes through the
// rows that see them, every p.parts-th tile of rows from the part's own on (p.parts > 1:
// sums to part_dk and part_dv, which softmax_dkv_join_kernel adds).
//
// Where both sums and operands fit into half of a SIMD's registers, a workgroup makes both
// (kDk | kDv); else one half of the workgroups makes dk and the other dv, scores twice: a wave alone on
// its SIMD, without another's products to fill its waits, took longer (16384 tokens of 8 heads, 2
// key heads, of 128 bf16 channels, both from registers: 1760 .. 1890 us against 1700 .. 1730;
// with keys and values in LDS and 8 waves, 1600 .. 1670, with DirectTile apart, 1500 .. 1540).
constexpr int kGradCols = 128;
constexpr int kDk = 1, kDv = 2;
template <typename T, int D> constexpr int kGradRows = D > 64 || (sizeof(T) == 4 && D > 32) ? (D == 96 ? 64 : 32) : 64;
template <typename T, int D> constexpr bool kGradsApart = sizeof(T) * D > 128;

template <typename T, int D, int kBuffers = 1> struct KeyGradShared {
    static constexpr int NP = kParts<T>, RB = kGradRows<T, D>;
    alignas(16) bf16_t tiles[kBuffers * 2 * NP * RB * D];
    alignas(16) float lses[kBuffers * RB], deltas[kBuffers * RB];
};

// kOwnDelta: delta is made here from o, by 256 / RB neighbouring lanes a row.
// kDirect: whole tiles of rows go straight to LDS, two ahead, in three buffers: registers of
// a tile on its way reach one tile ahead only, which is less than a load takes (16384 tokens, 2
// key heads of 128 bf16 channels: 1720 -> 1536 us).
template <typename T, int D, bool kWhole, int kGrads, bool kOwnDelta, bool kDirect = false>
__device__ __forceinline__ void key_grads(const SoftmaxArgs &p, int32_t block,
                                          KeyGradShared<T, D, (kDirect ? 3 : 1)> &lds) {
#pragma clang fp contract(off)
    constexpr int NP = kParts<T>, RB = kGradRows<T, D>, kSub = RB / 32, kPlane = RB * D;
    constexpr bool kDoK = kGrads & kDk, kDoV = kGrads & kDv;
    static_assert(!kDirect || (NP == 1 && kWhole && !kOwnDelta), "direct");
    const int32_t head_k = block % p.kv_heads;
    const int32_t part = block / p.kv_heads % p.parts;
    const int32_t x = block / p.kv_heads / p.parts;
    const int32_t group = p.group.d;
    auto begin = [&](int32_t b) { return k_split(p, b) / kGradCols + b; };
    const int32_t b = sequence_of(p.n_batch, x, begin);
    if (b < 0) return;
    const Sequence s = sequence_at<false>(p, b);
    const int32_t c0 = (x - begin(b)) * kGradCols;
    if (c0 >= s.lk) return;
    const int wave = wave_of_block(), lane = threadIdx.x & 63;
    const int32_t wave_key = c0 + 32 * wave, key = wave_key + (lane & 31);
    const bool there = key < s.lk;

    bf16x8 kf[D / 16][NP], vf[D / 16][NP];
    {
        const int64_t at = s.k0 + (there ? key : s.lk - 1);
        row_operand<T, D, kWhole>(static_cast<const T *>(p.k.data) + at * p.k.token_stride +
                                      head_k * p.k.head_stride,
                                  there, p.dk, kf);
        if constexpr (kDoK)
            row_operand<T, D, kWhole>(static_cast<const T *>(p.v.data) + at * p.v.token_stride +
                                          head_k * p.v.head_stride,
                                      there, p.dv, vf);
    }
    // the rows: from the first token that sees key c0 on
    const int32_t rows = s.lq * group;
    int32_t t0 = p.causal ? c0 - (s.lk - s.lq) : 0;
    if (t0 < 0) t0 = 0;
    const int32_t from = t0 < s.lq ? t0 * group / RB * RB : rows;
    // From the last rows back: the workgroups that run at a time then read the same rows, whichever
    // keys they begin with, and find them in the XCDs' caches (16384 tokens, 2 key heads of 128
    // bf16 channels: 1692 us from the first row that sees a workgroup's keys on, reading 6.9 GB; 1636).
    const int32_t step = RB * p.parts;

    const T *const qbase = static_cast<const T *>(p.q.data) + s.q0 * p.q.token_stride +
                           (int64_t)head_k * group * p.q.head_stride;
    const T *const gbase = static_cast<const T *>(p.d_o.data) + s.q0 * p.d_o.token_stride +
                           (int64_t)head_k * group * p.d_o.head_stride;
    TileLoad<T, D, RB, kGradThreads, kWhole> sq, sg;
    DirectTile<(kDirect ? D : 64), (kDirect ? RB : 64), kGradThreads> dq, dg;
    float next_lse = 0.f, next_delta = 0.f;
    constexpr int kAcross = kOwnDelta ? kGradThreads / RB : 1, kMine = D / kAcross;
    const int stat_row = threadIdx.x / kAcross;
    u32x4v next_g[kMine / kVec<T>], next_o[kMine / kVec<T>];  // (kOwnDelta)
    if (kWhole && p.even_rows) {
        auto place = [&](const sbc_heads &x) {
            return [&](int r) {
                const int32_t token = divide(r, p.group);
                return (uint32_t)token * (uint32_t)x.token_stride +
                       (uint32_t)(r - token * group) * (uint32_t)x.head_stride;
            };
        };
        if constexpr (kDirect) {
            dq.places(place(p.q));
            dg.places(place(p.d_o));
        } else {
            sq.places(place(p.q), p.dk);
            sg.places(place(p.d_o), p.dv);
        }
    }
    auto put_tile = [&](bf16_t *buffer) {
        sq.settle(p.dk);
        sg.settle(p.dv);
        sq.store(buffer);
        sg.store(buffer + NP * kPlane);
    };
    // what the rows' weights need, to place `slot`
    auto put_stats = [&](int slot) {
        if constexpr (kOwnDelta && kDoK) {
            next_delta = 0.f;
#pragma unroll
            for (int i = 0; i < kMine / kVec<T>; ++i) {
                float a[kVec<T>], c[kVec<T>];
                unpack<T>(__builtin_bit_cast(raw16, next_g[i]), a);
                unpack<T>(__builtin_bit_cast(raw16, next_o[i]), c);
#pragma unroll
                for (int e = 0; e < kVec<T>; ++e) next_delta = fmaf(a[e], c[e], next_delta);
            }
            next_delta = group_sum<kAcross>(next_delta);
        }
        if (threadIdx.x % kAcross == 0 && (kOwnDelta || threadIdx.x < RB)) {
            lds.lses[slot * RB + stat_row] = next_lse;
            lds.deltas[slot * RB + stat_row] = next_delta;
        }
    };
    // a tile into registers, or (kDirect) to LDS
    auto fetch = [&](int32_t r0, int slot) {
        auto row_of = [&](const T *base, const sbc_heads &x, int r) -> const T * {
            if (r0 + r >= rows) return nullptr;
            const int32_t token = divide(r0 + r, p.group);
            return base + token * x.token_stride + (r0 + r - token * group) * x.head_stride;
        };
        // (no weight for rows that do not exist)
        const int32_t r = r0 + stat_row;
        if constexpr (kOwnDelta) {
            next_lse = INFINITY;
            const int32_t token = divide(r < rows ? r : rows - 1, p.group);
            const int32_t head = head_k * group + (r < rows ? r - token * group : 0);
            if (r < rows) {
                next_lse = p.lse_in[(int64_t)(s.q0 + token) * p.heads + head] * kLog2E;
                if (next_lse == -INFINITY) next_lse = INFINITY;
            }
            if constexpr (kDoK) {
                const int c0 = threadIdx.x % kAcross * kMine;
                auto row = [&](const sbc_heads &x) {
                    return static_cast<const T *>(x.data) + (s.q0 + token) * x.token_stride +
                           (int64_t)head * x.head_stride;
                };
                const T *g = row(p.d_o), *o = row(p.o);
#pragma unroll
                for (int i = 0; i < kMine / kVec<T>; ++i) {
                    next_g[i] = load_elements<T>(g, c0 + i * kVec<T>, p.dv, r < rows);
                    next_o[i] = load_elements<T>(o, c0 + i * kVec<T>, p.dv, r < rows);
                }
            }
        } else if (threadIdx.x < RB && !(kDirect && r0 + RB <= rows)) {
            next_lse = INFINITY;
            next_delta = 0.f;
            if (r < rows) {
                next_lse = p.row_lse[packed_row(p, head_k, s.q0, r)];
                next_delta = p.row_delta[packed_row(p, head_k, s.q0, r)];
            }
        }
        if (kWhole && p.even_rows && r0 + RB <= rows) {
            const int32_t token = divide(r0, p.group);
            const T *const q0 = qbase + token * p.q.token_stride, *const g0 = gbase + token * p.d_o.token_stride;
            if constexpr (kDirect) {
                bf16_t *const buffer = lds.tiles + slot * 2 * kPlane;
                dq.load(q0, buffer);
                dg.load(g0, buffer + kPlane);
                // (each wave one of them, so that all have as many loads on their way)
                const int64_t at = packed_row(p, head_k, s.q0, r0);
                if (wave & 1)
                    direct_floats(p.row_delta + at, lds.deltas + slot * RB, RB);
                else
                    direct_floats(p.row_lse + at, lds.lses + slot * RB, RB);
            } else {
                sq.load_all(q0);
                sg.load_all(g0);
            }
        } else {
            sq.load([&](int r) { return row_of(qbase, p.q, r); }, qbase, p.dk);
            sg.load([&](int r) { return row_of(gbase, p.d_o, r); }, gbase, p.dv);
            if constexpr (kDirect) {
                put_tile(lds.tiles + slot * 2 * kPlane);
                put_stats(slot);
            }
        }
    };
    const LaneAt32<D> places;
    const int half = lane >> 5;
    floatx16 dk[D / 32], dv[D / 32];
    clear(dk);
    clear(dv);
    constexpr int kBuffer = 2 * NP * kPlane;
    int32_t r0 = from + ((rows - from + RB - 1) / RB - 1 - part) * RB;
    int slot = 0;
    if (r0 >= from) fetch(r0, 0);
    if (kDirect && r0 - step >= from) fetch(r0 - step, 1);
    for (; r0 >= from; r0 -= step) {
        if constexpr (kDirect) {
            // this tile's loads are done where none but the next one's are left (which is whole)
            if (r0 - step >= from)
                wait_direct<2 * decltype(dq)::kSteps + 1>();
            else
                wait_direct<0>();
            __syncthreads();  // (and the tile before has been read)
            if (r0 - 2 * step >= from) fetch(r0 - 2 * step, slot == 0 ? 2 : slot - 1);
        } else {
            __syncthreads();
            put_tile(lds.tiles);
            put_stats(0);
            __syncthreads();
            if (r0 - step >= from) fetch(r0 - step, 0);
        }
        const bf16_t *const qt = lds.tiles + slot * kBuffer, *const gt = qt + NP * kPlane;
        const float *const lses = lds.lses + slot * RB, *const deltas = lds.deltas + slot * RB;
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const LaneAt32<D> at(places);
            // (limits do not fall along the rows that there are; the others see nothing, also not by
            // a product of their zeros with an infinity)
            auto limit_of = [&](int32_t r) {
                return r < rows ? s.limit(divide(r, p.group), p.causal) : 0;
            };
            const int32_t first = __builtin_amdgcn_readfirstlane(limit_of(r0 + 32 * u));
            floatx16 w[kDoK ? 2 : 1];  // scores, and dO v
            clear(w);
            row_products<T, D, (kDoK ? 2 : 1), (NP == 1 && !kDoK ? 4 : 2)>(
                [&](int k, int j, bf16x8(&f)[NP]) {
                    frag_row32<D, NP>(j ? gt : qt, kPlane, u, k, at, f);
                },
                [&](int k, int j) -> const bf16x8(&)[NP] { return j ? vf[k] : kf[k]; }, w);
            ColumnProducts<T, D, 32, (NP == 3 ? 1 : 2)> grads;
            ColumnProducts<T, D, 32, (NP == 3 ? 1 : 2), kGradParts<T>> queries;
            if constexpr (kDoV) grads.read(gt, kPlane, 32 * u, at);
            else queries.read(qt, kPlane, 32 * u, at);
            const bool masked = first < wave_key + 32 || r0 + 32 * u + 32 > rows;
            floatx16 e[1], ds[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 32 * u + 8 * j + 4 * half;
                const floatx4 lse4 = *reinterpret_cast<const floatx4 *>(lses + r);
                floatx4 delta4{0.f, 0.f, 0.f, 0.f};
                if (kDoK) delta4 = *reinterpret_cast<const floatx4 *>(deltas + r);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[0][4 * j + i] = __builtin_amdgcn_exp2f(fmaf(w[0][4 * j + i], p.scale2, -lse4[i]));
                    if constexpr (kDoK) ds[0][4 * j + i] = e[0][4 * j + i] * (w[1][4 * j + i] - delta4[i]);
                }
            }
            if (masked) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool ok = key < limit_of(r0 + 32 * u + 8 * j + 4 * half + i);
                        if constexpr (kDoV) e[0][4 * j + i] = ok ? e[0][4 * j + i] : 0.f;
                        if constexpr (kDoK) ds[0][4 * j + i] = ok ? ds[0][4 * j + i] : 0.f;
                    }
            }
            if constexpr (kDoV) grads.add(e, gt, kPlane, 32 * u, at, dv);
            if constexpr (kDoK) {
                if constexpr (kDoV) queries.read(qt, kPlane, 32 * u, at);
                queries.add(ds, qt, kPlane, 32 * u, at, dk);
            }
        }
        if constexpr (kDirect) slot = slot == 2 ? 0 : slot + 1;
    }
    if (!there) return;
    const int64_t place = s.k0 + key;
    const int64_t flat = ((int64_t)part * p.m + place) * p.kv_heads + head_k;
    auto put = [&](const floatx16(&acc)[D / 32], float scale, float *parts, const sbc_heads &out,
                   int32_t d) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = 32 * t + 8 * j + 4 * half;
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = acc[t][4 * j + i] * scale;
                if (p.parts > 1)
                    put4<float, kWhole>(parts + flat * d, c, d, y);
                else
                    put4<T, kWhole>(static_cast<T *>(out.data) + place * out.token_stride +
                                        head_k * out.head_stride,
                                    c, d, y);
            }
    };
    if constexpr (kDoK) put(dk, p.scale, p.part_dk, p.dk_out, p.dk);
    if constexpr (kDoV) put(dv, 1.f, p.part_dv, p.dv_out, p.dv);
}

template <typename T, int D, bool kWhole, bool kDirect>
__global__ __launch_bounds__(kGradThreads, (kKeyGradWaves<T, D>)) void softmax_dkv_kernel(SoftmaxArgs p) {
    __shared__ KeyGradShared<T, D, (kDirect ? 3 : 1)> lds;
    if constexpr (kGradsApart<T, D>) {
        const int32_t half = gridDim.x / 2;  // (dk first: it takes longer)
        if ((int32_t)blockIdx.x < half)
            key_grads<T, D, kWhole, kDk, false, kDirect>(p, blockIdx.x, lds);
        else
            key_grads<T, D, kWhole, kDv, false, kDirect>(p, blockIdx.x - half, lds);
    } else {
        key_grads<T, D, kWhole, kDk | kDv, false, kDirect>(p, blockIdx.x, lds);
    }
}

// All three in one launch, for small problems, where a launch is most of the time: dq's
// workgroups first, each of the others making the deltas that it needs (8 tokens of 4 heads of 64
// bf16 channels: 20 us a call with two launches, 16 with one).
template <typename T, int D, bool kWhole>
__global__ __launch_bounds__(kGradThreads, (kKeyGradWaves<T, D>)) void softmax_grads_kernel(
    SoftmaxArgs p, int32_t dq_blocks, int32_t dkv_blocks) {
    __shared__ union Shared {
        RowGradShared<T, D> rows;
        KeyGradShared<T, D> keys;
        __device__ Shared() {}
    } lds;
    const int32_t block = (int32_t)blockIdx.x - dq_blocks;
    if (block < 0)
        row_grads<T, D, kWhole>(p, blockIdx.x, lds.rows);
    else if constexpr (!kGradsApart<T, D>)
        key_grads<T, D, kWhole, kDk | kDv, true>(p, block, lds.keys);
    else if (block < dkv_blocks)
        key_grads<T, D, kWhole, kDk, true>(p, block, lds.keys);
    else
        key_grads<T, D, kWhole, kDv, true>(p, block - dkv_blocks, lds.keys);
}

// The parts' sums of dk (blockIdx.y 0) and dv (1), in the parts' order; keys that lie in no
// sequence have none and are left alone.
template <typename T>
__global__ __launch_bounds__(256) void softmax_dkv_join_kernel(SoftmaxArgs p) {
    const bool values = blockIdx.y != 0;
    const int32_t d = values ? p.dv : p.dk, pieces = (d + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t flat = i / pieces;
    const int c = (int)(i - flat * pieces) * 4;
    const int64_t total = (int64_t)p.m * p.kv_heads;
    if (flat >= total) return;
    const int32_t place = (int32_t)(flat / p.kv_heads), head = (int32_t)(flat - (int64_t)place * p.kv_heads);
    if (place < k_split(p, 0) || place >= k_split(p, p.n_batch)) return;
    const float *from = (values ? p.part_dv : p.part_dk) + flat * d + c;
    float y[4] = {0.f, 0.f, 0.f, 0.f};
    const int have = d - c;
#pragma unroll 4
    for (int part = 0; part < p.parts; ++part) {
        float z[4];
        load_f32<4>(from + part * total * d, have, z);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] += z[e];
    }
    const sbc_heads &out = values ? p.dv_out : p.dk_out;
    put4<T, false>(static_cast<T *>(out.data) + place * out.token_stride + head * out.head_stride, c, d, y);
}

}  // namespace sbc
