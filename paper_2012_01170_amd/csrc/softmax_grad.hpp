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

// dq: a workgroup has 128 rows, 32 a wave, as softmax_tile_kernel.
template <typename T, int D> constexpr int kGradKeys = sizeof(T) == 4 && D > 64 ? 32 : 64;
// Waves a SIMD: the rows' operands and sums of wide heads in float32 fill its registers alone
template <typename T, int D> constexpr int kGradWaves = sizeof(T) == 4 && D > 32 ? 1 : 2;
template <typename T, int D> constexpr int kKeyGradWaves = sizeof(T) == 4 && D > 32 ? 1 : 2;

template <typename T, int D, bool kWhole>
__global__ __launch_bounds__(kGradThreads, (kGradWaves<T, D>)) void softmax_dq_kernel(SoftmaxArgs p) {
#pragma clang fp contract(off)
    constexpr int NP = kParts<T>, KB = kGradKeys<T, D>, kSub = KB / 32, kPlane = KB * D;
    // (one array, so that both tiles are at constant distances from a lane's places)
    __shared__ __attribute__((aligned(16))) bf16_t lds[2 * NP * kPlane];
    bf16_t *const kt = lds, *const vt = lds + NP * kPlane;
    const int32_t head_k = blockIdx.x % p.kv_heads;
    const int32_t x = p.slots - 1 - blockIdx.x / p.kv_heads;
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
    if (there && lane < 32) p.delta[flat] = delta;
    // (of a row whose scores are all -inf no key has a weight)
    float lse2 = there ? p.lse_in[flat] * kLog2E : 0.f;
    if (lse2 == -INFINITY) lse2 = INFINITY;

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
        sk.settle();
        sv.settle();
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
            ColumnProducts<T, D, 32> keys;
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

// dk and dv: a workgroup has 128 keys of one key head, 32 a wave, and goes through the
// rows that see them, every p.parts-th tile of rows from the part's own on (p.parts > 1:
// sums to part_dk and part_dv, which softmax_dkv_join_kernel adds).
// Threads of a workgroup, 32 keys a wave: 
template <typename T, int D> constexpr int kKeyGradThreads = sizeof(T) == 2 && D > 96 ? 512 : 256;
// Of the workgroup's keys and values, how many are kept in LDS rather than in registers
#ifndef KK
#define KK 2
#endif
template <typename T, int D> constexpr int kKeptKeys = sizeof(T) == 2 && D > 96 ? KK : 0;
template <typename T, int D> constexpr int kGradCols = kKeyGradThreads<T, D> / 2;
template <typename T, int D> constexpr int kGradRows = D > 96 || (sizeof(T) == 4 && D > 64) ? 32 : 64;

template <typename T, int D, bool kWhole>
__global__ __launch_bounds__((kKeyGradThreads<T, D>), (kKeyGradWaves<T, D>)) void softmax_dkv_kernel(SoftmaxArgs p) {
#pragma clang fp contract(off)
    constexpr int NP = kParts<T>, RB = kGradRows<T, D>, kSub = RB / 32, kPlane = RB * D;
    __shared__ __attribute__((aligned(16))) bf16_t lds[2 * NP * kPlane];
    bf16_t *const qt = lds, *const gt = lds + NP * kPlane;
    constexpr int kKept = kKeptKeys<T, D> * kGradCols<T, D> * D;
    __shared__ __attribute__((aligned(16))) bf16_t kept[kKept > 0 ? kKept : 1];
    __shared__ __attribute__((aligned(16))) float lses[RB], deltas[RB];
    __shared__ __attribute__((aligned(16))) int32_t limits[RB];
    const int32_t head_k = blockIdx.x % p.kv_heads;
    const int32_t part = blockIdx.x / p.kv_heads % p.parts;
    const int32_t x = blockIdx.x / p.kv_heads / p.parts;
    const int32_t group = p.group.d;
    constexpr int kThreads = kKeyGradThreads<T, D>, kCols = kGradCols<T, D>;
    auto begin = [&](int32_t b) { return k_split(p, b) / kCols + b; };
    const int32_t b = sequence_of(p.n_batch, x, begin);
    if (b < 0) return;
    const Sequence s = sequence_at<false>(p, b);
    const int32_t c0 = (x - begin(b)) * kCols;
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
        row_operand<T, D, kWhole>(static_cast<const T *>(p.v.data) + at * p.v.token_stride +
                                      head_k * p.v.head_stride,
                                  there, p.dv, vf);
    }
    const LaneAt32<D> places;
    if constexpr (kKept > 0) {  // (each wave reads its own only)
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            *reinterpret_cast<bf16x8 *>(kept + 32 * wave * D + LaneAt32<D>::along(places.row0, 2 * k)) = kf[k][0];
            if (kKeptKeys<T, D> > 1)
                *reinterpret_cast<bf16x8 *>(kept + (kCols + 32 * wave) * D +
                                            LaneAt32<D>::along(places.row0, 2 * k)) = vf[k][0];
        }
    }
    // the rows: from the first token that sees key c0 on
    const int32_t rows = s.lq * group;
    int32_t t0 = p.causal ? c0 - (s.lk - s.lq) : 0;
    if (t0 < 0) t0 = 0;
    const int32_t from = t0 < s.lq ? t0 * group / RB * RB : rows;
    const int32_t step = RB * p.parts;

    const T *const qbase = static_cast<const T *>(p.q.data) + s.q0 * p.q.token_stride +
                           (int64_t)head_k * group * p.q.head_stride;
    const T *const gbase = static_cast<const T *>(p.d_o.data) + s.q0 * p.d_o.token_stride +
                           (int64_t)head_k * group * p.d_o.head_stride;
    TileLoad<T, D, RB, kThreads, kWhole> sq, sg;
    float next_lse = 0.f, next_delta = 0.f;
    int32_t next_limit = 0;
    if (kWhole && p.even_rows) {
        auto place = [&](const sbc_heads &x) {
            return [&](int r) {
                const int32_t token = divide(r, p.group);
                return (uint32_t)token * (uint32_t)x.token_stride +
                       (uint32_t)(r - token * group) * (uint32_t)x.head_stride;
            };
        };
        sq.places(place(p.q), p.dk);
        sg.places(place(p.d_o), p.dv);
    }
    auto fetch = [&](int32_t r0) {
        auto row_of = [&](const T *base, const sbc_heads &x, int r) -> const T * {
            if (r0 + r >= rows) return nullptr;
            const int32_t token = divide(r0 + r, p.group);
            return base + token * x.token_stride + (r0 + r - token * group) * x.head_stride;
        };
        if (kWhole && p.even_rows && r0 + RB <= rows) {
            const int32_t token = divide(r0, p.group);
            sq.load_all(qbase + token * p.q.token_stride);
            sg.load_all(gbase + token * p.d_o.token_stride);
        } else {
            sq.load([&](int r) { return row_of(qbase, p.q, r); }, qbase, p.dk);
            sg.load([&](int r) { return row_of(gbase, p.d_o, r); }, gbase, p.dv);
        }
        if (threadIdx.x < RB) {
            const int32_t r = r0 + threadIdx.x;
            // (no weight for rows that do not exist or have no keys)
            next_lse = INFINITY;
            next_delta = 0.f;
            next_limit = 0;
            if (r < rows) {
                const int32_t token = divide(r, p.group);
                const int64_t flat = (int64_t)(s.q0 + token) * p.heads + head_k * group + r - token * group;
                next_limit = s.limit(token, p.causal);
                if (next_limit > 0) {
                    next_lse = p.lse_in[flat] * kLog2E;
                    if (next_lse == -INFINITY) next_lse = INFINITY;
                    next_delta = p.delta[flat];
                }
            }
        }
    };
    const int half = lane >> 5;
    floatx16 dk[D / 32], dv[D / 32];
    clear(dk);
    clear(dv);
    int32_t r0 = from + part * RB;
    if (r0 < rows) fetch(r0);
    for (; r0 < rows; r0 += step) {
        __syncthreads();
        sq.settle();
        sg.settle();
        sq.store(qt);
        sg.store(gt);
        if (threadIdx.x < RB) {
            lses[threadIdx.x] = next_lse;
            deltas[threadIdx.x] = next_delta;
            limits[threadIdx.x] = next_limit;
        }
        __syncthreads();
        if (r0 + step < rows) fetch(r0 + step);
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const LaneAt32<D> at(places);
            // (limits do not fall along the rows that there are; the others' sums are infinite)
            const int32_t first = __builtin_amdgcn_readfirstlane(limits[32 * u]);
            floatx16 w[2];
            clear(w);
            if constexpr (kKept > 0) {
                const bf16_t *const own = kept + 32 * wave * D;
                bf16x8 f[4][1];
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    frag_row32<D, 1>(qt, kPlane, u, k, at, reinterpret_cast<bf16x8(&)[1]>(f[0]));
                    frag_row32<D, 1>(own, 0, 0, k, at, reinterpret_cast<bf16x8(&)[1]>(f[1]));
                    frag_row32<D, 1>(gt, kPlane, u, k, at, reinterpret_cast<bf16x8(&)[1]>(f[2]));
                    if (kKeptKeys<T, D> > 1)
                        frag_row32<D, 1>(own + kCols * D, 0, 0, k, at, reinterpret_cast<bf16x8(&)[1]>(f[3]));
                    mma32<1, 1>(f[0], f[1], w[0]);
                    if (kKeptKeys<T, D> > 1)
                        mma32<1, 1>(f[2], f[3], w[1]);
                    else
                        mma32<1, 1>(f[2], reinterpret_cast<const bf16x8(&)[1]>(vf[k][0]), w[1]);
                }
            } else {
                row_products<T, D, 2, 2>(
                    [&](int k, int j, bf16x8(&f)[NP]) {
                        frag_row32<D, NP>(j ? gt : qt, kPlane, u, k, at, f);
                    },
                    [&](int k, int j) -> const bf16x8(&)[NP] { return j ? vf[k] : kf[k]; }, w);
            }
            ColumnProducts<T, D, 32, (NP == 1 && D > 96 ? 1 : 2)> grads, queries;
            grads.read(gt, kPlane, 32 * u, at);
            const bool masked = first < wave_key + 32;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 32 * u + 8 * j + 4 * half;
                const floatx4 lse4 = *reinterpret_cast<const floatx4 *>(lses + r);
                const floatx4 delta4 = *reinterpret_cast<const floatx4 *>(deltas + r);
                typedef int32_t i4 __attribute__((ext_vector_type(4)));
                i4 limit4{0, 0, 0, 0};
                if (masked) limit4 = *reinterpret_cast<const i4 *>(limits + r);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(w[0][4 * j + i], p.scale2, -lse4[i]));
                    const float d = e * (w[1][4 * j + i] - delta4[i]);
                    const bool ok = !masked || key < limit4[i];
                    w[0][4 * j + i] = ok ? e : 0.f;
                    w[1][4 * j + i] = ok ? d : 0.f;
                }
            }
            grads.add(reinterpret_cast<const floatx16(&)[1]>(w[0]), gt, kPlane, 32 * u, at, dv);
            queries.read(qt, kPlane, 32 * u, at);
            queries.add(reinterpret_cast<const floatx16(&)[1]>(w[1]), qt, kPlane, 32 * u, at, dk);
        }
    }
    if (!there) return;
    const int64_t place = s.k0 + key;
    const int64_t flat = ((int64_t)part * p.m + place) * p.kv_heads + head_k;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 32 * t + 8 * j + 4 * half;
            float y[4], z[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = dk[t][4 * j + i] * p.scale;
                z[i] = dv[t][4 * j + i];
            }
            if (p.parts > 1) {
                put4<float, false>(p.part_dk + flat * p.dk, c, p.dk, y);
                put4<float, false>(p.part_dv + flat * p.dv, c, p.dv, z);
            } else {
                put4<T, kWhole>(static_cast<T *>(p.dk_out.data) + place * p.dk_out.token_stride +
                                    head_k * p.dk_out.head_stride,
                                c, p.dk, y);
                put4<T, kWhole>(static_cast<T *>(p.dv_out.data) + place * p.dv_out.token_stride +
                                    head_k * p.dv_out.head_stride,
                                c, p.dv, z);
            }
        }
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
