// Both gradients behind the tokens, dk and dv, in one pass back along the sequences
// (attention.hpp), for states of up to 64 x 64.
//
//   dk: a = v, b = dO, c = q      dv: a = k, b = q, c = dO
//
// share the tiles of q and dO, the decays, and the state R = sum D q dO^T [dk, dv]
// (dk_j takes R v_j, dv_j takes R^T k_j): its columns lie in LDS one after another,
// read along for R^T k and across, by the transposing reads, for R v.  As passes of
// their own they stage the tiles, decay and update the state twice.
#pragma once

#include "attention_kernels.hpp"

namespace sbc {
namespace {

struct GradPass {
    AttnPass p;  // b = q, c = dO, da = dk, dc = dv, tiles = 1; x is not read
    sbc_heads k, v, dk, dv;
};

// kDots: dk's part of the rates' gradient, as in attn_pass_kernel (2) against k; the pairs
// of a chunk have both of their products here
template <typename T, int DK, int DV, bool kWhole, bool kDots>
__device__ __forceinline__ void grad_body(const GradPass &args, int block,
                                          PassShared<T, DK, DV, 3> &lds) {
#pragma clang fp contract(off)
    using S = StateTiles<DK, DV>;
    constexpr int NP = kParts<T>;
    constexpr int NS = 3;                        // parts of the state
    constexpr int NO = sizeof(T) == 4 ? 3 : 2;   // of what reaches the outputs alone
    constexpr bool kRev = true;
    const AttnPass &p = args.p;
    bf16_t *const qt = lds.tiles, *const gt = lds.tiles + NP * kChunk * DK;
    bf16_t *const st = lds.tiles + NP * kChunk * (DK + DV);
    int32_t *const tj = lds.tj;
    float *const wj = lds.wj;
    const LaneAt<DK> at_k;
    const LaneAt<DV> at_v;
    const int at_mine = at_v.col(S::col0() / 16);
    const int head = block % p.heads;
    const int seg = block / p.heads;
    const int32_t g0 = seg * p.seg_len;
    const int32_t g1 = seg == p.n_seg - 1 ? p.n : g0 + p.seg_len;
    const float rate = p.rates[head], rate2 = rate * kLog2E;
    const int wave = wave_of_block(), l = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    const int mine = 16 * wave + l;  // this lane's token of a chunk
    const Rows<T> rk(args.k, head, 0), rv(args.v, head, 0), rq(p.b, head, 0), rg(p.c, head, 0);
    const Rows<T> rdk(args.dk, head, 0), rdv(args.dv, head, 0);
    Staged<T, DK, kWhole, kRev> sq(rq, p.da);
    Staged<T, DV, kWhole, kRev> sg(rg, p.dc);
    RowFrag<T, DK, kWhole, kRev, true> sk;
    RowFrag<T, DV, kWhole, kRev, true> sv;
    double slope = 0.0;

    for (int32_t b = first_from(p, g1) - 1; b >= 0; --b) {
        const int32_t s = split_at(p, b), e = split_at(p, b + 1);
        if (e <= g0) break;
        const int32_t lo = s > g0 ? s : g0, hi = e < g1 ? e : g1;
        const bool came_in = e > g1 && seg < p.n_seg - 1;
        const int32_t length = hi > lo ? hi - lo : 0;
        if (length == 0) continue;

        int32_t t_next = 0;
        const int32_t chunks = (length + kChunk - 1) / kChunk;
        // the pass' chunk i (cut from the piece's first token on, as in attn_pass_kernel)
        auto lowest_of = [&](int32_t i) { return lo + (chunks - 1 - i) * kChunk; };
        auto count_from = [&](int32_t lowest) {
            return hi - lowest < kChunk ? hi - lowest : kChunk;
        };
        auto fetch = [&](int32_t i) {
            const int32_t lowest = lowest_of(i);
            const int count = count_from(lowest);
            sq.load(rq, lowest, count, p.da);
            sg.load(rg, lowest, count, p.dc);
            sk.load(rk, lowest, count, p.da, mine);
            sv.load(rv, lowest, count, p.dc, mine);
            if (threadIdx.x < kChunk) {
                const int l = (int)threadIdx.x < count ? threadIdx.x : 0;
                t_next = time_at(p, lowest + count - 1 - l);
            }
        };
        fetch(0);

        floatx4 acc[S::kTiles];
        bool some = came_in;  // whether there is a state
        int32_t ref = time_at(p, came_in ? g1 : hi - 1);  // its time
        {
            const float *from = p.carry + ((int64_t)seg * p.heads + head) * p.state_stride;
            const int col = S::col(), row0 = in_loop(S::row(0));
#pragma unroll
            for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = row0 + 16 * u + r;
                    acc[u][r] = some && row < p.da && col < p.dc ? from[row * p.dc + col] : 0.f;
                }
        }

        for (int32_t i = 0; i < chunks; ++i) {
            const int32_t lowest = lowest_of(i);
            const int count = count_from(lowest);
            const bool more = i + 1 < chunks;
            const bool there = mine < count;

            __syncthreads();  // the last chunk's tiles are done with
            if (threadIdx.x < kChunk) {
                const int32_t last = __shfl(t_next, count - 1);  // (the first wave has all 64)
                tj[threadIdx.x] = t_next;
                wj[threadIdx.x] =
                    (int)threadIdx.x < count ? decay(rate2, elapsed<kRev>(last, t_next)) : 0.f;
            }
            sq.store(qt, count, p.da);
            sg.store(gt, count, p.dc);
            if (some) store_state<DK, DV, NS>(st, acc);
            bf16x8 ak[DK / 32][NP], av[DV / 32][NP];
            sk.parts(ak, count, p.da, mine);
            sv.parts(av, count, p.dc, mine);
            __syncthreads();
            if (more) fetch(i + 1);

            const int32_t t_mine = tj[mine], t_last = __builtin_amdgcn_readfirstlane(tj[count - 1]);
            const float since = decay(rate2, elapsed<kRev>(t_mine, ref)) * p.scale;
            const int64_t token = lowest + (there ? count - 1 - mine : 0);
            // Products of one of the tiles with the lane's row, of the tokens 16 kt + 4 g + r
            // up to the lane's own
            auto products = [&](auto width, const bf16_t *tile, const auto &at, const auto &row,
                                float(&x)[kChunk / 16][4]) {
                constexpr int D = decltype(width)::value;
#pragma unroll
                for (int kt = 0; kt < kChunk / 16; ++kt) {
                    floatx4 d{0.f, 0.f, 0.f, 0.f};
                    if (kt <= wave) {
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) {
                            bf16x8 f[NP];
                            frag_row_split<D, NP>(tile, kChunk * D, kt, k, at, f);
                            mma<NP, NP>(f, row[k], d);
                        }
                        if (kt == wave) {
                            const int behind = in_loop(l - 4 * g);
#pragma unroll
                            for (int r = 0; r < 4; ++r) d[r] = r <= behind ? d[r] : 0.f;
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[kt][r] = d[r];
                }
            };
            // x = D dO . v and w = D q . k, and the pairs' own part of the rates' gradient
            float x[kChunk / 16][4], w[kChunk / 16][4], pairs = 0.f;
            products(std::integral_constant<int, DV>{}, gt, at_v, av, x);
            products(std::integral_constant<int, DK>{}, qt, at_k, ak, w);
#pragma unroll
            for (int kt = 0; kt < kChunk / 16; ++kt) {
                if (kt > wave) break;  // (both are 0 from there on)
                const int4 t = *reinterpret_cast<const int4 *>(tj + 16 * kt + 4 * g);
                const int32_t tk[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float dt = elapsed<kRev>(t_mine, tk[r]);
                    const float d = decay(rate2, dt);
                    w[kt][r] *= d;
                    if constexpr (kDots) pairs = fmaf(w[kt][r] * dt, x[kt][r], pairs);
                    x[kt][r] *= d;
                }
            }
            const RowOut<T, kWhole> out_k(rdk, token, p.da, there), out_v(rdv, token, p.dc, there);
            {  // dv
                bf16x8 px[kChunk / 32][NO];
#pragma unroll
                for (int s2 = 0; s2 < kChunk / 32; ++s2)
                    split8<NO>(reinterpret_cast<const float(&)[8]>(w[2 * s2]), px[s2]);
#pragma unroll
                for (int ti = 0; ti < DV / 16; ++ti) {
                    floatx4 o{0.f, 0.f, 0.f, 0.f}, in = o;
                    if (some) {
#pragma unroll
                        for (int k = 0; k < DK / 32; ++k) {
                            bf16x8 sf[NO];
                            frag_row_split<DK, NO>(st, DK * DV, ti, k, at_k, sf);
                            mma<NO, NP>(sf, ak[k], in);
                        }
                    }
#pragma unroll
                    for (int s2 = 0; s2 < kChunk / 32; ++s2) {
                        if (2 * s2 > wave) break;
                        bf16x8 cf[NP];
                        frag_col<DV, NP>(gt, kChunk * DV, s2, at_v.col(ti), cf);
                        mma<NP, NO>(cf, px[s2], o);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[r] = fmaf(o[r], p.scale, in[r] * since);
                    out_v.put(ti, o);
                }
            }
            {  // dk, and its products with k, whose channels `ak` holds
                bf16x8 py[kChunk / 32][NO];
#pragma unroll
                for (int s2 = 0; s2 < kChunk / 32; ++s2)
                    split8<NO>(reinterpret_cast<const float(&)[8]>(x[2 * s2]), py[s2]);
                float dot = 0.f;
#pragma unroll
                for (int ti = 0; ti < DK / 16; ++ti) {
                    floatx4 o{0.f, 0.f, 0.f, 0.f}, in = o;
                    if (some) {
#pragma unroll
                        for (int k = 0; k < DV / 32; ++k) {
                            bf16x8 sf[NS];
                            frag_col<DK, NS>(st, DK * DV, k, at_k.col(ti), sf);
                            mma<NS, NP>(sf, av[k], in);
                        }
                    }
#pragma unroll
                    for (int s2 = 0; s2 < kChunk / 32; ++s2) {
                        if (2 * s2 > wave) break;
                        bf16x8 cf[NP];
                        frag_col<DK, NP>(qt, kChunk * DK, s2, at_k.col(ti), cf);
                        mma<NP, NO>(cf, py[s2], o);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        in[r] *= since;
                        if constexpr (kDots)
                            dot = fmaf(part_sum<NP>(ak[ti / 2], 4 * (ti % 2) + r), in[r], dot);
                        o[r] = fmaf(o[r], p.scale, in[r]);
                    }
                    out_k.put(ti, o);
                }
                if constexpr (kDots)  // (the chunk's end comes first in the pass' order)
                    slope += (double)dot * (double)elapsed<kRev>(t_mine, tj[0]) +
                             (double)pairs * (double)p.scale;
            }
            if (more) {
                if (some) decay_state(step_factor(rate, elapsed<kRev>(t_last, ref)), acc);
                add_chunk<T, DK, DV>(qt, gt, at_k, at_mine, wj, acc);
                some = true;
                ref = t_last;
            }
        }
    }
    if constexpr (kDots) put_slope(p, slope, 0, seg, head);
}

// (Three workgroups a CU in bf16.)
template <typename T, int DK, int DV, bool kWhole, bool kDots>
__global__ __launch_bounds__(kAttnThreads, sizeof(T) == 2 ? 3 : 1) void attn_grad_kernel(
    GradPass args) {
    __shared__ PassShared<T, DK, DV, 3> lds;
    grad_body<T, DK, DV, kWhole, kDots>(args, blockIdx.x, lds);
}

// All gradients in one launch, for problems whose passes leave CUs without work: dq's
// workgroups, then those of dk and dv together, or of dv and of dk.  kDots: with the
// rates' gradient.
template <typename T, int D, bool kDots>
__global__ __launch_bounds__(kAttnThreads) void attn_grads_kernel(AttnPass dq, GradPass both) {
    __shared__ PassShared<T, D, D, 3> lds;
    const int first = dq.n_seg * dq.heads * dq.tiles;
    if ((int)blockIdx.x < first)
        pass_body<T, D, D, true, false, 3, kDots ? 1 : 0>(dq, blockIdx.x, lds);
    else
        grad_body<T, D, D, true, kDots>(both, blockIdx.x - first, lds);
}
template <typename T, int D, bool kDots>
__global__ __launch_bounds__(kAttnThreads) void attn_wide_grads_kernel(AttnPass dq, AttnPass dv,
                                                                       AttnPass dk) {
    constexpr int NO = sizeof(T) == 4 ? 3 : 2;
    __shared__ PassShared<T, D, 64, 3> lds;
    const int first = dq.n_seg * dq.heads * dq.tiles, second = first + dv.n_seg * dv.heads * dv.tiles;
    if ((int)blockIdx.x < first)
        pass_body<T, D, 64, true, false, 3, kDots ? 1 : 0>(dq, blockIdx.x, lds);
    else if ((int)blockIdx.x < second)
        pass_body<T, D, 64, true, true, NO, 0>(dv, blockIdx.x - first,
                                               reinterpret_cast<PassShared<T, D, 64, NO> &>(lds));
    else
        pass_body<T, D, 64, true, true, 3, kDots ? 2 : 0>(dk, blockIdx.x - second, lds);
}

}  // namespace
}  // namespace sbc
