// The kernels of a pass (attention.hpp).
#pragma once

#include <type_traits>

#include "attention_host.hpp"

namespace sbc {
namespace {

// One segment's part of the state that it hands on: the sum over the tokens of
// the sequence that goes on past the segment's end (kRev: past its start), at
// the time of the last of them.  Grid: segments x heads x column tiles.  A
// sequence's tokens are taken from the end back, and no further than their decay
// lasts: the weights of earlier ones are exactly 0.
template <typename T, int DA, int DCT> struct StateShared {
    alignas(16) bf16_t tiles[kParts<T> * kChunk * (DA + DCT)];
    alignas(16) float wj[kChunk];
    float last_w;
};
template <typename T, int DA, int DCT, bool kWhole, bool kRev>
__device__ __forceinline__ void state_body(const AttnPass &p, int block,
                                           StateShared<T, DA, DCT> &lds) {
    using S = StateTiles<DA, DCT>;
    constexpr int NP = kParts<T>;
    bf16_t *const bt = lds.tiles, *const ct = lds.tiles + NP * kChunk * DA;
    float *const wj = lds.wj;
    const LaneAt<DA> at_b;
    const int at_c = LaneAt<DCT>().col(S::col0() / 16);
    const int tile = block % p.tiles;
    const int head = (block / p.tiles) % p.heads;
    const int seg = block / p.tiles / p.heads;
    const int32_t g0 = seg * p.seg_len;
    const int32_t g1 = seg == p.n_seg - 1 ? p.n : g0 + p.seg_len;
    const float rate = p.rates[head], rate2 = rate * kLog2E;
    const int dc0 = tile * DCT;
    const bool first = tile == 0 && threadIdx.x == 0;
    float *factor = p.factor + (int64_t)seg * p.heads + head;

    // the sequence that goes on, and its tokens here
    int32_t b, lo, hi;
    bool goes_on, passes;
    if constexpr (!kRev) {
        b = first_from(p, g1) - 1;
        goes_on = b >= 0 && split_at(p, b + 1) > g1;
        lo = goes_on ? split_at(p, b) : g1;
        passes = lo < g0 && seg > 0;
        lo = lo > g0 ? lo : g0;
        hi = g1;
    } else {
        b = first_from(p, g0) - 1;
        goes_on = b >= 0 && split_at(p, b + 1) > g0;
        hi = goes_on ? split_at(p, b + 1) : g0;
        passes = hi > g1 && seg < p.n_seg - 1;
        hi = hi < g1 ? hi : g1;
        lo = g0;
    }
    if (!goes_on || lo >= hi) {
        if (first) *factor = kFresh;
        return;
    }
    const int32_t end = time_at(p, kRev ? g0 : g1 - 1);  // the time of the sum
    if (first)
        *factor = !passes ? kFresh
                          : step_factor(rate, elapsed<kRev>(end, time_at(p, kRev ? g1 : g0 - 1)));

    floatx4 acc[S::kTiles];
#pragma unroll
    for (int u = 0; u < S::kTiles; ++u) acc[u] = floatx4{0.f, 0.f, 0.f, 0.f};
    // row l of a chunk is l tokens before the chunk's last in the pass' order
    const Rows<T> rb(p.b, head, 0), rc(p.c, head, dc0);
    Staged<T, DA, kWhole, !kRev> sb(rb, p.da);
    Staged<T, DCT, kWhole, !kRev> sc(rc, p.dc - dc0);
    int32_t t_next = 0;
    auto fetch = [&](int32_t at) {  // the chunk whose last token lies `at` before the end
        const int32_t left = hi - lo - at;
        const int count = left < kChunk ? left : kChunk;
        const int32_t lowest = kRev ? lo + at : hi - at - count;
        sb.load(rb, lowest, count, p.da);
        sc.load(rc, lowest, count, p.dc - dc0);
        if ((int)threadIdx.x < count)
            t_next = time_at(p, kRev ? lowest + threadIdx.x : lowest + count - 1 - threadIdx.x);
    };
    fetch(0);
    for (int32_t at = 0; at < hi - lo; at += kChunk) {
        const int count = hi - lo - at < kChunk ? hi - lo - at : kChunk;
        if (threadIdx.x < kChunk) {
            const int l = threadIdx.x;
            const float w = l < count ? decay(rate2, elapsed<kRev>(end, t_next)) : 0.f;
            wj[l] = w;
            if (l == count - 1) lds.last_w = w;
        }
        sb.store(bt, count, p.da);
        sc.store(ct, count, p.dc - dc0);
        __syncthreads();
        const bool spent = lds.last_w == 0.f;
        if (at + kChunk < hi - lo && !spent) fetch(at + kChunk);
        add_chunk<T, DA, DCT>(bt, ct, at_b, at_c, wj, acc);
        __syncthreads();
        if (spent) break;
    }
    const int64_t place = ((int64_t)seg * p.heads + head) * p.state_stride;
    const int col = dc0 + S::col();
    const float *s0 = nullptr;
    float kept = 0.f;
    if (!kRev && !passes && p.state_in) {
        s0 = p.state_in + ((int64_t)b * p.heads + head) * p.da * p.dc;
        kept = decay(rate2, elapsed<kRev>(end, p.t ? p.state_time[b] : lo - 1));
    }
    if (col < p.dc) {
#pragma unroll
        for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = S::row(u) + r;
                if (row < p.da) {
                    float v = acc[u][r];
                    if (s0) v += kept * s0[(int64_t)row * p.dc + col];
                    p.carry[place + (int64_t)row * p.carry_i + (int64_t)col * p.carry_j] = v;
                }
            }
    }
}

template <typename T, int DA, int DCT, bool kWhole, bool kRev>
__global__ __launch_bounds__(kAttnThreads) void attn_state_kernel(AttnPass p) {
    __shared__ StateShared<T, DA, DCT> lds;
    state_body<T, DA, DCT, kWhole, kRev>(p, blockIdx.x, lds);
}
// Both directions in one launch, the first half of the workgroups along the sequences
template <typename T, int DA, int DCT, bool kWhole>
__global__ __launch_bounds__(kAttnThreads) void attn_states_kernel(AttnPass along, AttnPass back) {
    __shared__ StateShared<T, DA, DCT> lds;
    const int half = gridDim.x / 2;
    if ((int)blockIdx.x < half)
        state_body<T, DA, DCT, kWhole, false>(along, blockIdx.x, lds);
    else
        state_body<T, DA, DCT, kWhole, true>(back, blockIdx.x - half, lds);
}

// The states that segments start from, from the sums that they hand on, in place:
// carry[next] = sum[g] + carry[g] decayed by factor[g], the first term alone where
// a sequence starts in g.  16 groups of 16 lanes share the segments of 4 x 16
// values: each joins its run of segments, the runs are joined in LDS, and each
// run is gone through again from what comes in.  (A place that nothing hands on
// to holds whatever its sum's place held; nothing starts from it.)
template <bool kRev> __device__ __forceinline__ void scan_body(const AttnPass &p) {
    __shared__ floatx4 sums[16][16];
    __shared__ float through[16];
    const int lane = threadIdx.x % 16, run = threadIdx.x / 16;
    const int head = blockIdx.y;
    const int64_t e = ((int64_t)blockIdx.x * 16 + lane) * 4;
    const bool there = e < p.state_stride;
    const int per = (p.n_seg + 15) / 16;
    const int s0 = run * per, s1 = s0 + per < p.n_seg ? s0 + per : p.n_seg;
    auto place = [&](int s) { return (int64_t)(kRev ? p.n_seg - 1 - s : s) * p.heads + head; };
    auto at = [&](int s) {
        return reinterpret_cast<floatx4 *>(p.carry + place(s) * p.state_stride + e);
    };
    auto step = [](const floatx4 &c, floatx4 sum, float f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += apply_factor(f, c[i]);
        return sum;
    };
    constexpr int kAhead = 8;
    floatx4 v[kAhead];
    float f[kAhead];
    auto fetch = [&](int s) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (s + k < s1) {
                v[k] = *at(s + k);
                f[k] = p.factor[place(s + k)];
            }
    };
    floatx4 c{0.f, 0.f, 0.f, 0.f};
    float f_run = 0.f;  // the run's decay
    if (there) {
        for (int s = s0; s < s1; s += kAhead) {
            fetch(s);
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (s + k < s1) {
                    c = step(c, v[k], f[k]);
                    f_run = join_factors(f_run, f[k]);
                }
        }
        sums[run][lane] = c;
        through[run] = f_run;
    }
    __syncthreads();
    if (!there) return;
    c = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < run; ++r) c = step(c, sums[r][lane], through[r]);
    for (int s = s0; s < s1; s += kAhead) {
        fetch(s);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (s + k < s1) {
                *at(s + k) = c;
                c = step(c, v[k], f[k]);
            }
    }
}

// The scan along (blockIdx.z 0) and back (1)
__global__ __launch_bounds__(256) void attn_scan_kernel(AttnPass along, AttnPass back) {
    if (blockIdx.z == 0)
        scan_body<false>(along);
    else
        scan_body<true>(back);
}

// This lane's part of the product of two states at the end of a segment: `acc`, at the
// time t_last of its last token, and the one that comes in from behind, p.behind (laid
// out alike), at the time of the next token
template <int DA, int DCT>
__device__ __forceinline__ double meet_behind(const AttnPass &p,
                                              const floatx4 (&acc)[StateTiles<DA, DCT>::kTiles],
                                              float rate2, int seg, int head, int dc0, int32_t g1,
                                              int32_t t_last) {
    using S = StateTiles<DA, DCT>;
    const float *behind = p.behind + ((int64_t)seg * p.heads + head) * p.state_stride;
    const int col = dc0 + S::col(), row0 = in_loop(S::row(0));
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = row0 + 16 * u + r;
            if (row < p.da && col < p.dc)
                sum = fmaf(acc[u][r], behind[row * p.carry_i + col * p.carry_j], sum);
        }
    return (double)(sum * p.scale * decay(rate2, elapsed<false>(time_at(p, g1), t_last)));
}

// The sum of a workgroup's lanes to its place in p.slope
__device__ __forceinline__ void put_slope(const AttnPass &p, double slope, int tile, int seg,
                                          int head) {
    __shared__ double sums[kWaves];
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) slope += __shfl_xor(slope, m);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = slope;
    __syncthreads();
    if (threadIdx.x == 0)
        p.slope[((int64_t)tile * p.n_seg + seg) * p.heads + head] =
            (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// The pass over one segment's tokens.  (Rows and times are read inside the segment, and
// beside it only where there is another, whatever the splits say.)  Grid: segments x
// heads x column tiles.
// Wave w has the chunk's tokens 16 w .. + 15 as columns of its products (b a^T,
// S^T a^T and c^T P^T: a lane then holds keys and channels of one token, the
// masked products P go from one product's result to the next one's operand
// without LDS), and its tiles of the state.  NS: parts that P and S are split
// into, two where they only reach bf16 outputs (2^-17 of them, beside the
// output's rounding of 2^-8; with three the forward of 300k tokens, 4 heads takes 249 us
// against 236, and is as far from float64).
//
// A product with a masked weight is 0 times c, and NaN where c is infinite or NaN.
// kCareful, the forward pass: a chunk with such values in c is taken token by token, so
// that none reaches a token before its own; looking for them takes 1 % of the forward
// (300k tokens in bf16, 4 heads: 236 us against 233).
//
// kDots: what the pass adds to the rates' gradient (attention_bwd.hip).  1, along the
// sequence: products of x with y's part from the state S, times the time since S, and
// with that of a second state, S1, whose terms are those of S times the time from their
// chunk's end (or the segment's start) to the time of S; S1 takes the place of S in LDS
// behind S's products.  2, back along it: products of x with y's part from the state,
// times the time from the token to its chunk's end, and with that within the chunk, with
// every pair's own gap.
template <typename T, int DA, int DCT, int NS> struct PassShared {
    // (one array, so that all tiles are at constant distances from a lane's places)
    alignas(16) bf16_t tiles[kParts<T> * kChunk * (DA + DCT) + NS * DCT * DA];
    alignas(16) int32_t tj[kChunk];
    alignas(16) float wj[kChunk];
    int32_t bad[2];  // of a chunk and the one before
};
template <typename T, int DA, int DCT, bool kWhole, bool kRev, int NS, int kDots,
          bool kCareful = false>
__device__ __forceinline__ void pass_body(const AttnPass &p, int block,
                                          PassShared<T, DA, DCT, NS> &lds) {
#pragma clang fp contract(off)
    using S = StateTiles<DA, DCT>;
    constexpr int NP = kParts<T>;
    bf16_t *const bt = lds.tiles, *const ct = lds.tiles + NP * kChunk * DA;
    bf16_t *const st = lds.tiles + NP * kChunk * (DA + DCT);
    int32_t *const tj = lds.tj;
    float *const wj = lds.wj;
    const LaneAt<DA> at_a;
    const LaneAt<DCT> at_c;
    const int at_mine = at_c.col(S::col0() / 16);
    const int tile = block % p.tiles;
    const int head = (block / p.tiles) % p.heads;
    const int seg = block / p.tiles / p.heads;
    const int32_t g0 = seg * p.seg_len;
    const int32_t g1 = seg == p.n_seg - 1 ? p.n : g0 + p.seg_len;
    const float rate = p.rates[head], rate2 = rate * kLog2E;
    const int dc0 = tile * DCT;
    const int wave = wave_of_block(), l = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    const int mine = 16 * wave + l;  // this lane's token of a chunk
    const Rows<T> ra(p.a, head, 0), rb(p.b, head, 0), rc(p.c, head, dc0), ry(p.y, head, dc0);
    Staged<T, DA, kWhole, kRev> sb(rb, p.da);
    Staged<T, DCT, kWhole, kRev> sc(rc, p.dc - dc0);
    RowFrag<T, DA, kWhole, kRev> sa;
    // (columns 16 ti + 4 g .. + 3: loaded with the others, since a load behind them would
    // wait for them all)
    RowFrag<T, DCT, kWhole, kRev, true> sx;
    const Rows<T> rx(p.x, head, dc0);
    double slope = 0.0;
    static_assert(!kCareful || (!kRev && kDots == 0), "single tokens: along the sequence, alone");
    int turn = 0;
    if (kCareful && threadIdx.x == 0) lds.bad[0] = lds.bad[1] = 0;  // (a barrier follows)

    const int32_t b_new = first_from(p, kRev ? g1 : g0);  // the first sequence that starts here
    int32_t b = b_new;
    if (kRev || (seg > 0 && b > 0 && split_at(p, b) > g0)) --b;  // or one that came in
    while (kRev ? b >= 0 : b < p.n_batch) {
        const int32_t s = split_at(p, b), e = split_at(p, b + 1);
        if (kRev ? e <= g0 : (b >= b_new && s >= g1 && seg != p.n_seg - 1)) break;
        const int32_t lo = s > g0 ? s : g0, hi = e < g1 ? e : g1;
        const bool came_in = kRev ? e > g1 && seg < p.n_seg - 1 : b < b_new;
        const bool ends = !kRev && e <= g1;
        const int32_t length = hi > lo ? hi - lo : 0;

        int32_t t_next = 0;
        // Chunks are cut from the piece's first token on, also where the pass goes back
        // (passes must agree on what is a chunk's own pair).
        int32_t singly_to = lo;  // up to here token by token
        auto count_from = [&](int32_t lowest) {
            if (kCareful && lowest < singly_to) return 1;
            return hi - lowest < kChunk ? hi - lowest : kChunk;
        };
        auto fetch = [&](int32_t lowest) {
            const int count = count_from(lowest);
            sb.load(rb, lowest, count, p.da);
            sc.load(rc, lowest, count, p.dc - dc0);
            sa.load(ra, lowest, count, p.da, mine);
            if constexpr (kDots > 0) sx.load(rx, lowest, count, p.dc - dc0, mine);
            if (threadIdx.x < kChunk) {
                const int l = (int)threadIdx.x < count ? threadIdx.x : 0;
                t_next = time_at(p, kRev ? lowest + count - 1 - l : lowest + l);
            }
        };
        const int32_t start = kRev ? lo + (length - 1) / kChunk * kChunk : lo;
        if (length > 0) fetch(start);

        const bool goes_on = kDots == 1 && e > g1 && seg < p.n_seg - 1;
        floatx4 acc[S::kTiles], acc1[S::kTiles];  // S, and of kDots 1 S1
        bool some = false, some1 = false;  // whether there is a state, and one in S1
        int32_t ref = 0;    // its time
        {
            const float *from = nullptr;
            int64_t si = 0, sj = 0;
            if (came_in) {
                from = p.carry + ((int64_t)seg * p.heads + head) * p.state_stride;
                si = p.carry_i;
                sj = p.carry_j;
                ref = time_at(p, kRev ? g1 : g0 - 1);
            } else if (!kRev && p.state_in) {
                from = p.state_in + ((int64_t)b * p.heads + head) * p.da * p.dc;
                si = p.dc;
                sj = 1;
                ref = p.t ? p.state_time[b] : lo - 1;
            } else if (length > 0) {
                ref = time_at(p, kRev ? hi - 1 : lo);
            }
            some = from != nullptr;
            const int col = dc0 + S::col(), row0 = in_loop(S::row(0));
#pragma unroll
            for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = row0 + 16 * u + r;
                    acc[u][r] = some && row < p.da && col < p.dc ? from[row * si + col * sj] : 0.f;
                    acc1[u][r] = 0.f;
                }
        }

        int32_t next;
        for (int32_t lowest = start; length > 0 && (kRev ? lowest >= lo : lowest < hi);
             lowest = next) {
            const int count = count_from(lowest);
            next = kRev ? lowest - kChunk : lowest + count;
            const bool more = kRev ? next >= lo : next < hi;
            const bool update = more || (ends && p.state_out);
            const bool there = mine < count;

            __syncthreads();  // the last chunk's tiles are done with
            if (threadIdx.x < kChunk) {
                const int32_t last = __shfl(t_next, count - 1);  // (the first wave has all 64)
                tj[threadIdx.x] = t_next;
                wj[threadIdx.x] =
                    (int)threadIdx.x < count ? decay(rate2, elapsed<kRev>(last, t_next)) : 0.f;
            }
            sb.store(bt, count, p.da);
            sc.store(ct, count, p.dc - dc0);
            if constexpr (kCareful) {
                if (sc.not_finite()) lds.bad[turn] = 1;
                if (threadIdx.x == 0) lds.bad[turn ^ 1] = 0;
            }
            if (some) store_state<DA, DCT, NS>(st, acc);
            bf16x8 a[DA / 32][NP];  // the rows of a, as an operand
            sa.parts(a, count, p.da, mine);
            bf16x8 xv[DCT / 32][NP];
            if constexpr (kDots > 0) sx.parts(xv, count, p.dc - dc0, mine);
            __syncthreads();
            if constexpr (kCareful) {
                const bool again = count > 1 && __builtin_amdgcn_readfirstlane(lds.bad[turn]);
                turn ^= 1;
                if (again) {
                    singly_to = lowest + count;
                    next = lowest;
                    fetch(lowest);
                    continue;
                }
            }
            if (more) fetch(next);

            // P^T: keys 16 kt + 4 g + r of the lane's token, masked and decayed
            const int32_t t_mine = tj[mine], t_last = __builtin_amdgcn_readfirstlane(tj[count - 1]);
            bf16x8 pf[kChunk / 32][NS], pf1[kChunk / 32][NS];
#pragma unroll
            for (int s2 = 0; s2 < kChunk / 32; ++s2) {
                float x[8], x1[8];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int kt = 2 * s2 + half;
                    floatx4 d{0.f, 0.f, 0.f, 0.f}, d1{0.f, 0.f, 0.f, 0.f};
                    if (kt <= wave) {
#pragma unroll
                        for (int k = 0; k < DA / 32; ++k) {
                            bf16x8 bk[NP];
                            frag_row<DA, NP>(bt, kChunk * DA, kt, k, at_a, bk);
                            mma<NP, NP>(bk, a[k], d);
                        }
                        const int4 t = *reinterpret_cast<const int4 *>(tj + 16 * kt + 4 * g);
                        const int32_t tk[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float dt = elapsed<kRev>(t_mine, tk[r]);
                            d[r] *= decay(rate2, dt);
                            if constexpr (kDots == 2) d1[r] = d[r] * dt;
                        }
                        if (kt == wave) {
                            const int behind = in_loop(l - 4 * g);
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                d[r] = r <= behind ? d[r] : 0.f;
                                if constexpr (kDots == 2) d1[r] = r <= behind ? d1[r] : 0.f;
                            }
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        x[4 * half + r] = d[r];
                        x1[4 * half + r] = d1[r];
                    }
                }
                split8<NS>(x, pf[s2]);
                if constexpr (kDots == 2) split8<NS>(x1, pf1[s2]);
            }
            const float since = decay(rate2, elapsed<kRev>(t_mine, ref)) * p.scale;
            const RowOut<T, kWhole> out(ry, (int64_t)lowest + (kRev ? count - 1 - mine : mine),
                                        p.dc - dc0, there);
            float dot = 0.f, dot1 = 0.f;
#pragma unroll
            for (int ti = 0; ti < DCT / 16; ++ti) {
                floatx4 o{0.f, 0.f, 0.f, 0.f}, o1 = o, in = o;
                if (some) {
#pragma unroll
                    for (int k = 0; k < DA / 32; ++k) {
                        bf16x8 sf[NS];
                        frag_row<DA, NS>(st, DCT * DA, ti, k, at_a, sf);
                        mma<NS, NP>(sf, a[k], in);
                    }
                }
#pragma unroll
                for (int s2 = 0; s2 < kChunk / 32; ++s2) {
                    if (2 * s2 > wave) break;
                    bf16x8 cf[NP];
                    frag_col<DCT, NP>(ct, kChunk * DCT, s2, at_c.col(ti), cf);
                    mma<NP, NS>(cf, pf[s2], o);
                    if constexpr (kDots == 2) mma<NP, NS>(cf, pf1[s2], o1);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    in[r] *= since;
                    o[r] = fmaf(o[r], p.scale, in[r]);
                }
                out.put(ti, o);
                if constexpr (kDots > 0) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = part_sum<NP>(xv[ti / 2], 4 * (ti % 2) + r);
                        dot = fmaf(x, in[r], dot);
                        if constexpr (kDots == 2) dot1 = fmaf(x, o1[r], dot1);
                    }
                }
            }
            if constexpr (kDots == 2)  // (the chunk's end comes first in the pass' order)
                slope += (double)dot * (double)elapsed<kRev>(t_mine, tj[0]) +
                         (double)dot1 * (double)p.scale;
            if constexpr (kDots == 1) {
                slope += (double)dot * (double)elapsed<kRev>(t_mine, ref);
                if (some1) {
                    __syncthreads();  // the products with S are done with
                    store_state<DA, DCT, NS>(st, acc1);
                    __syncthreads();
#pragma unroll
                    for (int ti = 0; ti < DCT / 16; ++ti) {
                        floatx4 in{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = 0; k < DA / 32; ++k) {
                            bf16x8 sf[NS];
                            frag_row<DA, NS>(st, DCT * DA, ti, k, at_a, sf);
                            mma<NS, NP>(sf, a[k], in);
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            dot1 = fmaf(part_sum<NP>(xv[ti / 2], 4 * (ti % 2) + r), in[r], dot1);
                    }
                    slope += (double)(dot1 * since);
                }
                if (some && (more || goes_on)) {
                    const float dt = elapsed<kRev>(t_last, ref), f = step_factor(rate, dt);
#pragma unroll
                    for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc1[u][r] = fmaf(dt, acc[u][r], acc1[u][r]);
                    decay_state(f, acc1);
                    some1 = true;
                }
            }
            if (update) {
                if (some) decay_state(step_factor(rate, elapsed<kRev>(t_last, ref)), acc);
                add_chunk<T, DA, DCT>(bt, ct, at_a, at_mine, wj, acc);
                some = true;
                ref = t_last;
            }
        }
        if constexpr (kDots == 1)
            if (goes_on && some1)
                slope += meet_behind<DA, DCT>(p, acc1, rate2, seg, head, dc0, g1,
                                              time_at(p, g1 - 1));
        if (ends && p.state_out) {
            const int col = dc0 + S::col(), row0 = in_loop(S::row(0));
            float *to = p.state_out + ((int64_t)b * p.heads + head) * p.da * p.dc;
#pragma unroll
            for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = row0 + 16 * u + r;
                    if (row < p.da && col < p.dc) to[(int64_t)row * p.dc + col] = acc[u][r];
                }
            if (p.time_out && tile == 0 && head == 0 && threadIdx.x == 0)
                p.time_out[b] =
                    length > 0 ? time_at(p, hi - 1) : (p.state_in ? p.state_time[b] : 0);
        }
        b += kRev ? -1 : 1;
    }
    if constexpr (kDots > 0) put_slope(p, slope, tile, seg, head);
}

// Workgroups a CU that the registers are to hold: three in bf16 up to 64 channels, but for
// the products of kDots 2; two in float32 with S1, which would take the second's registers
// (all gradients of 100k tokens, 4 heads: 543 us against 588).
template <typename T, int DA, int kDots>
constexpr int kPassBlocks = DA > 64 ? 1 : sizeof(T) == 2 ? (kDots < 2 ? 3 : 1) : kDots == 1 ? 2 : 1;
template <typename T, int DA, int DCT, bool kWhole, bool kRev, int NS, int kDots,
          bool kCareful = false>
__global__ __launch_bounds__(kAttnThreads, (kPassBlocks<T, DA, kDots>)) void attn_pass_kernel(
    AttnPass p) {
    __shared__ PassShared<T, DA, DCT, NS> lds;
    pass_body<T, DA, DCT, kWhole, kRev, NS, kDots, kCareful>(p, blockIdx.x, lds);
}

// ---------------------------------------------------------------- launches
// Calls f with the padded channels of a, the columns of a tile of c, and whether rows
// are whole 16-byte pieces.  (Rows that are not take the sizes up to 64 or 128.)
template <typename T, typename F> void pass_dispatch(int32_t da, int32_t dct, bool whole, F &&f) {
#define SBC_PASS(x, y, w)                                                        \
    f(std::integral_constant<int, x>{}, std::integral_constant<int, y>{},        \
      std::integral_constant<bool, w>{})
    if (!whole) {
        if (dct == 32 && da <= 64) SBC_PASS(64, 32, false);
        else if (dct == 32) SBC_PASS(128, 32, false);
        else if (da <= 64) SBC_PASS(64, 64, false);
        else SBC_PASS(128, 64, false);
    } else if (dct == 32) {
        if (da <= 32) SBC_PASS(32, 32, true);
        else if (da <= 64) SBC_PASS(64, 32, true);
        else if (da <= 96) SBC_PASS(96, 32, true);
        else SBC_PASS(128, 32, true);
    } else {
        if (da <= 32) SBC_PASS(32, 64, true);
        else if (da <= 64) SBC_PASS(64, 64, true);
        else if (da <= 96) SBC_PASS(96, 64, true);
        else SBC_PASS(128, 64, true);
    }
#undef SBC_PASS
}

inline dim3 scan_grid(const AttnPass &p) {
    return dim3((unsigned)grid_for(p.state_stride, 64), (unsigned)p.heads, 1);
}
inline dim3 pass_grid(const AttnPass &p) {
    return dim3((unsigned)((int64_t)p.n_seg * p.heads * p.tiles));
}

}  // namespace
}  // namespace sbc
