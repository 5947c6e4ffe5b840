// The kernels of a pass (attention.hpp).
#pragma once

#include <type_traits>

#include "attention.hpp"

namespace sbc {
namespace {

// One segment's part of the state that it hands on: the sum over the tokens of
// the sequence that goes on past the segment's end (kRev: past its start), at
// the time of the last of them.  Grid: segments x heads x column tiles.  A
// sequence's tokens are taken from the end back, and no further than their decay
// lasts: the weights of earlier ones are exactly 0.
template <typename T, int DA, int DCT, bool kRev>
__global__ __launch_bounds__(kAttnThreads) void attn_state_kernel(AttnPass p) {
    using S = StateTiles<DA, DCT>;
    constexpr int NP = kParts<T>;
    __shared__ alignas(16) bf16_t bt[NP * kChunk * DA];
    __shared__ alignas(16) bf16_t ct[NP * kChunk * DCT];
    __shared__ float wj[kChunk];
    __shared__ float last_w;
    const int tile = blockIdx.x % p.tiles;
    const int head = (blockIdx.x / p.tiles) % p.heads;
    const int seg = blockIdx.x / p.tiles / p.heads;
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
        passes = lo < g0;
        lo = lo > g0 ? lo : g0;
        hi = g1;
    } else {
        b = first_from(p, g0) - 1;
        goes_on = b >= 0 && split_at(p, b + 1) > g0;
        hi = goes_on ? split_at(p, b + 1) : g0;
        passes = hi > g1;
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
    Staged<T, DA> sb;
    Staged<T, DCT> sc;
    // chunks from the end of the sum: the last in the pass' order, from its last token
    for (int32_t done = 0; done < hi - lo; done += kChunk) {
        const int32_t left = hi - lo - done;
        const int count = left < kChunk ? left : kChunk;
        const int32_t newest = kRev ? lo + done : hi - 1 - done;
        // (token l of the chunk is l tokens before the newest in the pass' order)
        sb.template load<!kRev>(p.b, head, newest, count, 0, p.da);
        sc.template load<!kRev>(p.c, head, newest, count, dc0, p.dc);
        if (threadIdx.x < kChunk) {
            const int l = threadIdx.x;
            float w = 0.f;
            if (l < count)
                w = decay(rate2, elapsed<kRev>(end, time_at(p, (int32_t)token_of<!kRev>(newest, l))));
            wj[l] = w;
            if (l == count - 1) last_w = w;
        }
        sb.store(bt);
        sc.store(ct);
        __syncthreads();
        const bool spent = last_w == 0.f;
        add_chunk<T, DA, DCT>(bt, ct, wj, acc);
        __syncthreads();
        if (spent) break;
    }
    float *out = p.carry + ((int64_t)seg * p.heads + head) * p.state_stride;
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
                    out[(int64_t)row * p.carry_i + (int64_t)col * p.carry_j] = v;
                }
            }
    }
}

// The states that segments start from, from the sums that they hand on, in place:
// carry[next] = sum[g] + carry[g] decayed by factor[g], the first term alone where
// a sequence starts in g.  16 groups of 16 lanes share the segments of 4 x 16
// values: each joins its run of segments, the runs are joined in LDS, and each
// run is gone through again from what comes in.  (A place that nothing hands on
// to holds whatever its sum's place held; nothing starts from it.)
template <bool kRev>
__global__ __launch_bounds__(256) void attn_scan_kernel(float *__restrict__ carry,
                                                        const float *__restrict__ factor,
                                                        int32_t n_seg, int32_t heads,
                                                        int64_t state_stride) {
    __shared__ floatx4 sums[16][16];
    __shared__ float through[16][16];
    const int lane = threadIdx.x % 16, run = threadIdx.x / 16;
    const int head = blockIdx.y;
    const int64_t e = ((int64_t)blockIdx.x * 16 + lane) * 4;
    const bool there = e < state_stride;
    const int per = (n_seg + 15) / 16;
    const int s0 = run * per, s1 = s0 + per < n_seg ? s0 + per : n_seg;
    auto place = [&](int s) { return (int64_t)(kRev ? n_seg - 1 - s : s) * heads + head; };
    auto step = [](floatx4 c, floatx4 sum, float f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += apply_factor(f, c[i]);
        return sum;
    };
    constexpr int kAhead = 8;
    floatx4 c{0.f, 0.f, 0.f, 0.f};
    float f_run = 0.f;  // the run's decay
    if (there) {
        for (int s = s0; s < s1; s += kAhead) {
            floatx4 v[kAhead];
            float f[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (s + k < s1) {
                    v[k] = *reinterpret_cast<const floatx4 *>(carry + place(s + k) * state_stride + e);
                    f[k] = factor[place(s + k)];
                }
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (s + k < s1) {
                    c = step(c, v[k], f[k]);
                    f_run = join_factors(f_run, f[k]);
                }
        }
        sums[run][lane] = c;
        through[run][lane] = f_run;
    }
    __syncthreads();
    if (!there) return;
    c = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < run; ++r) c = step(c, sums[r][lane], through[r][lane]);
    for (int s = s0; s < s1; s += kAhead) {
        floatx4 v[kAhead];
        float f[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (s + k < s1) {
                v[k] = *reinterpret_cast<const floatx4 *>(carry + place(s + k) * state_stride + e);
                f[k] = factor[place(s + k)];
            }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (s + k < s1) {
                *reinterpret_cast<floatx4 *>(carry + place(s + k) * state_stride + e) = c;
                c = step(c, v[k], f[k]);
            }
    }
}

// The pass over one segment's tokens.  Grid: segments x heads x column tiles.
// Wave w has the chunk's tokens 16 w .. + 15 as columns of its products (b a^T,
// S^T a^T and c^T P^T: a lane then holds keys and channels of one token, the
// masked products P go from one product's result to the next one's operand
// without LDS), and its tiles of the state.  NS: parts that P and S are split
// into, two where they only reach bf16 outputs (2^-17 of them, beside the
// output's rounding of 2^-8).
template <typename T, int DA, int DCT, bool kRev, int NS>
__global__ __launch_bounds__(kAttnThreads) void attn_pass_kernel(AttnPass p) {
    using S = StateTiles<DA, DCT>;
    constexpr int NP = kParts<T>;
    __shared__ alignas(16) bf16_t bt[NP * kChunk * DA];
    __shared__ alignas(16) bf16_t ct[NP * kChunk * DCT];
    __shared__ alignas(16) bf16_t st[NS * DCT * DA];
    __shared__ alignas(16) int32_t tj[kChunk];
    __shared__ float wj[kChunk];
    const int tile = blockIdx.x % p.tiles;
    const int head = (blockIdx.x / p.tiles) % p.heads;
    const int seg = blockIdx.x / p.tiles / p.heads;
    const int32_t g0 = seg * p.seg_len;
    const int32_t g1 = seg == p.n_seg - 1 ? p.n : g0 + p.seg_len;
    const float rate = p.rates[head], rate2 = rate * kLog2E;
    const int dc0 = tile * DCT;
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    const int mine = 16 * wave + l;  // this lane's token of a chunk
    const T *a_data = static_cast<const T *>(p.a.data) + (int64_t)head * p.a.head_stride;
    T *y_data = static_cast<T *>(p.y.data) + (int64_t)head * p.y.head_stride + dc0;

    const int32_t b_new = first_from(p, kRev ? g1 : g0);  // the first sequence that starts here
    int32_t b = b_new;
    if (kRev || (b > 0 && split_at(p, b) > g0)) --b;      // or one that came in
    while (kRev ? b >= 0 : b < p.n_batch) {
        const int32_t s = split_at(p, b), e = split_at(p, b + 1);
        if (kRev ? e <= g0 : (b >= b_new && s >= g1 && seg != p.n_seg - 1)) break;
        const int32_t lo = s > g0 ? s : g0, hi = e < g1 ? e : g1;
        const bool came_in = kRev ? e > g1 : b < b_new;
        const bool ends = !kRev && e <= g1;
        const int32_t length = hi > lo ? hi - lo : 0;

        floatx4 acc[S::kTiles];
        bool some = false;  // whether there is a state
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
            const int col = dc0 + S::col();
#pragma unroll
            for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = S::row(u) + r;
                    acc[u][r] = some && row < p.da && col < p.dc ? from[row * si + col * sj] : 0.f;
                }
        }

        Staged<T, DA> sb;
        Staged<T, DCT> sc;
        auto fetch = [&](int32_t at) {  // the chunk `at` tokens into the piece
            const int32_t left = length - at;
            const int count = left < kChunk ? left : kChunk;
            const int32_t first = kRev ? hi - 1 - at : lo + at;
            sb.template load<kRev>(p.b, head, first, count, 0, p.da);
            sc.template load<kRev>(p.c, head, first, count, dc0, p.dc);
        };
        if (length > 0) fetch(0);
        for (int32_t at = 0; at < length; at += kChunk) {
            const int count = length - at < kChunk ? length - at : kChunk;
            const int32_t first = kRev ? hi - 1 - at : lo + at;
            const bool more = at + kChunk < length;
            const bool update = more || (ends && p.state_out);
            const int64_t token = token_of<kRev>(first, mine);
            const bool there = mine < count;
            const int32_t t_last = time_at(p, (int32_t)token_of<kRev>(first, count - 1));

            __syncthreads();  // the last chunk's tiles are done with
            sb.store(bt);
            sc.store(ct);
            if (threadIdx.x < kChunk) {
                const int32_t t = time_at(
                    p, (int32_t)token_of<kRev>(first, (int)threadIdx.x < count ? threadIdx.x : 0));
                tj[threadIdx.x] = t;
                wj[threadIdx.x] =
                    (int)threadIdx.x < count ? decay(rate2, elapsed<kRev>(t_last, t)) : 0.f;
            }
            if (some) {
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
            // the rows of a, as an operand
            bf16x8 a[DA / 32][NP];
            const T *a_row = a_data + (there ? token : 0) * p.a.token_stride;
#pragma unroll
            for (int k = 0; k < DA / 32; ++k)
                frag_global<T>(a_row, 32 * k + 8 * g, p.da, there, a[k]);
            __syncthreads();
            if (more) fetch(at + kChunk);

            // P^T: keys 16 kt + 4 g + r of the lane's token, masked and decayed
            const int32_t t_mine = tj[mine];
            float pk[kChunk / 16][4];
#pragma unroll
            for (int kt = 0; kt < kChunk / 16; ++kt) {
                floatx4 d{0.f, 0.f, 0.f, 0.f};
                if (kt <= wave) {
#pragma unroll
                    for (int k = 0; k < DA / 32; ++k) {
                        bf16x8 bk[NP];
                        frag_row<DA, NP>(bt, kChunk * DA, 16 * kt + l, 32 * k + 8 * g, bk);
                        mma<NP, NP>(bk, a[k], d);
                    }
                    const int4 t = *reinterpret_cast<const int4 *>(tj + 16 * kt + 4 * g);
                    const int32_t tk[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = d[r] * decay(rate2, elapsed<kRev>(t_mine, tk[r]));
                        d[r] = 16 * kt + 4 * g + r <= mine ? x : 0.f;
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) pk[kt][r] = d[r];
            }
            bf16x8 pf[kChunk / 32][NS];
#pragma unroll
            for (int s2 = 0; s2 < kChunk / 32; ++s2) {
                float x[8];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] = pk[2 * s2][r];
                    x[4 + r] = pk[2 * s2 + 1][r];
                }
                split8<NS>(x, pf[s2]);
            }
            const float since = some ? decay(rate2, elapsed<kRev>(t_mine, ref)) : 0.f;
            float dot = 0.f;
#pragma unroll
            for (int ti = 0; ti < DCT / 16; ++ti) {
                floatx4 o{0.f, 0.f, 0.f, 0.f};
                if (some) {
#pragma unroll
                    for (int k = 0; k < DA / 32; ++k) {
                        bf16x8 sf[NS];
                        frag_row<DA, NS>(st, DCT * DA, 16 * ti + l, 32 * k + 8 * g, sf);
                        mma<NS, NP>(sf, a[k], o);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[r] *= since;
                }
#pragma unroll
                for (int s2 = 0; s2 < kChunk / 32; ++s2) {
                    if (2 * s2 > wave) break;
                    bf16x8 cf[NP];
                    frag_col<DCT, NP>(ct, kChunk * DCT, 32 * s2, 16 * ti, cf);
                    mma<NP, NS>(cf, pf[s2], o);
                }
                const int c = 16 * ti + 4 * g;  // the lane's channels c .. + 3 of its token
                if (there && dc0 + c < p.dc) {
                    const int have = p.dc - dc0 - c;
                    T raw[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        o[r] *= p.scale;
                        raw[r] = from_f32<T>(o[r]);
                    }
                    T *dst = y_data + token * p.y.token_stride + c;
                    if (have >= 4) {
                        __builtin_memcpy(dst, raw, sizeof(raw));
                    } else {
#pragma unroll
                        for (int r = 0; r < 3; ++r)
                            if (r < have) dst[r] = raw[r];
                    }
                    if (p.dots) {
                        const T *x = static_cast<const T *>(p.x.data) + token * p.x.token_stride +
                                     (int64_t)head * p.x.head_stride + dc0 + c;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (r < have) dot += o[r] * to_f32(x[r]);
                    }
                }
            }
            if (p.dots) {
                dot += __shfl_xor(dot, 16);
                dot += __shfl_xor(dot, 32);
                if (there && g == 0)
                    p.dots[((int64_t)tile * p.heads + head) * p.n + token] = dot;
            }
            if (update) {
                const float f = step_factor(rate, elapsed<kRev>(t_last, ref));
                if (some) {
#pragma unroll
                    for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[u][r] = apply_factor(f, acc[u][r]);
                }
                add_chunk<T, DA, DCT>(bt, ct, wj, acc);
                some = true;
                ref = t_last;
            }
        }
        if (ends && p.state_out) {
            const int col = dc0 + S::col();
            float *to = p.state_out + ((int64_t)b * p.heads + head) * p.da * p.dc;
#pragma unroll
            for (int u = 0; u < S::kTiles; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = S::row(u) + r;
                    if (row < p.da && col < p.dc) to[(int64_t)row * p.dc + col] = acc[u][r];
                }
            if (p.time_out && tile == 0 && head == 0 && threadIdx.x == 0)
                p.time_out[b] = length > 0 || came_in ? time_at(p, hi - 1)
                                                      : (p.state_in ? p.state_time[b] : 0);
        }
        b += kRev ? -1 : 1;
    }
}

// ---------------------------------------------------------------- launches
// Calls f with the padded channels of a (32, 64 or 128) and the columns of a tile
// of c (32 or 64).
template <typename F> void pass_dispatch(int32_t da, int32_t dct, F &&f) {
#define SBC_PASS(x, y) f(std::integral_constant<int, x>{}, std::integral_constant<int, y>{})
    if (dct == 32) {
        if (da <= 32) SBC_PASS(32, 32);
        else if (da <= 64) SBC_PASS(64, 32);
        else SBC_PASS(128, 32);
    } else {
        if (da <= 32) SBC_PASS(32, 64);
        else if (da <= 64) SBC_PASS(64, 64);
        else SBC_PASS(128, 64);
    }
#undef SBC_PASS
}

inline dim3 pass_grid(const AttnPass &p) {
    return dim3((unsigned)((int64_t)p.n_seg * p.heads * p.tiles));
}

}  // namespace
}  // namespace sbc
