// Norms of queries and keys for each head with the rotation by their positions, forward and
// backward.
//
// As the rotation alone (rotary.hip), memory bounds it: a lane has a vector of pairs of one
// token, makes their sines and cosines once and takes the token's heads of both arrays, kBatch
// at a time.  A token's lanes are neighbours within a wave, padded to a power of two, so that
// the mean square of a head is a sum over them in registers.
//
// Backward, with g = R(-pos) dy and rstd = 1 / sqrt(mean(x^2) + eps):
//   dw = sum over tokens and heads of g x rstd,  dx = rstd (g w - x rstd^2 mean(g w x)).
// A lane's part of dw stays in registers over its tokens; a workgroup adds its lanes' in LDS,
// and a second kernel the workgroups', both in a fixed order.
#include <type_traits>

#include "rotary.hpp"

namespace sbc {
namespace {

constexpr int kThreads = 256;
constexpr int kMostBlocks = 768;  // of the backward pass: rows of the weights' partial sums

struct QkNormArgs {
    sbc_heads in[2], out[2], dy[2];
    int32_t heads[2];
    const float *weight[2];
    int32_t n, d, pairs, units, lanes;  // lanes: of a token, a power of two
    const void *positions;
    int64_t pos_stride;
    int32_t float_positions;
    const float *freqs;
    int32_t n_axes;
    int32_t upto[SBC_MAX_AXES];
    float eps;
    float *partial;  // [blocks, 2, d]
    float *dw[2];
    int32_t blocks;
};

// What a lane has of a token: its vectors' first channels and how many of each exist
template <typename T, bool kInterleaved> struct LaneChannels {
    static constexpr int V = kVec<T>, N = kPairs<T, kInterleaved>, kVecs = kInterleaved ? 1 : 2;
    int c[2], width[2], have, p0;
    bool copies;  // channels past the last pair
    __device__ __forceinline__ LaneChannels(const QkNormArgs &a, int unit) {
        const int turning = (a.pairs + N - 1) / N;
        copies = unit >= turning;
        p0 = unit * N;
        have = copies ? 0 : a.pairs - p0;
        const int past = 2 * a.pairs + (unit - turning) * V;
        c[0] = copies ? past : kInterleaved ? 2 * p0 : p0;
        c[1] = a.pairs + p0;
        width[0] = unit >= a.units ? 0 : copies ? a.d - past : kInterleaved ? 2 * have : have;
        width[1] = copies ? 0 : have;
#pragma unroll
        for (int w = 0; w < 2; ++w) width[w] = width[w] < 0 ? 0 : width[w] > V ? V : width[w];
        if (kInterleaved) width[1] = 0;
    }
    __device__ __forceinline__ void turns(const QkNormArgs &a, int64_t i, float sign,
                                          float (&cs)[N], float (&sn)[N]) const {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            cs[k] = 1.f;
            sn[k] = 0.f;
            if (k < have) {
                int axis = 0;
                for (int y = 0; y + 1 < a.n_axes; ++y) axis += p0 + k >= a.upto[y];
                const int64_t at = i * a.pos_stride + axis;
                const double pos = a.float_positions
                                       ? (double)static_cast<const float *>(a.positions)[at]
                                       : (double)static_cast<const int32_t *>(a.positions)[at];
                float s;
                turn_of(pos, a.freqs[p0 + k], cs[k], s);
                sn[k] = sign * s;
            }
        }
    }
    __device__ __forceinline__ void turn(float (&x)[kVecs][V], const float (&cs)[N],
                                         const float (&sn)[N]) const {
        if (copies) return;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float &p = kInterleaved ? x[0][2 * k] : x[0][k];
            float &q = kInterleaved ? x[0][2 * k + 1] : x[kVecs - 1][k];
            const float turned = p * cs[k] - q * sn[k];
            q = q * cs[k] + p * sn[k];
            p = turned;
        }
    }
};

template <typename T>
__device__ __forceinline__ T *head_at(const sbc_heads (&x)[2], const int32_t (&heads)[2], int64_t i,
                                      int j) {
    const int w = j >= heads[0], h = w ? j - heads[0] : j;
    return static_cast<T *>(x[w].data) + i * x[w].token_stride + h * x[w].head_stride;
}

// Raw vectors of a head on their way
// (kEven: a lane's vectors are whole or none, and no branch lies between the loads)
template <typename T, bool kInterleaved, bool kEven> struct HeadLoad {
    using L = LaneChannels<T, kInterleaved>;
    raw16 raw[L::kVecs];
    __device__ __forceinline__ void load(const T *from, const L &lane) {
#pragma unroll
        for (int w = 0; w < L::kVecs; ++w) {
            if constexpr (kEven)
                __builtin_memcpy(&raw[w], from + (lane.width[w] > 0 ? lane.c[w] : 0), 16);
            else
                raw[w] = load_raw16<T>(from + lane.c[w], lane.width[w]);
        }
    }
    __device__ __forceinline__ void get(const L &lane, float (&x)[L::kVecs][L::V]) const {
#pragma unroll
        for (int w = 0; w < L::kVecs; ++w) {
            unpack<T>(raw[w], x[w]);
            if constexpr (kEven) {
#pragma unroll
                for (int e = 0; e < L::V; ++e) x[w][e] = lane.width[w] > 0 ? x[w][e] : 0.f;
            }
        }
    }
    __device__ __forceinline__ static void put(T *to, const L &lane, const float (&x)[L::kVecs][L::V]) {
#pragma unroll
        for (int w = 0; w < L::kVecs; ++w) {
            if constexpr (kEven) {
                if (lane.width[w] > 0) store_vec<T>(to + lane.c[w], L::V, x[w]);
            } else {
                store_vec<T>(to + lane.c[w], lane.width[w], x[w]);
            }
        }
    }
};

// kLanes of a token.  (The next kBatch heads are on their way while a batch is computed.)
template <typename T, bool kInterleaved, bool kEven, int kLanes>
__global__ __launch_bounds__(kThreads) void qk_norm_kernel(QkNormArgs a) {
    using L = LaneChannels<T, kInterleaved>;
    constexpr int V = L::V, N = L::N, kVecs = L::kVecs, kBatch = kInterleaved ? 4 : 2;
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t i = at / kLanes;
    const int unit = (int)(at & (kLanes - 1));
    if (i >= a.n) return;  // (all lanes of a token)
    const L lane(a, unit);
    const int total = a.heads[0] + a.heads[1];
    HeadLoad<T, kInterleaved, kEven> next[kBatch];
    auto fetch = [&](int j0) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (j0 + u < total) next[u].load(head_at<T>(a.in, a.heads, i, j0 + u), lane);
    };
    fetch(0);
    float weight[2][kVecs][V];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int w = 0; w < kVecs; ++w) {
#pragma unroll
            for (int e = 0; e < V; ++e) weight[y][w][e] = 1.f;
            if (a.weight[y]) load_f32<V>(a.weight[y] + lane.c[w], lane.width[w], weight[y][w]);
        }
    float cs[N], sn[N];
    lane.turns(a, i, 1.f, cs, sn);
    const float per = 1.f / a.d;
    for (int j0 = 0; j0 < total; j0 += kBatch) {
        float x[kBatch][kVecs][V];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) next[u].get(lane, x[u]);
        if (j0 + kBatch < total) fetch(j0 + kBatch);
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (j0 + u < total) {
                float square = 0.f;
#pragma unroll
                for (int w = 0; w < kVecs; ++w)
#pragma unroll
                    for (int e = 0; e < V; ++e) square = fmaf(x[u][w][e], x[u][w][e], square);
                square = group_sum<kLanes>(square);
                const float rstd = 1.f / sqrtf(fmaf(square, per, a.eps));
                const bool keys = j0 + u >= a.heads[0];
#pragma unroll
                for (int w = 0; w < kVecs; ++w)
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        x[u][w][e] *= rstd * (keys ? weight[1][w][e] : weight[0][w][e]);
                lane.turn(x[u], cs, sn);
                T *to = head_at<T>(a.out, a.heads, i, j0 + u);
                HeadLoad<T, kInterleaved, kEven>::put(to, lane, x[u]);
            }
    }
}

template <typename T, bool kInterleaved, bool kEven, int kLanes>
__global__ __launch_bounds__(kThreads) void qk_norm_grad_kernel(QkNormArgs a) {
    using L = LaneChannels<T, kInterleaved>;
    constexpr int V = L::V, N = L::N, kVecs = L::kVecs;
    __shared__ float sums[kThreads * kVecs * V];
    constexpr int kGroups = kThreads / kLanes;
    const int group = threadIdx.x / kLanes, unit = threadIdx.x & (kLanes - 1);
    const L lane(a, unit);
    float weight[2][kVecs][V], dw[2][kVecs][V];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int w = 0; w < kVecs; ++w) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                weight[y][w][e] = 1.f;
                dw[y][w][e] = 0.f;
            }
            if (a.weight[y]) load_f32<V>(a.weight[y] + lane.c[w], lane.width[w], weight[y][w]);
        }
    const float per = 1.f / a.d;
    for (int64_t i = (int64_t)blockIdx.x * kGroups + group; i < a.n; i += (int64_t)gridDim.x * kGroups) {
        float cs[N], sn[N];
        HeadLoad<T, kInterleaved, kEven> next_x, next_g;
        auto fetch = [&](int y, int h) {
            next_x.load(static_cast<const T *>(a.in[y].data) + i * a.in[y].token_stride +
                            h * a.in[y].head_stride,
                        lane);
            next_g.load(static_cast<const T *>(a.dy[y].data) + i * a.dy[y].token_stride +
                            h * a.dy[y].head_stride,
                        lane);
        };
        fetch(a.heads[0] > 0 ? 0 : 1, 0);
        lane.turns(a, i, -1.f, cs, sn);
#pragma unroll
        for (int y = 0; y < 2; ++y)
            for (int h = 0; h < a.heads[y]; ++h) {
                float x[kVecs][V], g[kVecs][V];
                next_x.get(lane, x);
                next_g.get(lane, g);
                if (h + 1 < a.heads[y])
                    fetch(y, h + 1);
                else if (y == 0 && a.heads[1] > 0)
                    fetch(1, 0);
                lane.turn(g, cs, sn);
                float square = 0.f, dot = 0.f;
#pragma unroll
                for (int w = 0; w < kVecs; ++w)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        square = fmaf(x[w][e], x[w][e], square);
                        dot = fmaf(g[w][e] * weight[y][w][e], x[w][e], dot);
                    }
                square = group_sum<kLanes>(square);
                dot = group_sum<kLanes>(dot);
                const float rstd = 1.f / sqrtf(fmaf(square, per, a.eps));
                const float back = dot * per * rstd * rstd;
#pragma unroll
                for (int w = 0; w < kVecs; ++w)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float z = x[w][e];
                        dw[y][w][e] = fmaf(g[w][e], z * rstd, dw[y][w][e]);
                        x[w][e] = rstd * fmaf(-back, z, g[w][e] * weight[y][w][e]);
                    }
                T *to = static_cast<T *>(a.out[y].data) + i * a.out[y].token_stride +
                        h * a.out[y].head_stride;
                HeadLoad<T, kInterleaved, kEven>::put(to, lane, x);
            }
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        if (!a.dw[y]) continue;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kVecs; ++w)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < lane.width[w]) sums[group * a.d + lane.c[w] + e] = dw[y][w][e];
        __syncthreads();
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            float s = 0.f;
#pragma unroll 8
            for (int g = 0; g < kGroups; ++g) s += sums[g * a.d + c];
            if (gridDim.x == 1)
                a.dw[y][c] = s;  // (nothing to add it to)
            else
                a.partial[((int64_t)blockIdx.x * 2 + y) * a.d + c] = s;
        }
    }
}

// dw: the workgroups' sums of 16 channels, every sixteenth of them a thread's
__global__ __launch_bounds__(kThreads) void qk_norm_reduce_kernel(QkNormArgs a) {
    __shared__ float sums[16][17];
    const int y = blockIdx.y, c = blockIdx.x * 16 + threadIdx.x % 16, part = threadIdx.x / 16;
    if (!a.dw[y]) return;
    float s = 0.f;
    if (c < a.d) {
#pragma unroll 8
        for (int b = part; b < a.blocks; b += 16) s += a.partial[((int64_t)b * 2 + y) * a.d + c];
    }
    sums[part][threadIdx.x % 16] = s;
    __syncthreads();
    if (part == 0 && c < a.d) {
        s = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) s += sums[r][threadIdx.x];
        a.dw[y][c] = s;
    }
}

template <typename T, bool kInterleaved, typename F> void dispatch_lanes(const QkNormArgs &a, F f) {
    using L = LaneChannels<T, kInterleaved>;
    const bool even = a.pairs % L::N == 0 && (a.d - 2 * a.pairs) % L::V == 0;
    auto by_even = [&](auto lanes) {
        even ? f(T{}, std::bool_constant<kInterleaved>{}, std::true_type{}, lanes)
             : f(T{}, std::bool_constant<kInterleaved>{}, std::false_type{}, lanes);
    };
    switch (a.lanes) {
        case 1: return by_even(std::integral_constant<int, 1>{});
        case 2: return by_even(std::integral_constant<int, 2>{});
        case 4: return by_even(std::integral_constant<int, 4>{});
        case 8: return by_even(std::integral_constant<int, 8>{});
        case 16: return by_even(std::integral_constant<int, 16>{});
        case 32: return by_even(std::integral_constant<int, 32>{});
        default: return by_even(std::integral_constant<int, 64>{});
    }
}
template <typename F> void dispatch(sbc_dtype dtype, bool interleaved, const QkNormArgs &a, F f) {
    if (dtype == SBC_F32)
        interleaved ? dispatch_lanes<float, true>(a, f) : dispatch_lanes<float, false>(a, f);
    else
        interleaved ? dispatch_lanes<bf16_t, true>(a, f) : dispatch_lanes<bf16_t, false>(a, f);
}

int32_t grad_blocks(int32_t n, int32_t lanes) {
    const int64_t b = ((int64_t)n * lanes + kThreads - 1) / kThreads;
    return (int32_t)(b < kMostBlocks ? b : kMostBlocks);
}

// Checks of both directions, and the arguments that they share
sbc_status arguments(const sbc_rotary_plan *plan, const sbc_heads *q, int32_t q_heads,
                     const sbc_heads *k, int32_t k_heads, const float *q_weight,
                     const float *k_weight, sbc_dtype dtype, int32_t n, int32_t d, float eps,
                     QkNormArgs *a) {
    if (!plan) return fail(SBC_ERR_INVALID_ARG, "plan is null");
    if (n < 0 || d <= 0) return fail(SBC_ERR_INVALID_ARG, "n must be >= 0 and d > 0");
    if (!known_dtype(dtype)) return fail(SBC_ERR_INVALID_ARG, "unknown dtype");
    if (!(eps >= 0.f)) return fail(SBC_ERR_INVALID_ARG, "eps must be >= 0");
    int64_t pairs;
    SBC_TRY(check_rotary(plan, d, &pairs, a->upto));
    if (q_heads < 0 || k_heads < 0) return fail(SBC_ERR_INVALID_ARG, "negative number of heads");
    if (q_heads > 65535 || k_heads > 65535)
        return fail(SBC_ERR_UNSUPPORTED, "the heads must be <= 65535");
    const int64_t units = rotary_units(dtype, plan->interleaved, pairs, d);
    if (d > 256 || units > 64)
        return fail(SBC_ERR_UNSUPPORTED, "d must be <= 256, in 64 pieces of 16 bytes at most");
    a->lanes = 1;
    while (a->lanes < units) a->lanes *= 2;
    if ((int64_t)n * a->lanes > (int64_t)1 << 31)
        return fail(SBC_ERR_UNSUPPORTED, "n and d need more than 2^31 lanes");
    if (n > 0 && (q_heads > 0 || k_heads > 0)) {
        if (!plan->positions || !plan->freqs)
            return fail(SBC_ERR_INVALID_ARG, "positions or freqs is null");
        SBC_TRY(check_heads(q, q_heads, n, d, dtype, "q"));
        SBC_TRY(check_heads(k, k_heads, n, d, dtype, "k"));
    }
    const sbc_heads none{};
    a->in[0] = q_heads && q ? *q : none;
    a->in[1] = k_heads && k ? *k : none;
    a->heads[0] = q_heads;
    a->heads[1] = k_heads;
    a->weight[0] = q_weight;
    a->weight[1] = k_weight;
    a->n = n;
    a->d = d;
    a->pairs = (int32_t)pairs;
    a->units = (int32_t)units;
    a->positions = plan->positions;
    a->pos_stride = plan->position_stride;
    a->float_positions = plan->float_positions != 0;
    a->freqs = plan->freqs;
    a->n_axes = plan->n_axes;
    a->eps = eps;
    return SBC_OK;
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" sbc_status sbc_qk_norm_rotary_forward(
    const sbc_rotary_plan *plan, const sbc_heads *q, int32_t q_heads, const sbc_heads *k,
    int32_t k_heads, const float *q_weight, const float *k_weight, sbc_dtype dtype, int32_t n,
    int32_t d, float eps, const sbc_heads *q_out, const sbc_heads *k_out, hipStream_t stream) {
    clear_error();
    QkNormArgs a{};
    SBC_TRY(arguments(plan, q, q_heads, k, k_heads, q_weight, k_weight, dtype, n, d, eps, &a));
    if (n == 0 || (q_heads == 0 && k_heads == 0)) return SBC_OK;
    SBC_TRY(check_out_heads(q_out, q_heads, n, d, dtype, "q_out"));
    SBC_TRY(check_out_heads(k_out, k_heads, n, d, dtype, "k_out"));
    if (q_heads) a.out[0] = *q_out;
    if (k_heads) a.out[1] = *k_out;
    for (int w = 0; w < 2; ++w)
        for (int u = 0; u < 2; ++u) {
            const bool same = w == u && a.in[u].data == a.out[w].data &&
                              a.in[u].token_stride == a.out[w].token_stride &&
                              a.in[u].head_stride == a.out[w].head_stride;
            if (!same && meet(region_heads(&a.out[w], a.heads[w], n, d, dtype),
                              region_heads(&a.in[u], a.heads[u], n, d, dtype)))
                return fail(SBC_ERR_INVALID_ARG, "an output overlaps an input that is not its own");
        }
    SBC_TRY(check_apart({region_heads(&a.out[0], q_heads, n, d, dtype),
                         region_heads(&a.out[1], k_heads, n, d, dtype)},
                        {region_rows(plan->positions, n, plan->n_axes, plan->position_stride, SBC_F32),
                         region(plan->freqs, a.pairs, 4), region(q_weight, d, 4),
                         region(k_weight, d, 4)}));
    trace_before("qk_norm_fwd", stream);
    dispatch(dtype, plan->interleaved, a, [&](auto t, auto inter, auto even, auto lanes) {
        hipLaunchKernelGGL((qk_norm_kernel<decltype(t), decltype(inter)::value, decltype(even)::value,
                            decltype(lanes)::value>),
                           dim3((unsigned)grid_for((int64_t)n * a.lanes, kThreads)), dim3(kThreads), 0,
                           stream, a);
    });
    SBC_LAUNCH_CHECK();
    trace_after("qk_norm_fwd", stream);
    return SBC_OK;
}

extern "C" size_t sbc_qk_norm_rotary_workspace_size(int32_t n, int32_t d) {
    if (n < 0 || d <= 0 || d > 256) return 0;
    return align_up((size_t)grad_blocks(n, 64) * 2 * d * sizeof(float) + 1);
}

extern "C" sbc_status sbc_qk_norm_rotary_backward(
    const sbc_rotary_plan *plan, const sbc_heads *dq, const sbc_heads *dk, const sbc_heads *q,
    int32_t q_heads, const sbc_heads *k, int32_t k_heads, const float *q_weight,
    const float *k_weight, sbc_dtype dtype, int32_t n, int32_t d, float eps,
    const sbc_heads *dq_out, const sbc_heads *dk_out, float *dq_weight, float *dk_weight,
    void *workspace, size_t workspace_bytes, hipStream_t stream) {
    clear_error();
    QkNormArgs a{};
    SBC_TRY(arguments(plan, q, q_heads, k, k_heads, q_weight, k_weight, dtype, n, d, eps, &a));
    SBC_TRY(check_heads(dq, q_heads, n, d, dtype, "dq"));
    SBC_TRY(check_heads(dk, k_heads, n, d, dtype, "dk"));
    SBC_TRY(check_out_heads(dq_out, q_heads, n, d, dtype, "dq_out"));
    SBC_TRY(check_out_heads(dk_out, k_heads, n, d, dtype, "dk_out"));
    const bool work = n > 0 && (q_heads > 0 || k_heads > 0);
    if (!work && !dq_weight && !dk_weight) return SBC_OK;
    if (n > 0) {
        if (q_heads) {
            a.dy[0] = *dq;
            a.out[0] = *dq_out;
        }
        if (k_heads) {
            a.dy[1] = *dk;
            a.out[1] = *dk_out;
        }
    }
    SBC_TRY(check_apart({region_heads(&a.out[0], q_heads, n, d, dtype),
                         region_heads(&a.out[1], k_heads, n, d, dtype), region(dq_weight, d, 4),
                         region(dk_weight, d, 4)},
                        {region_heads(&a.in[0], q_heads, n, d, dtype),
                         region_heads(&a.in[1], k_heads, n, d, dtype),
                         region_heads(&a.dy[0], q_heads, n, d, dtype),
                         region_heads(&a.dy[1], k_heads, n, d, dtype),
                         region_rows(plan->positions, n, plan->n_axes, plan->position_stride, SBC_F32),
                         region(plan->freqs, a.pairs, 4), region(q_weight, d, 4),
                         region(k_weight, d, 4)}));
    const bool sums = dq_weight || dk_weight;
    if (sums && (!workspace || workspace_bytes < sbc_qk_norm_rotary_workspace_size(n, d)))
        return fail(SBC_ERR_WORKSPACE, "workspace smaller than sbc_qk_norm_rotary_workspace_size()");
    a.dw[0] = dq_weight;
    a.dw[1] = dk_weight;
    a.partial = sums ? static_cast<float *>(workspace) : nullptr;
    a.blocks = work ? grad_blocks(n, a.lanes) : 0;
    if (work) {
        trace_before("qk_norm_bwd", stream);
        dispatch(dtype, plan->interleaved, a, [&](auto t, auto inter, auto even, auto lanes) {
            hipLaunchKernelGGL((qk_norm_grad_kernel<decltype(t), decltype(inter)::value, decltype(even)::value,
                            decltype(lanes)::value>),
                               dim3((unsigned)a.blocks), dim3(kThreads), 0, stream, a);
        });
        SBC_LAUNCH_CHECK();
        trace_after("qk_norm_bwd", stream);
    }
    if (sums && a.blocks != 1) {
        trace_before("qk_norm_reduce", stream);
        hipLaunchKernelGGL(qk_norm_reduce_kernel, dim3((unsigned)((d + 15) / 16), 2), dim3(kThreads),
                           0, stream, a);
        SBC_LAUNCH_CHECK();
        trace_after("qk_norm_reduce", stream);
    }
    return SBC_OK;
}
