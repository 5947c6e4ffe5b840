// Rotary positions with several axes (time and pixel of an event, coordinates
// of a point), forward and backward.
//
// Pair p of a head's channels turns by the angle positions[i, axis(p)] freqs[p]:
//   (a, b) -> (a cos - b sin, b cos + a sin),
// the gradient by the opposite angle.  Every value is moved twice and turned with
// four products, so memory bounds it as long as the angle's sine and cosine are
// not made for every head: a lane makes those of some pairs of a token once and
// takes the token's heads, of both arrays, kBatch at a time, so that their loads are
// in flight together (and the first ones while it makes them).
//
// The angle is taken in revolutions in float64, where the product of two float32
// is exact and 1 / 2 pi costs 2^-53 of it, and reduced before sine and cosine in
// float32: angles of 1e6 (timestamps) are as good as small ones.
#include "common.hpp"
#include "seq.hpp"

namespace sbc {
namespace {

constexpr int kThreads = 256;

struct RotaryArgs {
    sbc_heads in[2], out[2];
    int32_t heads[2];
    int32_t n, d, pairs, units;  // units: lanes that a token takes
    const void *positions;
    int64_t pos_stride;
    const float *freqs;
    int32_t n_axes;
    int32_t upto[SBC_MAX_AXES];  // pairs of the axes so far
    float sign;
};

// Pairs of a lane: one vector of them, or of each of their halves
template <typename T, bool kInterleaved> constexpr int kPairs = kInterleaved ? kVec<T> / 2 : kVec<T>;

// kTail: there are channels past the last pair (300k events: 112 us without such lanes'
// conditions, 139 with them)
template <typename T, typename P, bool kInterleaved, bool kTail>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
    constexpr int V = kVec<T>, N = kPairs<T, kInterleaved>;
    constexpr int kVecs = kInterleaved ? 1 : 2, kBatch = kInterleaved ? 4 : 2;
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t i = at / a.units;
    if (i >= a.n) return;
    const int unit = (int)(at - i * a.units);
    const int turning = (a.pairs + N - 1) / N;
    const int total = a.heads[0] + a.heads[1];
    auto source = [&](int j) {
        const int w = j >= a.heads[0], h = w ? j - a.heads[0] : j;
        return static_cast<const T *>(a.in[w].data) + i * a.in[w].token_stride +
               h * a.in[w].head_stride;
    };
    auto target = [&](int j) {
        const int w = j >= a.heads[0], h = w ? j - a.heads[0] : j;
        return static_cast<T *>(a.out[w].data) + i * a.out[w].token_stride +
               h * a.out[w].head_stride;
    };
    // A lane's vectors: of pairs (of the pairs themselves, or of their first and second
    // halves), or of channels past the last pair, which are copied.  (By a way of their
    // own the copies' loads, one head after another, had the whole wave wait.)
    const bool copies = kTail && unit >= turning;
    const int p0 = unit * N;
    const int have = a.pairs - p0;  // pairs of this lane, if fewer than N
    const int past = 2 * a.pairs + (unit - turning) * V;
    const int c[2] = {copies ? past : kInterleaved ? 2 * p0 : p0, a.pairs + p0};
    const int width[2] = {copies ? a.d - past : kInterleaved ? 2 * have : have, copies ? 0 : have};
    float x[kBatch][kVecs][V];
    auto fetch = [&](int j0) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (j0 + u < total) {
#pragma unroll
                for (int w = 0; w < kVecs; ++w)
                    load_vec<T>(source(j0 + u) + c[w], width[w], x[u][w]);
            }
    };
    fetch(0);
    float cs[N], sn[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        cs[k] = 1.f;
        sn[k] = 0.f;
        if (!copies && k < have) {
            int axis = 0;
            for (int y = 0; y + 1 < a.n_axes; ++y) axis += p0 + k >= a.upto[y];
            const double pos = (double)static_cast<const P *>(a.positions)[i * a.pos_stride + axis];
            double rev = pos * (double)a.freqs[p0 + k] * 0.15915494309189533577;
            rev -= rint(rev);
            float s, co;
            sincospif((float)(2.0 * rev), &s, &co);
            cs[k] = co;
            sn[k] = a.sign * s;
        }
    }
    for (int j0 = 0; j0 < total; j0 += kBatch) {
        if (j0 > 0) fetch(j0);
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (j0 + u < total) {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    if (copies) break;
                    float &p = kInterleaved ? x[u][0][2 * k] : x[u][0][k];
                    float &q = kInterleaved ? x[u][0][2 * k + 1] : x[u][kVecs - 1][k];
                    const float turned = p * cs[k] - q * sn[k];
                    q = q * cs[k] + p * sn[k];
                    p = turned;
                }
#pragma unroll
                for (int w = 0; w < kVecs; ++w) store_vec<T>(target(j0 + u) + c[w], width[w], x[u][w]);
            }
    }
}

template <typename T, typename P>
void launch(const RotaryArgs &a, bool interleaved, bool tail, hipStream_t stream) {
    const dim3 grid((unsigned)grid_for((int64_t)a.n * a.units, kThreads)), block(kThreads);
#define SBC_ROTARY(I, L) hipLaunchKernelGGL((rotary_kernel<T, P, I, L>), grid, block, 0, stream, a)
    if (interleaved && tail)
        SBC_ROTARY(true, true);
    else if (interleaved)
        SBC_ROTARY(true, false);
    else if (tail)
        SBC_ROTARY(false, true);
    else
        SBC_ROTARY(false, false);
#undef SBC_ROTARY
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" sbc_status sbc_rotary(const sbc_rotary_plan *plan, const sbc_heads *q, int32_t q_heads,
                                 const sbc_heads *k, int32_t k_heads, sbc_dtype dtype, int32_t n,
                                 int32_t d, int32_t backward, const sbc_heads *q_out,
                                 const sbc_heads *k_out, hipStream_t stream) {
    clear_error();
    if (!plan) return fail(SBC_ERR_INVALID_ARG, "plan is null");
    if (n < 0 || d <= 0) return fail(SBC_ERR_INVALID_ARG, "n must be >= 0 and d > 0");
    if (!known_dtype(dtype)) return fail(SBC_ERR_INVALID_ARG, "unknown dtype");
    if (plan->n_axes < 1 || plan->n_axes > SBC_MAX_AXES)
        return fail(SBC_ERR_INVALID_ARG, "n_axes must be 1 .. SBC_MAX_AXES");
    RotaryArgs a{};
    int64_t pairs = 0;
    for (int x = 0; x < plan->n_axes; ++x) {
        if (plan->sections[x] < 0) return fail(SBC_ERR_INVALID_ARG, "a section is negative");
        pairs += plan->sections[x];
        a.upto[x] = (int32_t)(pairs <= d ? pairs : d);
    }
    if (pairs < 1 || 2 * pairs > d)
        return fail(SBC_ERR_INVALID_ARG, "the sections must sum to 1 .. d / 2 pairs");
    if (plan->position_stride < plan->n_axes)
        return fail(SBC_ERR_INVALID_ARG, "position_stride is smaller than n_axes");
    if (q_heads < 0 || k_heads < 0) return fail(SBC_ERR_INVALID_ARG, "negative number of heads");
    if (n == 0 || (q_heads == 0 && k_heads == 0)) return SBC_OK;
    if (!plan->positions || !plan->freqs)
        return fail(SBC_ERR_INVALID_ARG, "positions or freqs is null");
    SBC_TRY(check_heads(q, q_heads, n, d, dtype, "q"));
    SBC_TRY(check_heads(k, k_heads, n, d, dtype, "k"));
    SBC_TRY(check_out_heads(q_out, q_heads, n, d, dtype, "q_out"));
    SBC_TRY(check_out_heads(k_out, k_heads, n, d, dtype, "k_out"));
    const sbc_heads none{};
    const sbc_heads *in[2] = {q_heads ? q : &none, k_heads ? k : &none};
    const sbc_heads *out[2] = {q_heads ? q_out : &none, k_heads ? k_out : &none};
    const int32_t heads[2] = {q_heads, k_heads};
    for (int w = 0; w < 2; ++w) {
        for (int u = 0; u < 2; ++u) {
            const bool same = w == u && in[u]->data == out[w]->data &&
                              in[u]->token_stride == out[w]->token_stride &&
                              in[u]->head_stride == out[w]->head_stride;
            if (!same && meet(region_heads(out[w], heads[w], n, d, dtype),
                              region_heads(in[u], heads[u], n, d, dtype)))
                return fail(SBC_ERR_INVALID_ARG, "an output overlaps an input that is not its own");
        }
        a.in[w] = *in[w];
        a.out[w] = *out[w];
        a.heads[w] = heads[w];
    }
    SBC_TRY(check_apart({region_heads(out[0], heads[0], n, d, dtype),
                         region_heads(out[1], heads[1], n, d, dtype)},
                        {region_rows(plan->positions, n, plan->n_axes, plan->position_stride, SBC_F32),
                         region(plan->freqs, pairs, 4)}));
    const int V = dtype == SBC_F32 ? 4 : 8;
    const int N = plan->interleaved ? V / 2 : V;  // (kPairs)
    a.n = n;
    a.d = d;
    a.pairs = (int32_t)pairs;
    a.units = (int32_t)((pairs + N - 1) / N + (d - 2 * pairs + V - 1) / V);
    a.positions = plan->positions;
    a.pos_stride = plan->position_stride;
    a.freqs = plan->freqs;
    a.n_axes = plan->n_axes;
    a.sign = backward ? -1.f : 1.f;
    if ((int64_t)n * a.units > (int64_t)1 << 31)
        return fail(SBC_ERR_UNSUPPORTED, "n and d need more than 2^31 lanes");
    trace_before("rotary", stream);
    const bool interleaved = plan->interleaved, tail = 2 * pairs < d;
    if (dtype == SBC_F32 && plan->float_positions)
        launch<float, float>(a, interleaved, tail, stream);
    else if (dtype == SBC_F32)
        launch<float, int32_t>(a, interleaved, tail, stream);
    else if (plan->float_positions)
        launch<bf16_t, float>(a, interleaved, tail, stream);
    else
        launch<bf16_t, int32_t>(a, interleaved, tail, stream);
    SBC_LAUNCH_CHECK();
    trace_after("rotary", stream);
    return SBC_OK;
}
