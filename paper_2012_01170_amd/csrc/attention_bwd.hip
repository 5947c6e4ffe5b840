// Gradients of the linear attention with decays: three passes of attention.hpp.
//
//   dq: (dO, v, k) along the sequence       dk: (v, dO, q) back along it
//   dv: (k, q, dO) back along it
//
// The rates' gradient.  With P_ij the term of a pair (its decay, both products
// and the scale), drate = - sum of (t_i - t_j) P_ij.  The sum of P_ij over the
// pairs that cross a point between two tokens is a flow: it grows by
// k_j . dk_j = sum over i of P_ij behind token j and falls by q_i . dq_i = sum
// over j of P_ij behind token i, so that
//   sum of (t_i - t_j) P_ij = sum over gaps of gap * flow
//     = X (t_end - t_before) + sum over m of (k_m . dk_m - q_m . dq_m) (t_end - t_m)
// for a segment's tokens m of one sequence, t_end the last one's time, with the
// flow X into the segment, the product of the states that meet there (the sum
// of k v^T from before it and of q dO^T from behind).  The passes leave the
// products of a token; starting anew from X in each segment keeps their rounding
// from adding up along the sequence.
#include "attention_host.hpp"
#include "attention_kernels.hpp"

namespace sbc {
namespace {

constexpr int kBwdPerCu = 2;

struct RatesArgs {
    AttnPass p;                  // the sequences, times and segments
    const float *before, *behind;  // states that come into segments along and back
    int32_t elements;            // of a state
    const float *dot_q, *dot_k;  // [tiles, heads, n]
    int32_t tiles;
    double *part;                // [n_seg, heads]
};

// Sum over a workgroup of 256 in its first thread.
__device__ __forceinline__ double block_sum(double x, double *buf) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
    __syncthreads();
    return (buf[0] + buf[1]) + (buf[2] + buf[3]);
}

__global__ __launch_bounds__(256) void attn_rates_kernel(RatesArgs r) {
    __shared__ double buf[4];
    const AttnPass &p = r.p;
    const int head = blockIdx.x % p.heads, seg = blockIdx.x / p.heads;
    const int32_t g0 = seg * p.seg_len;
    const int32_t g1 = seg == p.n_seg - 1 ? p.n : g0 + p.seg_len;
    const int32_t b_new = first_from(p, g0);
    const bool came_in = b_new > 0 && split_at(p, b_new) > g0;
    const float rate2 = p.rates[head] * kLog2E;
    double x = 0.0;
    if (came_in) {
        const float *f = r.before + ((int64_t)seg * p.heads + head) * p.state_stride;
        const float *d = r.behind + ((int64_t)(seg - 1) * p.heads + head) * p.state_stride;
        for (int i = threadIdx.x; i < r.elements; i += 256) x += (double)f[i] * (double)d[i];
        x = block_sum(x, buf) *
            (double)(p.scale * decay(rate2, elapsed<false>(time_at(p, g0), time_at(p, g0 - 1))));
    }
    double sum = 0.0;
    for (int32_t b = came_in ? b_new - 1 : b_new; b < p.n_batch; ++b) {
        const int32_t s = split_at(p, b), e = split_at(p, b + 1);
        if (b >= b_new && s >= g1) break;
        const int32_t lo = s > g0 ? s : g0, hi = e < g1 ? e : g1;
        if (lo >= hi) continue;
        const int32_t t_end = time_at(p, hi - 1);
        if (b < b_new && threadIdx.x == 0)
            sum += x * (double)elapsed<false>(t_end, time_at(p, g0 - 1));
        for (int32_t m = lo + (int32_t)threadIdx.x; m < hi; m += 256) {
            float c = 0.f;
            for (int ti = 0; ti < r.tiles; ++ti) {
                const int64_t at = ((int64_t)ti * p.heads + head) * p.n + m;
                c += r.dot_k[at] - r.dot_q[at];
            }
            sum += (double)c * (double)elapsed<false>(t_end, time_at(p, m));
        }
    }
    sum = block_sum(sum, buf);
    if (threadIdx.x == 0) r.part[(int64_t)seg * p.heads + head] = sum;
}

__global__ __launch_bounds__(256) void attn_rates_sum_kernel(const double *__restrict__ part,
                                                             int32_t n_seg, int32_t heads,
                                                             float *__restrict__ drates) {
    __shared__ double buf[4];
    double s = 0.0;
    for (int g = threadIdx.x; g < n_seg; g += 256) s += part[(int64_t)g * heads + blockIdx.x];
    s = block_sum(s, buf);
    if (threadIdx.x == 0) drates[blockIdx.x] = (float)-s;
}

void backward_segments(int32_t n, int32_t heads, int32_t dk, int32_t dv, int32_t *seg_len,
                       int32_t *n_seg) {
    const int32_t tiles = attn_tiles(dk < dv ? dk : dv);
    attn_segments(n, (int64_t)heads * tiles, kBwdPerCu, seg_len, n_seg);
}

struct BwdSpace {
    float *before, *behind, *f_before, *f_behind, *dot_q, *dot_k;
    double *part;
    size_t bytes;
};
BwdSpace carve(void *ws, int32_t n, int32_t heads, int32_t dk, int32_t dv, int32_t n_seg) {
    Carver c(ws);
    BwdSpace s;
    const size_t states = (size_t)n_seg * heads * state_stride(dk, dv);
    s.before = c.take<float>(states);
    s.behind = c.take<float>(states);
    s.f_before = c.take<float>((size_t)n_seg * heads);
    s.f_behind = c.take<float>((size_t)n_seg * heads);
    s.dot_q = c.take<float>((size_t)attn_tiles(dk) * heads * n);
    s.dot_k = c.take<float>((size_t)attn_tiles(dk) * heads * n);
    s.part = c.take<double>((size_t)n_seg * heads);
    s.bytes = c.used;
    return s;
}

template <typename T, bool kRev> void states(const AttnPass &p, hipStream_t stream) {
    pass_dispatch(p.da, attn_tile(p.dc), [&](auto da, auto dct) {
        hipLaunchKernelGGL((attn_state_kernel<T, decltype(da)::value, decltype(dct)::value, kRev>),
                           pass_grid(p), dim3(kAttnThreads), 0, stream, p);
    });
    hipLaunchKernelGGL(attn_scan_kernel<kRev>,
                       dim3((unsigned)grid_for(p.state_stride, 64), (unsigned)p.heads), dim3(256),
                       0, stream, p.carry, p.factor, p.n_seg, p.heads, p.state_stride);
}

template <typename T, bool kRev> void pass(const AttnPass &p, hipStream_t stream) {
    pass_dispatch(p.da, attn_tile(p.dc), [&](auto da, auto dct) {
        hipLaunchKernelGGL(
            (attn_pass_kernel<T, decltype(da)::value, decltype(dct)::value, kRev, 3>),
            pass_grid(p), dim3(kAttnThreads), 0, stream, p);
    });
}

template <typename T>
sbc_status backward(const sbc_attention *a, const sbc_heads &dO, const sbc_heads &q,
                    const sbc_heads &k, const sbc_heads &v, const sbc_heads &dq,
                    const sbc_heads &dk, const sbc_heads &dv, float *drates, void *workspace,
                    hipStream_t stream) {
    AttnPass base{};
    base.n = a->n;
    base.n_batch = a->n_batch;
    base.heads = a->heads;
    base.scale = a->scale;
    base.rates = a->rates;
    base.splits = a->splits;
    base.t = a->t;
    base.state_stride = state_stride(a->dk, a->dv);
    backward_segments(a->n, a->heads, a->dk, a->dv, &base.seg_len, &base.n_seg);
    const BwdSpace s = carve(workspace, a->n, a->heads, a->dk, a->dv, base.n_seg);

    auto make = [&](const sbc_heads &x, const sbc_heads &y, const sbc_heads &z,
                    const sbc_heads &out, bool keys, bool back) {
        // keys: x and y have the channels of the keys, z and out those of the values
        AttnPass p = base;
        p.a = x;
        p.b = y;
        p.c = z;
        p.y = out;
        p.da = keys ? a->dk : a->dv;
        p.dc = keys ? a->dv : a->dk;
        p.tiles = attn_tiles(p.dc);
        p.carry = back ? s.behind : s.before;
        p.factor = back ? s.f_behind : s.f_before;
        // states lie as [dk, dv]
        p.carry_i = keys ? a->dv : 1;
        p.carry_j = keys ? 1 : a->dv;
        return p;
    };
    if (base.n_seg > 1) {
        trace_before("attn_bwd_state", stream);
        states<T, false>(make(q, k, v, q, true, false), stream);
        states<T, true>(make(k, q, dO, k, true, true), stream);
        trace_after("attn_bwd_state", stream);
    }
    AttnPass pq = make(dO, v, k, dq, false, false);
    AttnPass pk = make(v, dO, q, dk, false, true);
    AttnPass pv = make(k, q, dO, dv, true, true);
    if (drates) {
        pq.x = q;
        pq.dots = s.dot_q;
        pk.x = k;
        pk.dots = s.dot_k;
    }
    trace_before("attn_bwd", stream);
    pass<T, false>(pq, stream);
    pass<T, true>(pk, stream);
    pass<T, true>(pv, stream);
    trace_after("attn_bwd", stream);
    if (drates) {
        trace_before("attn_rates", stream);
        RatesArgs r{base, s.before, s.behind, a->dk * a->dv, s.dot_q, s.dot_k, pq.tiles, s.part};
        hipLaunchKernelGGL(attn_rates_kernel, dim3((unsigned)(base.n_seg * base.heads)), dim3(256),
                           0, stream, r);
        hipLaunchKernelGGL(attn_rates_sum_kernel, dim3((unsigned)base.heads), dim3(256), 0, stream,
                           s.part, base.n_seg, base.heads, drates);
        trace_after("attn_rates", stream);
    }
    SBC_LAUNCH_CHECK();
    return SBC_OK;
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" size_t sbc_linear_attention_backward_workspace_size(int32_t n, int32_t heads,
                                                               int32_t dk, int32_t dv) {
    if (n < 0 || heads <= 0 || dk <= 0 || dv <= 0 || dk > 128 || dv > 128) return 0;
    int32_t seg_len, n_seg;
    backward_segments(n, heads, dk, dv, &seg_len, &n_seg);
    return carve(nullptr, n, heads, dk, dv, n_seg).bytes;
}

extern "C" sbc_status sbc_linear_attention_backward(const sbc_attention *a, const sbc_heads *dO,
                                                    const sbc_heads *q, const sbc_heads *k,
                                                    const sbc_heads *v, const sbc_heads *dq,
                                                    const sbc_heads *dk, const sbc_heads *dv,
                                                    float *drates, void *workspace,
                                                    size_t workspace_bytes, hipStream_t stream) {
    clear_error();
    SBC_TRY(check_sequences(a));
    const int32_t n = a->n, H = a->heads;
    SBC_TRY(check_heads(dO, H, n, a->dv, a->dtype, "dO"));
    SBC_TRY(check_heads(q, H, n, a->dk, a->dtype, "q"));
    SBC_TRY(check_heads(k, H, n, a->dk, a->dtype, "k"));
    SBC_TRY(check_heads(v, H, n, a->dv, a->dtype, "v"));
    SBC_TRY(check_out_heads(dq, H, n, a->dk, a->dtype, "dq"));
    SBC_TRY(check_out_heads(dk, H, n, a->dk, a->dtype, "dk"));
    SBC_TRY(check_out_heads(dv, H, n, a->dv, a->dtype, "dv"));
    if (n == 0)
        return drates ? fill_i32(reinterpret_cast<int32_t *>(drates), 0, H, stream) : SBC_OK;
    const sbc_heads *in[4] = {dO, q, k, v}, *out[3] = {dq, dk, dv};
    const int32_t in_d[4] = {a->dv, a->dk, a->dk, a->dv}, out_d[3] = {a->dk, a->dk, a->dv};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 4; ++j)
            if (heads_overlap(*out[i], H, out_d[i], *in[j], H, in_d[j], n, a->dtype))
                return fail(SBC_ERR_INVALID_ARG, "a gradient overlaps an input");
        for (int j = 0; j < i; ++j)
            if (heads_overlap(*out[i], H, out_d[i], *out[j], H, out_d[j], n, a->dtype))
                return fail(SBC_ERR_INVALID_ARG, "two gradients overlap");
    }
    if (!workspace ||
        workspace_bytes < sbc_linear_attention_backward_workspace_size(n, H, a->dk, a->dv))
        return fail(SBC_ERR_WORKSPACE,
                    "workspace smaller than sbc_linear_attention_backward_workspace_size()");
    return a->dtype == SBC_F32
               ? backward<float>(a, *dO, *q, *k, *v, *dq, *dk, *dv, drates, workspace, stream)
               : backward<bf16_t>(a, *dO, *q, *k, *v, *dq, *dk, *dv, drates, workspace, stream);
}
