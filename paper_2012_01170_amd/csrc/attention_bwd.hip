// Gradients of the linear attention with decays: three passes of attention.hpp.
//
//   dq: (dO, v, k) along the sequence       dk: (v, dO, q) back along it
//   dv: (k, q, dO) back along it
// and the rates' gradient beside dk: drate = - sum of (t_i - t_j) times the terms of
// y = dk summed over j against k_j, the pass' kSlope.  (From the products k . dk and
// q . dq of the tokens alone, as a flow that each token adds to and takes from, it
// would lose what the flow's rounding gains over a segment: 4e-6 to 1e-5.)
#include "attention_host.hpp"
#include "attention_kernels.hpp"

namespace sbc {
namespace {

constexpr int kBwdPerCu = 2;

// drates[h] = - the sum of the workgroups' parts [parts, heads], in order
__global__ __launch_bounds__(256) void attn_rates_kernel(const double *__restrict__ part,
                                                         int32_t parts, int32_t heads,
                                                         float *__restrict__ drates) {
    __shared__ double buf[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += part[(int64_t)i * heads + blockIdx.x];
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) drates[blockIdx.x] = (float)-((buf[0] + buf[1]) + (buf[2] + buf[3]));
}

// Columns of a tile: of float32 and 128 channels, a state and its derivative leave
// LDS room for 32.
int bwd_tile(int32_t da, int32_t dc, bool slope, sbc_dtype dtype) {
    return slope && dtype == SBC_F32 && da > 96 ? 32 : attn_tile(dc);
}

void backward_segments(int32_t n, int32_t heads, int32_t dk, int32_t dv, int32_t *seg_len,
                       int32_t *n_seg) {
    const int32_t tiles = attn_tiles(dk < dv ? dk : dv);
    attn_segments(n, (int64_t)heads * tiles, kBwdPerCu, seg_len, n_seg);
}

struct BwdSpace {
    float *before, *behind, *behind1, *f_before, *f_behind, *gap;
    double *slope;
    size_t bytes;
};
BwdSpace carve(void *ws, int32_t n, int32_t heads, int32_t dk, int32_t dv, int32_t n_seg) {
    Carver c(ws);
    BwdSpace s;
    const size_t states = (size_t)n_seg * heads * state_stride(dk, dv);
    s.before = c.take<float>(states);
    s.behind = c.take<float>(states);
    s.behind1 = c.take<float>(states);
    s.f_before = c.take<float>((size_t)n_seg * heads);
    s.f_behind = c.take<float>((size_t)n_seg * heads);
    s.gap = c.take<float>(n_seg);
    s.slope = c.take<double>((size_t)((dk + 31) / 32) * n_seg * heads);
    s.bytes = c.used;
    return s;
}

template <typename T, bool kRev, bool kSlope>
void states(AttnPass p, bool whole_rows, hipStream_t stream) {
    p.tiles = attn_tiles(p.dc);
    pass_dispatch<T>(p.da, attn_tile(p.dc), whole_rows, [&](auto da, auto dct, auto whole) {
        hipLaunchKernelGGL((attn_state_kernel<T, decltype(da)::value, decltype(dct)::value,
                                              decltype(whole)::value, kRev, kSlope>),
                           pass_grid(p), dim3(kAttnThreads), 0, stream, p);
    });
    hipLaunchKernelGGL((attn_scan_kernel<kRev, kSlope>), scan_grid(p), dim3(256), 0, stream, p);
}

// (dk takes three parts also without the rates' gradient, which must not change it)
template <typename T, bool kRev, int NS, bool kSlope>
void pass(AttnPass p, bool whole_rows, hipStream_t stream) {
    const int dct = bwd_tile(p.da, p.dc, kSlope, sizeof(T) == 4 ? SBC_F32 : SBC_BF16);
    p.tiles = (p.dc + dct - 1) / dct;
    pass_dispatch<T>(p.da, dct, whole_rows, [&](auto da, auto dct, auto whole) {
        constexpr int DA = decltype(da)::value, DCT = decltype(dct)::value;
        if constexpr (!(kSlope && sizeof(T) == 4 && DA > 96 && DCT > 32))
            hipLaunchKernelGGL(
                (attn_pass_kernel<T, DA, DCT, decltype(whole)::value, kRev, NS, kSlope>),
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
    const bool whole = whole_rows(a, {&dO, &q, &k, &v});

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
        p.carry = back ? s.behind : s.before;
        p.carry1 = s.behind1;
        p.factor = back ? s.f_behind : s.f_before;
        p.gap = s.gap;
        // states lie as [dk, dv]
        p.carry_i = keys ? a->dv : 1;
        p.carry_j = keys ? 1 : a->dv;
        return p;
    };
    if (base.n_seg > 1) {
        trace_before("attn_bwd_state", stream);
        states<T, false, false>(make(q, k, v, q, true, false), whole, stream);
        const AttnPass back = make(k, q, dO, k, true, true);
        if (drates)
            states<T, true, true>(back, whole, stream);
        else
            states<T, true, false>(back, whole, stream);
        trace_after("attn_bwd_state", stream);
    }
    constexpr int NS = sizeof(T) == 4 ? 3 : 2;
    trace_before("attn_bwd", stream);
    pass<T, false, NS, false>(make(dO, v, k, dq, false, false), whole, stream);
    pass<T, true, NS, false>(make(k, q, dO, dv, true, true), whole, stream);
    AttnPass pk = make(v, dO, q, dk, false, true);
    if (drates) {
        pk.x = k;
        pk.slope = s.slope;
        pass<T, true, 3, true>(pk, whole, stream);
    } else {
        pass<T, true, 3, false>(pk, whole, stream);
    }
    trace_after("attn_bwd", stream);
    if (drates) {
        trace_before("attn_rates", stream);
        const int dct = bwd_tile(a->dv, a->dk, true, a->dtype);
        hipLaunchKernelGGL(attn_rates_kernel, dim3((unsigned)base.heads), dim3(256), 0, stream,
                           s.slope, (a->dk + dct - 1) / dct * base.n_seg, base.heads, drates);
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
