// Gradients of the linear attention with decays: passes of attention.hpp,
//
//   dq: (dO, v, k) along the sequence       dk: (v, dO, q) back along it
//   dv: (k, q, dO) back along it
//
// the last two in one (attention_grad.hpp) where a state is 64 x 64 or smaller.
//
// The rates' gradient.  With P_ij the term of a pair (its decay, both products and the
// scale), drate = - sum of (t_i - t_j) P_ij.  A chunk's own pairs are summed as they
// are.  The gap of any other is cut at the ends T of the chunks between:
//   t_i - t_j = (T_c(j) - t_j) + (T_{c(i)-1} - T_c(j)) + (t_i - T_{c(i)-1}).
// Of the first, dk's pass makes sum over j of (T - t_j) k_j . dk_j, with the part of dk_j
// from the state, and dq's pass makes sum over i of (t_i - T) q_i . dq_i of the last.
// The middle is carried by a second state of dq's pass along each segment,
//   S1 <- D (S1 + dt S)  from chunk to chunk,
// whose product with dO and q is summed for every token, and at the segment's end with
// the state that comes in from behind; the next segment goes on with S alone, from the
// time of this one's last token.  So every part of a gap is a factor of a term that its
// own decay has weakened, and nothing is left to cancel: a pause, however long, adds
// nothing to the error.  (300k tokens in bf16, 4 heads: 666 us for all gradients.  647 with
// sums that cancel, of k . dk less q . dq times the time to the segment's end; but where 190
// tokens with a rate of 0.05 hold pauses of 1.5e8, these are off by 4 to 11 %.)
#include "attention_host.hpp"
#include "attention_grad.hpp"

namespace sbc {
namespace {

// drates[h] = - the sums of both passes' workgroups, [parts, heads], in order
__global__ __launch_bounds__(256) void attn_rates_kernel(const double *__restrict__ along,
                                                         int32_t n_along,
                                                         const double *__restrict__ back,
                                                         int32_t n_back, int32_t heads,
                                                         float *__restrict__ drates) {
    __shared__ double buf[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < n_along; i += 256) s -= along[(int64_t)i * heads + blockIdx.x];
    for (int i = threadIdx.x; i < n_back; i += 256) s -= back[(int64_t)i * heads + blockIdx.x];
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) drates[blockIdx.x] = (float)((buf[0] + buf[1]) + (buf[2] + buf[3]));
}

// Workgroups a CU: what its registers hold of the passes up to 64 channels in bf16 (300k
// tokens, 4 heads: 666 us at 3, 683 at 2 with the registers for 2), else two.
void backward_segments(int32_t n, int32_t heads, int32_t dk, int32_t dv, sbc_dtype dtype,
                       int32_t *seg_len, int32_t *n_seg) {
    const bool three = dtype == SBC_BF16 && dk <= 64 && dv <= 64;
    const int32_t tiles = attn_tiles(dk < dv ? dk : dv);
    attn_segments(n, (int64_t)heads * tiles, three ? 3 : 2, seg_len, n_seg);
}

struct BwdSpace {
    float *before, *behind, *f_before, *f_behind;
    double *slope;
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
    s.slope = c.take<double>((size_t)2 * attn_tiles(dk) * n_seg * heads);
    s.bytes = c.used;
    return s;
}

// The states that the segments start from, along the sequences and back
template <typename T>
void states(AttnPass along, AttnPass back, bool whole_rows, hipStream_t stream) {
    along.tiles = back.tiles = attn_tiles(along.dc);
    pass_dispatch<T>(along.da, attn_tile(along.dc), whole_rows, [&](auto da, auto dct, auto whole) {
        dim3 grid = pass_grid(along);
        grid.x *= 2;
        hipLaunchKernelGGL((attn_states_kernel<T, decltype(da)::value, decltype(dct)::value,
                                               decltype(whole)::value>),
                           grid, dim3(kAttnThreads), 0, stream, along, back);
    });
    dim3 grid = scan_grid(along);
    grid.z = 2;
    hipLaunchKernelGGL(attn_scan_kernel, grid, dim3(256), 0, stream, along, back);
}

template <typename T, bool kRev, int NS, int kDots>
void pass(AttnPass p, bool whole_rows, hipStream_t stream) {
    p.tiles = attn_tiles(p.dc);
    pass_dispatch<T>(p.da, attn_tile(p.dc), whole_rows, [&](auto da, auto dct, auto whole) {
        hipLaunchKernelGGL((attn_pass_kernel<T, decltype(da)::value, decltype(dct)::value,
                                             decltype(whole)::value, kRev, NS, kDots>),
                           pass_grid(p), dim3(kAttnThreads), 0, stream, p);
    });
}

template <typename T, bool kDots>
void grad(const GradPass &g, bool whole_rows, hipStream_t stream) {
    const dim3 grid = pass_grid(g.p), block(kAttnThreads);
    if (!whole_rows)
        hipLaunchKernelGGL((attn_grad_kernel<T, 64, 64, false, kDots>), grid, block, 0, stream, g);
    else if (g.p.da <= 32 && g.p.dc <= 32)
        hipLaunchKernelGGL((attn_grad_kernel<T, 32, 32, true, kDots>), grid, block, 0, stream, g);
    else
        hipLaunchKernelGGL((attn_grad_kernel<T, 64, 64, true, kDots>), grid, block, 0, stream, g);
}

template <typename T, bool kDots>
void grads(const AttnPass &pq, const GradPass &both, hipStream_t stream) {
    const dim3 grid(pass_grid(pq).x + pass_grid(both.p).x), block(kAttnThreads);
    if (pq.da <= 32 && pq.dc <= 32)
        hipLaunchKernelGGL((attn_grads_kernel<T, 32, kDots>), grid, block, 0, stream, pq, both);
    else
        hipLaunchKernelGGL((attn_grads_kernel<T, 64, kDots>), grid, block, 0, stream, pq, both);
}

template <typename T, bool kDots>
void wide_grads(const AttnPass &pq, const AttnPass &pv, const AttnPass &pk, hipStream_t stream) {
    const dim3 grid(pass_grid(pq).x + pass_grid(pv).x + pass_grid(pk).x), block(kAttnThreads);
    if (pq.da <= 96 && pq.dc <= 96)
        hipLaunchKernelGGL((attn_wide_grads_kernel<T, 96, kDots>), grid, block, 0, stream, pq, pv,
                           pk);
    else
        hipLaunchKernelGGL((attn_wide_grads_kernel<T, 128, kDots>), grid, block, 0, stream, pq, pv,
                           pk);
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
    backward_segments(a->n, a->heads, a->dk, a->dv, a->dtype, &base.seg_len, &base.n_seg);
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
        p.factor = back ? s.f_behind : s.f_before;
        p.behind = s.behind;
        // states lie as [dk, dv]
        p.carry_i = keys ? a->dv : 1;
        p.carry_j = keys ? 1 : a->dv;
        return p;
    };
    if (base.n_seg > 1) {
        trace_before("attn_bwd_state", stream);
        states<T>(make(q, k, v, q, true, false), make(k, q, dO, k, true, true), whole, stream);
        trace_after("attn_bwd_state", stream);
    }
    // The states that meet the rates' gradient have three parts (and have them without it,
    // so that it changes no other gradient); dv has nothing to do with it.
    trace_before("attn_bwd", stream);
    const int32_t parts = attn_tiles(a->dk) * base.n_seg;
    double *back = s.slope + (size_t)parts * base.heads;
    AttnPass pq = make(dO, v, k, dq, false, false);
    AttnPass pv = make(k, q, dO, dv, true, true), pk = make(v, dO, q, dk, false, true);
    pq.tiles = pk.tiles = attn_tiles(a->dk);
    pv.tiles = attn_tiles(a->dv);
    pq.x = q;
    pq.slope = s.slope;
    pk.x = k;
    pk.slope = back;
    const bool narrow = a->dk <= 64 && a->dv <= 64;
    GradPass both{pv, k, v, dk, dv};
    both.p.tiles = 1;
    both.p.slope = back;
    // Together in one launch where dq's workgroups are at most three for two CUs: of 258
    // (11003 tokens, 3 heads) 51 us against 77 in bf16 and 145 against 150 at 40 and 72
    // channels in float32; of 64 31 against 47; of 512 150 against 133 at 128 channels in
    // bf16, where the joint kernel's registers leave fewer workgroups on a CU.
    const bool together = whole && 2 * (int64_t)parts * base.heads <= 3 * (int64_t)device_cus();
    auto run = [&](auto dots) {
        constexpr bool kDots = decltype(dots)::value;
        if (together && narrow)
            grads<T, kDots>(pq, both, stream);
        else if (together)
            wide_grads<T, kDots>(pq, pv, pk, stream);
        else
            pass<T, false, 3, kDots ? 1 : 0>(pq, whole, stream);
        if (!together && narrow) grad<T, kDots>(both, whole, stream);
        if (!together && !narrow) {
            pass<T, true, sizeof(T) == 4 ? 3 : 2, 0>(pv, whole, stream);
            pass<T, true, 3, kDots ? 2 : 0>(pk, whole, stream);
        }
    };
    if (drates)
        run(std::true_type{});
    else
        run(std::false_type{});
    trace_after("attn_bwd", stream);
    if (drates) {
        trace_before("attn_rates", stream);
        hipLaunchKernelGGL(attn_rates_kernel, dim3((unsigned)base.heads), dim3(256), 0, stream,
                           s.slope, parts, back, narrow ? base.n_seg : parts, base.heads,
                           drates);
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
    backward_segments(n, heads, dk, dv, SBC_BF16, &seg_len, &n_seg);  // (float32 has no more)
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
    auto heads = [&](const sbc_heads *x, int32_t d) { return region_heads(x, H, n, d, a->dtype); };
    SBC_TRY(check_apart({heads(dq, a->dk), heads(dk, a->dk), heads(dv, a->dv), region(drates, H, 4)},
                        {heads(dO, a->dv), heads(q, a->dk), heads(k, a->dk), heads(v, a->dv),
                         region(a->rates, H, 4), region(a->splits, (int64_t)a->n_batch + 1, 4),
                         region(a->t, n, 4)}));
    if (!workspace ||
        workspace_bytes < sbc_linear_attention_backward_workspace_size(n, H, a->dk, a->dv))
        return fail(SBC_ERR_WORKSPACE,
                    "workspace smaller than sbc_linear_attention_backward_workspace_size()");
    return a->dtype == SBC_F32
               ? backward<float>(a, *dO, *q, *k, *v, *dq, *dk, *dv, drates, workspace, stream)
               : backward<bf16_t>(a, *dO, *q, *k, *v, *dq, *dk, *dv, drates, workspace, stream);
}
