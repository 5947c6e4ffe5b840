// Linear attention with decays, forward over whole sequences (attention.hpp).
#include "attention_host.hpp"
#include "attention_kernels.hpp"

namespace sbc {
namespace {

// Workgroups a CU: what its registers (bf16) or LDS (float32) hold of 64 channels.
// 300k tokens in bf16, 4 heads: 240 us at 2, 231 at 3, 243 at 4; 32768 in float32: 83
// at 2, 91 at 3.
void forward_segments(int32_t n, int32_t heads, int32_t dv, sbc_dtype dtype, int32_t *seg_len,
                      int32_t *n_seg) {
    attn_segments(n, (int64_t)heads * attn_tiles(dv), dtype == SBC_F32 ? 2 : 3, seg_len, n_seg);
}

template <typename T> sbc_status forward(const AttnPass &p, bool whole_rows, hipStream_t stream) {
    constexpr int NS = sizeof(T) == 4 ? 3 : 2;
    pass_dispatch<T>(p.da, attn_tile(p.dc), whole_rows, [&](auto da, auto dct, auto whole) {
        constexpr int DA = decltype(da)::value, DCT = decltype(dct)::value;
        constexpr bool W = decltype(whole)::value;
        if (p.n_seg > 1) {
            trace_before("attn_state", stream);
            hipLaunchKernelGGL((attn_state_kernel<T, DA, DCT, W, false>), pass_grid(p),
                               dim3(kAttnThreads), 0, stream, p);
            trace_after("attn_state", stream);
            trace_before("attn_scan", stream);
            hipLaunchKernelGGL(attn_scan_kernel, scan_grid(p), dim3(256), 0, stream, p, p);
            trace_after("attn_scan", stream);
        }
        trace_before("attn_fwd", stream);
        hipLaunchKernelGGL((attn_pass_kernel<T, DA, DCT, W, false, NS, 0, true>), pass_grid(p),
                           dim3(kAttnThreads), 0, stream, p);
        trace_after("attn_fwd", stream);
    });
    SBC_LAUNCH_CHECK();
    return SBC_OK;
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" size_t sbc_linear_attention_workspace_size(int32_t n, int32_t heads, int32_t dk,
                                                      int32_t dv) {
    if (n < 0 || heads <= 0 || dk <= 0 || dv <= 0 || dk > 128 || dv > 128) return 0;
    int32_t seg_len, n_seg;
    forward_segments(n, heads, dv, SBC_BF16, &seg_len, &n_seg);  // (float32 has no more)
    Carver c(nullptr);
    c.take<float>((size_t)n_seg * heads * state_stride(dk, dv));
    c.take<float>((size_t)n_seg * heads);
    return c.used;
}

extern "C" sbc_status sbc_linear_attention_forward(const sbc_attention *a, const sbc_heads *q,
                                                   const sbc_heads *k, const sbc_heads *v,
                                                   const float *state_in,
                                                   const int32_t *state_time, const sbc_heads *o,
                                                   float *state_out, int32_t *time_out,
                                                   void *workspace, size_t workspace_bytes,
                                                   hipStream_t stream) {
    clear_error();
    SBC_TRY(check_sequences(a));
    const int32_t n = a->n, H = a->heads;
    SBC_TRY(check_heads(q, H, n, a->dk, a->dtype, "q"));
    SBC_TRY(check_heads(k, H, n, a->dk, a->dtype, "k"));
    SBC_TRY(check_heads(v, H, n, a->dv, a->dtype, "v"));
    SBC_TRY(check_out_heads(o, H, n, a->dv, a->dtype, "o"));
    if (a->t && state_in && !state_time)
        return fail(SBC_ERR_INVALID_ARG, "a state needs its time (state_time) where t is given");
    if (a->t && (state_out != nullptr) != (time_out != nullptr))
        return fail(SBC_ERR_INVALID_ARG, "with t, state_out and time_out go together");
    if (n == 0 && (a->n_batch == 0 || !state_out)) return SBC_OK;
    const int64_t states = (int64_t)a->n_batch * H * a->dk * a->dv;
    if (!a->t) state_time = time_out = nullptr;
    SBC_TRY(check_apart({region_heads(o, H, n, a->dv, a->dtype), region(state_out, states, 4),
                         region(time_out, a->n_batch, 4)},
                        {region_heads(q, H, n, a->dk, a->dtype), region_heads(k, H, n, a->dk, a->dtype),
                         region_heads(v, H, n, a->dv, a->dtype), region(state_in, states, 4),
                         region(state_time, a->n_batch, 4), region(a->rates, H, 4),
                         region(a->splits, (int64_t)a->n_batch + 1, 4), region(a->t, n, 4)}));
    if (!a->rates) return fail(SBC_ERR_INVALID_ARG, "rates is null");
    if (!workspace || workspace_bytes < sbc_linear_attention_workspace_size(n, H, a->dk, a->dv))
        return fail(SBC_ERR_WORKSPACE,
                    "workspace smaller than sbc_linear_attention_workspace_size()");
    AttnPass p{};
    p.n = n;
    p.n_batch = a->n_batch;
    p.heads = H;
    p.da = a->dk;
    p.dc = a->dv;
    forward_segments(n, H, a->dv, a->dtype, &p.seg_len, &p.n_seg);
    p.tiles = attn_tiles(a->dv);
    p.scale = a->scale;
    p.rates = a->rates;
    p.splits = a->splits;
    p.t = a->t;
    if (n > 0) {
        p.a = *q;
        p.b = *k;
        p.c = *v;
        p.y = *o;
    }
    Carver c(workspace);
    p.state_stride = state_stride(a->dk, a->dv);
    p.carry = c.take<float>((size_t)p.n_seg * H * p.state_stride);
    p.factor = c.take<float>((size_t)p.n_seg * H);
    p.carry_i = a->dv;
    p.carry_j = 1;
    p.state_in = state_in;
    p.state_time = state_time;
    p.state_out = state_out;
    p.time_out = time_out;
    const bool whole = n > 0 && whole_rows(a, {q, k, v});
    return a->dtype == SBC_F32 ? forward<float>(p, whole, stream)
                               : forward<bf16_t>(p, whole, stream);
}
