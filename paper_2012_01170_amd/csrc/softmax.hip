// Softmax attention over packed sequences, forward.
#include "softmax_launch.hpp"

using namespace sbc;

extern "C" size_t sbc_softmax_attention_workspace_size(const sbc_softmax_attention *a) {
    if (check_softmax_sequences(a) != SBC_OK) return 0;
    return softmax_workspace(a, softmax_plan(a, a->m));
}

extern "C" sbc_status sbc_softmax_attention_forward(const sbc_softmax_attention *a,
                                                    const sbc_heads *q, const sbc_heads *k,
                                                    const sbc_heads *v, const sbc_heads *o,
                                                    float *lse, void *workspace,
                                                    size_t workspace_bytes, hipStream_t stream) {
    clear_error();
    SBC_TRY(check_softmax_sequences(a));
    const int32_t n = a->n, m = a->m, H = a->heads, G = a->kv_heads;
    const sbc_dtype dt = a->dtype;
    SBC_TRY(check_heads(q, H, n, a->dk, dt, "q"));
    SBC_TRY(check_heads(k, G, m, a->dk, dt, "k"));
    SBC_TRY(check_heads(v, G, m, a->dv, dt, "v"));
    SBC_TRY(check_out_heads(o, H, n, a->dv, dt, "o"));
    if (n == 0) return SBC_OK;
    SBC_TRY(check_apart({region_heads(o, H, n, a->dv, dt), region(lse, (int64_t)n * H, 4)},
                        {region_heads(q, H, n, a->dk, dt), region_heads(k, G, m, a->dk, dt),
                         region_heads(v, G, m, a->dv, dt),
                         region(a->splits, (int64_t)a->n_batch + 1, 4),
                         region(a->k_splits, (int64_t)a->n_batch + 1, 4)}));
    const SoftmaxPlan plan = softmax_plan(a, m);
    const size_t needed = softmax_workspace(a, plan);
    if (needed > 0 && (!workspace || workspace_bytes < needed))
        return fail(SBC_ERR_WORKSPACE,
                    "workspace smaller than sbc_softmax_attention_workspace_size()");
    SoftmaxArgs p = softmax_args(a);
    p.q = *q;
    if (m > 0) {
        p.k = *k;
        p.v = *v;
    }
    p.o = *o;
    p.lse = lse;
    return dt == SBC_F32 ? softmax_forward<float, false>(p, a, plan, workspace, stream)
                         : softmax_forward<bf16_t, false>(p, a, plan, workspace, stream);
}
