// Softmax attention over packed sequences, gradients.
#include "softmax_grad.hpp"
#include "softmax_host.hpp"

namespace sbc {
namespace {

// Parts of the rows for dk and dv: as many as give every CU three workgroups, of 128 rows or more
// (a causal sequence's first keys are seen by all rows, its last by few)
int32_t grad_parts(const sbc_softmax_attention *a) {
    const int64_t tiles = ((int64_t)a->m / kGradCols + a->n_batch) * a->kv_heads;
    const int64_t rows = (int64_t)a->n * (a->heads / a->kv_heads) / (a->n_batch > 0 ? a->n_batch : 1);
    int64_t parts = ((int64_t)3 * device_cus() + tiles - 1) / (tiles > 0 ? tiles : 1);
    if (parts > rows / 128) parts = rows / 128;
    if (parts > 16) parts = 16;
    // so many that each of the 8 XCDs has key heads and parts, and their rows, of its own
    int32_t even = 8;
    while (even > 1 && a->kv_heads % (8 / even * 2) == 0) even /= 2;
    const int64_t up = (parts + even - 1) / even * even;
    if (parts > 1 && up <= 2 * parts && up <= 16) parts = up;
    return parts < 1 ? 1 : (int32_t)parts;
}
// One launch for all: while its workgroups are all on the CUs at once
bool grads_joint(const sbc_softmax_attention *a) {
    const int64_t rows = softmax_places(a, 128), keys = (int64_t)a->m / kGradCols + a->n_batch;
    return a->n > 0 && a->m > 0 && (rows + 2 * keys * grad_parts(a)) * a->kv_heads <= 2 * device_cus();
}
void carve(const sbc_softmax_attention *a, void *workspace, SoftmaxArgs *p, size_t *used) {
    Carver c(workspace);
    p->parts = grad_parts(a);
    if (!grads_joint(a)) {
        p->row_delta = c.take<float>((size_t)a->n * a->heads);
        p->row_lse = c.take<float>((size_t)a->n * a->heads);
    }
    if (p->parts > 1) {
        p->part_dk = c.take<float>((size_t)p->parts * a->m * a->kv_heads * a->dk);
        p->part_dv = c.take<float>((size_t)p->parts * a->m * a->kv_heads * a->dv);
    }
    *used = c.used;
}

template <typename T, bool kWhole>
sbc_status backward(SoftmaxArgs p, const sbc_softmax_attention *a, hipStream_t stream) {
    const int64_t dq_blocks = softmax_places(a, 128) * a->kv_heads;
    const int64_t cols = (int64_t)a->m / kGradCols + a->n_batch;
    const int64_t dkv_blocks = cols * a->kv_heads * p.parts;
    const int64_t join = ((int64_t)a->m * a->kv_heads * ((a->dk > a->dv ? a->dk : a->dv) + 3) / 4 + 255) / 256 + 1;
    if (dq_blocks >= (int64_t)1 << 24 || dkv_blocks >= (int64_t)1 << 23 ||
        (p.parts > 1 && join >= (int64_t)1 << 24))
        return fail(SBC_ERR_UNSUPPORTED, "more than 2^24 workgroups needed");
    softmax_dispatch(a->dk > a->dv ? a->dk : a->dv, [&](auto d) {
        constexpr int D = decltype(d)::value;
        constexpr int kRows = kGradRows<T, D>;
        const int32_t group = a->heads / a->kv_heads;
        p.even_rows = kRows % group == 0;
        for (const sbc_heads *x : {&p.q, &p.d_o})
            if (x->token_stride >= 1 << 22 || x->head_stride > ((int64_t)1 << 28) / group)
                p.even_rows = 0;
        const int32_t dkv_kinds = kGradsApart<T, D> ? 2 : 1;
        p.slots = (int32_t)softmax_places(a, 128);  // (of rows)
        if (grads_joint(a)) {
            trace_before("softmax_grads", stream);
            hipLaunchKernelGGL((softmax_grads_kernel<T, D, kWhole>),
                               dim3((unsigned)(dq_blocks + dkv_blocks * dkv_kinds)),
                               dim3(kGradThreads), 0, stream, p, (int32_t)dq_blocks,
                               (int32_t)dkv_blocks);
            trace_after("softmax_grads", stream);
            return;
        }
        if (a->n > 0) {
            trace_before("softmax_dq", stream);
            hipLaunchKernelGGL((softmax_dq_kernel<T, D, kWhole>), dim3((unsigned)dq_blocks),
                               dim3(kGradThreads), 0, stream, p);
            trace_after("softmax_dq", stream);
        }
        if (a->m > 0) {
            trace_before("softmax_dkv", stream);
            const dim3 grid((unsigned)(dkv_blocks * dkv_kinds)), block(kGradThreads);
            constexpr bool kCan = sizeof(T) == 2 && D % 64 == 0 && kWhole;
            if (kCan && p.even_rows && a->dk == D && softmax_direct(a, {&p.q, &p.d_o}))
                hipLaunchKernelGGL((softmax_dkv_kernel<T, D, kWhole, kCan>), grid, block, 0, stream, p);
            else
                hipLaunchKernelGGL((softmax_dkv_kernel<T, D, kWhole, false>), grid, block, 0, stream, p);
            trace_after("softmax_dkv", stream);
        }
    });
    SBC_LAUNCH_CHECK();
    if (p.parts > 1 && a->m > 0) {
        trace_before("softmax_dkv_join", stream);
        hipLaunchKernelGGL(softmax_dkv_join_kernel<T>, dim3((unsigned)join, 2), dim3(256), 0, stream, p);
        SBC_LAUNCH_CHECK();
        trace_after("softmax_dkv_join", stream);
    }
    return SBC_OK;
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" size_t sbc_softmax_attention_backward_workspace_size(const sbc_softmax_attention *a) {
    if (check_softmax_sequences(a) != SBC_OK) return 0;
    SoftmaxArgs p{};
    size_t used = 0;
    carve(a, nullptr, &p, &used);
    return used;
}

extern "C" sbc_status sbc_softmax_attention_backward(
    const sbc_softmax_attention *a, const sbc_heads *dO, const sbc_heads *q, const sbc_heads *k,
    const sbc_heads *v, const sbc_heads *o, const float *lse, const sbc_heads *dq,
    const sbc_heads *dk, const sbc_heads *dv, void *workspace, size_t workspace_bytes,
    hipStream_t stream) {
    clear_error();
    SBC_TRY(check_softmax_sequences(a));
    const int32_t n = a->n, m = a->m, H = a->heads, G = a->kv_heads;
    const sbc_dtype dt = a->dtype;
    SBC_TRY(check_heads(dO, H, n, a->dv, dt, "dO"));
    SBC_TRY(check_heads(q, H, n, a->dk, dt, "q"));
    SBC_TRY(check_heads(k, G, m, a->dk, dt, "k"));
    SBC_TRY(check_heads(v, G, m, a->dv, dt, "v"));
    SBC_TRY(check_heads(o, H, n, a->dv, dt, "o"));
    SBC_TRY(check_out_heads(dq, H, n, a->dk, dt, "dq"));
    SBC_TRY(check_out_heads(dk, G, m, a->dk, dt, "dk"));
    SBC_TRY(check_out_heads(dv, G, m, a->dv, dt, "dv"));
    if (n == 0 && m == 0) return SBC_OK;
    if (n > 0 && !lse) return fail(SBC_ERR_INVALID_ARG, "lse is null");
    SBC_TRY(check_apart({region_heads(dq, H, n, a->dk, dt), region_heads(dk, G, m, a->dk, dt),
                         region_heads(dv, G, m, a->dv, dt)},
                        {region_heads(dO, H, n, a->dv, dt), region_heads(q, H, n, a->dk, dt),
                         region_heads(k, G, m, a->dk, dt), region_heads(v, G, m, a->dv, dt),
                         region_heads(o, H, n, a->dv, dt), region(lse, (int64_t)n * H, 4),
                         region(a->splits, (int64_t)a->n_batch + 1, 4),
                         region(a->k_splits, (int64_t)a->n_batch + 1, 4)}));
    SoftmaxArgs p = softmax_args(a);
    size_t used = 0;
    carve(a, workspace, &p, &used);
    if (used > 0 && (!workspace || workspace_bytes < used))
        return fail(SBC_ERR_WORKSPACE,
                    "workspace smaller than sbc_softmax_attention_backward_workspace_size()");
    if (n > 0) {
        p.d_o = *dO;
        p.q = *q;
        p.o = *o;
        p.dq = *dq;
    }
    if (m > 0) {
        p.k = *k;
        p.v = *v;
        p.dk_out = *dk;
        p.dv_out = *dv;
    }
    p.lse_in = lse;
    const bool whole = softmax_whole(a, {&p.k, &p.v});
    if (dt == SBC_F32)
        return whole ? backward<float, true>(p, a, stream) : backward<float, false>(p, a, stream);
    return whole ? backward<bf16_t, true>(p, a, stream) : backward<bf16_t, false>(p, a, stream);
}
