// Softmax attention of new tokens over a paged cache.
#include "softmax_launch.hpp"

namespace sbc {
namespace {

// Fields that the call does not read are taken as 0 from here on
sbc_status check_paged(const sbc_softmax_attention *&a, sbc_softmax_attention *read, int32_t n_pages,
                       int32_t page, int32_t width) {
    if (a) {
        *read = *a;
        read->m = read->causal = 0;
        read->k_splits = nullptr;
        a = read;
    }
    SBC_TRY(check_softmax(a));
    if (!a->splits && a->n != a->n_batch)
        return fail(SBC_ERR_INVALID_ARG, "without splits every sequence has one new token (n = n_batch)");
    if (a->n > 0 && a->n_batch == 0)
        return fail(SBC_ERR_INVALID_ARG, "tokens without a sequence (n_batch 0)");
    if (n_pages < 0 || page <= 0 || width < 0)
        return fail(SBC_ERR_INVALID_ARG, "n_pages and width must be >= 0 and page > 0");
    return SBC_OK;
}
int64_t most_keys(int32_t page, int32_t width) {
    const int64_t keys = (int64_t)page * width;
    return keys > INT32_MAX ? INT32_MAX : keys;
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" size_t sbc_softmax_attention_paged_workspace_size(const sbc_softmax_attention *a,
                                                             int32_t page, int32_t width) {
    sbc_softmax_attention read;
    if (check_paged(a, &read, 0, page, width) != SBC_OK) return 0;
    return softmax_workspace(a, softmax_plan(a, most_keys(page, width)));
}

extern "C" sbc_status sbc_softmax_attention_paged(const sbc_softmax_attention *a, const sbc_heads *q,
                                                  const sbc_pages *k, const sbc_pages *v,
                                                  int32_t n_pages, int32_t page,
                                                  const int32_t *table, int32_t width,
                                                  const int32_t *lengths, const sbc_heads *o,
                                                  float *lse, void *workspace,
                                                  size_t workspace_bytes, hipStream_t stream) {
    clear_error();
    sbc_softmax_attention read;
    SBC_TRY(check_paged(a, &read, n_pages, page, width));
    const int32_t n = a->n, H = a->heads, G = a->kv_heads;
    const sbc_dtype dt = a->dtype;
    SBC_TRY(check_heads(q, H, n, a->dk, dt, "q"));
    SBC_TRY(check_out_heads(o, H, n, a->dv, dt, "o"));
    SBC_TRY(check_pages(k, n_pages, page, G, a->dk, dt, "k_pages"));
    SBC_TRY(check_pages(v, n_pages, page, G, a->dv, dt, "v_pages"));
    if (n == 0) return SBC_OK;
    if (!table || !lengths) return fail(SBC_ERR_INVALID_ARG, "table or lengths is null");
    SBC_TRY(check_apart({region_heads(o, H, n, a->dv, dt), region(lse, (int64_t)n * H, 4)},
                        {region_heads(q, H, n, a->dk, dt), region_pages(k, n_pages, page, G, a->dk, dt),
                         region_pages(v, n_pages, page, G, a->dv, dt),
                         region(table, (int64_t)a->n_batch * width, 4), region(lengths, a->n_batch, 4),
                         region(a->splits, (int64_t)a->n_batch + 1, 4)}));
    const SoftmaxPlan plan = softmax_plan(a, most_keys(page, width));
    const size_t needed = softmax_workspace(a, plan);
    if (needed > 0 && (!workspace || workspace_bytes < needed))
        return fail(SBC_ERR_WORKSPACE,
                    "workspace smaller than sbc_softmax_attention_paged_workspace_size()");
    SoftmaxArgs p = softmax_args(a);
    p.causal = 1;
    p.q = *q;
    p.o = *o;
    p.lse = lse;
    if (n_pages > 0) {
        p.pages.k = *k;
        p.pages.v = *v;
    }
    p.pages.n_pages = n_pages;
    p.pages.width = n_pages > 0 ? width : 0;
    p.pages.page = divisor(page);
    p.pages.table = table;
    p.pages.lengths = lengths;
    return dt == SBC_F32 ? softmax_forward<float, true>(p, a, plan, workspace, stream)
                         : softmax_forward<bf16_t, true>(p, a, plan, workspace, stream);
}
