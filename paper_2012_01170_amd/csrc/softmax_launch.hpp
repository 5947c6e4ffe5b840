// Launches of softmax attention's forward pass.
#pragma once

#include "softmax_host.hpp"
#include "softmax_kernels.hpp"

namespace sbc {

template <typename T, bool kPaged>
sbc_status softmax_forward(SoftmaxArgs p, const sbc_softmax_attention *a, const SoftmaxPlan &plan,
                           void *workspace, hipStream_t stream) {
    if (plan.blocks >= (int64_t)1 << 24)  // (a launch holds fewer than 2^32 work-items)
        return fail(SBC_ERR_UNSUPPORTED, "more than 2^24 workgroups needed");
    p.slots = (int32_t)softmax_places(a, plan.few ? kFewRows : kTileRows);
    p.parts = plan.parts;
    if (plan.parts > 1) {
        Carver c(workspace);
        p.part_o = c.take<float>((size_t)plan.parts * a->n * a->heads * a->dv);
        p.part_lse = c.take<float>((size_t)plan.parts * a->n * a->heads);
    }
    const dim3 grid((unsigned)plan.blocks), block(kSoftmaxThreads);
    const bool whole = softmax_whole(a, {&p.k, &p.v});
    trace_before("softmax_fwd", stream);
    softmax_dispatch(a->dk > a->dv ? a->dk : a->dv, [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (plan.few && whole)
            hipLaunchKernelGGL((softmax_rows_kernel<T, D, true, kPaged>), grid, block, 0, stream, p);
        else if (plan.few)
            hipLaunchKernelGGL((softmax_rows_kernel<T, D, false, kPaged>), grid, block, 0, stream, p);
        else if (constexpr bool kCan = sizeof(T) == 2 && D % 64 == 0 && !kPaged;
                 kCan && whole && a->dk == D && softmax_direct(a, {&p.k, &p.v}))
            hipLaunchKernelGGL((softmax_tile_kernel<T, D, true, kPaged, kCan>), grid, block, 0, stream,
                               p);
        else if (whole)
            hipLaunchKernelGGL((softmax_tile_kernel<T, D, true, kPaged>), grid, block, 0, stream, p);
        else
            hipLaunchKernelGGL((softmax_tile_kernel<T, D, false, kPaged>), grid, block, 0, stream, p);
    });
    SBC_LAUNCH_CHECK();
    trace_after("softmax_fwd", stream);
    if (plan.parts > 1) {
        trace_before("softmax_join", stream);
        const int64_t rows = (int64_t)a->n * a->heads;
        if (plan.parts > 8)
            hipLaunchKernelGGL((softmax_join_kernel<T, kPaged, 4>), dim3((unsigned)rows), dim3(256), 0,
                               stream, p);
        else
            hipLaunchKernelGGL((softmax_join_kernel<T, kPaged, 1>), dim3((unsigned)((rows + 3) / 4)),
                               dim3(256), 0, stream, p);
        SBC_LAUNCH_CHECK();
        trace_after("softmax_join", stream);
    }
    return SBC_OK;
}

}  // namespace sbc
