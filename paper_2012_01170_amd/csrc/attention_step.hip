// Linear attention with decays, one token for each of many streams:
//   S = exp(-rate dt) S + k v^T,  o = scale q S.
// A state is read and written once (8 bytes a value, three operations), so
// memory bounds it, and for few streams the launch.  The columns of a state do
// not meet: a workgroup has a tile of kCols of them, 4 a lane, and 256 / (kCols
// / 4) lanes down a column, whose parts of o are added in LDS.
#include "attention_host.hpp"

namespace sbc {
namespace {

struct StepArgs {
    int32_t n, heads, dk, dv, tiles;
    float scale;
    const float *rates;
    const int32_t *t, *state_time;
    sbc_heads q, k, v, o;
    const float *state_in;
    float *state_out;
    int32_t *time_out;
};

constexpr int kCols = 64;
constexpr int kAcross = kCols / 4;
constexpr int kDown = 256 / kAcross;

template <typename T>
__global__ __launch_bounds__(256) void attn_step_kernel(StepArgs p) {
    __shared__ float part[kDown][kCols + 4];
    const int tile = blockIdx.x % p.tiles;
    const int head = (blockIdx.x / p.tiles) % p.heads;
    const int64_t i = blockIdx.x / p.tiles / p.heads;
    const int across = threadIdx.x % kAcross, down = threadIdx.x / kAcross;
    const int c = tile * kCols + 4 * across;
    const int have = p.dv - c;
    const T *q = static_cast<const T *>(p.q.data) + i * p.q.token_stride + head * p.q.head_stride;
    const T *k = static_cast<const T *>(p.k.data) + i * p.k.token_stride + head * p.k.head_stride;
    const T *v = static_cast<const T *>(p.v.data) + i * p.v.token_stride + head * p.v.head_stride;
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = j < have ? to_f32(v[c + j]) : 0.f;
    float dt = 1.f;
    if (p.t) dt = (float)((uint32_t)p.t[i] - (uint32_t)p.state_time[i]);
    const float keep = expf(-p.rates[head] * dt);
    const int64_t base = (i * p.heads + head) * (int64_t)p.dk * p.dv + c;
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    if (have > 0) {
#pragma unroll 4
        for (int r = down; r < p.dk; r += kDown) {
            float s[4];
            load_f32<4>(p.state_in + base + (int64_t)r * p.dv, have, s);
            const float kr = to_f32(k[r]), qr = to_f32(q[r]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j] = fmaf(kr, x[j], keep * s[j]);
                o[j] = fmaf(qr, s[j], o[j]);
            }
            store_vec<float>(p.state_out + base + (int64_t)r * p.dv, have, s);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) part[down][4 * across + j] = o[j];
    __syncthreads();
    if (threadIdx.x < kCols && tile * kCols + (int)threadIdx.x < p.dv) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < kDown; ++r) sum += part[r][threadIdx.x];
        static_cast<T *>(p.o.data)[i * p.o.token_stride + head * p.o.head_stride + tile * kCols +
                                   threadIdx.x] = from_f32<T>(sum * p.scale);
    }
    if (p.time_out && tile == 0 && head == 0 && threadIdx.x == 0) p.time_out[i] = p.t[i];
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" sbc_status sbc_linear_attention_step(const sbc_attention *a, const sbc_heads *q,
                                                const sbc_heads *k, const sbc_heads *v,
                                                const float *state_in, const int32_t *state_time,
                                                const sbc_heads *o, float *state_out,
                                                int32_t *time_out, hipStream_t stream) {
    clear_error();
    SBC_TRY(check_attention(a));
    const int32_t n = a->n, H = a->heads;
    SBC_TRY(check_heads(q, H, n, a->dk, a->dtype, "q"));
    SBC_TRY(check_heads(k, H, n, a->dk, a->dtype, "k"));
    SBC_TRY(check_heads(v, H, n, a->dv, a->dtype, "v"));
    SBC_TRY(check_out_heads(o, H, n, a->dv, a->dtype, "o"));
    if (n == 0) return SBC_OK;
    if (!state_in || !state_out) return fail(SBC_ERR_INVALID_ARG, "state_in or state_out is null");
    if (a->t && (!state_time || !time_out))
        return fail(SBC_ERR_INVALID_ARG, "with t, state_time and time_out are needed");
    const Region tokens = region_heads(o, H, n, a->dv, a->dtype);
    const Region state = region(state_out, (int64_t)n * H * a->dk * a->dv, 4);
    const Region times = region(a->t ? time_out : nullptr, n, 4);
    const Region before = region(state_in, (int64_t)n * H * a->dk * a->dv, 4);
    if (state_in != state_out && meet(state, before))
        return fail(SBC_ERR_INVALID_ARG, "state_out overlaps state_in and is not state_in itself");
    SBC_TRY(check_apart({tokens, state, times},
                        {region_heads(q, H, n, a->dk, a->dtype), region_heads(k, H, n, a->dk, a->dtype),
                         region_heads(v, H, n, a->dv, a->dtype), region(a->rates, H, 4),
                         region(a->t, n, 4), region(a->t ? state_time : nullptr, n, 4)}));
    SBC_TRY(check_apart({tokens, times}, {before}));
    StepArgs p{n, H, a->dk, a->dv, (a->dv + kCols - 1) / kCols, a->scale, a->rates, a->t,
               state_time, *q, *k, *v, *o, state_in, state_out, a->t ? time_out : nullptr};
    const int64_t blocks = (int64_t)n * H * p.tiles;
    if (blocks >= (int64_t)1 << 24)  // (a launch holds fewer than 2^32 work-items)
        return fail(SBC_ERR_UNSUPPORTED, "n * heads * ceil(dv / 64) must be below 2^24");
    trace_before("attn_step", stream);
    if (a->dtype == SBC_F32)
        hipLaunchKernelGGL(attn_step_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(attn_step_kernel<bf16_t>, dim3((unsigned)blocks), dim3(256), 0, stream,
                           p);
    SBC_LAUNCH_CHECK();
    trace_after("attn_step", stream);
    return SBC_OK;
}
