// Layer norm over the channels of a row, forward and backward.
//
//   y = (x - mean) rstd w + b,   rstd = 1 / sqrt(var + eps)
//   with xn = (x - mean) rstd and g = dy w:
//   dx = rstd (g - <g> - xn <g xn>),   dw = sum over rows dy xn,   db = sum dy
//
// Both passes move each value once (forward 2, backward 3 elements a value) and
// compute little, so memory bounds them.  A row belongs to a group of G lanes,
// as few as hold it at kVec elements a lane (several rows share a wave where
// they are short; longer rows take K vectors a lane, then a whole workgroup);
// it is read once and stays in registers, so the variance is that of the
// differences from the mean.
//
// A float32 sum leaves the mean m off by some roundings, and with it all differences;
// where the spread is small beside the mean this is most of y.  So the differences'
// own mean, delta (they are exact where it matters), is taken off again:
//   mean = m + delta,   var = <(x - m)^2> - delta^2,   x - mean = (x - m) - delta,
// one sum more beside that of the squares.  Equal values leave exactly zero.
//
// Rows that do not fit a workgroup's registers are
// read again from the cache instead (wide_* kernels), and summed in float64: a lane
// adds up to 2^16 of their values, where float32 loses 6e-4 of the sum.
//
// dw and db: a lane keeps the sums of its channels over the rows that it takes,
// the workgroup adds its groups in LDS, and norm_reduce_kernel adds the
// workgroups' parts in float64, all in a fixed order.
#include "common.hpp"
#include "seq.hpp"

namespace sbc {
namespace {

constexpr int kThreads = 256;
constexpr int kMostK = 4;  // vectors of a row that a lane holds

// Sum over the lanes that share a row, in each of them.  G = kThreads: the
// workgroup, by way of LDS (two buffers in turn, so one barrier a sum).
template <int G> struct RowSum {
    __device__ __forceinline__ float operator()(float x) { return group_sum<G>(x); }
};
template <> struct RowSum<kThreads> {
    float *buf;
    int turn = 0;
    __device__ __forceinline__ float operator()(float x) {
        x = group_sum<64>(x);
        float *b = buf + 4 * turn;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = x;
        __syncthreads();
        return (b[0] + b[1]) + (b[2] + b[3]);
    }
};

template <int G> __device__ __forceinline__ RowSum<G> row_sum(float *buf) {
    if constexpr (G == kThreads)
        return RowSum<G>{buf};
    else
        return RowSum<G>{};
}

// rstd from the mean square of the differences from a mean that is off by delta.  (A NaN
// stays one: fmaxf would drop it.)
__device__ __forceinline__ float spread(float square, float delta, float eps) {
    const float var = square - delta * delta;
    return 1.0f / sqrtf((var < 0.f ? 0.f : var) + eps);
}

template <typename T, int G, int K>
__global__ __launch_bounds__(kThreads) void norm_fwd_kernel(
    const T *__restrict__ x, int64_t x_stride, const float *__restrict__ w,
    const float *__restrict__ b, int32_t n, int32_t C, float eps, T *__restrict__ y,
    int64_t y_stride, float *__restrict__ mean, float *__restrict__ rstd) {
    constexpr int V = kVec<T>;
    __shared__ float buf[8];
    constexpr int kRows = kThreads / G;
    const int lane = threadIdx.x % G;
    auto sum = row_sum<G>(buf);
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
    raw16 next[K];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * V;
            next[k] = load_raw16<T>(x + row * x_stride + c, C - c);
        }
    };
    if (r < n) fetch(r);
    for (; r < n; r += step) {
        float v[K][V];
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            unpack<T>(next[k], v[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) s += v[k][i];
        }
        if (r + step < n) fetch(r + step);
        const float mu = sum(s) / (float)C;
        s = 0.f;
        float left = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] -= mu;
                left += c + i < C ? v[k][i] : 0.f;
                s += c + i < C ? v[k][i] * v[k][i] : 0.f;
            }
        }
        const float delta = sum(left) / (float)C;
        const float rs = spread(sum(s) / (float)C, delta, eps);
        if (lane == 0) {
            if (mean) mean[r] = mu + delta;
            if (rstd) rstd[r] = rs;
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * V;
            if (c >= C) break;
            float wv[V], bv[V];
            if (w) load_f32<V>(w + c, C - c, wv);
            if (b) load_f32<V>(b + c, C - c, bv);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float o = (v[k][i] - delta) * rs;
                if (w) o *= wv[i];
                if (b) o += bv[i];
                v[k][i] = o;
            }
            store_vec<T>(y + r * y_stride + c, C - c, v[k]);
        }
    }
}

// The same sum over a workgroup in float64.
struct WideSum {
    double *buf;
    int turn = 0;
    __device__ __forceinline__ double operator()(double x) {
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m);
        double *b = buf + 4 * turn;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = x;
        __syncthreads();
        return (b[0] + b[1]) + (b[2] + b[3]);
    }
};

// Rows longer than a workgroup's registers: a workgroup a row, read three times.
template <typename T>
__global__ __launch_bounds__(kThreads) void wide_fwd_kernel(
    const T *__restrict__ x, int64_t x_stride, const float *__restrict__ w,
    const float *__restrict__ b, int32_t n, int32_t C, float eps, T *__restrict__ y,
    int64_t y_stride, float *__restrict__ mean, float *__restrict__ rstd) {
    constexpr int V = kVec<T>;
    __shared__ double buf[8];
    WideSum sum{buf};
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const T *xr = x + r * x_stride;
        float v[V];
        double s = 0.0;
        for (int c = threadIdx.x * V; c < C; c += kThreads * V) {
            load_vec<T>(xr + c, C - c, v);
#pragma unroll
            for (int i = 0; i < V; ++i) s += v[i];
        }
        s = sum(s) / C;
        const float mu = (float)s, delta = (float)(s - mu);
        s = 0.0;
        for (int c = threadIdx.x * V; c < C; c += kThreads * V) {
            load_vec<T>(xr + c, C - c, v);
#pragma unroll
            for (int i = 0; i < V; ++i) s += c + i < C ? (v[i] - mu) * (v[i] - mu) : 0.f;
        }
        const float rs = spread((float)(sum(s) / C), delta, eps);
        if (threadIdx.x == 0) {
            if (mean) mean[r] = mu;
            if (rstd) rstd[r] = rs;
        }
        for (int c = threadIdx.x * V; c < C; c += kThreads * V) {
            load_vec<T>(xr + c, C - c, v);
            float wv[V], bv[V];
            if (w) load_f32<V>(w + c, C - c, wv);
            if (b) load_f32<V>(b + c, C - c, bv);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float o = ((v[i] - mu) - delta) * rs;
                if (w) o *= wv[i];
                if (b) o += bv[i];
                v[i] = o;
            }
            store_vec<T>(y + r * y_stride + c, C - c, v);
        }
    }
}

// part [gridDim.x, 2, C]: the workgroup's sums of dy xn and of dy (null: not wanted)
template <typename T, int G, int K>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(
    const T *__restrict__ dy, int64_t dy_stride, const T *__restrict__ x, int64_t x_stride,
    const float *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
    int32_t n, int32_t C, T *__restrict__ dx, int64_t dx_stride, float *__restrict__ part) {
    constexpr int V = kVec<T>;
    constexpr int kRows = kThreads / G;
    __shared__ float buf[8];
    // the groups' sums, a slab of V channels at a time (banks: a row of kThreads + 1)
    __shared__ float red[G == kThreads ? 1 : V * (kThreads + 1)];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    auto sum = row_sum<G>(buf);
    const float inv_c = 1.0f / (float)C;
    float wv[K][V], dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * G + lane) * V;
        if (w) load_f32<V>(w + c, C - c, wv[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!w) wv[k][i] = 1.f;
            dw[k][i] = db[k][i] = 0.f;
        }
    }
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t r = (int64_t)blockIdx.x * kRows + group;
    raw16 next_x[K], next_g[K];
    float next_mu = 0.f, next_rs = 0.f;
    auto fetch = [&](int64_t row) {
        next_mu = mean[row];
        next_rs = rstd[row];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * V;
            next_x[k] = load_raw16<T>(x + row * x_stride + c, C - c);
            next_g[k] = load_raw16<T>(dy + row * dy_stride + c, C - c);
        }
    };
    if (r < n) fetch(r);
    for (; r < n; r += step) {
        const float mu = next_mu, rs = next_rs;
        float xn[K][V], g[K][V];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            unpack<T>(next_x[k], xn[k]);
            unpack<T>(next_g[k], g[k]);
        }
        if (r + step < n) fetch(r + step);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xn[k][i] = c + i < C ? (xn[k][i] - mu) * rs : 0.f;
                dw[k][i] += g[k][i] * xn[k][i];
                db[k][i] += g[k][i];
                g[k][i] *= wv[k][i];
                s1 += g[k][i];
                s2 += g[k][i] * xn[k][i];
            }
        }
        if (!dx) continue;
        s1 = sum(s1) * inv_c;
        s2 = sum(s2) * inv_c;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * V;
            if (c >= C) break;
#pragma unroll
            for (int i = 0; i < V; ++i) g[k][i] = rs * (g[k][i] - s1 - xn[k][i] * s2);
            store_vec<T>(dx + r * dx_stride + c, C - c, g[k]);
        }
    }
    if (!part) return;
    float *mine = part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + lane) * V;
            float(&acc)[V] = which ? db[k] : dw[k];
            if constexpr (G == kThreads) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (c + i < C) mine[(int64_t)which * C + c + i] = acc[i];
            } else {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < V; ++i) red[i * (kThreads + 1) + threadIdx.x] = acc[i];
                __syncthreads();
                for (int j = threadIdx.x; j < G * V; j += kThreads) {
                    const int l = j / V, i = j % V;
                    const int cc = (k * G + l) * V + i;
                    float t = 0.f;
                    for (int q = 0; q < kRows; ++q) t += red[i * (kThreads + 1) + q * G + l];
                    if (cc < C) mine[(int64_t)which * C + cc] = t;
                }
            }
        }
    }
}

// dx of rows longer than a workgroup's registers: a workgroup a row.
template <typename T>
__global__ __launch_bounds__(kThreads) void wide_dx_kernel(
    const T *__restrict__ dy, int64_t dy_stride, const T *__restrict__ x, int64_t x_stride,
    const float *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
    int32_t n, int32_t C, T *__restrict__ dx, int64_t dx_stride) {
    constexpr int V = kVec<T>;
    __shared__ double buf[8];
    WideSum sum{buf};
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const float mu = mean[r], rs = rstd[r];
        double d1 = 0.0, d2 = 0.0;
        float s1 = 0.f, s2 = 0.f;
        for (int pass = 0; pass < 2; ++pass) {
            for (int c = threadIdx.x * V; c < C; c += kThreads * V) {
                float xn[V], g[V], wv[V];
                load_vec<T>(x + r * x_stride + c, C - c, xn);
                load_vec<T>(dy + r * dy_stride + c, C - c, g);
                if (w) load_f32<V>(w + c, C - c, wv);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    xn[i] = c + i < C ? (xn[i] - mu) * rs : 0.f;
                    if (w) g[i] *= wv[i];
                    if (pass == 0) {
                        d1 += g[i];
                        d2 += g[i] * xn[i];
                    } else {
                        g[i] = rs * (g[i] - s1 - xn[i] * s2);
                    }
                }
                if (pass == 1) store_vec<T>(dx + r * dx_stride + c, C - c, g);
            }
            if (pass == 0) {
                s1 = (float)(sum(d1) / C);
                s2 = (float)(sum(d2) / C);
            }
        }
    }
}

// The sums of dy xn and dy for such rows: a lane kVec channels (blockIdx.y), a
// workgroup every gridDim.x-th row.
template <typename T>
__global__ __launch_bounds__(kThreads) void wide_dw_kernel(
    const T *__restrict__ dy, int64_t dy_stride, const T *__restrict__ x, int64_t x_stride,
    const float *__restrict__ mean, const float *__restrict__ rstd, int32_t n, int32_t C,
    float *__restrict__ part) {
    constexpr int V = kVec<T>;
    const int64_t c = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * V;
    if (c >= C) return;
    const int have = (int)(C - c);
    float dw[V] = {}, db[V] = {};
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const float mu = mean[r], rs = rstd[r];
        float xn[V], g[V];
        load_vec<T>(x + r * x_stride + c, have, xn);
        load_vec<T>(dy + r * dy_stride + c, have, g);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            dw[i] += g[i] * ((xn[i] - mu) * rs);
            db[i] += g[i];
        }
    }
    float *mine = part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < have) {
            mine[c + i] = dw[i];
            mine[(int64_t)C + c + i] = db[i];
        }
}

// dw and db from `parts` workgroups' sums: 16 channels a workgroup, 64 lanes a
// channel, in float64.  (A round of loads takes 1.7 us here, from what other XCDs
// have just written: with 16 lanes a channel 512 parts of 64 channels took 7 us.)
constexpr int kReduceThreads = 1024;
__global__ __launch_bounds__(kReduceThreads) void norm_reduce_kernel(
    const float *__restrict__ part, int32_t parts, int32_t C, float *__restrict__ dw,
    float *__restrict__ db) {
    constexpr int kDown = kReduceThreads / 16, kAhead = 8;  // loads in flight
    __shared__ double red[kDown][17];
    const int cl = threadIdx.x % 16, pl = threadIdx.x / 16;
    const int64_t j = (int64_t)blockIdx.x * 16 + cl, width = 2 * (int64_t)C;
    double s = 0.0;
    if (j < width) {
        for (int p0 = pl; p0 < parts; p0 += kDown * kAhead) {
            float v[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                v[k] = p0 + kDown * k < parts ? part[(p0 + kDown * k) * width + j] : 0.f;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) s += (double)v[k];
        }
    }
    red[pl][cl] = s;
    for (int half = kDown / 2; half > 0; half /= 2) {
        __syncthreads();
        if (pl < half) red[pl][cl] += red[pl + half][cl];
    }
    if (pl == 0 && j < width) {
        if (j < C) {
            if (dw) dw[j] = (float)red[0][cl];
        } else if (db) {
            db[j - C] = (float)red[0][cl];
        }
    }
}

// Calls f(G, K) for the lanes a row takes and the vectors a lane holds; false if
// a workgroup's registers do not hold the row.
template <int V, typename F> bool row_dispatch(int32_t C, F &&f) {
    const int nv = (C + V - 1) / V;
#define SBC_ROW(g, k) f(std::integral_constant<int, g>{}, std::integral_constant<int, k>{})
    if (nv <= 1) SBC_ROW(1, 1);
    else if (nv <= 2) SBC_ROW(2, 1);
    else if (nv <= 4) SBC_ROW(4, 1);
    else if (nv <= 8) SBC_ROW(8, 1);
    else if (nv <= 16) SBC_ROW(16, 1);
    else if (nv <= 32) SBC_ROW(32, 1);
    else if (nv <= 64) SBC_ROW(64, 1);
    else if (nv <= 128) SBC_ROW(64, 2);
    else if (nv <= 256) SBC_ROW(64, 4);
    else if (nv <= 512) SBC_ROW(256, 2);
    else if (nv <= 1024) SBC_ROW(256, 4);
    else return false;
#undef SBC_ROW
    return true;
}

// Workgroups of the forward pass (and of dx in wide rows), one for the rows that it
// takes at once; rows past 2^22 workgroups' are taken in turn.  (A launch holds fewer
// than 2^32 work-items.  1M rows of 64 bf16 take 72.6 us so, 73.2 in 8192 workgroups.)
constexpr int64_t kMostBlocks = 1 << 22;
unsigned row_blocks(int64_t n, int rows) {
    const int64_t b = (n + rows - 1) / rows;
    return (unsigned)(b < kMostBlocks ? b : kMostBlocks);
}

// Workgroups of the backward pass: at most 2 a CU (12007 rows of 1001 bf16: 29 us, 39 at
// one a CU), and one for 16 rows, since each leaves 2 C sums to be read again (4000 rows of
// 4096 float32: 44 us, 47 at 8 rows, 58 at 32; 4000 of 1001 bf16: 18, 18, 23).  Few wide
// rows would rather have more: 256 of 4096 take 30 us, 20 at 8 rows.
int32_t bwd_blocks(int32_t n) {
    const int64_t most = 2 * (int64_t)device_cus();
    int64_t b = ((int64_t)n + 15) / 16;
    if (b > most) b = most;
    return (int32_t)(b < 1 ? 1 : b);
}

sbc_status check_norm(int32_t n, int32_t C, sbc_dtype dtype) {
    if (n < 0) return fail(SBC_ERR_INVALID_ARG, "n must be >= 0");
    if (C <= 0) return fail(SBC_ERR_INVALID_ARG, "C must be > 0");
    if (C > 1 << 24) return fail(SBC_ERR_UNSUPPORTED, "C must be <= 2^24");
    if (!known_dtype(dtype)) return fail(SBC_ERR_INVALID_ARG, "unknown dtype");
    return SBC_OK;
}

template <typename T>
sbc_status forward(const void *x, int64_t xs, const float *w, const float *b, int32_t n, int32_t C,
                   float eps, void *y, int64_t ys, float *mean, float *rstd, hipStream_t stream) {
    const T *xp = static_cast<const T *>(x);
    T *yp = static_cast<T *>(y);
    const bool held = row_dispatch<kVec<T>>(C, [&](auto g, auto k) {
        constexpr int G = decltype(g)::value, K = decltype(k)::value;
        hipLaunchKernelGGL((norm_fwd_kernel<T, G, K>), dim3(row_blocks(n, kThreads / G)),
                           dim3(kThreads), 0, stream, xp, xs, w, b, n, C, eps, yp, ys, mean, rstd);
    });
    if (!held)
        hipLaunchKernelGGL(wide_fwd_kernel<T>, dim3(row_blocks(n, 1)), dim3(kThreads), 0, stream, xp,
                           xs, w, b, n, C, eps, yp, ys, mean, rstd);
    SBC_LAUNCH_CHECK();
    return SBC_OK;
}

template <typename T>
sbc_status backward(const void *dy, int64_t dys, const void *x, int64_t xs, const float *w,
                    const float *mean, const float *rstd, int32_t n, int32_t C, void *dx,
                    int64_t dxs, float *part, int32_t parts, hipStream_t stream) {
    const T *dyp = static_cast<const T *>(dy), *xp = static_cast<const T *>(x);
    T *dxp = static_cast<T *>(dx);
    const bool held = row_dispatch<kVec<T>>(C, [&](auto g, auto k) {
        constexpr int G = decltype(g)::value, K = decltype(k)::value;
        hipLaunchKernelGGL((norm_bwd_kernel<T, G, K>), dim3((unsigned)parts), dim3(kThreads), 0,
                           stream, dyp, dys, xp, xs, w, mean, rstd, n, C, dxp, dxs, part);
    });
    if (!held) {
        if (dx)
            hipLaunchKernelGGL(wide_dx_kernel<T>, dim3(row_blocks(n, 1)), dim3(kThreads), 0, stream,
                               dyp, dys, xp, xs, w, mean, rstd, n, C, dxp, dxs);
        if (part)
            hipLaunchKernelGGL(wide_dw_kernel<T>,
                               dim3((unsigned)parts, (unsigned)grid_for(C, kThreads * kVec<T>)),
                               dim3(kThreads), 0, stream, dyp, dys, xp, xs, mean, rstd, n, C, part);
    }
    SBC_LAUNCH_CHECK();
    return SBC_OK;
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" sbc_status sbc_layer_norm_forward(const void *x, int64_t x_stride, const float *weight,
                                             const float *bias, sbc_dtype dtype, int32_t n,
                                             int32_t C, float eps, void *y, int64_t y_stride,
                                             float *mean, float *rstd, hipStream_t stream) {
    clear_error();
    SBC_TRY(check_norm(n, C, dtype));
    if (!(eps >= 0.f)) return fail(SBC_ERR_INVALID_ARG, "eps must be >= 0");
    if (x_stride < C || y_stride < C)
        return fail(SBC_ERR_INVALID_ARG, "a row stride is smaller than C");
    if (n == 0) return SBC_OK;
    if (!x || !y) return fail(SBC_ERR_INVALID_ARG, "x or y is null");
    SBC_TRY(check_apart({region_rows(y, n, C, y_stride, dtype), region(mean, n, 4), region(rstd, n, 4)},
                        {region_rows(x, n, C, x_stride, dtype), region(weight, C, 4),
                         region(bias, C, 4)}));
    trace_before("norm_fwd", stream);
    SBC_TRY(dtype == SBC_F32 ? forward<float>(x, x_stride, weight, bias, n, C, eps, y, y_stride,
                                              mean, rstd, stream)
                             : forward<bf16_t>(x, x_stride, weight, bias, n, C, eps, y, y_stride,
                                               mean, rstd, stream));
    trace_after("norm_fwd", stream);
    return SBC_OK;
}

extern "C" size_t sbc_layer_norm_workspace_size(int32_t n, int32_t C) {
    if (n < 0 || C <= 0) return 0;
    return align_up((size_t)bwd_blocks(n) * 2 * (size_t)C * 4);
}

extern "C" sbc_status sbc_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x,
                                              int64_t x_stride, const float *weight,
                                              const float *mean, const float *rstd,
                                              sbc_dtype dtype, int32_t n, int32_t C, void *dx,
                                              int64_t dx_stride, float *dweight, float *dbias,
                                              void *workspace, size_t workspace_bytes,
                                              hipStream_t stream) {
    clear_error();
    SBC_TRY(check_norm(n, C, dtype));
    if (dy_stride < C || x_stride < C || (dx && dx_stride < C))
        return fail(SBC_ERR_INVALID_ARG, "a row stride is smaller than C");
    const bool sums = dweight || dbias;
    if (!dx && !sums) return SBC_OK;
    if (n == 0) {
        if (dweight) SBC_TRY(fill_i32(reinterpret_cast<int32_t *>(dweight), 0, C, stream));
        if (dbias) SBC_TRY(fill_i32(reinterpret_cast<int32_t *>(dbias), 0, C, stream));
        return SBC_OK;
    }
    if (!dy || !x || !mean || !rstd)
        return fail(SBC_ERR_INVALID_ARG, "dy, x, mean or rstd is null");
    SBC_TRY(check_apart({region_rows(dx, n, C, dx_stride, dtype), region(dweight, C, 4),
                         region(dbias, C, 4)},
                        {region_rows(dy, n, C, dy_stride, dtype), region_rows(x, n, C, x_stride, dtype),
                         region(weight, C, 4), region(mean, n, 4), region(rstd, n, 4)}));
    if (sums && (!workspace || workspace_bytes < sbc_layer_norm_workspace_size(n, C)))
        return fail(SBC_ERR_WORKSPACE, "workspace smaller than sbc_layer_norm_workspace_size()");
    float *part = sums ? static_cast<float *>(workspace) : nullptr;
    const int32_t parts = bwd_blocks(n);
    trace_before("norm_bwd", stream);
    SBC_TRY(dtype == SBC_F32 ? backward<float>(dy, dy_stride, x, x_stride, weight, mean, rstd, n, C,
                                               dx, dx_stride, part, parts, stream)
                             : backward<bf16_t>(dy, dy_stride, x, x_stride, weight, mean, rstd, n,
                                                C, dx, dx_stride, part, parts, stream));
    trace_after("norm_bwd", stream);
    if (!sums) return SBC_OK;
    trace_before("norm_reduce", stream);
    hipLaunchKernelGGL(norm_reduce_kernel, dim3(grid_for(2 * (int64_t)C, 16)),
                       dim3(kReduceThreads), 0, stream, part, parts, C, dweight, dbias);
    SBC_LAUNCH_CHECK();
    trace_after("norm_reduce", stream);
    return SBC_OK;
}
