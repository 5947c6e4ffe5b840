// A cache of keys and values in pages: pages and places for new tokens, and the rows' way
// into them.
//
// sbc_cache_slots is a sum over the streams (which pages are whose) and then a word or two for
// each entry of the table and each token: a launch bounds it.  Up to kFew streams every
// workgroup makes the sums itself, in LDS, so that there is one launch; more streams take the
// library's scan before.
#include "softmax.hpp"

namespace sbc {
namespace {

constexpr int kThreads = 256;
constexpr int kFew = 1024;

struct SlotArgs {
    const int32_t *lengths, *splits;
    int32_t n, n_batch, width, n_free;
    Divisor page, by_width;
    const int32_t *table, *free_pages;
    int32_t *table_out;
    int64_t *slots;
    int32_t *lengths_out, *needed;
    int32_t *counts, *ranks;  // of many streams
};

struct Stream {
    int32_t before, fresh, held, need;  // tokens, new tokens, pages, new pages
};
__device__ __forceinline__ int32_t pages_of(int64_t tokens, const SlotArgs &a) {
    const int64_t p = tokens / a.page.d + (tokens % a.page.d != 0);
    return p < a.width ? (int32_t)p : a.width;
}
__device__ __forceinline__ int32_t split_of(const SlotArgs &a, int32_t b) {
    return a.splits ? clamp_i(a.splits[b], 0, a.n) : b;
}
__device__ __forceinline__ Stream stream_at(const SlotArgs &a, int32_t b) {
    Stream s;
    s.before = a.lengths[b] > 0 ? a.lengths[b] : 0;
    s.fresh = split_of(a, b + 1) - split_of(a, b);
    if (s.fresh < 0) s.fresh = 0;
    s.held = pages_of(s.before, a);
    s.need = pages_of((int64_t)s.before + s.fresh, a) - s.held;
    return s;
}

__global__ __launch_bounds__(kThreads) void cache_need_kernel(SlotArgs a) {
    const int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (b < a.n_batch) a.counts[b] = stream_at(a, (int32_t)b).need;
}

// Items: the table's entries, then the tokens, then the streams
template <bool kScan>
__global__ __launch_bounds__(kThreads) void cache_slots_kernel(SlotArgs a) {
    __shared__ int32_t ranks[kScan ? kFew + 1 : 1], waves[kThreads / 64];
    if constexpr (kScan) {
        constexpr int kEach = kFew / kThreads;
        int32_t need[kEach], sum = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int b = threadIdx.x * kEach + e;
            need[e] = b < a.n_batch ? stream_at(a, b).need : 0;
            sum += need[e];
        }
        int32_t upto = sum;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int32_t y = __shfl_up(upto, m);
            if ((int)(threadIdx.x & 63) >= m) upto += y;
        }
        if ((threadIdx.x & 63) == 63) waves[threadIdx.x >> 6] = upto;
        __syncthreads();
        upto -= sum;
        for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) upto += waves[w];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            ranks[threadIdx.x * kEach + e] = upto;
            upto += need[e];
        }
        if (threadIdx.x == kThreads - 1) ranks[kFew] = upto;
        __syncthreads();
    }
    auto rank_of = [&](int32_t b) { return kScan ? ranks[b] : a.ranks[b]; };
    // entry j of stream b
    auto entry = [&](const Stream &s, int32_t b, int32_t j) -> int32_t {
        if (j < s.held || j >= s.held + s.need) return a.table[(int64_t)b * a.width + j];
        const int32_t r = rank_of(b) + j - s.held;
        return r < a.n_free ? a.free_pages[r] : -1;
    };
    const int64_t entries = (int64_t)a.n_batch * a.width, all = entries + a.n + a.n_batch;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < all;
         i += (int64_t)gridDim.x * kThreads) {
        if (i < entries) {
            const int32_t b = divide((int32_t)i, a.by_width), j = (int32_t)i - b * a.width;
            const Stream s = stream_at(a, b);
            if (a.table_out != a.table || (j >= s.held && j < s.held + s.need))
                a.table_out[i] = entry(s, b, j);
        } else if (i < entries + a.n) {
            const int32_t t = (int32_t)(i - entries);
            int32_t lo = 0, hi = a.n_batch;  // the streams that begin at or before t
            if (!a.splits) {
                lo = t + 1;
            } else {
                while (lo < hi) {
                    const int32_t mid = lo + (hi - lo) / 2;
                    if (split_of(a, mid) <= t) lo = mid + 1;
                    else hi = mid;
                }
            }
            const int32_t b = lo - 1;
            int64_t slot = -1;
            if (b >= 0 && t < split_of(a, b + 1)) {
                const Stream s = stream_at(a, b);
                const int64_t pos = (int64_t)s.before + (t - split_of(a, b));
                const int64_t j = pos / a.page.d;
                if (j < a.width) {
                    const int32_t g = entry(s, b, (int32_t)j);
                    if (g >= 0) slot = (int64_t)g * a.page.d + (pos - j * a.page.d);
                }
            }
            a.slots[t] = slot;
        } else {
            const int32_t b = (int32_t)(i - entries - a.n);
            const Stream s = stream_at(a, b);
            const int64_t after = (int64_t)s.before + s.fresh;
            a.lengths_out[b] = after > INT32_MAX ? INT32_MAX : (int32_t)after;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *a.needed = kScan ? ranks[kFew] : a.n_batch > 0 ? a.ranks[a.n_batch] : 0;
}

struct AppendArgs {
    sbc_heads x[2];
    sbc_pages to[2];
    int32_t d[2], n, heads, n_pages, page;
    Divisor units, first, pieces[2];  // of a token, of its key part, of a head
    const int64_t *slots;
};

// A lane has 16 bytes of a head of a token, of the keys and then of the values.
template <typename T>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(AppendArgs a) {
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (at >= (int64_t)a.n * a.units.d) return;
    const int32_t i = divide((int32_t)at, a.units);
    int32_t unit = (int32_t)at - i * (int32_t)a.units.d;
    const int64_t slot = a.slots[i];
    if (slot < 0 || slot >= (int64_t)a.n_pages * a.page) return;
    const int w = unit >= (int32_t)a.first.d;
    if (w) unit -= a.first.d;
    const int32_t h = divide(unit, a.pieces[w]), c = (unit - h * (int32_t)a.pieces[w].d) * kVec<T>;
    const int64_t g = slot / a.page, place = slot - g * a.page;
    const T *from = static_cast<const T *>(a.x[w].data) + i * a.x[w].token_stride + h * a.x[w].head_stride + c;
    T *to = static_cast<T *>(a.to[w].data) + g * a.to[w].page_stride + place * a.to[w].token_stride +
            h * a.to[w].head_stride + c;
    const int have = a.d[w] - c;
    if (have >= kVec<T>) {
        raw16 r;
        __builtin_memcpy(&r, from, 16);
        __builtin_memcpy(to, &r, 16);
    } else {
        for (int e = 0; e < have; ++e) to[e] = from[e];
    }
}

}  // namespace
}  // namespace sbc

using namespace sbc;

extern "C" size_t sbc_cache_slots_workspace_size(int32_t n_batch) {
    if (n_batch <= kFew) return 0;
    Carver c(nullptr);
    c.take<int32_t>(n_batch);
    c.take<int32_t>((size_t)n_batch + 1);
    c.take<char>(scan_workspace_bytes(n_batch));
    return c.used;
}

extern "C" sbc_status sbc_cache_slots(const int32_t *lengths, const int32_t *splits, int32_t n,
                                      int32_t n_batch, const int32_t *table, int32_t width,
                                      int32_t page, const int32_t *free_pages, int32_t n_free,
                                      int32_t *table_out, int64_t *slots, int32_t *lengths_out,
                                      int32_t *needed, void *workspace, size_t workspace_bytes,
                                      hipStream_t stream) {
    clear_error();
    if (n < 0 || n_batch < 0 || width < 0 || n_free < 0)
        return fail(SBC_ERR_INVALID_ARG, "n, n_batch, width and n_free must be >= 0");
    if (page <= 0) return fail(SBC_ERR_INVALID_ARG, "page must be > 0");
    if (!splits && n != n_batch)
        return fail(SBC_ERR_INVALID_ARG, "without splits every stream has one new token (n = n_batch)");
    const int64_t entries = (int64_t)n_batch * width;
    if (entries >= (int64_t)1 << 31)
        return fail(SBC_ERR_UNSUPPORTED, "n_batch * width must be below 2^31");
    if (!needed || (n_batch > 0 && (!lengths || !lengths_out)) || (n > 0 && !slots) ||
        (entries > 0 && (!table || !table_out)) || (n_free > 0 && !free_pages))
        return fail(SBC_ERR_INVALID_ARG, "an array is null");
    const Region to = region(table_out, entries, 4), from = region(table, entries, 4);
    if (table_out != table && meet(to, from))
        return fail(SBC_ERR_INVALID_ARG, "table_out overlaps table and is not table itself");
    const Region others[3] = {region(slots, n, 8), region(lengths_out, n_batch, 4), region(needed, 1, 4)};
    SBC_TRY(check_apart({to, others[0], others[1], others[2]},
                        {region(lengths, n_batch, 4), region(splits, (int64_t)n_batch + 1, 4),
                         region(free_pages, n_free, 4)}));
    SBC_TRY(check_apart({others[0], others[1], others[2]}, {from}));
    const size_t bytes = sbc_cache_slots_workspace_size(n_batch);
    if (bytes > 0 && (!workspace || workspace_bytes < bytes))
        return fail(SBC_ERR_WORKSPACE, "workspace smaller than sbc_cache_slots_workspace_size()");
    SlotArgs a{lengths, splits, n, n_batch, width, n_free, divisor(page), divisor(width > 0 ? width : 1),
               table, free_pages, table_out, slots, lengths_out, needed, nullptr, nullptr};
    const int64_t items = entries + n + n_batch;
    const int64_t want = (items + kThreads - 1) / kThreads;
    const int32_t most = 8 * device_cus();
    const dim3 grid((unsigned)(want < 1 ? 1 : want < most ? want : most)), block(kThreads);
    trace_before("cache_slots", stream);
    if (n_batch <= kFew) {
        hipLaunchKernelGGL(cache_slots_kernel<true>, grid, block, 0, stream, a);
    } else {
        Carver c(workspace);
        a.counts = c.take<int32_t>(n_batch);
        a.ranks = c.take<int32_t>((size_t)n_batch + 1);
        void *ws = c.take<char>(scan_workspace_bytes(n_batch));
        hipLaunchKernelGGL(cache_need_kernel, dim3((unsigned)grid_for(n_batch, kThreads)), block, 0,
                           stream, a);
        SBC_LAUNCH_CHECK();
        SBC_TRY(exclusive_scan_i32(a.counts, a.ranks, n_batch, nullptr, ws, stream));
        hipLaunchKernelGGL(cache_slots_kernel<false>, grid, block, 0, stream, a);
    }
    SBC_LAUNCH_CHECK();
    trace_after("cache_slots", stream);
    return SBC_OK;
}

extern "C" sbc_status sbc_cache_append(const sbc_heads *k, const sbc_heads *v, int32_t n,
                                       int32_t kv_heads, int32_t dk, int32_t dv, sbc_dtype dtype,
                                       const int64_t *slots, const sbc_pages *k_pages,
                                       const sbc_pages *v_pages, int32_t n_pages, int32_t page,
                                       hipStream_t stream) {
    clear_error();
    if (n < 0 || n_pages < 0) return fail(SBC_ERR_INVALID_ARG, "n and n_pages must be >= 0");
    if (kv_heads <= 0 || page <= 0 || (k && dk <= 0) || (v && dv <= 0))
        return fail(SBC_ERR_INVALID_ARG, "kv_heads, page, dk and dv must be > 0");
    if (!known_dtype(dtype)) return fail(SBC_ERR_INVALID_ARG, "unknown dtype");
    if ((k != nullptr) != (k_pages != nullptr) || (v != nullptr) != (v_pages != nullptr))
        return fail(SBC_ERR_INVALID_ARG, "rows and their pages go together");
    if (n == 0 || (!k && !v)) return SBC_OK;
    if (!slots) return fail(SBC_ERR_INVALID_ARG, "slots is null");
    AppendArgs a{};
    const int V = dtype == SBC_F32 ? 4 : 8;
    int64_t units[2] = {0, 0};
    Region rows[2] = {}, pages[2] = {};
    for (int w = 0; w < 2; ++w) {
        const sbc_heads *x = w ? v : k;
        const sbc_pages *to = w ? v_pages : k_pages;
        const int32_t d = w ? dv : dk;
        a.pieces[w] = divisor(1);
        if (!x) continue;
        SBC_TRY(check_heads(x, kv_heads, n, d, dtype, w ? "v" : "k"));
        SBC_TRY(check_out_pages(to, n_pages, page, kv_heads, d, dtype, w ? "v_pages" : "k_pages"));
        a.x[w] = *x;
        a.to[w] = *to;
        a.d[w] = d;
        a.pieces[w] = divisor((d + V - 1) / V);
        units[w] = (int64_t)kv_heads * a.pieces[w].d;
        rows[w] = region_heads(x, kv_heads, n, d, dtype);
        pages[w] = region_pages(to, n_pages, page, kv_heads, d, dtype);
    }
    for (const Region &to : pages)
        SBC_TRY(check_apart({to}, {rows[0], rows[1], region(slots, n, 8)}));
    if (n_pages == 0) return SBC_OK;
    if (k && v && meet_pages(k_pages, dk, v_pages, dv, n_pages, page, kv_heads, dtype))
        return fail(SBC_ERR_INVALID_ARG, "two outputs overlap");
    if ((units[0] + units[1]) * n >= (int64_t)1 << 31)
        return fail(SBC_ERR_UNSUPPORTED, "the rows must be fewer than 2^31 pieces of 16 bytes");
    a.n = n;
    a.heads = kv_heads;
    a.n_pages = n_pages;
    a.page = page;
    a.units = divisor((int32_t)(units[0] + units[1]));
    a.first = Divisor{0, (uint32_t)units[0], 0};
    a.slots = slots;
    trace_before("cache_append", stream);
    const dim3 grid((unsigned)grid_for(n * (units[0] + units[1]), kThreads)), block(kThreads);
    if (dtype == SBC_F32)
        hipLaunchKernelGGL(cache_append_kernel<float>, grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL(cache_append_kernel<bf16_t>, grid, block, 0, stream, a);
    SBC_LAUNCH_CHECK();
    trace_after("cache_append", stream);
    return SBC_OK;
}
