// The kernels of softmax attention's forward pass (softmax.hpp), over packed sequences or a
// paged cache.
#pragma once

#include "softmax.hpp"

namespace sbc {

constexpr int kSoftmaxThreads = 256;

// The keys of a tile in LDS: 64, or 32 of wide float32 heads, whose three parts
// would fill more than the 64 KB that let two workgroups share a CU's LDS.
template <typename T, int D> constexpr int kTileKeys = sizeof(T) == 4 && D > 64 ? 32 : 64;

// 32s of keys that a wave takes at once, as its registers allow
template <typename T, int D> constexpr int kTogether = sizeof(T) == 2 && D <= 64 ? 2 : 1;
// Waves a SIMD: wide float32 heads fill its registers alone
template <typename T, int D> constexpr int kTileWaves = sizeof(T) == 4 && D > 64 ? 1 : 2;

constexpr int kTileRows = 128;  // of softmax_tile_kernel: 32 a wave
constexpr int kFewRows = 32;    // of softmax_rows_kernel

// A sequence's keys in p.parts parts: as even ones as multiples of 128 keys (a round of the
// four waves of softmax_rows_kernel) allow
constexpr int32_t part_keys(int32_t lk, int32_t parts) {
    return (int32_t)(((int64_t)lk + parts - 1) / parts + 127) / 128 * 128;
}
// Where the keys of a part that begins at `first` end, of those up to `limit` (the last part's
// first + size may lie past 2^31)
constexpr int32_t part_end(int32_t first, int32_t size, int32_t limit) {
    return limit - first > size ? first + size : limit;
}
// Parts that hold keys below `limit`
constexpr int32_t parts_below(int32_t limit, int32_t size) {
    return limit > 0 ? (limit - 1) / size + 1 : 0;
}

// ---------------------------------------------------------------- many rows
// A workgroup has 128 rows, 32 a wave, and goes through the keys that they see in tiles,
// which its waves share in LDS.  The next tile is on its way into registers meanwhile; or
// (kDirect, whole bf16 pieces) two tiles straight to LDS, in three buffers: 32768 events of 4 heads
// of 64 channels 655 -> 630 us, 32 prompts of some 1024 tokens, 8 heads of 128, 125 -> 121.
//
// The vector ALU bounds it with the matrix cores: a tile of 64 keys of 64 channels takes a wave 512
// cycles of products and some 800 of exponentials (8 cycles each), sums and conversions.  A SIMD
// overlaps those of different waves only as they happen to meet (39 % and 62 % of its time at two
// and three waves); making the next tile's scores between this one's exponentials, in one wave,
// took more registers than it gave (746 us), as did four waves of 32 keys at once (710).
template <typename T, int D, bool kWhole, bool kPaged, bool kDirect = false>
__global__ __launch_bounds__(kSoftmaxThreads, (kTileWaves<T, D>)) void softmax_tile_kernel(SoftmaxArgs p) {
    constexpr int NP = kParts<T>, KB = kDirect && D > 64 ? 32 : kTileKeys<T, D>, kPlane = KB * D;
    constexpr int kSub = KB < 32 * kTogether<T, D> ? 1 : kTogether<T, D>;
    constexpr int kBuffer = 2 * NP * kPlane;  // keys, then values
    __shared__ __attribute__((aligned(16))) bf16_t lds[(kDirect ? 3 : 1) * kBuffer];
    static_assert(!kDirect || (NP == 1 && kWhole && !kPaged), "direct");
    __shared__ int32_t first_bad[D];  // (TileLoad::put_bad_apart)
    const int32_t head_k = blockIdx.x % p.kv_heads;
    const int32_t part = blockIdx.x / p.kv_heads % p.parts;
    // (from the back: a causal sequence's last tiles are its longest)
    const int32_t x = p.slots - 1 - blockIdx.x / p.kv_heads / p.parts;
    const int32_t group = p.group.d;
    auto begin = [&](int32_t b) {
        return (int32_t)((int64_t)q_split(p, b) * group / kTileRows) + b;
    };
    const int32_t b = sequence_of(p.n_batch, x, begin);
    if (b < 0) return;
    const Sequence s = sequence_at<kPaged>(p, b);
    const int32_t r0 = (x - begin(b)) * kTileRows, rows = s.lq * group;
    if (r0 >= rows) return;
    const int wave = wave_of_block(), lane = threadIdx.x & 63;
    // this lane's row (the last one in place of those that do not exist)
    const int32_t wave_row = r0 + 32 * wave, row = wave_row + (lane & 31);
    const bool there = row < rows;
    const int32_t token = divide(there ? row : rows - 1, p.group);
    const int32_t head = head_k * group + (there ? row - token * group : 0);
    const int32_t limit = s.limit(token, p.causal);
    auto limit_of = [&](int32_t r) {
        return s.limit(divide(r < rows ? r : rows - 1, p.group), p.causal);
    };
    const int32_t least = __builtin_amdgcn_readfirstlane(limit_of(r0));
    const int32_t most = __builtin_amdgcn_readfirstlane(limit_of(r0 + kTileRows - 1));
    // the part's keys
    const int32_t size = p.parts > 1 ? part_keys(s.lk, p.parts) : s.lk;
    const int32_t first = part * size;
    const int32_t end = p.parts > 1 ? part_end(first, size, most) : most;
    if (part > 0 && first >= most) return;  // (softmax_join_kernel knows)
    const int32_t wave_least = __builtin_amdgcn_readfirstlane(limit_of(wave_row));

    bf16x8 q[D / 16][NP];
    {
        const T *at = static_cast<const T *>(p.q.data) + (int64_t)(s.q0 + token) * p.q.token_stride +
                      (int64_t)head * p.q.head_stride;
        row_operand<T, D, kWhole>(at, there, p.dk, q);
    }
    const T *kbase, *vbase;
    if constexpr (kPaged) {
        kbase = static_cast<const T *>(p.pages.k.data);
        vbase = static_cast<const T *>(p.pages.v.data);
    } else {
        kbase = static_cast<const T *>(p.k.data) + s.k0 * p.k.token_stride + head_k * p.k.head_stride;
        vbase = static_cast<const T *>(p.v.data) + s.k0 * p.v.token_stride + head_k * p.v.head_stride;
    }
    constexpr uint64_t kAll = KB == 64 ? ~0ull : 0xFFFFFFFFull;
    TileLoad<T, D, KB, kSoftmaxThreads, kWhole> sk, sv;
    DirectTile<(kDirect ? D : 64), (kDirect ? KB : 64), kSoftmaxThreads> dk, dv;
    KeyPlaces where;  // of the tile that is fetched next
    uint64_t known = kAll, next_known = kAll;
    auto put_tile = [&](int32_t k0, bf16_t *buffer) {
        sk.settle(p.dk);
        sv.settle(p.dv);
        if (k0 + KB > least) sv.put_bad_apart(k0, first_bad);
        sk.store(buffer);
        sv.store(buffer + NP * kPlane);
    };
    // a tile into registers, or (kDirect) to LDS
    auto fetch = [&](int32_t k0, bf16_t *buffer) {
        if constexpr (kPaged) {
            where.template settle<KB>(p);
            sk.load([&](int r) { return where.row<T>(p.pages.k, head_k, r); }, kbase, p.dk);
            sv.load([&](int r) { return where.row<T>(p.pages.v, head_k, r); }, vbase, p.dv);
            next_known = where.there;
            where.template look<KB>(p, s, k0 + KB, s.lk);
        } else {
            if (kWhole && k0 + KB <= s.lk) {
                const T *const k = kbase + k0 * p.k.token_stride, *const v = vbase + k0 * p.v.token_stride;
                if constexpr (kDirect) {
                    dk.load(k, buffer);
                    dv.load(v, buffer + kPlane);
                } else {
                    sk.load_all(k);
                    sv.load_all(v);
                }
                return;
            }
            sk.load([&](int r) { return k0 + r < s.lk ? kbase + (k0 + r) * p.k.token_stride : nullptr; },
                    kbase, p.dk);
            sv.load([&](int r) { return k0 + r < s.lk ? vbase + (k0 + r) * p.v.token_stride : nullptr; },
                    vbase, p.dv);
            if constexpr (kDirect) put_tile(k0, buffer);
        }
    };
    if constexpr (kDirect) {
        dk.places([&](int r) { return (uint32_t)r * (uint32_t)p.k.token_stride; });
        dv.places([&](int r) { return (uint32_t)r * (uint32_t)p.v.token_stride; });
    } else if (kWhole && !kPaged) {
        sk.places(p.k.token_stride, p.dk);
        sv.places(p.v.token_stride, p.dv);
    }
    const LaneAt32<D> at;
    RowSums<D> sums;
    if (threadIdx.x < D) first_bad[threadIdx.x] = INT32_MAX;
    __syncthreads();
    if (first < end) {
        if constexpr (kPaged) where.template look<KB>(p, s, first, s.lk);
        fetch(first, lds);
        if (kDirect && first + KB < end) fetch(first + KB, lds + kBuffer);
    }
    int slot = 0;
    for (int32_t k0 = first; k0 < end; k0 += KB) {
        if constexpr (kDirect) {
            // this tile's loads are done where none but the next one's are left
            if (k0 + KB < end && k0 + 2 * KB <= s.lk)
                wait_direct<2 * decltype(dk)::kSteps>();
            else
                wait_direct<0>();
            __syncthreads();  // (and the tile before has been read)
            if (k0 + KB > least) {
                decltype(dv)::put_bad_apart(lds + slot * kBuffer + kPlane, k0, first_bad);
                __syncthreads();
            }
            if (k0 + 2 * KB < end) fetch(k0 + 2 * KB, lds + (slot == 0 ? 2 : slot - 1) * kBuffer);
        } else {
            __syncthreads();  // the last tile has been read
            put_tile(k0, lds);
            known = next_known;
            __syncthreads();
            if (k0 + KB < end) fetch(k0 + KB, lds);
        }
        const bf16_t *const kt = lds + slot * kBuffer, *const vt = kt + NP * kPlane;
        // (tiles that hold nothing for this wave, behind the diagonal, are gone through as well: with a
        // branch around them the sums were copied from registers to registers in every tile)
#pragma unroll
        for (int u0 = 0; u0 < KB / 32; u0 += kSub) {
            floatx16 x[kSub];
            clear(x);
            row_products<T, D, kSub, (NP == 1 && kSub == 1 ? 4 : 2)>(
                [&](int k, int j, bf16x8(&f)[NP]) { frag_row32<D, NP>(kt, kPlane, u0 + j, k, at, f); },
                [&](int k, int j) -> const bf16x8(&)[NP] { return q[k]; }, x);
            ColumnProducts<T, D, 32 * kSub> values;
            values.read(vt, kPlane, 32 * u0, at);
            if (k0 + 32 * (u0 + kSub) > wave_least || known != kAll) {
#pragma unroll
                for (int u = 0; u < kSub; ++u) {
                    const uint32_t seen = seen_bits(known, u0 + u, limit - k0);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        x[u][r] = seen >> (8 * (r / 4) + r % 4) & 1u ? x[u][r] : -INFINITY;
                }
            }
            softmax_weights<D, kSub>(x, p.scale2, sums);
            values.add(x, vt, kPlane, 32 * u0, at, sums.o);
        }
        if constexpr (kDirect) slot = slot == 2 ? 0 : slot + 1;
    }
    if (!there) return;
    const float l = halves_sum(sums.l);
    const int64_t place = s.q0 + token, flat = place * p.heads + head;
    const int64_t in_part = (int64_t)part * p.n * p.heads + flat;
    if (lane < 32) {
        const float lse2 = l == 0.f ? -INFINITY : sums.m + log2f(l);
        if (p.parts > 1)
            p.part_lse[in_part] = lse2;
        else if (p.lse)
            p.lse[flat] = lse2 * kLn2;
    }
    const float scale = 1.f / l;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float y[4];
            const int c = 32 * t + 8 * j + 4 * (lane >> 5);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = l == 0.f ? 0.f : sums.o[t][4 * j + i] * scale;
                if (first_bad[c + i] < limit) y[i] = NAN;
            }
            if (p.parts > 1)
                put4<float, kWhole>(p.part_o + in_part * p.dv, c, p.dv, y);
            else
                put4<T, kWhole>(static_cast<T *>(p.o.data) + place * p.o.token_stride +
                                    (int64_t)head * p.o.head_stride,
                                c, p.dv, y);
        }
}

// ---------------------------------------------------------------- few rows
// The parts of a weight where it meets v (kWeights of ColumnProducts).  Over a cache, which memory
// bounds, a bf16 call's have two (2^-17): o is as near as with float32 weights, and one part was
// 1e-3 .. 1.8e-3 away from that (a token each over 1 x 4095 and 64 x 8000: 14.5 and 121 us with
// either; 64 streams of 16 tokens, 8 heads of 128: 111 us, 113; 32 of 64 tokens, 8 of 64: 32, 34).
// One where it costs more: packed keys of 128 channels lack the registers (32 sequences of 64
// tokens over 2000 keys: 78 us, 92), and workgroups of 128 rows are bound by products (32768 events
// 615 us, 838; 32 prompts 124, 146; chunks over a cache 58, 65; dv in the gradients 2595, 2750).
template <typename T, bool kPaged> constexpr int kFewWeights = sizeof(T) == 4 ? 3 : kPaged ? 2 : 1;

// A workgroup has 32 rows and one part of the keys; each wave takes every fourth 32 of
// these keys by itself (keys from memory to registers, values through LDS of its own),
// and the waves' sums are joined at the end.  Memory bounds it where a row or few meet a long cache:
// the next 32 keys and values are always on their way.
template <typename T, int D, bool kWhole, bool kPaged>
__global__ __launch_bounds__(kSoftmaxThreads, (sizeof(T) == 4 && D > 32 ? 1 : 2)) void softmax_rows_kernel(SoftmaxArgs p) {
    constexpr int NP = kParts<T>, kPlane = 32 * D;
    constexpr int kJoin = 4 * 32 * 36 * 2;  // (bf16 elements of [4][32][36] float32)
    constexpr int kTiles = 4 * NP * kPlane;
    __shared__ __attribute__((aligned(16))) bf16_t lds[kTiles > kJoin ? kTiles : kJoin];
    __shared__ float wave_m[4][32], wave_l[4][32];
    __shared__ int32_t first_bad[D];
    const int32_t head_k = blockIdx.x % p.kv_heads;
    const int32_t part = blockIdx.x / p.kv_heads % p.parts;
    const int32_t x = p.slots - 1 - blockIdx.x / p.kv_heads / p.parts;
    const int32_t group = p.group.d;
    auto begin = [&](int32_t b) {
        return (int32_t)((int64_t)q_split(p, b) * group / kFewRows) + b;
    };
    const int32_t b = sequence_of(p.n_batch, x, begin);
    if (b < 0) return;
    const Sequence s = sequence_at<kPaged>(p, b);
    const int32_t r0 = (x - begin(b)) * kFewRows, rows = s.lq * group;
    if (r0 >= rows) return;
    const int wave = wave_of_block(), lane = threadIdx.x & 63;
    const int32_t row = r0 + (lane & 31);
    const bool there = row < rows;
    const int32_t token = divide(there ? row : rows - 1, p.group);
    const int32_t head = head_k * group + (there ? row - token * group : 0);
    const int32_t limit = s.limit(token, p.causal);
    auto limit_of = [&](int32_t r) {
        return s.limit(divide(r < rows ? r : rows - 1, p.group), p.causal);
    };
    const int32_t least = __builtin_amdgcn_readfirstlane(limit_of(r0));
    const int32_t most = __builtin_amdgcn_readfirstlane(limit_of(r0 + kFewRows - 1));
    const int32_t size = p.parts > 1 ? part_keys(s.lk, p.parts) : s.lk;
    const int32_t first = part * size;
    const int32_t end = p.parts > 1 ? part_end(first, size, most) : most;
    if (part > 0 && first >= most) return;  // (softmax_join_kernel knows)

    bf16x8 q[D / 16][NP];
    {
        const T *at = static_cast<const T *>(p.q.data) + (int64_t)(s.q0 + token) * p.q.token_stride +
                      (int64_t)head * p.q.head_stride;
        row_operand<T, D, kWhole>(at, there, p.dk, q);
    }
    const T *kbase, *vbase;
    if constexpr (kPaged) {
        kbase = static_cast<const T *>(p.pages.k.data);
        vbase = static_cast<const T *>(p.pages.v.data);
    } else {
        kbase = static_cast<const T *>(p.k.data) + s.k0 * p.k.token_stride + head_k * p.k.head_stride;
        vbase = static_cast<const T *>(p.v.data) + s.k0 * p.v.token_stride + head_k * p.v.head_stride;
    }
    u32x4v kraw[D / 16][8 / kVec<T>];
    TileLoad<T, D, 32, 64, kWhole> sv;
    KeyPlaces where;  // of the keys that are fetched next
    uint64_t known = 0xFFFFFFFFull, next_known = known;
    auto fetch = [&](int32_t k0) {
        if constexpr (kPaged) {
            where.template settle<32>(p);
            const T *at = where.row<T>(p.pages.k, head_k, lane & 31);
            load_row<T, D, kWhole>(at ? at : kbase, at != nullptr, p.dk, kraw);
            sv.load([&](int r) { return where.row<T>(p.pages.v, head_k, r); }, vbase, p.dv);
            next_known = where.there;
            where.template look<32>(p, s, k0 + 128, s.lk);
        } else {
            const int32_t key = k0 + (lane & 31);
            const bool ok = key < s.lk;
            load_row<T, D, kWhole>(kbase + (ok ? key : 0) * p.k.token_stride, ok, p.dk, kraw);
            if (kWhole && k0 + 32 <= s.lk)
                sv.load_all(vbase + k0 * p.v.token_stride);
            else
                sv.load([&](int r) { return k0 + r < s.lk ? vbase + (k0 + r) * p.v.token_stride : nullptr; },
                        vbase, p.dv);
        }
    };
    if (kWhole && !kPaged) sv.places(p.v.token_stride, p.dv);
    const LaneAt32<D> lane_at;
    RowSums<D> sums;
    bf16_t *const vt = lds + wave * NP * kPlane;
    if (threadIdx.x < D) first_bad[threadIdx.x] = INT32_MAX;
    __syncthreads();
    int32_t k0 = first + 32 * wave;
    if (k0 < end) {
        if constexpr (kPaged) where.template look<32>(p, s, k0, s.lk);
        fetch(k0);
    }
    for (; k0 < end; k0 += 128) {
        const LaneAt32<D> at(lane_at);
        floatx16 w[1];
        clear(w);
        settle_row<T, D, kWhole>(true, p.dk, kraw);  // (scores of keys that are not there are hidden)
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            bf16x8 f[NP];
            raw_parts<T>(kraw[k], f);
            mma32<NP, NP>(f, q[k], w[0]);
        }
        sv.settle(p.dv);
        if (k0 + 32 > least) sv.put_bad_apart(k0, first_bad);
        sv.store(vt);
        known = next_known;
        if (k0 + 128 < end) fetch(k0 + 128);
        const int32_t visible = limit < end ? limit : end;
        const uint32_t seen = seen_bits(known, 0, visible - k0);
#pragma unroll
        for (int r = 0; r < 16; ++r)
            w[0][r] = seen >> (8 * (r / 4) + r % 4) & 1u ? w[0][r] : -INFINITY;
        softmax_weights<D, 1>(w, p.scale2, sums);
        // (the wave's own LDS, which it reads in the order of its writes)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        ColumnProducts<T, D, 32, 2, kFewWeights<T, kPaged>> values;
        values.read(vt, kPlane, 0, at);
        values.add(w, vt, kPlane, 0, at, sums.o);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    // joined: the waves' sums as weights of the largest maximum
    const float l = halves_sum(sums.l);
    if (lane < 32) {
        wave_m[wave][lane] = sums.m;
        wave_l[wave][lane] = l;
    }
    __syncthreads();  // (all tiles have been read besides)
    const int r = lane & 31;
    const float top = fmaxf(fmaxf(wave_m[0][r], wave_m[1][r]), fmaxf(wave_m[2][r], wave_m[3][r]));
    // (without a maximum the sums are zero, or NaN of scores that are NaN)
    auto weight = [](float m, float top) {
        return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);
    };
    const float f = weight(sums.m, top);
    float *const join = reinterpret_cast<float *>(lds);
    // this thread's part of the sums: a row and four channels of each tile
    const int32_t jr = threadIdx.x / 8, jc = threadIdx.x % 8 * 4;
    const int32_t out_row = r0 + jr;
    const int32_t out_token = divide(out_row < rows ? out_row : rows - 1, p.group);
    const int64_t place = s.q0 + out_token;
    const int32_t out_head = head_k * group + (out_row < rows ? out_row - out_token * group : 0);
    const float out_top = fmaxf(fmaxf(wave_m[0][jr], wave_m[1][jr]), fmaxf(wave_m[2][jr], wave_m[3][jr]));
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        total += wave_l[i][jr] * weight(wave_m[i][jr], out_top);
    const float inverse = 1.f / total;
    const int32_t out_limit = limit_of(out_row);
    const int64_t flat = place * p.heads + out_head;
    if (out_row < rows && jc == 0) {
        const float lse2 = total == 0.f ? -INFINITY : out_top + log2f(total);
        if (p.parts > 1)
            p.part_lse[(int64_t)part * p.n * p.heads + flat] = lse2;
        else if (p.lse)
            p.lse[flat] = lse2 * kLn2;
    }
#pragma unroll
    for (int t = 0; t < D / 32; ++t) {
        if (t > 0) __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            floatx4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = sums.o[t][4 * j + i] * f;
            *reinterpret_cast<floatx4 *>(join + (wave * 32 + r) * 36 + 8 * j + 4 * (lane >> 5)) = y;
        }
        __syncthreads();
        float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const floatx4 z = *reinterpret_cast<const floatx4 *>(join + (w * 32 + jr) * 36 + jc);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] += z[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = total == 0.f ? 0.f : y[i] * inverse;
            if (first_bad[32 * t + jc + i] < out_limit) y[i] = NAN;
        }
        if (out_row < rows) {
            if (p.parts > 1)
                put4<float, kWhole>(p.part_o + ((int64_t)part * p.n * p.heads + flat) * p.dv, 32 * t + jc,
                                   p.dv, y);
            else
                put4<T, kWhole>(static_cast<T *>(p.o.data) + place * p.o.token_stride +
                                    (int64_t)out_head * p.o.head_stride,
                                32 * t + jc, p.dv, y);
        }
    }
}

// The parts' sums joined, kAcross waves a token and head, each of them every kAcross-th part:
// each part's own softmax weighs by its sum.  Only parts that begin before the row's limit have been
// written.  Few parts take a wave (12984 rows of 4: 10 us, 24 with four waves each), many
// four (8 rows of 63: 4 us, 15 with one).
template <typename T, bool kPaged, int kAcross>
__global__ __launch_bounds__(256) void softmax_join_kernel(SoftmaxArgs p) {
    constexpr int kRows = 4 / kAcross;
    __shared__ float sums[4][128];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), across = wave % kAcross;
    const int64_t stride = (int64_t)p.n * p.heads;
    const int64_t flat = (int64_t)blockIdx.x * kRows + wave / kAcross;
    const bool row = flat < stride;
    const int32_t token = row ? (int32_t)(flat / p.heads) : 0;
    const int32_t head = row ? (int32_t)(flat - (int64_t)token * p.heads) : 0;
    const float found = row && lane < p.parts ? p.part_lse[lane * stride + flat] : 0.f;  // (parts <= 64)
    const int32_t b = sequence_of(p.n_batch, token, [&](int32_t i) { return q_split(p, i); });
    Sequence s{};
    if (b >= 0) s = sequence_at<kPaged>(p, b);
    const bool there = row && b >= 0 && token - s.q0 < s.lq;  // (not behind the last sequence)
    const int32_t limit = there ? s.limit(token - s.q0, p.causal) : 0;
    const int32_t size = part_keys(s.lk, p.parts);
    const float lse2 = lane < p.parts && (int64_t)lane * size < limit ? found : -INFINITY;
    float top = lse2;
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    const float w = lse2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(lse2 - top);
    const float total = group_sum<64>(w);
    const int32_t parts = parts_below(limit, size);
    float y[2] = {0.f, 0.f};
    const int c = 2 * lane;
#pragma unroll 8
    for (int i = across; i < parts; i += kAcross) {
        const float u = __shfl(w, i);
        float z[2];
        load_f32<2>(p.part_o + (i * stride + flat) * p.dv + c, p.dv - c, z);
        y[0] = fmaf(u, z[0], y[0]);
        y[1] = fmaf(u, z[1], y[1]);
    }
    if constexpr (kAcross > 1) {
        sums[wave][c] = y[0];
        sums[wave][c + 1] = y[1];
        __syncthreads();
        if (across > 0) return;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            y[e] = (sums[wave][c + e] + sums[wave + 1][c + e]) +
                   (sums[wave + 2][c + e] + sums[wave + 3][c + e]);
    }
    if (!there) return;
    T *out = static_cast<T *>(p.o.data) + token * p.o.token_stride + (int64_t)head * p.o.head_stride;
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (c + e < p.dv) out[c + e] = from_f32<T>(total == 0.f ? 0.f : y[e] / total);
    if (p.lse && lane == 0) p.lse[flat] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
}

}  // namespace sbc
