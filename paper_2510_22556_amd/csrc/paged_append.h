// New tokens' rows into the pages: the kernel that copies K and V, rotates K and q on the way, and, with NormedAppendArgs, divides both by their
// root mean square in front of that.
#pragma once

#include "paged_rows.h"

#include <type_traits>

namespace sablock {
namespace {

constexpr int ANGLES = 4096;                   // (token, pair) whose sine and cosine LDS holds at a time
constexpr int BATCH = 4;                       // rows of a thread in flight, twice
// Workgroups per compute unit, if the head rows allow: the same angles in each of them against an even end (the prompts by 8, 12, 16 and
// 24: 75, 70, 71 and 73 us)
constexpr int APPEND_WGS = 12;

struct AppendArgs {
    PageDims d;
    TokenDims t;
    PageView pv;
    const char *q, *k, *v;
    const int32_t *counts, *positions;
    const float *inv_freq;
    char *q_out;
    int slots, per;             // head rows: K's heads, V's, q's; of a workgroup
    int chunks, lanes;          // 16-byte chunks of a row, the next power of two
    int groups, side;           // rows and head rows that a workgroup does at a time
    int tile;                   // tokens whose angles LDS holds
};
struct NormedAppendArgs : AppendArgs {
    const float *q_weight, *k_weight;
    int64_t q_layer, k_layer, head;                            // steps of the weights, in elements; head 0: all heads of a layer have the same
    float eps, per_element;                                    // 1 / D
};

// sums over the lanes of a row, a power of two of them, for B rows at a time
template <int B> __device__ __forceinline__ void over_row(float (&x)[B], int lanes)
{
#define SABLOCK_OVER(M)                                        \
    if (lanes > M) {                                           \
        _Pragma("unroll") for (int i = 0; i < B; ++i) x[i] += xor_lane<M>(x[i]); \
    }
    SABLOCK_OVER(1) SABLOCK_OVER(2) SABLOCK_OVER(4) SABLOCK_OVER(8) SABLOCK_OVER(16) SABLOCK_OVER(32)
#undef SABLOCK_OVER
}

// numbers of the lane `apart` lanes on or back: where that is one bit of the lane's number, without LDS
template <int N> __device__ __forceinline__ void from_partner(float (&z)[N], const float (&y)[N], int apart, int partner)
{
    if (apart == 8) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = xor_lane<8>(y[e]);
    } else if (apart == 4) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = xor_lane<4>(y[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = __shfl(y[e], partner);
    }
}

// grid (touched pages, sequences x layers, parts of the head rows).  The angle of a (token, pair) is the same for all heads: formed
// once per workgroup, position * inv_freq in fp64 (at position 131 072 an angle in fp32 is off by up to 2^-8), see turn() of either
// type.  A thread has one chunk of every groups-th row of a head, a row's chunks lie in the lanes of one wavefront, where
// the other halves of pairs come from.  The rows of the next step are on their way while one is turned and stored, the first
// ones while the angles are formed.
// ONE: a token per sequence, and a workgroup has no more head rows than it does at a time.  SPLIT: the two elements of a pair lie half a rotation
// apart, in different chunks.
// Loads of a step are issued whatever the lane has to do there (at the nearest place that exists): behind a branch the compiler could
// not count the loads in flight and would wait for all of them.  A step whose rows all exist stores without a branch for the same reason.
template <bool BF16, bool ONE, bool SPLIT, typename Args>
__global__ void __launch_bounds__(NT, ONE || (std::is_same_v<Args, AppendArgs> ? SPLIT : !BF16) ? 4 : 3)
append_paged_kernel(Args a)
{
    using E = Elem<BF16>;
    constexpr bool NORM = std::is_same_v<Args, NormedAppendArgs>;
    constexpr int B = ONE ? 1 : BATCH;
    __shared__ __attribute__((aligned(16))) uint32_t sh[ONE ? 1 : NT * 8];
    __shared__ __attribute__((aligned(16))) float2 turn[ONE ? 128 : ANGLES];               // cosine, sine
    const PageDims &d = a.d;
    const int s = blockIdx.y / d.n_layers, layer = blockIdx.y - s * d.n_layers, tid = threadIdx.x;
    // Not rows_of: behind a full table the new tokens are rows that no page holds, not the last ones that have a page.  A length that leaves
    // them all there is as good as any larger one.
    const int len = (int)min((uint32_t)max(a.pv.lengths[s], 0), ((uint32_t)d.max_pages << d.shift) + a.t.n_new);
    const int count = min(a.counts ? min(max(a.counts[s], 0), a.t.n_new) : a.t.n_new, len);
    const int first = len - count, page = (first >> d.shift) + (int)blockIdx.x;
    if ((int64_t)page << d.shift >= len) return;
    const int page_begin = page << d.shift, begin = max(first, page_begin), end = page_begin + min(len - page_begin, d.page);
    if (begin >= end) return;
    const int id = page < d.max_pages ? page_at(d, a.pv.table, s, page) : -1;
    // K and V of a page that does not exist go nowhere
    const int slot0 = id < 0 ? max((int)blockIdx.z * a.per, 2 * d.Hkv) : blockIdx.z * a.per, slot_end = min(a.slots, ((int)blockIdx.z + 1) * a.per);
    if (slot0 >= slot_end) return;
    const int half = a.t.R / 2, pair_chunks = half / E::N;
    const int c = tid & (a.lanes - 1), place = tid / a.lanes, group = place % a.groups, lane_slot = place / a.groups;
    const bool active = lane_slot < a.side && c < a.chunks;
    const int64_t position0 = a.t.R ? (int64_t)a.positions[s] : 0;
    // this chunk's part in the rotation: where its angles lie, and the chunk of the other elements of its pairs
    const bool turned = c < 2 * pair_chunks, upper = SPLIT && turned && c >= pair_chunks;
    const int angle = SPLIT ? (upper ? c - pair_chunks : c) * E::N : c * (E::N / 2);
    const int partner = !turned ? tid : upper ? tid - pair_chunks : tid + pair_chunks;     // lane

    struct Source { const char *at; int64_t step; };
    auto source = [&](int base) {
        const int slot = min(base + lane_slot, slot_end - 1);
        const bool is_k = slot < d.Hkv, is_v = !is_k && slot < 2 * d.Hkv;
        const int head = is_k ? slot : is_v ? slot - d.Hkv : slot - 2 * d.Hkv;
        const int64_t *st = is_k ? a.t.ks : is_v ? a.t.vs : a.t.qs;
        return Source{(is_k ? a.k : is_v ? a.v : a.q) + (s * st[0] + layer * st[1] + head * st[2]) * E::BYTES + min(c, a.chunks - 1) * 16, st[3] * E::BYTES};
    };
    // weights of this chunk's elements; V's lanes load q's or K's, and do not use them
    struct Weights { float own[NORM ? E::N : 1]; };
    auto load_weights = [&](int base, Weights &w) {
        if constexpr (NORM) {
            const int slot = min(base + lane_slot, slot_end - 1);
            const bool is_q = slot >= 2 * d.Hkv;
            const float *at = is_q ? a.q_weight + layer * a.q_layer + (slot - 2 * d.Hkv) * a.head : a.k_weight + layer * a.k_layer + min(slot, d.Hkv - 1) * a.head;
#pragma unroll
            for (int e = 0; e < E::N; e += 4) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(at + min(c, a.chunks - 1) * E::N + e);
#pragma unroll
                for (int j = 0; j < 4; ++j) w.own[e + j] = x[j];
            }
        }
    };
    // the thread's pair of the angles, which it forms for every angle_step-th token
    const int angle_step = half ? NT / half : 1, pair = half ? tid % half : 0, angle_tok = half ? tid / half : angle_step;
    float freq = 0.f;
    if (angle_tok < angle_step) freq = a.inv_freq[pair];
    for (int t0 = begin;; t0 += a.tile) {
        const int n = min(a.tile, end - t0), rows = B * a.groups, batches = (n + rows - 1) / rows;
        u32x4 x[B];
        auto load = [&](int base, int b, u32x4 (&x)[B]) {
            const Source r = source(base);
            const char *from = r.at + (t0 - first) * r.step;
#pragma unroll
            for (int i = 0; i < B; ++i) x[i] = *reinterpret_cast<const u32x4 *>(from + min(group + (b * B + i) * a.groups, n - 1) * r.step);
        };
        load(slot0, 0, x);
        if (a.t.R) {
            if (t0 > begin) __syncthreads();
            if (angle_tok < angle_step)
                for (int tok = angle_tok; tok < n; tok += angle_step)
                    turn[tok * half + pair] = E::turn((double)(position0 + t0 - first + tok), freq);
            __syncthreads();
        }
        Bounds<BF16> b;
        b.clear();
        for (int base = slot0, bt = 0;;) {
            const bool slot_done = bt + 1 == batches;
            const int next_base = slot_done ? base + a.side : base, next_bt = slot_done ? 0 : bt + 1;
            Weights weights;
            load_weights(base, weights);                       // in front of the next rows, and so not waited for with them
            u32x4 xn[B];
            if constexpr (!ONE) load(next_base, next_bt, xn);  // behind the last: the last again
            const int slot = base + lane_slot;
            const bool is_k = slot < d.Hkv, is_v = !is_k && slot < 2 * d.Hkv, live = active && slot < slot_end;
            const int head = is_k ? slot : is_v ? slot - d.Hkv : slot - 2 * d.Hkv;
            char *dst;                                         // row t0
            int64_t step;
            if (is_k || is_v) {
                const int64_t *ps = is_k ? d.ks : d.vs;
                step = ps[3] * E::BYTES;
                dst = (is_k ? a.pv.k : a.pv.v) + (layer * ps[0] + id * ps[1] + head * ps[2]) * E::BYTES + (t0 & (d.page - 1)) * step + c * 16;
            } else {
                step = d.D * E::BYTES;
                dst = a.q_out + ((((int64_t)s * d.n_layers + layer) * d.Hq + head) * a.t.n_new + t0 - first) * step + c * 16;
            }
            float over[NORM ? B : 1];                          // 1 / root mean square of the rows, for all of them at a time: each is a chain of lane exchanges
            if constexpr (NORM) {
                if (__ballot(!is_v)) {
#pragma unroll
                    for (int i = 0; i < B; ++i) {
                        over[i] = 0.f;
#pragma unroll
                        for (int e = 0; e < E::N; ++e) over[i] = fmaf(E::get(x[i], e), E::get(x[i], e), over[i]);
                        over[i] = c < a.chunks ? over[i] : 0.f;
                    }
                    over_row<B>(over, a.lanes);
                    bool beyond = false;
#pragma unroll
                    for (int i = 0; i < B; ++i) {
                        over[i] = __builtin_amdgcn_rsqf(fmaf(over[i], a.per_element, a.eps));
                        beyond |= over[i] == 0.f;
                    }
                    if (__ballot(beyond && !is_v)) {           // squares that pass fp32: zeros now, as a product with a weight may be infinite
#pragma unroll
                        for (int i = 0; i < B; ++i) {
                            float y[E::N];
#pragma unroll
                            for (int e = 0; e < E::N; ++e) y[e] = E::get(x[i], e) * 0.f;       // what is infinite becomes no number
                            if (over[i] == 0.f && !is_v) x[i] = E::pack(y);
                        }
                    }
                }
            }
            auto turn_row = [&](int i) {
                u32x4 w = x[i], o{0, 0, 0, 0};
                if constexpr (SPLIT && !NORM) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = (uint32_t)__shfl((int)w[e], partner);
                }
                float y[E::N];
                if constexpr (NORM) {
                    if (is_v) return w;
#pragma unroll
                    for (int e = 0; e < E::N; ++e) y[e] = E::get(w, e) * weights.own[e];
                    float z[SPLIT ? E::N : 1];                 // the pairs' other elements
                    if constexpr (SPLIT) from_partner(z, y, pair_chunks, partner);
                    if (turned) {
                        const float4 *angles = reinterpret_cast<const float4 *>(turn + min(group + (bt * B + i) * a.groups, n - 1) * half + angle);
                        if constexpr (SPLIT) {
                            const float sign = upper ? 1.f : -1.f;
#pragma unroll
                            for (int e = 0; e < E::N; e += 2) {
                                const float4 t = angles[e / 2];
                                y[e] = fmaf(z[e], sign * t.y, y[e] * t.x);
                                y[e + 1] = fmaf(z[e + 1], sign * t.w, y[e + 1] * t.z);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < E::N; e += 2) {
                                const float4 t = angles[e / 4];
                                const float u = y[e], v = y[e + 1], cs = e % 4 ? t.z : t.x, sn = e % 4 ? t.w : t.y;
                                y[e] = u * cs - v * sn;
                                y[e + 1] = v * cs + u * sn;
                            }
                        }
                    }
#pragma unroll
                    for (int e = 0; e < E::N; ++e) y[e] *= over[i];
                    return E::pack(y);
                }
                if (!turned || is_v) return w;
                const float4 *angles = reinterpret_cast<const float4 *>(turn + min(group + (bt * B + i) * a.groups, n - 1) * half + angle);
                if constexpr (SPLIT) {
#pragma unroll
                    for (int e = 0; e < E::N; e += 2) {
                        const float4 t = angles[e / 2];
                        const float z0 = E::get(o, e), z1 = E::get(o, e + 1);
                        y[e] = E::get(w, e) * t.x + (upper ? z0 : -z0) * t.y;
                        y[e + 1] = E::get(w, e + 1) * t.z + (upper ? z1 : -z1) * t.w;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E::N; e += 4) {
                        const float4 t = angles[e / 4];
                        const float u0 = E::get(w, e), z0 = E::get(w, e + 1), u1 = E::get(w, e + 2), z1 = E::get(w, e + 3);
                        y[e] = u0 * t.x - z0 * t.y;
                        y[e + 1] = z0 * t.x + u0 * t.y;
                        y[e + 2] = u1 * t.z - z1 * t.w;
                        y[e + 3] = z1 * t.z + u1 * t.w;
                    }
                }
                return E::pack(y);
            };
            if (!ONE && a.side * a.chunks * a.groups == NT && base + a.side <= slot_end && (bt + 1) * rows <= n) {
#pragma unroll
                for (int i = 0; i < B; ++i) {
                    x[i] = turn_row(i);
                    *reinterpret_cast<u32x4 *>(dst + (group + (bt * B + i) * a.groups) * step) = x[i];
                }
                if (is_k) {
#pragma unroll
                    for (int i = 0; i < B; ++i) b.add(x[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < B; ++i) {
                    const int at = group + (bt * B + i) * a.groups;
                    const u32x4 w = turn_row(i);
                    if (live && at < n) {
                        *reinterpret_cast<u32x4 *>(dst + at * step) = w;
                        if (is_k) b.add(w);
                    }
                }
            }
            if (slot_done && a.pv.bounds && base < d.Hkv) {    // the same for the whole workgroup
                const bool extend = t0 & (d.page - 1);         // rows in front of these
                if constexpr (ONE) {
                    if (live && is_k) {
                        char *at = bounds_at(d, a.pv, layer, id, head) + c * 16;
                        if (extend) b.merge_stored(*reinterpret_cast<const u32x4 *>(at), *reinterpret_cast<const u32x4 *>(at + d.D * E::BYTES));
                        b.store(at, d.D * E::BYTES);
                    }
                } else {
                    store_joined<BF16>(b, sh, a.groups, a.chunks * a.side, group, lane_slot * a.chunks + c, active, d.D * E::BYTES, extend, [&](int place) {
                        const int slot = base + place / a.chunks;
                        return slot < min(slot_end, d.Hkv) ? bounds_at(d, a.pv, layer, id, slot) + place % a.chunks * 16 : nullptr;
                    });
                }
                b.clear();
            }
            if constexpr (ONE) break;
            if (next_base >= slot_end) break;
#pragma unroll
            for (int i = 0; i < B; ++i) x[i] = xn[i];
            base = next_base;
            bt = next_bt;
        }
        if (end - t0 <= a.tile) break;                         // in front of the step, which may pass 2^31
    }
}

// What the launch of either kernel makes of a call: the rest of the arguments, and the grid
inline dim3 plan_append(AppendArgs &a, const PageDims &pd, const TokenDims &td, const void *q, const void *k, const void *v, const int32_t *counts,
                        const int32_t *positions, const float *inv_freq, const PageView &pv, void *q_out, bool *one_out)
{
    a.d = pd;
    a.t = td;
    a.pv = pv;
    a.q = static_cast<const char *>(q);
    a.k = static_cast<const char *>(k);
    a.v = static_cast<const char *>(v);
    a.counts = counts;
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.q_out = static_cast<char *>(q_out);
    a.chunks = pd.D * elt_bytes(pd) / 16;
    a.lanes = 1;
    while (a.lanes < a.chunks) a.lanes *= 2;
    a.groups = std::min(std::min(td.n_new, pd.page / BATCH), NT / a.lanes);    // BATCH rows per thread in a whole page
    a.side = NT / (a.lanes * a.groups);
    a.tile = td.R ? std::min(pd.page, ANGLES / (td.R / 2)) : pd.page;
    a.slots = 2 * pd.Hkv + (q ? pd.Hq : 0);
    const int64_t pages = (td.n_new + (int64_t)pd.page - 2) / pd.page + 1, units = pages * pd.n_seq * pd.n_layers;
    const int steps = (a.slots + a.side - 1) / a.side;         // of a workgroup that had them all
    const bool one = *one_out = td.n_new == 1 && steps <= (int)GRID_Y_MOST;    // a grid's third axis has as many places
    const int parts = one ? steps : (int)std::max<int64_t>(1, std::min<int64_t>(std::min(steps, (int)GRID_Y_MOST), APPEND_WGS * pd.cus / units));
    a.per = (steps + parts - 1) / parts * a.side;
    return dim3((unsigned)pages, pd.n_seq * pd.n_layers, (a.slots + a.per - 1) / a.per);
}

template <typename Args> hipError_t launch_append(const Args &a, dim3 grid, bool one, hipStream_t st)
{
    const bool split = a.t.R > 0 && !a.t.interleaved, bf = a.d.dtype == SABLOCK_BF16;
#define SABLOCK_APPEND(SV) (one ? (bf ? append_paged_kernel<true, true, SV, Args> : append_paged_kernel<false, true, SV, Args>) \
                                : (bf ? append_paged_kernel<true, false, SV, Args> : append_paged_kernel<false, false, SV, Args>))
    const auto fn = split ? SABLOCK_APPEND(true) : SABLOCK_APPEND(false);
#undef SABLOCK_APPEND
    hipLaunchKernelGGL(fn, grid, dim3(NT), 0, st, a);
    return hipGetLastError();
}

}  // namespace
}  // namespace sablock
