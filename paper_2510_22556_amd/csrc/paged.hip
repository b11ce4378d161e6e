// The paged cache's writers: the retained rows of a compression into pages (end of Sec. 3.3), and new tokens behind them with
// the position rotation of queries and keys on the way.  Both are copies, 16 bytes per lane, and both keep the page bounds: the
// least and the largest value of every element of K over a page's rows, taken on order-preserving whole numbers (a
// packed 16-bit minimum serves two bf16 elements) and joined over the rows of a workgroup through LDS.
#include "sablock_internal.h"

namespace sablock {
namespace {

constexpr int NT = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <bool BF16> struct Elem;
template <> struct Elem<true> {
    static constexpr int N = 8, BYTES = 2;                     // per 16 bytes, of one
    // signed whole numbers in the order of the values; its own inverse
    static __device__ uint32_t ordered(uint32_t w)
    {
        const s16x2 x = __builtin_bit_cast(s16x2, w);
        return __builtin_bit_cast(uint32_t, x ^ ((x >> 15) & (short)0x7fff));
    }
    static __device__ uint32_t lower(uint32_t a, uint32_t b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
    }
    static __device__ uint32_t upper(uint32_t a, uint32_t b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
    }
    static constexpr uint32_t LEAST = 0x80008000u, MOST = 0x7fff7fffu;
    static __device__ float get(const u32x4 &v, int e) { return __uint_as_float((e & 1) ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
    static __device__ u32x4 pack(const float (&x)[8])          // rounded to nearest, ties to even
    {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
        return o;
    }
};
template <> struct Elem<false> {
    static constexpr int N = 4, BYTES = 4;
    static __device__ uint32_t ordered(uint32_t w) { return w ^ ((uint32_t)((int32_t)w >> 31) & 0x7fffffffu); }
    static __device__ uint32_t lower(uint32_t a, uint32_t b) { return (uint32_t)min((int32_t)a, (int32_t)b); }
    static __device__ uint32_t upper(uint32_t a, uint32_t b) { return (uint32_t)max((int32_t)a, (int32_t)b); }
    static constexpr uint32_t LEAST = 0x80000000u, MOST = 0x7fffffffu;
    static __device__ float get(const u32x4 &v, int e) { return __uint_as_float(v[e]); }
    static __device__ u32x4 pack(const float (&x)[4])
    {
        return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};

template <bool BF16> struct Bounds {                           // of the elements of one 16-byte chunk, as ordered whole numbers
    using E = Elem<BF16>;
    u32x4 lo, hi;
    __device__ void clear()
    {
        lo = u32x4{E::MOST, E::MOST, E::MOST, E::MOST};
        hi = u32x4{E::LEAST, E::LEAST, E::LEAST, E::LEAST};
    }
    __device__ void add(const u32x4 &v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = E::ordered(v[i]);
            lo[i] = E::lower(lo[i], x);
            hi[i] = E::upper(hi[i], x);
        }
    }
    __device__ void merge_stored(const u32x4 &l, const u32x4 &h)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = E::lower(lo[i], E::ordered(l[i]));
            hi[i] = E::upper(hi[i], E::ordered(h[i]));
        }
    }
    __device__ void store(char *b, int row_bytes) const
    {
        u32x4 l, h;
#pragma unroll
        for (int i = 0; i < 4; ++i) { l[i] = E::ordered(lo[i]); h[i] = E::ordered(hi[i]); }
        *reinterpret_cast<u32x4 *>(b) = l;
        *reinterpret_cast<u32x4 *>(b + row_bytes) = h;
    }
};

// bounds of a chunk over the row groups of a workgroup: sh[group][chunk]; what the first group's threads get is joined
template <bool BF16>
__device__ void join_groups(Bounds<BF16> &b, Bounds<BF16> *sh, int groups, int per_group, int group, int place, bool active)
{
    __syncthreads();
    if (active) sh[group * per_group + place] = b;
    __syncthreads();
    if (active && group == 0)
        for (int g = 1; g < groups; ++g) {
            const Bounds<BF16> o = sh[g * per_group + place];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                b.lo[i] = Elem<BF16>::lower(b.lo[i], o.lo[i]);
                b.hi[i] = Elem<BF16>::upper(b.hi[i], o.hi[i]);
            }
        }
}

__device__ __forceinline__ char *bounds_at(const PageDims &d, const PageView &v, int32_t layer, int32_t id, int32_t head)
{
    return v.bounds + (((int64_t)layer * d.n_pages + id) * d.Hkv + head) * 2 * d.D * elt_bytes(d);
}

// grid (pages of a sequence, problems): a workgroup fills one page of one problem.  A thread has one chunk of every groups-th row.
template <bool BF16>
__global__ void __launch_bounds__(NT)
compact_paged_kernel(Dims d, PageDims pd, PageView pv, const char *k, const char *v, const int32_t *idx, int budget, int kept, int rows,
                     int chunks, int32_t *lengths_out)
{
    using E = Elem<BF16>;
    __shared__ Bounds<BF16> sh[NT];
    const int p = blockIdx.y, s = seq_of_problem(pd, p), layer = layer_of_problem(pd, p), head = head_of_problem(pd, p);
    if (lengths_out && blockIdx.x == 0 && layer == 0 && head == 0 && threadIdx.x == 0) lengths_out[s] = rows;
    const int r0 = blockIdx.x << pd.shift, n = min(pd.page, rows - r0);
    const int groups = NT / chunks, group = threadIdx.x / chunks, c = threadIdx.x - group * chunks;
    const bool active = group < groups;
    if (n <= 0) return;
    const int id = page_at(pd, pv.table, s, blockIdx.x);
    if (id < 0) return;
    const char *ksrc = k + k_problem_offset(d, p) * E::BYTES + (int64_t)c * 16, *vsrc = v + v_problem_offset(d, p) * E::BYTES + (int64_t)c * 16;
    char *kdst = pv.k + (layer * pd.ks[0] + id * pd.ks[1] + head * pd.ks[2]) * E::BYTES + (int64_t)c * 16;
    char *vdst = pv.v + (layer * pd.vs[0] + id * pd.vs[1] + head * pd.vs[2]) * E::BYTES + (int64_t)c * 16;
    Bounds<BF16> b;
    b.clear();
    if (active)
        for (int r = group; r < n; r += groups) {
            const int at = r0 + r, t = at < kept ? idx[(int64_t)p * budget + at] : d.T + at - kept;
            u32x4 x{0, 0, 0, 0}, y{0, 0, 0, 0};
            if (t >= 0 && t < d.L) {
                x = *reinterpret_cast<const u32x4 *>(ksrc + t * d.ks[3] * E::BYTES);
                y = *reinterpret_cast<const u32x4 *>(vsrc + t * d.vs[3] * E::BYTES);
            }
            *reinterpret_cast<u32x4 *>(kdst + r * pd.ks[3] * E::BYTES) = x;
            *reinterpret_cast<u32x4 *>(vdst + r * pd.vs[3] * E::BYTES) = y;
            b.add(x);
        }
    if (!pv.bounds) return;
    join_groups<BF16>(b, sh, groups, chunks, group, c, active);
    if (group == 0) b.store(bounds_at(pd, pv, layer, id, head) + c * 16, pd.D * E::BYTES);
}

constexpr int ANGLES = 4096;                   // (token, pair) whose sine and cosine LDS holds at a time

struct AppendArgs {
    PageDims d;
    TokenDims t;
    PageView pv;
    const char *q, *k, *v;
    const int32_t *counts, *positions;
    const float *inv_freq;
    char *q_out;
    int slots, per;             // head rows: K's heads, V's, q's; of a workgroup
    int chunks, groups, side;   // 16-byte chunks of a row; rows and head rows that a workgroup does at a time
    int tile;                   // tokens whose angles LDS holds
};

// grid (touched pages, sequences x layers, parts of the head rows).  The angle of a (token, pair) is the same for all heads: formed
// once per workgroup, position * inv_freq in whole turns in fp64 (at position 131 072 an angle in fp32 is off by up to 2^-8), the
// fraction of a turn in fp32.
template <bool BF16>
__global__ void __launch_bounds__(NT)
append_paged_kernel(AppendArgs a)
{
    using E = Elem<BF16>;
    __shared__ Bounds<BF16> sh[NT];
    __shared__ float2 turn[ANGLES];                            // cosine, sine
    const PageDims &d = a.d;
    const int s = blockIdx.y / d.n_layers, layer = blockIdx.y - s * d.n_layers, tid = threadIdx.x;
    const int len = rows_of(d, a.pv.lengths, s);
    const int count = min(a.counts ? min(max(a.counts[s], 0), a.t.n_new) : a.t.n_new, len);
    const int first = len - count, page = (first >> d.shift) + (int)blockIdx.x;
    if ((int64_t)page << d.shift >= len) return;
    const int begin = max(first, page << d.shift), end = min(len, (page + 1) << d.shift);
    if (begin >= end) return;
    const int id = page_at(d, a.pv.table, s, page);
    const int half = a.t.R / 2, pair_chunks = half / E::N, rotated = a.t.R / E::N;
    const int c = tid % a.chunks, at = tid / a.chunks, group = at % a.groups, lane_slot = at / a.groups;
    const bool active = lane_slot < a.side;
    const int slot_end = min(a.slots, ((int)blockIdx.z + 1) * a.per);
    const int64_t position0 = a.t.R ? (int64_t)a.positions[s] : 0;
    for (int t0 = begin; t0 < end; t0 += a.tile) {
        const int n = min(a.tile, end - t0);
        if (a.t.R) {
            __syncthreads();
            for (int i = tid; i < n * half; i += NT) {
                const int tok = i / half, pair = i - tok * half;
                const double turns = (double)(position0 + t0 - first + tok) * ((double)a.inv_freq[pair] * 0.15915494309189535);
                float sn, cs;
                sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
                turn[i] = make_float2(cs, sn);
            }
            __syncthreads();
        }
        for (int base = blockIdx.z * a.per; base < slot_end; base += a.side) {
            const int slot = base + lane_slot;
            const bool live = active && slot < slot_end, is_k = slot < d.Hkv, is_v = !is_k && slot < 2 * d.Hkv;
            const int head = is_k ? slot : is_v ? slot - d.Hkv : slot - 2 * d.Hkv;
            const int64_t *st = is_k ? a.t.ks : is_v ? a.t.vs : a.t.qs;
            const char *src = (is_k ? a.k : is_v ? a.v : a.q) + (s * st[0] + layer * st[1] + head * st[2]) * E::BYTES;
            Bounds<BF16> b;
            b.clear();
            if (live)
                for (int r = group; r < n; r += a.groups) {
                    const int row = t0 + r, tok = row - first;
                    const char *x_at = src + tok * st[3] * E::BYTES;
                    u32x4 x = *reinterpret_cast<const u32x4 *>(x_at + c * 16);
                    if (!is_v && c < rotated) {
                        float y[E::N];
                        if (a.t.interleaved) {
#pragma unroll
                            for (int e = 0; e < E::N; e += 2) {
                                const float2 w = turn[r * half + (c * E::N + e) / 2];
                                const float u = E::get(x, e), z = E::get(x, e + 1);
                                y[e] = u * w.x - z * w.y;
                                y[e + 1] = z * w.x + u * w.y;
                            }
                        } else {
                            const bool up = c >= pair_chunks;
                            const u32x4 o = *reinterpret_cast<const u32x4 *>(x_at + (up ? c - pair_chunks : c + pair_chunks) * 16);
#pragma unroll
                            for (int e = 0; e < E::N; ++e) {
                                const float2 w = turn[r * half + (up ? c - pair_chunks : c) * E::N + e];
                                const float u = E::get(x, e), z = E::get(o, e);
                                y[e] = u * w.x + (up ? z : -z) * w.y;
                            }
                        }
                        x = E::pack(y);
                    }
                    if (is_k || is_v) {
                        if (id < 0) continue;
                        const int64_t *ps = is_k ? d.ks : d.vs;
                        char *dst = (is_k ? a.pv.k : a.pv.v) + (layer * ps[0] + id * ps[1] + head * ps[2] + (row & (d.page - 1)) * ps[3]) * E::BYTES;
                        *reinterpret_cast<u32x4 *>(dst + c * 16) = x;
                        if (is_k) b.add(x);
                    } else {
                        const int64_t out_row = (((int64_t)s * d.n_layers + layer) * d.Hq + head) * a.t.n_new + tok;
                        *reinterpret_cast<u32x4 *>(a.q_out + out_row * d.D * E::BYTES + c * 16) = x;
                    }
                }
            if (!a.pv.bounds || base >= d.Hkv) continue;       // the same for the whole workgroup
            if (a.groups > 1) join_groups<BF16>(b, sh, a.groups, a.chunks * a.side, group, lane_slot * a.chunks + c, active);
            if (live && is_k && group == 0 && id >= 0) {
                char *at_bounds = bounds_at(d, a.pv, layer, id, head) + c * 16;
                if (t0 & (d.page - 1))                         // rows in front of these
                    b.merge_stored(*reinterpret_cast<const u32x4 *>(at_bounds), *reinterpret_cast<const u32x4 *>(at_bounds + d.D * E::BYTES));
                b.store(at_bounds, d.D * E::BYTES);
            }
        }
    }
}

}  // namespace

hipError_t launch_compact_paged(const Dims &d, const void *k, const void *v, const int32_t *idx, int32_t budget, int32_t rows,
                                const PageDims &pd, const PageView &pv, int32_t *lengths_out, hipStream_t st)
{
    const int chunks = pd.D * elt_bytes(pd) / 16, kept = std::min(budget, d.T);
    const dim3 grid(std::max(1, (rows + pd.page - 1) >> pd.shift), pd.P);
    hipLaunchKernelGGL(pd.dtype == SABLOCK_BF16 ? compact_paged_kernel<true> : compact_paged_kernel<false>, grid, dim3(NT), 0, st, d, pd, pv,
                       static_cast<const char *>(k), static_cast<const char *>(v), idx, budget, kept, rows, chunks, lengths_out);
    return hipGetLastError();
}

hipError_t launch_append_paged(const PageDims &pd, const TokenDims &td, const void *q, const void *k, const void *v, const int32_t *counts,
                               const int32_t *positions, const float *inv_freq, const PageView &pv, void *q_out, hipStream_t st)
{
    AppendArgs a;
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
    a.groups = std::min(std::min(td.n_new, pd.page), NT / a.chunks);
    a.side = NT / (a.chunks * a.groups);
    a.tile = td.R ? std::min(pd.page, ANGLES / (td.R / 2)) : pd.page;
    a.slots = 2 * pd.Hkv + (q ? pd.Hq : 0);
    const int64_t pages = (td.n_new + (int64_t)pd.page - 2) / pd.page + 1, units = pages * pd.n_seq * pd.n_layers;
    const int steps = (a.slots + a.side - 1) / a.side;         // of a workgroup that had them all
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(steps, 4 * pd.cus / units));
    a.per = (steps + parts - 1) / parts * a.side;
    const dim3 grid((unsigned)pages, pd.n_seq * pd.n_layers, (a.slots + a.per - 1) / a.per);
    hipLaunchKernelGGL(pd.dtype == SABLOCK_BF16 ? append_paged_kernel<true> : append_paged_kernel<false>, grid, dim3(NT), 0, st, a);
    return hipGetLastError();
}

}  // namespace sablock
