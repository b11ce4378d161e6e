// The paged cache's writers: the retained rows of a compression into pages (end of Sec. 3.3), and new tokens behind them with
// the position rotation of queries and keys on the way.  Both are copies, 16 bytes per lane, and both keep the page bounds: the
// least and the largest value of every element of K over a page's rows, taken on order-preserving whole numbers (a
// packed 16-bit minimum serves two bf16 elements) and joined over the rows of a workgroup through LDS.
//
// What bounds them: the copy.  A large device copy reaches 5.0-5.3 TB/s here, read and written.  Compaction of 32 layers x 8 heads,
// 1 024 rows of 256 bytes each out of 32 768 (272 MB in and out): 61 us, 4.6 TB/s; several rows per thread in flight gain
// nothing over one and eight workgroups per compute unit (61.1, 60.2 us).  Appended prompts, 11 300 tokens x 48 heads (278 MB): 69 us,
// 4.0 TB/s, the rotation's vector instructions a third of that time beside it; without a rotation 68; fp32 130 us.  One token: 4.4 us in a graph, as
// good as one launch and three dependent loads; 256 sequences, a token each, 5.9 us.
#include "sablock_internal.h"

namespace sablock {
namespace {

constexpr int NT = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr double TURN = 0.15915494309189535, TURN_REST = -9.839338337591243e-18;                // 1 / (2 pi), and what fp64 leaves of it

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
    // cosine and sine of position * freq.  The fraction of a turn, sine and cosine in fp32: off by 2^-22, which rows of 8 bits do not show
    static __device__ float2 turn(double position, float freq)
    {
        const double turns = position * ((double)freq * TURN);
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        return make_float2(cs, sn);
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
    // The angle as the fp64 number that it is, its fraction of a turn to 2^-53 of one however many there are, less the nearest quarter.  What is left, at
    // most pi / 4, as the sum h + l of two fp32 numbers; sine and cosine by the first terms of their series (the next are below 2^-32 of them), with
    // what l and the roundings of the large terms leave out put back: off by 0.75 and 0.6 units in the last place at most, on average by as much as fp64
    // rounded once.  (In fp64 throughout, the registers would leave room for a workgroup less.)
    static __device__ float2 turn(double position, float freq)
    {
        const double angle = position * (double)freq, part = fma(angle, TURN_REST, fma(angle, TURN, -rint(angle * TURN)));
        const double quarters = rint(4.0 * part), r = (part - 0.25 * quarters) * 6.283185307179586;
        const float h = (float)r, l = (float)(r - (double)h), z = h * h, zl = fmaf(h, h, -z) + 2.f * h * l;
        float sn = fmaf(z, -1.f / 39916800, 1.f / 362880), cs = fmaf(z, -1.f / 3628800, 1.f / 40320);
        sn = fmaf(z, sn, -1.f / 5040);
        cs = fmaf(z, cs, -1.f / 720);
        sn = fmaf(z, sn, 1.f / 120);
        cs = fmaf(z, cs, 1.f / 24);
        sn = fmaf(z, sn, -1.f / 6);
        const float most = fmaf(z, -0.5f, 1.f), rest = (1.f - most) - 0.5f * z;
        const float s = h + fmaf(h * z, sn, l * most), c = most + (fmaf(zl, -0.5f, rest) + z * z * cs);
        const int q = (int)quarters & 3;                       // the pair turned by a quarter: (c, s) -> (-s, c)
        const float x = q & 1 ? s : c, y = q & 1 ? c : s;
        return make_float2(q == 1 || q == 2 ? -x : x, q & 2 ? -y : y);
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

// Bounds of a workgroup's chunks over its row groups, sh[group][place], written where at(place) says (nullptr: nowhere), joined with what is
// there if `extend`.  A thread joins one dword of one place: consecutive lanes, consecutive banks.
template <bool BF16, typename At>
__device__ void store_joined(const Bounds<BF16> &b, uint32_t *sh, int groups, int places, int group, int place, bool active, int row_bytes, bool extend, At &&at)
{
    using E = Elem<BF16>;
    __syncthreads();
    if (active) {
        u32x4 *o = reinterpret_cast<u32x4 *>(sh) + (group * places + place) * 2;
        o[0] = b.lo;
        o[1] = b.hi;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < places * 8; i += NT) {
        const int w = i & 7;
        char *dst = at(i >> 3);
        if (!dst) continue;
        uint32_t x = sh[i];
        auto join = [&](uint32_t y) { x = w < 4 ? E::lower(x, y) : E::upper(x, y); };
#pragma unroll 4
        for (int g = 1; g < groups; ++g) join(sh[g * places * 8 + i]);
        uint32_t *word = reinterpret_cast<uint32_t *>(dst + (w < 4 ? 0 : row_bytes)) + (w & 3);
        if (extend) join(E::ordered(*word));
        *word = E::ordered(x);
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
    __shared__ __attribute__((aligned(16))) uint32_t sh[NT * 8];
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
    char *at = bounds_at(pd, pv, layer, id, head);
    store_joined<BF16>(b, sh, groups, chunks, group, c, active, pd.D * E::BYTES, false, [&](int place) { return at + place * 16; });
}

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

// grid (touched pages, sequences x layers, parts of the head rows).  The angle of a (token, pair) is the same for all heads: formed
// once per workgroup, position * inv_freq in fp64 (at position 131 072 an angle in fp32 is off by up to 2^-8), see turn() of either
// type.  A thread has one chunk of every groups-th row of a head, a row's chunks lie in the lanes of one wavefront, where
// the other halves of pairs come from.  The rows of the next step are on their way while one is turned and stored, the first
// ones while the angles are formed.
// ONE: a token per sequence, and a workgroup has no more head rows than it does at a time.  SPLIT: the two elements of a pair lie half a rotation
// apart, in different chunks.
// Loads of a step are issued whatever the lane has to do there (at the nearest place that exists): behind a branch the compiler could
// not count the loads in flight and would wait for all of them.  A step whose rows all exist stores without a branch for the same reason.
template <bool BF16, bool ONE, bool SPLIT>
__global__ void __launch_bounds__(NT, ONE || SPLIT ? 4 : 3)
append_paged_kernel(AppendArgs a)
{
    using E = Elem<BF16>;
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
            auto turn_row = [&](int i) {
                u32x4 w = x[i], o{0, 0, 0, 0};
                if constexpr (SPLIT) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = (uint32_t)__shfl((int)w[e], partner);
                }
                if (!turned || is_v) return w;
                float y[E::N];
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
    a.lanes = 1;
    while (a.lanes < a.chunks) a.lanes *= 2;
    a.groups = std::min(std::min(td.n_new, pd.page / BATCH), NT / a.lanes);    // BATCH rows per thread in a whole page
    a.side = NT / (a.lanes * a.groups);
    a.tile = td.R ? std::min(pd.page, ANGLES / (td.R / 2)) : pd.page;
    a.slots = 2 * pd.Hkv + (q ? pd.Hq : 0);
    const int64_t pages = (td.n_new + (int64_t)pd.page - 2) / pd.page + 1, units = pages * pd.n_seq * pd.n_layers;
    const int steps = (a.slots + a.side - 1) / a.side;         // of a workgroup that had them all
    const bool one = td.n_new == 1 && steps <= (int)GRID_Y_MOST, bf = pd.dtype == SABLOCK_BF16;               // a grid's third axis has as many places
    const int parts = one ? steps : (int)std::max<int64_t>(1, std::min<int64_t>(std::min(steps, (int)GRID_Y_MOST), APPEND_WGS * pd.cus / units));
    a.per = (steps + parts - 1) / parts * a.side;
    const dim3 grid((unsigned)pages, pd.n_seq * pd.n_layers, (a.slots + a.per - 1) / a.per);
    const bool split = td.R > 0 && !td.interleaved;
#define SABLOCK_APPEND(SV) (one ? (bf ? append_paged_kernel<true, true, SV> : append_paged_kernel<false, true, SV>) \
                                : (bf ? append_paged_kernel<true, false, SV> : append_paged_kernel<false, false, SV>))
    const auto fn = split ? SABLOCK_APPEND(true) : SABLOCK_APPEND(false);
#undef SABLOCK_APPEND
    hipLaunchKernelGGL(fn, grid, dim3(NT), 0, st, a);
    return hipGetLastError();
}

}  // namespace sablock
