// The pages that a decode step over a paged cache reads when it may not read all: a score per page from the bounds of its keys,
// then the best of them per KV head.
//
//   page_scores_kernel   max(q lo, q hi) is q+ hi + q- lo with q+ = max(q, 0), q- = min(q, 0): two products per element and head,
//       formed and summed in fp64.  The products of two bf16 values and their sum over a head are exact there (but for
//       elements some 2^30 apart), so that which of two pages comes first does not hang on the order of a sum.  A page's row of bounds
//       is spread over LP lanes, 16 bytes of lo and of hi each, several pages in flight; the sums of up to four heads over the
//       lanes hand each lane one head, which it rounds to fp32 and turns into a whole number of the same order, and the maximum
//       over the heads is one of whole numbers, in which what is no number can be the largest.
//       What bounds it: 8 heads x 8 192 pages of 512 bytes of bounds, four query heads: 12.4 us, of which 5.1 are the bytes at 6.6 TB/s
//       and 5.7 the vector pipe (two fp64 products per element and head); the rest is the chain length, table, bounds.  With the
//       next pages' bounds on their way 13.4 in place of 14.7.
//   pick_pages_kernel    a workgroup per problem; the keys stay in registers.  The last key that is taken is found digit by digit, 11 bits
//       of its distance from the least key at a time (the keys of a problem share their upper bits) until 64 are left, which a wavefront
//       ranks, and one prefix sum places the pages in order.  8 192 pages: 7.3 us, a chain of a dozen barriers.
#include "sablock_internal.h"

namespace sablock {
namespace {

constexpr int NT = 256, PICK_NT = 1024;
constexpr int SCORE_WGS = 2;                   // workgroups of the scores per compute unit: as many as run at a time
constexpr uint32_t NOT_A_NUMBER = 0xfffffffeu; // above every number's key

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <bool BF16> struct Piece;             // 16 bytes of a row
template <> struct Piece<true> {
    static constexpr int N = 8;
    static __device__ float value(const u32x4 &v, int e) { return __uint_as_float((e & 1) ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
};
template <> struct Piece<false> {
    static constexpr int N = 4;
    static __device__ float value(const u32x4 &v, int e) { return __uint_as_float(v[e]); }
};

template <int M> __device__ __forceinline__ uint32_t xor_lane_u(uint32_t x) { return __float_as_uint(xor_lane<M>(__uint_as_float(x))); }
template <int M> __device__ __forceinline__ double xor_lane_d(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)xor_lane_u<M>((uint32_t)(u >> 32)) << 32 | xor_lane_u<M>((uint32_t)u));
}

// x[0 .. N) summed over LP lanes: lane l gets the entries l % S + S j, S = min(N, LP), in x[j]
template <int B, int S, int LP, int N>
__device__ __forceinline__ void sum_lanes(double (&x)[N])
{
    if constexpr (B < LP) {
        if constexpr (B < S) {
            const bool up = threadIdx.x & B;
#pragma unroll
            for (int i = 0; i < N / (2 * B); ++i) {
                const double own = up ? x[2 * i + 1] : x[2 * i], other = up ? x[2 * i] : x[2 * i + 1];
                x[i] = own + xor_lane_d<B>(other);
            }
        } else {
#pragma unroll
            for (int j = 0; j < N / S; ++j) x[j] += xor_lane_d<B>(x[j]);
        }
        sum_lanes<2 * B, S, LP, N>(x);
    }
}
template <int B, int S> __device__ __forceinline__ uint32_t most_of_lanes(uint32_t x)
{
    if constexpr (B < S) return most_of_lanes<2 * B, S>(max(x, xor_lane_u<B>(x)));
    else return x;
}

// Pages in flight per lane: those of the next step besides, or so many more for one loading of the heads' registers
constexpr int flight_of(bool many) { return many ? 8 : 4; }

struct ScoreArgs {
    PageDims d;
    PageView pv;
    const char *q;
    int stride;                  // of a problem's keys
    uint32_t *keys;
};

// grid (parts of a sequence's pages, problems).  HB heads at a time, in registers; more heads (MANY) are more walks over the pages in
// flight.
template <bool BF16, int LP, int HB, bool MANY>
__global__ void __launch_bounds__(NT, 2)
page_scores_kernel(ScoreArgs a)
{
    using Pc = Piece<BF16>;
    constexpr int E = Pc::N, ELT = 16 / E, PW = 64 / LP, S = HB < LP ? HB : LP, FLIGHT = flight_of(MANY);
    const PageDims &d = a.d;
    const int p = blockIdx.y, s = seq_of_problem(d, p), layer = layer_of_problem(d, p), head = head_of_problem(d, p);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % LP, place = lane / LP;
    const int n = (rows_of(d, a.pv.lengths, s) + d.page - 1) >> d.shift;
    const bool mine = c * E < d.D;                             // lanes behind the row's end are padding
    const int64_t row = (int64_t)d.D * ELT;
    const char *q = a.q + (((int64_t)s * d.n_layers + layer) * d.Hq + head * d.G) * row + c * 16;
    __shared__ __attribute__((aligned(16))) char q_sh[MANY ? 16 * 256 * ELT : 16];         // all heads: read for every walk, beside loads in flight
    const char *bounds = a.pv.bounds + ((int64_t)layer * d.n_pages * d.Hkv + head) * 2 * row + (mine ? c : 0) * 16;
    double up[HB][E], down[HB][E];                             // q+ and q-
    auto load_heads = [&](int g0) {
#pragma unroll
        for (int g = 0; g < HB; ++g) {
            u32x4 x{0, 0, 0, 0};
            if (mine && g0 + g < d.G) x = *reinterpret_cast<const u32x4 *>(MANY ? q_sh + c * 16 + (g0 + g) * (int)row : q + (g0 + g) * row);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float v = Pc::value(x, e);
                up[g][e] = (double)(v < 0.f ? 0.f : v);        // what is no number stays one
                down[g][e] = (double)(v < 0.f ? v : 0.f);
            }
        }
    };
    struct Flight { int id[FLIGHT]; u32x4 lo[FLIGHT], hi[FLIGHT]; };
    // Nothing is loaded behind a branch (what does not exist is replaced by what does, and not used): the compiler could not count
    // the loads in flight there.
    auto load_ids = [&](int i0, int (&id)[FLIGHT]) {
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) id[u] = page_at(d, a.pv.table, s, min(i0 + u * PW + place, n - 1));
    };
    auto load_bounds = [&](Flight &f) {
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const char *b = bounds + (int64_t)max(f.id[u], 0) * d.Hkv * 2 * row;
            f.lo[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(b));
            f.hi[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(b + row));
        }
    };
    if constexpr (MANY) {
        for (int i = threadIdx.x * 16; i < d.G * (int)row; i += NT * 16)
            *reinterpret_cast<u32x4 *>(q_sh + i) = *reinterpret_cast<const u32x4 *>(q - c * 16 + i);
        __syncthreads();
    }
    const int step = gridDim.x * (NT / 64) * PW * FLIGHT, start = (blockIdx.x * (NT / 64) + wave) * PW * FLIGHT;
    if (start >= n) return;
    Flight now, next;
    load_ids(start, now.id);
    if constexpr (!MANY) load_ids(start + step, next.id);
    load_bounds(now);
    if constexpr (!MANY) load_heads(0);
    for (int i0 = start; i0 < n; i0 += step) {
        uint32_t key[FLIGHT];
        int later[FLIGHT];
        if constexpr (!MANY) {
            load_bounds(next);
            load_ids(i0 + 2 * step, later);
        } else load_ids(i0 + step, later);
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            key[u] = 0;
            if (!mine) now.lo[u] = now.hi[u] = u32x4{0, 0, 0, 0};
        }
        for (int g0 = 0; g0 < (MANY ? d.G : 1); g0 += HB) {
            if constexpr (MANY) {
                load_heads(g0);
#pragma unroll
                for (int u = 0; u < FLIGHT; ++u)               // converted anew for every walk: in fp64 they would not fit the registers
#pragma unroll
                    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(now.lo[u][i]), "+v"(now.hi[u][i]));
            }
#pragma unroll
            for (int u = 0; u < FLIGHT; ++u) {
                double x[HB];
#pragma unroll
                for (int g = 0; g < HB; ++g) x[g] = 0.0;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const double l = (double)Pc::value(now.lo[u], e), h = (double)Pc::value(now.hi[u], e);
#pragma unroll
                    for (int g = 0; g < HB; ++g) x[g] = fma(up[g][e], h, fma(down[g][e], l, x[g]));
                }
                sum_lanes<1, S, LP, HB>(x);
#pragma unroll
                for (int j = 0; j < HB / S; ++j)
                    if (g0 + c % S + S * j < d.G) key[u] = max(key[u], x[j] == x[j] ? ordered_key((float)x[j]) : NOT_A_NUMBER);
            }
        }
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const int i = i0 + u * PW + place;
            const uint32_t x = most_of_lanes<1, S>(key[u]);
            if (c == 0 && i < n) a.keys[(int64_t)p * a.stride + i] = now.id[u] >= 0 ? x : ordered_key(-INFINITY);
        }
        if constexpr (!MANY) {
            now = next;
#pragma unroll
            for (int u = 0; u < FLIGHT; ++u) next.id[u] = later[u];
        } else {
#pragma unroll
            for (int u = 0; u < FLIGHT; ++u) now.id[u] = later[u];
            load_bounds(now);
        }
    }
}

__device__ __forceinline__ int sum_upto(int x, int lane)       // inclusive, over the lanes
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(x, o);
        if (lane >= o) x += u;
    }
    return x;
}

constexpr int DIGIT = 11, BINS = 1 << DIGIT;
constexpr int FEW = 64;                        // keys that one wavefront ranks

// grid P: the first and the last pages and the best of the others, the lower page first where keys are equal.  A thread has RUN consecutive pages,
// or (RUN = 0) as many as it takes, read again in every pass.
template <int RUN>
__global__ void __launch_bounds__(PICK_NT)
pick_pages_kernel(PageDims d, PageView pv, int n_pick, int n_first, int n_last, const uint32_t *keys_all, int stride, int32_t *list_all)
{
    constexpr int NWV = PICK_NT / 64;
    __shared__ int hist[BINS], red[NWV], few_at[FEW], n_few;
    __shared__ uint32_t extreme[2 * NWV], few_key[FEW];
    __shared__ int found[3];                                   // bin, taken from it, its size; then the last key and page that are taken
    const int p = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t *keys = keys_all + (int64_t)p * stride;
    const int full = RUN ? RUN : 0;
    uint32_t own[RUN ? RUN : 1];
    if constexpr (RUN > 0) {                                   // before the length is known; the row's end is padded
#pragma unroll
        for (int j = 0; j < RUN; j += 4) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(keys + min(tid * full + j, stride - 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) own[j + i] = x[i];
        }
    }
    const int n = (rows_of(d, pv.lengths, seq_of_problem(d, p)) + d.page - 1) >> d.shift;
    int32_t *list = list_all + (int64_t)p * n_pick;
    if (n <= n_pick) {
        for (int i = tid; i < n_pick; i += PICK_NT) list[i] = i < n ? i : -1;
        return;
    }
    const int run = RUN ? RUN : ((n + PICK_NT - 1) / PICK_NT + 3) & ~3, from = (int)min((int64_t)n, (int64_t)tid * run), to = min(n, from + run);
    const int rest0 = n_first, rest1 = n - n_last;             // the pages that have to be ranked
    auto ranked = [&](auto &&f) {                              // f(key, page) for the thread's pages that have to be ranked
        if constexpr (RUN > 0) {
#pragma unroll
            for (int j = 0; j < RUN; ++j)
                if (from + j >= rest0 && from + j < min(to, rest1)) f(own[j], from + j);
        } else {
#pragma unroll 4
            for (int i = from; i < to; i += 4) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(keys + i);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (i + j >= rest0 && i + j < min(to, rest1)) f(x[j], i + j);
            }
        }
    };
    uint32_t least = 0xffffffffu, most = 0;
    ranked([&](uint32_t x, int) { least = min(least, x); most = max(most, x); });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { least = min(least, (uint32_t)__shfl_xor((int)least, o)); most = max(most, (uint32_t)__shfl_xor((int)most, o)); }
    if (lane == 0) { extreme[wave] = least; extreme[NWV + wave] = most; }
    for (int i = tid; i < BINS; i += PICK_NT) hist[i] = 0;
    if (tid == 0) n_few = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NWV; ++w) { least = min(least, extreme[w]); most = max(most, extreme[NWV + w]); }
    // `left` of the `inside` keys in [least, least + 2^bits) are taken, and all above
    int left = n_pick - n_first - n_last, bits = most > least ? 32 - __clz((int)(most - least)) : 0, inside = rest1 - rest0;
    auto is_inside = [&](uint32_t x) { return x >= least && (bits == 32 || (x - least) >> bits == 0); };
    while (left > 0 && left < inside && bits > 0 && inside > FEW) {
        const int shift = max(0, bits - DIGIT);
        ranked([&](uint32_t x, int) {
            if (is_inside(x)) atomicAdd(&hist[(x - least) >> shift], 1);
        });
        __syncthreads();
        const int b0 = BINS - 1 - 2 * tid, h0 = hist[b0], h1 = hist[b0 - 1];   // two bins per thread, the largest first
        const int upto = sum_upto(h0 + h1, lane);
        if (lane == 63) red[wave] = upto;
        __syncthreads();
        int before = upto - h0 - h1;
#pragma unroll
        for (int w = 0; w < NWV; ++w) before += w < wave ? red[w] : 0;
        if (before < left && before + h0 >= left) { found[0] = b0; found[1] = left - before; found[2] = h0; }
        else if (before + h0 < left && before + h0 + h1 >= left) { found[0] = b0 - 1; found[1] = left - before - h0; found[2] = h1; }
        hist[b0] = hist[b0 - 1] = 0;
        __syncthreads();
        least += (uint32_t)found[0] << shift;
        left = found[1];
        inside = found[2];
        bits = shift;
        __syncthreads();
    }
    // the last that is taken, in the order of keys and of pages: key `cut`, page `cut_at`
    uint32_t cut = least;
    int cut_at = 0x7fffffff;
    if (left == 0) cut = 0xffffffffu;                          // none: above all keys
    else if (left < inside) {
        if (inside <= FEW) {
            ranked([&](uint32_t x, int i) {
                if (is_inside(x)) {
                    const int at = atomicAdd(&n_few, 1);       // their order is of no account
                    few_key[at] = x;
                    few_at[at] = i;
                }
            });
            __syncthreads();
            if (tid < inside) {
                const uint32_t x = few_key[tid];
                const int i = few_at[tid];
                int better = 0;
                for (int j = 0; j < inside; ++j) better += few_key[j] > x || (few_key[j] == x && few_at[j] < i);
                if (better == left - 1) { found[0] = (int)x; found[1] = i; }
            }
        } else {                                               // all inside are equal
            int eq = 0;
            ranked([&](uint32_t x, int) { eq += x == least; });
            const int upto = sum_upto(eq, lane);
            if (lane == 63) red[wave] = upto;
            __syncthreads();
            int before = upto - eq;
#pragma unroll
            for (int w = 0; w < NWV; ++w) before += w < wave ? red[w] : 0;
            ranked([&](uint32_t x, int i) {
                if (x == least && ++before == left) { found[0] = (int)x; found[1] = i; }
            });
        }
        __syncthreads();
        cut = (uint32_t)found[0];
        cut_at = found[1];
        __syncthreads();
    }
    auto taken = [&](uint32_t x, int i) { return x > cut || (x == cut && i <= cut_at); };
    int count = max(0, min(to, rest0) - from) + max(0, to - max(from, rest1));
    ranked([&](uint32_t x, int i) { count += taken(x, i); });
    const int upto = sum_upto(count, lane);
    if (lane == 63) red[wave] = upto;
    __syncthreads();
    int at = upto - count;
#pragma unroll
    for (int w = 0; w < NWV; ++w) at += w < wave ? red[w] : 0;
    for (int i = from; i < min(to, rest0); ++i) list[at++] = i;
    ranked([&](uint32_t x, int i) {
        if (taken(x, i)) list[at++] = i;
    });
    for (int i = max(from, rest1); i < to; ++i) list[at++] = i;
}

int key_stride(const PageDims &d) { return (d.max_pages + 3) & ~3; }

template <bool BF16, int LP>
void (*scores_for(int G))(ScoreArgs)
{
    return G == 1 ? page_scores_kernel<BF16, LP, 1, false> : G == 2 ? page_scores_kernel<BF16, LP, 2, false>
         : G <= 4 ? page_scores_kernel<BF16, LP, 4, false> : page_scores_kernel<BF16, LP, 4, true>;
}

}  // namespace

size_t select_pages_ws_bytes(const PageDims &d) { return align256((size_t)d.P * key_stride(d) * 4); }

hipError_t launch_select_pages(const PageDims &d, const void *q, const PageView &pv, int32_t n_pick, int32_t n_first, int32_t n_last,
                               int32_t *list, void *ws, hipStream_t st)
{
    ScoreArgs a;
    a.d = d;
    a.pv = pv;
    a.q = static_cast<const char *>(q);
    a.stride = key_stride(d);
    a.keys = static_cast<uint32_t *>(ws);
    if (d.max_pages > n_pick) {                                // otherwise every list is whole
        const int pieces = d.D * elt_bytes(d) / 16;
        int lp = 1;
        while (lp < pieces) lp *= 2;
        const bool bf = d.dtype == SABLOCK_BF16;
        void (*fn)(ScoreArgs) = nullptr;
        // bf16 rows of up to 32 pieces, fp32 rows of 2 to 64: twice as many for the same heads
#define SABLOCK_SCORES(LV) if (bf && lp == LV) fn = scores_for<true, LV>(d.G); if (!bf && lp == 2 * LV) fn = scores_for<false, 2 * LV>(d.G);
        SABLOCK_SCORES(1) SABLOCK_SCORES(2) SABLOCK_SCORES(4) SABLOCK_SCORES(8) SABLOCK_SCORES(16) SABLOCK_SCORES(32)
#undef SABLOCK_SCORES
        if (!fn) return hipErrorInvalidValue;
        const int pages = NT / lp * flight_of(d.G > 4);                    // of a workgroup at a time
        const int parts = std::max(1, std::min((d.max_pages + pages - 1) / pages, (SCORE_WGS * d.cus + d.P - 1) / d.P));
        hipLaunchKernelGGL(fn, dim3(parts, d.P), dim3(NT), 0, st, a);
    }
    const int run = (d.max_pages + PICK_NT - 1) / PICK_NT;     // per thread
    const auto pick = run <= 4 ? pick_pages_kernel<4> : run <= 8 ? pick_pages_kernel<8> : run <= 16 ? pick_pages_kernel<16> : pick_pages_kernel<0>;
    hipLaunchKernelGGL(pick, dim3(d.P), dim3(PICK_NT), 0, st, d, pv, n_pick, n_first, n_last, a.keys, a.stride, list);
    return hipGetLastError();
}

}  // namespace sablock
