// The pages that a decode step over a paged cache reads when it may not read all: a score per page from the bounds of its keys,
// then the best of them per KV head.
//
//   page_scores_kernel   max(q lo, q hi) is q+ hi + q- lo with q+ = max(q, 0), q- = min(q, 0) (finite lo and hi): two products per element and head,
//       formed and summed in fp64, on the matrix pipe.  The products of two bf16 values and their sum over a head are exact there (but for
//       elements some 2^30 apart), so that which of two pages comes first does not hang on the order of a sum.  A matrix
//       instruction of four products 4 x 4 x 4 has four pages in its rows, four heads in its columns and, in its four inner places
//       and in the four products, different 16-byte pieces of a row of bounds, one element of each at a time: a lane's
//       operand is an element of the piece that it loaded.  The products' sums are joined over the lanes, each lane then
//       has one page and head, whose score it rounds to fp32 and turns into a whole number of the same order; the maximum over the heads is
//       one of whole numbers, in which what is no number can be the largest.
//       What bounds it: loads.  8 heads x 8 192 pages of 512 bytes of bounds, four query heads: 10.2 us (at best 9.6), of which 5.1 are the bytes at 6.6 TB/s;
//       as long without the products, the rest is the launch and the chain length, table, bounds.  Formed on the vector pipe, by fp64
//       instructions and sums over 16 lanes, 12.3 at best; with 16 query heads, picking and reading with it, 36.3 in place of 46.3.
//   pick_pages_kernel    a workgroup per problem; the keys stay in registers.  The last key that is taken is found digit by digit, 11 bits
//       of its distance from the least key at a time (the keys of a problem share their upper bits) until 64 are left, which a wavefront
//       ranks, and one prefix sum places the pages in order.  8 192 pages: 7.2 us, at best 5.6, a chain of seven barriers and the reads between
//       them (with lane sums through LDS and nine barriers 6.5 at best).
#include "sablock_internal.h"

namespace sablock {
namespace {

constexpr int NT = 256, PICK_NT = 1024;
// Workgroups of the scores per compute unit that the launch plans for, as many as run at a time (with two 64 x 8 heads x 2 048 pages, scored, picked
// and read, 209 us in place of 199).  Not so for more than eight query heads and rows of more than 256 bytes in bf16, 512 in fp32: the heads' elements
// take 64 KB of LDS there, two run at a time, and the third comes behind them.
constexpr int SCORE_WGS = 3;
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

struct ScoreArgs {
    PageDims d;
    PageView pv;
    const char *q;
    int stride;                  // of a problem's keys
    uint32_t *keys;
};

// How page_scores_kernel spreads its work: a row's pieces over LP lanes, NP per lane, and HS sets of four heads
template <bool BF16, int LP, int NP, int HS> struct Spread {
    static constexpr int E = Piece<BF16>::N, PAGES = 64 / LP;  // pages of a wavefront's matrix instruction
    static constexpr int FLIGHT = NP < 2 ? 2 : 1;              // of those at a time, while as many are on their way (4: 30.2 us for 28.9, 8: 32)
    static constexpr bool IN_LDS = HS * NP * E > 16;           // the heads' elements do not fit the registers
    static constexpr int WG_PAGES = NT / 64 * PAGES * FLIGHT;
};

// grid (problems, parts of a sequence's pages): the heads' bounds of a page lie side by side and are read at one time
template <bool BF16, int LP, int NP, int HS>
__global__ void __launch_bounds__(NT, SCORE_WGS)
page_scores_kernel(ScoreArgs a)
{
    using Pc = Piece<BF16>;
    using Sp = Spread<BF16, LP, NP, HS>;
    constexpr int E = Pc::N, ELT = 16 / E, FLIGHT = Sp::FLIGHT, BLOCKS = LP / 4;              // BLOCKS: of the four small products, with one page's pieces
    const PageDims &d = a.d;
    const int p = blockIdx.x, s = seq_of_problem(d, p), layer = layer_of_problem(d, p), head = head_of_problem(d, p);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // as operand: a page's or a head's number within four, block, place in the inner dimension; a result has the page in the place of the latter
    const int four = lane & 3, block = lane >> 2 & 3, inner = lane >> 4;
    const int c = block % BLOCKS + BLOCKS * inner, place = four + 4 * (block / BLOCKS), result_place = inner + 4 * (block / BLOCKS);
    const int n = (rows_of(d, a.pv.lengths, s) + d.page - 1) >> d.shift;
    const int64_t row = (int64_t)d.D * ELT;
    const bool padded = d.D < LP * NP * E;
    auto mine = [&](int j) { return (c + LP * j) * E < d.D; }; // lanes behind the row's end are padding
    const char *q = a.q + (((int64_t)s * d.n_layers + layer) * d.Hq + head * d.G) * row;
    const char *bounds = a.pv.bounds + ((int64_t)layer * d.n_pages * d.Hkv + head) * 2 * row;
    int at[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) at[j] = mine(j) ? (c + LP * j) * 16 : 0;
    struct Flight { int id[FLIGHT]; u32x4 lo[FLIGHT][NP], hi[FLIGHT][NP]; };
    // Nothing is loaded behind a branch (what does not exist is replaced by what does, and not used): the compiler could not count
    // the loads in flight there.
    auto load_ids = [&](int i0, int (&id)[FLIGHT]) {
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) id[u] = page_at(d, a.pv.table, s, min(i0 + u * Sp::PAGES + place, n - 1));
    };
    auto load_bounds = [&](Flight &f) {
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const char *b = bounds + (int64_t)max(f.id[u], 0) * d.Hkv * 2 * row;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                f.lo[u][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(b + at[j]));
                f.hi[u][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(b + row + at[j]));
            }
        }
    };
    // q+ and q- of the heads; those behind the last are the last again
    typedef double pair __attribute__((ext_vector_type(2)));
    auto load_heads = [&](int set, int j, auto &&put) {        // put(e, {q+, q-})
        u32x4 x{0, 0, 0, 0};
        if (mine(j)) x = *reinterpret_cast<const u32x4 *>(q + min(4 * set + four, d.G - 1) * row + (c + LP * j) * 16);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float v = Pc::value(x, e);
            put(e, pair{(double)(v < 0.f ? 0.f : v), (double)(v < 0.f ? v : 0.f)});            // what is no number stays one
        }
    };
    __shared__ pair q_sh[Sp::IN_LDS ? HS * NP * E * 64 : 1];   // [set][piece][element][lane]
    pair q_own[Sp::IN_LDS ? 1 : HS * NP * E];
    const int step = gridDim.y * Sp::WG_PAGES, start = (blockIdx.y * (NT / 64) + wave) * Sp::PAGES * FLIGHT;
    if ((int)(blockIdx.y * Sp::WG_PAGES) >= n) return;
    Flight now, next;
    load_ids(start, now.id);
    load_ids(start + step, next.id);
    load_bounds(now);
    if constexpr (Sp::IN_LDS) {
        for (int i = wave; i < HS * NP; i += NT / 64)
            load_heads(i / NP, i % NP, [&](int e, pair x) { q_sh[(i * E + e) * 64 + lane] = x; });
        __syncthreads();
    } else {
#pragma unroll
        for (int i = 0; i < HS * NP; ++i) load_heads(i / NP, i % NP, [&](int e, pair x) { q_own[i * E + e] = x; });
    }
    for (int i0 = start; i0 < n; i0 += step) {
        int later[FLIGHT];
        load_bounds(next);
        load_ids(i0 + 2 * step, later);
        if (padded) {
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (!mine(j)) {
#pragma unroll
                    for (int u = 0; u < FLIGHT; ++u) now.lo[u][j] = now.hi[u][j] = u32x4{0, 0, 0, 0};
                }
        }
        double x[FLIGHT][HS];
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u)
#pragma unroll
            for (int g = 0; g < HS; ++g) x[u][g] = 0.0;
#pragma unroll
        for (int j = 0; j < NP; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                double l[FLIGHT], h[FLIGHT];
                if constexpr (Sp::IN_LDS) asm volatile("" ::: "memory");                      // not read sooner: all of them do not fit
#pragma unroll
                for (int u = 0; u < FLIGHT; ++u) { l[u] = (double)Pc::value(now.lo[u][j], e); h[u] = (double)Pc::value(now.hi[u][j], e); }
#pragma unroll
                for (int g = 0; g < HS; ++g) {
                    const int i = (g * NP + j) * E + e;
                    const pair w = Sp::IN_LDS ? q_sh[i * 64 + lane] : q_own[Sp::IN_LDS ? 0 : i];
#pragma unroll
                    for (int u = 0; u < FLIGHT; ++u) x[u][g] = __builtin_amdgcn_mfma_f64_4x4x4f64(h[u], w[0], x[u][g], 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < FLIGHT; ++u) x[u][g] = __builtin_amdgcn_mfma_f64_4x4x4f64(l[u], w[1], x[u][g], 0, 0, 0);
                }
            }
        // read before any branch, see the products of the decode kernel
        uint32_t key[FLIGHT];
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            key[u] = 0;
#pragma unroll
            for (int g = 0; g < HS; ++g) {
                double y = x[u][g];
                if constexpr (BLOCKS >= 2) y += xor_lane_d<4>(y);
                if constexpr (BLOCKS >= 4) y += xor_lane_d<8>(y);
                key[u] = max(key[u], y == y ? ordered_key((float)y) : NOT_A_NUMBER);
            }
            key[u] = max(key[u], xor_lane_u<1>(key[u]));
            key[u] = max(key[u], xor_lane_u<2>(key[u]));
            const uint64_t none = __ballot(now.id[u] < 0) >> (inner + 4 * block);             // the result's page in the lanes of operands
            if (none & 1) key[u] = ordered_key(-INFINITY);
        }
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const int i = i0 + u * Sp::PAGES + result_place;
            if (four == 0 && block % BLOCKS == 0 && i < n) a.keys[(int64_t)p * a.stride + i] = key[u];
        }
        now = next;
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) next.id[u] = later[u];
    }
}

template <int M> __device__ __forceinline__ uint32_t most_of_lanes(uint32_t x)
{
    if constexpr (M < 64) return most_of_lanes<2 * M>(max(x, xor_lane_u<M>(x)));
    else return x;
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
    least = ~most_of_lanes<1>(~least);
    most = most_of_lanes<1>(most);
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
        const int upto = sum_upto_lane(h0 + h1);
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
        left = found[1];                                       // written again only behind a barrier
        inside = found[2];
        bits = shift;
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
            const int upto = sum_upto_lane(eq);
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
    }
    auto taken = [&](uint32_t x, int i) { return x > cut || (x == cut && i <= cut_at); };
    int count = max(0, min(to, rest0) - from) + max(0, to - max(from, rest1));
    ranked([&](uint32_t x, int i) { count += taken(x, i); });
    const int upto = sum_upto_lane(count);
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

struct Scores { void (*fn)(ScoreArgs); int pages; };           // pages: of a workgroup at a time

template <bool BF16, int LP, int NP> Scores scores_for(int G)
{
    if (G <= 4) return {page_scores_kernel<BF16, LP, NP, 1>, Spread<BF16, LP, NP, 1>::WG_PAGES};
    if (G <= 8) return {page_scores_kernel<BF16, LP, NP, 2>, Spread<BF16, LP, NP, 2>::WG_PAGES};
    return {page_scores_kernel<BF16, LP, NP, 4>, Spread<BF16, LP, NP, 4>::WG_PAGES};
}

template <bool BF16> Scores scores_for(int G, int pieces)
{
    if (pieces <= 4) return scores_for<BF16, 4, 1>(G);
    if (pieces <= 8) return scores_for<BF16, 8, 1>(G);
    if (pieces <= 16) return scores_for<BF16, 16, 1>(G);
    if constexpr (!BF16)                                       // no bf16 head has more than 32
        if (pieces > 32) return scores_for<BF16, 16, 4>(G);
    return scores_for<BF16, 16, 2>(G);
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
        const Scores f = d.dtype == SABLOCK_BF16 ? scores_for<true>(d.G, pieces) : scores_for<false>(d.G, pieces);
        const int parts = std::min({(d.max_pages + f.pages - 1) / f.pages, (SCORE_WGS * d.cus + d.P - 1) / d.P, (int)GRID_Y_MOST});
        hipLaunchKernelGGL(f.fn, dim3(d.P, parts), dim3(NT), 0, st, a);
    }
    const int run = (d.max_pages + PICK_NT - 1) / PICK_NT;     // per thread
    const auto pick = run <= 4 ? pick_pages_kernel<4> : run <= 8 ? pick_pages_kernel<8> : run <= 16 ? pick_pages_kernel<16> : pick_pages_kernel<0>;
    hipLaunchKernelGGL(pick, dim3(d.P), dim3(PICK_NT), 0, st, d, pv, n_pick, n_first, n_last, a.keys, a.stride, list);
    return hipGetLastError();
}

}  // namespace sablock
