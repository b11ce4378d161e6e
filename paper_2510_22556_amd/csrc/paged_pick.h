// The choice among the numbered things of a problem (pages, or rows) by whole numbers in the order of their scores: the first ones, the last ones and, of the
// others, those with the largest keys, the lower number first where keys are equal.  A workgroup of PICK_NT threads; the last key that is taken
// is found digit by digit, 11 bits of its distance from the least key at a time (the keys of a problem share their upper bits) until 64
// are left, which a wavefront ranks, and one prefix sum places what is taken in order.
#pragma once

#include "sablock_internal.h"

namespace sablock {
namespace {

constexpr int PICK_NT = 1024;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int M> __device__ __forceinline__ uint32_t xor_lane_u(uint32_t x) { return __float_as_uint(xor_lane<M>(__uint_as_float(x))); }
template <int M> __device__ __forceinline__ uint32_t most_of_lanes(uint32_t x)
{
    if constexpr (M < 64) return most_of_lanes<2 * M>(max(x, xor_lane_u<M>(x)));
    else return x;
}

constexpr int DIGIT = 11, BINS = 1 << DIGIT;
constexpr int FEW = 64;                        // keys that one wavefront ranks

struct PickShared {
    static constexpr int NWV = PICK_NT / 64;
    int hist[BINS], red[NWV], few_at[FEW], n_few;
    uint32_t extreme[2 * NWV], few_key[FEW];
    int found[3];                                              // bin, taken from it, its size; then the last key and place that are taken
};

// put(at, i): i is the at-th that is taken, of n_pick; n > n_pick.  A thread has RUN consecutive ones, whose keys are in `own`, or (RUN = 0) as many as it takes,
// read again in every pass from `keys`.
template <int RUN, typename Put>
__device__ __forceinline__ void pick(PickShared &sh, const uint32_t (&own)[RUN ? RUN : 1], const uint32_t *keys, int n, int n_pick, int n_first, int n_last, Put &&put)
{
    constexpr int NWV = PickShared::NWV;
    auto &hist = sh.hist;
    auto &red = sh.red;
    auto &few_at = sh.few_at;
    auto &n_few = sh.n_few;
    auto &extreme = sh.extreme;
    auto &few_key = sh.few_key;
    auto &found = sh.found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
    for (int i = from; i < min(to, rest0); ++i) put(at++, i);
    ranked([&](uint32_t x, int i) {
        if (taken(x, i)) put(at++, i);
    });
    for (int i = max(from, rest1); i < to; ++i) put(at++, i);
}

}  // namespace
}  // namespace sablock
