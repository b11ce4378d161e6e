// The pages that a decode step over a paged cache reads when it may not read all: a score per page from the bounds of its keys,
// then the best of them per KV head.
#include "sablock_internal.h"

namespace sablock {
namespace {

constexpr int NT = 256, PICK_NT = 1024;
constexpr uint32_t FORCED = 0xffffffffu, NOT_A_NUMBER = 0xfffffffeu;       // above every number's key

template <bool BF16> __device__ double element(const char *p, int64_t i)
{
    if constexpr (BF16) return (double)__uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << 16);
    else return (double)reinterpret_cast<const float *>(p)[i];
}

// grid (parts of a sequence's pages, problems): keys [P][max_pages], in the order of the scores.  max(q lo, q hi) is q+ hi + q- lo; the sum of
// products of bf16 values in fp64 is exact but for values some 2^30 apart, so its order does not depend on how it is formed.
template <bool BF16>
__global__ void __launch_bounds__(NT)
page_scores_kernel(PageDims d, PageView pv, const char *q, int n_first, int n_last, uint32_t *keys)
{
    const int p = blockIdx.y, s = seq_of_problem(d, p), layer = layer_of_problem(d, p), head = head_of_problem(d, p);
    const int i = blockIdx.x * NT + threadIdx.x, n = (rows_of(d, pv.lengths, s) + d.page - 1) >> d.shift;
    if (i >= n) return;
    const int id = page_at(d, pv.table, s, i);
    uint32_t key = ordered_key(-INFINITY);
    if (i < n_first || i >= n - n_last) key = FORCED;
    else if (id >= 0) {
        const int64_t b = (((int64_t)layer * d.n_pages + id) * d.Hkv + head) * 2 * d.D;
        double most = -INFINITY;
        bool number = true;
        for (int g = 0; g < d.G; ++g) {
            const int64_t qrow = (((int64_t)s * d.n_layers + layer) * d.Hq + head * d.G + g) * d.D;
            double x = 0.0;
            for (int c = 0; c < d.D; ++c) {
                const double v = element<BF16>(q, qrow + c);
                x = fma(fmax(v, 0.0), element<BF16>(pv.bounds, b + d.D + c), fma(fmin(v, 0.0), element<BF16>(pv.bounds, b + c), x));
            }
            number = number && x == x;
            most = fmax(most, x);
        }
        key = number ? ordered_key((float)most) : NOT_A_NUMBER;
    }
    keys[(int64_t)p * d.max_pages + i] = key;
}

// grid P: the n_pick largest keys of a problem, the lower page first where they are equal.  The n_pick-th largest key is found digit by
// digit (8 bits, counts in LDS); a thread then has a run of consecutive pages, and one prefix sum over the threads places theirs.
__global__ void __launch_bounds__(PICK_NT)
pick_pages_kernel(PageDims d, PageView pv, int n_pick, const uint32_t *keys_all, int32_t *list_all)
{
    __shared__ int hist[256], wave_gt[PICK_NT / 64], wave_eq[PICK_NT / 64];
    __shared__ uint32_t s_prefix;
    __shared__ int s_left;
    const int p = blockIdx.x, tid = threadIdx.x, n = (rows_of(d, pv.lengths, seq_of_problem(d, p)) + d.page - 1) >> d.shift;
    int32_t *list = list_all + (int64_t)p * n_pick;
    if (n <= n_pick) {
        for (int i = tid; i < n_pick; i += PICK_NT) list[i] = i < n ? i : -1;
        return;
    }
    const uint32_t *keys = keys_all + (int64_t)p * d.max_pages;
    uint32_t prefix = 0;
    int left = n_pick;                                         // of the pages whose upper digits are the prefix's
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += PICK_NT) {
            const uint32_t x = keys[i];
            if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(x >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid < 64) {                                        // lane l has the digits 255 - 4 l .. 252 - 4 l
            int c[4], sum = 0;
            for (int j = 0; j < 4; ++j) { c[j] = hist[255 - 4 * tid - j]; sum += c[j]; }
            int upto = sum;
            for (int o = 1; o < 64; o <<= 1) {
                const int u = __shfl_up(upto, o);
                if (tid >= o) upto += u;
            }
            int before = upto - sum;
            if (before < left && upto >= left)                 // one lane
                for (int j = 0; j < 4; ++j) {
                    if (before < left && before + c[j] >= left) {
                        s_prefix = prefix | (uint32_t)(255 - 4 * tid - j) << shift;
                        s_left = left - before;
                    }
                    before += c[j];
                }
        }
        __syncthreads();
        prefix = s_prefix;
        left = s_left;
    }
    const int run = (n + PICK_NT - 1) / PICK_NT, from = min(n, tid * run), to = min(n, from + run);
    int gt = 0, eq = 0;
    for (int i = from; i < to; ++i) { gt += keys[i] > prefix; eq += keys[i] == prefix; }
    int gt_upto = gt, eq_upto = eq;
    for (int o = 1; o < 64; o <<= 1) {
        const int a = __shfl_up(gt_upto, o), b = __shfl_up(eq_upto, o);
        if ((tid & 63) >= o) { gt_upto += a; eq_upto += b; }
    }
    if ((tid & 63) == 63) { wave_gt[tid >> 6] = gt_upto; wave_eq[tid >> 6] = eq_upto; }
    __syncthreads();
    int gt_before = gt_upto - gt, eq_before = eq_upto - eq;
    for (int w = 0; w < tid >> 6; ++w) { gt_before += wave_gt[w]; eq_before += wave_eq[w]; }
    for (int i = from; i < to; ++i) {
        const uint32_t x = keys[i];
        if (x > prefix || (x == prefix && eq_before < left)) list[gt_before + min(eq_before, left)] = i;
        gt_before += x > prefix;
        eq_before += x == prefix;
    }
}

}  // namespace

size_t select_pages_ws_bytes(const PageDims &d) { return align256((size_t)d.P * d.max_pages * 4); }

hipError_t launch_select_pages(const PageDims &d, const void *q, const PageView &pv, int32_t n_pick, int32_t n_first, int32_t n_last,
                               int32_t *list, void *ws, hipStream_t st)
{
    uint32_t *keys = static_cast<uint32_t *>(ws);
    if (d.max_pages > n_pick)                                  // otherwise every list is whole
        hipLaunchKernelGGL(d.dtype == SABLOCK_BF16 ? page_scores_kernel<true> : page_scores_kernel<false>, dim3((d.max_pages + NT - 1) / NT, d.P),
                           dim3(NT), 0, st, d, pv, static_cast<const char *>(q), n_first, n_last, keys);
    hipLaunchKernelGGL(pick_pages_kernel, dim3(d.P), dim3(PICK_NT), 0, st, d, pv, n_pick, keys, list);
    return hipGetLastError();
}

}  // namespace sablock
