// New tokens into the paged cache with a norm per head in front of the rotation: every head of q and k over its root mean square,
//   y_d = x_d w_d / sqrt(mean(x^2) + eps),
// then rotated, in the kernel that appends without one (paged_append.h).  A row's pieces lie in consecutive lanes, which share the sum of its
// squares by lane exchange, a batch of rows' sums at a time.  x_d w_d is formed first, a pair's other one comes from its lane, and the row's factor is
// multiplied last, when it has long been there; rows whose squares pass fp32 are made zeros before that.  All in fp32, one rounding to the cache's type.
//
// What bounds it: the copy, and the vector instructions beside it, 190 per wavefront and row of 128 bf16 elements, a quarter of them the angles: half
// the time by themselves.  Prompts, 11 300 tokens x 48 heads (278 MB): 81.4 us, 3.4 TB/s (without a norm 67.5); pairs side by side, whose other elements need no
// exchange, 78.6.  bf16 runs three workgroups per compute unit (161 registers; four spill 13 of them, 85 us; two take 96), fp32 four (142 -> 133 us for the
// same prompts, 4.1 TB/s).  Batches of two rows 107 us; 5, 8 and 20 workgroups per compute unit to deal to 93, 84 and 87.  One token 4.6 us in a graph; 256
// sequences, a token each, 5.8.
#include "paged_append.h"

#include <cfloat>

namespace sablock {

hipError_t launch_append_normed_paged(const PageDims &pd, const TokenDims &td, const NormDims &nd, const void *q, const void *k, const void *v,
                                      const int32_t *counts, const int32_t *positions, const float *inv_freq, const PageView &pv, void *q_out, hipStream_t st)
{
    NormedAppendArgs a;
    bool one;
    const dim3 grid = plan_append(a, pd, td, q, k, v, counts, positions, inv_freq, pv, q_out, &one);
    a.q_weight = nd.q_weight;
    a.k_weight = nd.k_weight;
    a.q_layer = nd.per_head ? (int64_t)pd.Hq * pd.D : pd.D;
    a.k_layer = nd.per_head ? (int64_t)pd.Hkv * pd.D : pd.D;
    a.head = nd.per_head ? pd.D : 0;
    a.eps = std::max(nd.eps, FLT_MIN);                         // what the reciprocal root takes
    a.per_element = 1.f / (float)pd.D;
    return launch_append(a, grid, one, st);
}

}  // namespace sablock
