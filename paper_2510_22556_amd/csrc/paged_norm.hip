// New tokens into the paged cache with a norm per head in front of the rotation: every head of q and k over its root mean square,
//   y_d = x_d w_d / sqrt(mean(x^2) + eps),
// then rotated, in the kernel that appends without one (paged_append.h).  A row's pieces lie in consecutive lanes, which share the sum of its
// squares by lane exchange.  A pair's other element is exchanged as it came, 16 bits of it in bf16 caches, and weighted by the lane that needs it:
// a lane has the weights of both of its pairs' elements in registers, read again (from the L1 cache) with every batch of rows, so that they wait for
// nothing.  All in fp32, one rounding to the cache's type.
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
