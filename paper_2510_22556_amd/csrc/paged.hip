// The paged cache's writers (what they share is in paged_rows.h, the appending kernel in paged_append.h): the retained rows of a compression into
// pages (end of Sec. 3.3), and new tokens behind them with the position rotation of queries and keys on the way.  Both are copies, 16 bytes per lane, and both keep the page bounds: the
// least and the largest value of every element of K over a page's rows, taken on order-preserving whole numbers (a
// packed 16-bit minimum serves two bf16 elements) and joined over the rows of a workgroup through LDS.
//
// What bounds them: the copy.  A large device copy reaches 4.9-5.4 TB/s here, read and written (2 GB and 0.5 GB).  Compaction of 32 layers x 8 heads,
// 1 024 rows of 256 bytes each out of 32 768 (272 MB in and out): 61 us, 4.6 TB/s; several rows per thread in flight gain
// nothing over one and eight workgroups per compute unit (61.1, 60.2 us).  Appended prompts, 11 300 tokens x 48 heads (278 MB): 69 us,
// 4.0 TB/s, the rotation's vector instructions a third of that time beside it; without a rotation 68; fp32 130 us.  One token: 4.4 us in a graph, as
// good as one launch and three dependent loads; 256 sequences, a token each, 5.9 us.
#include "paged_append.h"

namespace sablock {
namespace {

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
    bool one;
    const dim3 grid = plan_append(a, pd, td, q, k, v, counts, positions, inv_freq, pv, q_out, &one);
    return launch_append(a, grid, one, st);
}

}  // namespace sablock
