// Decode attention that adds every row's share to what the row has gathered: w_r <- decay w_r + sum over the KV head's query heads of softmax_r.
//
// The attention is paged_decode.h's, whose lanes hold the logits.  A problem that one workgroup has alone is weighed by it as soon as its heads' references and
// denominators are known, 2^(logit - reference) / denominator, from the logits that its wavefronts keep in LDS.  Those that do not fit, and those
// of problems in pieces, go to the workspace, 4 bytes per row and query head, and the launch that joins the pieces has workgroups that weigh the rows.
//
// What bounds it: the attention's reads, and the writes among them, which cost far more than their bytes: 64 sequences of up to 8 192 rows, 8 heads of 128 bf16
// elements, four query heads each (1.07 GB read): the kernel takes 172 us without the logits' 34 MB, 228 with a store in every step, whatever its layout or
// cache policy, 224 with stores of eight steps at a time, 212-217 with as many logits in LDS as fit: 229 us in all, 18 of them the joining and weighing.  8 heads
// x 1 056 rows: 10.6 us in a graph, with a launch of its own for the weighing 14.3.
#include "paged_decode.h"

namespace sablock {
namespace {

struct WeighedArgs : DecodePagedArgs {
    float *logits;               // [P][stride][G], log2 domain, in the order of logit_place
    int64_t stride;              // rows
    float *gathered;             // [n_layers][n_pages][Hkv][page]
    const int32_t *counts;
    int n_new;
    float decay;
    static constexpr bool LOGITS = true;

    // rows r .. r + 3 of a problem, which lie in one page.  stats: reference and 1 / denominator of each head; logits(g): of these rows
    template <typename Logits>
    __device__ __forceinline__ void weigh(int s, int layer, int head, int r, int len, const f32x2 *stats, Logits &&logits_of) const
    {
        const int id = page_at(d, pv.table, s, r >> d.shift);
        // rows from here on have gathered nothing.  Not rows_of: new rows that the table has no room for are not the last ones that it has
        const int fresh = max(pv.lengths[s], 0) - (counts ? min(max(counts[s], 0), n_new) : n_new);
        if (id < 0) return;
        f32x4 *at = reinterpret_cast<f32x4 *>(gathered + weight_at(d, layer, id, head) + (r & (d.page - 1)));
        const f32x4 old = *at;
        f32x4 w{0.f, 0.f, 0.f, 0.f};
        for (int g = 0; g < d.G; ++g) {
            const f32x4 z = logits_of(g);
            const f32x2 x = stats[g];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = fmaf(__builtin_amdgcn_exp2f(z[i] - x[0]), x[1], w[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = r + i >= len ? old[i] : r + i >= fresh || decay == 0.f ? w[i] : fmaf(decay, old[i], w[i]);
        *at = w;
    }
};

constexpr int WEIGH_WGS = 8;                   // workgroups that weigh, per compute unit, at most

int64_t logits_stride(const PageDims &d) { return (((int64_t)d.max_pages << d.shift) + 31) & ~(int64_t)31; }
size_t logits_bytes(const PageDims &d) { return align256((size_t)d.P * d.G * logits_stride(d) * 4); }

}  // namespace

size_t decode_weighed_ws_bytes(const PageDims &d) { return decode_ws_bytes_of(d) + logits_bytes(d); }

hipError_t launch_decode_weighed(const PageDims &d, const void *q, const PageView &pv, const int32_t *counts, int32_t n_new, float decay, float *weights,
                                 float *out, void *ws, hipStream_t st)
{
    WeighedArgs a;
    a.logits = reinterpret_cast<float *>(static_cast<char *>(ws) + decode_ws_bytes_of(d));
    a.stride = logits_stride(d);
    a.gathered = weights;
    a.counts = counts;
    a.n_new = n_new;
    a.decay = decay;
    const int64_t most = (a.stride + 4 * MERGE_T - 1) / (4 * MERGE_T);
    return launch_decode_of(a, d, q, pv, nullptr, 0, out, ws, st, (int)std::min<int64_t>(most, (WEIGH_WGS * d.cus + d.P - 1) / d.P));
}

}  // namespace sablock
