// Decode attention that adds every row's share to what the row has gathered: w_r <- decay w_r + sum over the KV head's query heads of softmax_r.
//
// The attention is paged_decode.h's, whose lanes hold the logits; they go to the workspace, 4 bytes per row and query head, as do each
// head's reference and denominator once they are known.  A share is then 2^(logit - reference) / denominator.
#include "paged_decode.h"

namespace sablock {
namespace {

struct WeighedArgs : DecodePagedArgs {
    float *logits;               // [P][G][stride], log2 domain
    int64_t stride;
    float *stats;                // [P][G][2]: reference (log2 domain), 1 / denominator
    float *gathered;             // [n_layers][n_pages][Hkv][page]
    const int32_t *counts;
    int n_new;
    float decay;
    static constexpr bool STATS = true, LOGITS = true;
};

constexpr int WEIGH_ROWS = 4;                  // of a thread, in one page
constexpr int WEIGH_WGS = 8;                   // workgroups per compute unit, at most

// grid (parts, problems)
__global__ void __launch_bounds__(NT)
weigh_kernel(WeighedArgs a)
{
    const PageDims &d = a.d;
    const int p = blockIdx.y, s = seq_of_problem(d, p), layer = layer_of_problem(d, p), head = head_of_problem(d, p);
    const int len = rows_of(d, a.pv.lengths, s);
    const int fresh = len - (a.counts ? min(max(a.counts[s], 0), a.n_new) : a.n_new);          // rows from here on have gathered nothing
    const float *logits = a.logits + (int64_t)p * d.G * a.stride, *stats = a.stats + (int64_t)p * d.G * 2;
    const int64_t step = (int64_t)gridDim.x * NT * WEIGH_ROWS;
    for (int64_t r = ((int64_t)blockIdx.x * NT + threadIdx.x) * WEIGH_ROWS; r < len; r += step) {
        const int id = page_at(d, a.pv.table, s, (int)(r >> d.shift));
        if (id < 0) continue;
        f32x4 *at = reinterpret_cast<f32x4 *>(a.gathered + weight_at(d, layer, id, head) + (r & (d.page - 1)));
        f32x4 w{0.f, 0.f, 0.f, 0.f};
        const f32x4 old = *at;
        for (int g = 0; g < d.G; ++g) {
            const f32x4 z = *reinterpret_cast<const f32x4 *>(logits + g * a.stride + r);
            const float ref = stats[2 * g], over = stats[2 * g + 1];
#pragma unroll
            for (int i = 0; i < WEIGH_ROWS; ++i) w[i] = fmaf(__builtin_amdgcn_exp2f(z[i] - ref), over, w[i]);
        }
#pragma unroll
        for (int i = 0; i < WEIGH_ROWS; ++i)
            w[i] = r + i >= len ? old[i] : r + i >= fresh || a.decay == 0.f ? w[i] : fmaf(a.decay, old[i], w[i]);
        *at = w;
    }
}

int64_t logits_stride(const PageDims &d) { return (((int64_t)d.max_pages << d.shift) + 31) & ~(int64_t)31; }
size_t logits_bytes(const PageDims &d) { return align256((size_t)d.P * d.G * logits_stride(d) * 4); }
size_t stats_bytes(const PageDims &d) { return align256((size_t)d.P * d.G * 8); }

}  // namespace

size_t decode_weighed_ws_bytes(const PageDims &d) { return decode_ws_bytes_of(d) + stats_bytes(d) + logits_bytes(d); }

hipError_t launch_decode_weighed(const PageDims &d, const void *q, const PageView &pv, const int32_t *counts, int32_t n_new, float decay, float *weights,
                                 float *out, void *ws, hipStream_t st)
{
    WeighedArgs a;
    char *at = static_cast<char *>(ws) + decode_ws_bytes_of(d);
    a.stats = reinterpret_cast<float *>(at);
    a.logits = reinterpret_cast<float *>(at + stats_bytes(d));
    a.stride = logits_stride(d);
    a.gathered = weights;
    a.counts = counts;
    a.n_new = n_new;
    a.decay = decay;
    const hipError_t done = launch_decode_of(a, d, q, pv, nullptr, 0, out, ws, st);
    if (done != hipSuccess) return done;
    const int64_t most = (a.stride + NT * WEIGH_ROWS - 1) / (NT * WEIGH_ROWS), parts = std::min<int64_t>(most, (WEIGH_WGS * d.cus + d.P - 1) / d.P);
    hipLaunchKernelGGL(weigh_kernel, dim3((unsigned)parts, d.P), dim3(NT), 0, st, a);
    return hipGetLastError();
}

}  // namespace sablock
