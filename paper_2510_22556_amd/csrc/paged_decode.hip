// Decode-time attention of one new token per sequence over a paged cache (Sec. 2.1 Eq. 1 for a single query position), over all
// of a sequence's pages or over listed ones.
#include "sablock_internal.h"

namespace sablock {
namespace {

constexpr int NT = 256;

template <bool BF16> __device__ float element(const char *p, int64_t i)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << 16);
    else return reinterpret_cast<const float *>(p)[i];
}

// grid (query heads of a KV head, problems): 256 rows at a time, one per thread for the logits, one column per thread for the
// weighted sum
template <bool BF16>
__global__ void __launch_bounds__(NT)
decode_paged_kernel(PageDims d, PageView pv, const char *q, const int32_t *list, int n_listed, float qscale, float *out)
{
    __shared__ float qs[256], w[NT], red[NT / 64];
    __shared__ int64_t place[NT];
    const int p = blockIdx.y, s = seq_of_problem(d, p), layer = layer_of_problem(d, p), head = head_of_problem(d, p), tid = threadIdx.x;
    const int64_t qrow = (((int64_t)s * d.n_layers + layer) * d.Hq + head * d.G + blockIdx.x) * d.D;
    if (tid < d.D) qs[tid] = element<BF16>(q, qrow + tid) * qscale;
    const int len = rows_of(d, pv.lengths, s), pages = (len + d.page - 1) >> d.shift;
    const int total = list ? min(n_listed, pages) << d.shift : len;
    float m = -INFINITY, z = 0.f, acc = 0.f;
    for (int r0 = 0; r0 < total; r0 += NT) {
        const int r = r0 + tid;
        int at = -1;                                           // page of the sequence
        if (r < total) at = list ? list[(int64_t)p * n_listed + (r >> d.shift)] : r >> d.shift;
        int id = -1;
        if (at >= 0 && at < pages && (at << d.shift) + (r & (d.page - 1)) < len) id = page_at(d, pv.table, s, at);
        __syncthreads();
        place[tid] = id < 0 ? -1 : layer * d.vs[0] + id * d.vs[1] + head * d.vs[2] + (r & (d.page - 1)) * d.vs[3];
        float x = -INFINITY;
        if (id >= 0) {
            const int64_t k = layer * d.ks[0] + id * d.ks[1] + head * d.ks[2] + (r & (d.page - 1)) * d.ks[3];
            x = 0.f;
            for (int c = 0; c < d.D; ++c) x = fmaf(qs[c], element<BF16>(pv.k, k + c), x);
        }
        float mx = x;
        for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
        if ((tid & 63) == 0) red[tid >> 6] = mx;
        __syncthreads();
        for (int i = 0; i < NT / 64; ++i) mx = fmaxf(mx, red[i]);
        mx = fmaxf(mx, m);
        const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - mx) : 0.f;
        w[tid] = x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x - mx);
        m = mx;
        __syncthreads();
        z *= f;
        acc *= f;
        const int n = min(NT, total - r0);
        for (int i = 0; i < n; ++i) {
            if (place[i] < 0) continue;
            z += w[i];
            if (tid < d.D) acc = fmaf(w[i], element<BF16>(pv.v, place[i] + tid), acc);
        }
    }
    if (tid < d.D) out[qrow + tid] = z == 0.f ? 0.f : acc / z;
}

}  // namespace

bool decode_paged_supported(const PageDims &d) { return d.G <= 16 && d.D % (d.dtype == SABLOCK_F32 ? 16 : 32) == 0; }

size_t decode_paged_ws_bytes(const PageDims &) { return 256; }

hipError_t launch_decode_paged(const PageDims &d, const void *q, const PageView &pv, const int32_t *list, int32_t n_listed, float *out,
                               void *, hipStream_t st)
{
    const float qscale = (float)(1.4426950408889634 / sqrt((double)d.D));
    hipLaunchKernelGGL(d.dtype == SABLOCK_BF16 ? decode_paged_kernel<true> : decode_paged_kernel<false>, dim3(d.G, d.P), dim3(NT), 0, st, d, pv,
                       static_cast<const char *>(q), list, n_listed, qscale, out);
    return hipGetLastError();
}

}  // namespace sablock
