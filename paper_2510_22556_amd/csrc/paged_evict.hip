// Eviction from the paged cache: of every problem the rows that have gathered the most weight, with the first and the last ones, into the pages of
// another table, in their order.
//
//   pick_rows_kernel   the choice, by a workgroup per problem: a key per row in registers, out of the problem's pages.  Tables with room for up to 16 384 rows.
//   row_keys_kernel, pick_pages_kernel (paged_select.hip)   the same for larger tables: the weights of a problem's rows as whole numbers of the same order, side
//       by side, and the choice among those.
//   evict_kernel       a workgroup fills one page of one problem: K, V and weights of its rows, and the page's bounds.  The rows' places are found
//       once, by a thread each, and wait in LDS: list, table and row are loads that depend on each other.
//
// What bounds it: the copy.  32 layers x 8 heads of 4 sequences of up to 4 352 rows cut to 2 048 (1.75 GB moved and weighed): 377 us, 4.65 TB/s, where a copy
// of as much reaches 5.2; 358 of them the rows', 16.6 the choice.  A layer, 8 heads x 1 184 rows to 1 056: 11.0 us in a graph, two chains of dependent loads (6.8 and 5.1).
// The choice in three launches took 3 us more there; choice and rows in one kernel 14.7 and 395 us.  Larger tables, the choice still one workgroup per problem,
// which reads its keys again in every pass: 8 heads of 41 523 rows 41 us, of 131 072 97;
// one launch with up to 64 keys per thread 44 us for the first, 83 in place of 97 for 256 heads of 65 536 (37 registers spilled): not taken.
#include "paged_pick.h"
#include "paged_rows.h"

namespace sablock {
namespace {

constexpr int KEY_ROWS = 4;                    // of a thread, in one page
constexpr int KEY_WGS = 8;                     // workgroups of the keys per compute unit, at most

constexpr uint32_t NO_ROW = 0;                 // the key of a row whose page does not exist: below every number's, -infinity among them

__device__ __forceinline__ uint32_t row_key(float w) { return w == w ? ordered_key(w) : NOT_A_NUMBER; }

// grid (parts, problems)
__global__ void __launch_bounds__(NT)
row_keys_kernel(PageDims d, PageView pv, const float *weights, uint32_t *keys, int64_t stride)
{
    const int p = blockIdx.y, s = seq_of_problem(d, p), layer = layer_of_problem(d, p), head = head_of_problem(d, p);
    const int n = rows_of(d, pv.lengths, s);
    const int64_t step = (int64_t)gridDim.x * NT * KEY_ROWS;
    for (int64_t r = ((int64_t)blockIdx.x * NT + threadIdx.x) * KEY_ROWS; r < n; r += step) {
        const int id = page_at(d, pv.table, s, (int)(r >> d.shift));
        u32x4 key{NO_ROW, NO_ROW, NO_ROW, NO_ROW};
        if (id >= 0) {
            const f32x4 w = *reinterpret_cast<const f32x4 *>(weights + weight_at(d, layer, id, head) + (r & (d.page - 1)));
#pragma unroll
            for (int i = 0; i < KEY_ROWS; ++i) key[i] = row_key(w[i]);
        }
        *reinterpret_cast<u32x4 *>(keys + (int64_t)p * stride + r) = key;
    }
}

// grid (pages of the rows that stay, problems).  Where a sequence keeps all its rows in the pages that they lie in, every thread writes what it has read from there
// (not to do so costs the others' workgroups 2 %, 377 -> 383 us: they wait for the old page's number)
template <bool BF16>
__global__ void __launch_bounds__(NT)
evict_kernel(PageDims d, PageView pv, EvictDims ed, int chunks)
{
    using E = Elem<BF16>;
    __shared__ __attribute__((aligned(16))) uint32_t sh[NT * 8];
    __shared__ int2 from[NT];                                  // page, row in it
    const int p = blockIdx.y, s = seq_of_problem(d, p), layer = layer_of_problem(d, p), head = head_of_problem(d, p), tid = threadIdx.x;
    const int len = rows_of(d, pv.lengths, s), kept = min(len, ed.n_keep);
    if (blockIdx.x == 0 && layer == 0 && head == 0 && tid == 0) ed.lengths_out[s] = kept;
    const int r0 = blockIdx.x << d.shift, n = min(d.page, kept - r0);
    if (n <= 0) return;
    const int id = page_at(d, ed.table_out, s, blockIdx.x);
    if (id < 0) return;
    if (tid < n) {
        const int t = ed.rows_out[(int64_t)p * ed.n_keep + r0 + tid], at = t & (d.page - 1);
        const int source = page_at(d, pv.table, s, t >> d.shift);
        from[tid] = make_int2(source, at);
        ed.weights[weight_at(d, layer, id, head) + tid] = source < 0 ? 0.f : ed.weights[weight_at(d, layer, source, head) + at];
    }
    __syncthreads();
    const int groups = NT / chunks, group = tid / chunks, c = tid - group * chunks;
    const bool active = group < groups;
    const char *ksrc = pv.k + (layer * d.ks[0] + head * d.ks[2]) * E::BYTES + (int64_t)c * 16, *vsrc = pv.v + (layer * d.vs[0] + head * d.vs[2]) * E::BYTES + (int64_t)c * 16;
    char *kdst = pv.k + (layer * d.ks[0] + id * d.ks[1] + head * d.ks[2]) * E::BYTES + (int64_t)c * 16;
    char *vdst = pv.v + (layer * d.vs[0] + id * d.vs[1] + head * d.vs[2]) * E::BYTES + (int64_t)c * 16;
    Bounds<BF16> b;
    b.clear();
    if (active)
        for (int r = group; r < n; r += groups) {
            const int2 f = from[r];
            u32x4 x{0, 0, 0, 0}, y{0, 0, 0, 0};
            if (f.x >= 0) {
                x = *reinterpret_cast<const u32x4 *>(ksrc + (f.x * d.ks[1] + f.y * d.ks[3]) * E::BYTES);
                y = *reinterpret_cast<const u32x4 *>(vsrc + (f.x * d.vs[1] + f.y * d.vs[3]) * E::BYTES);
            }
            *reinterpret_cast<u32x4 *>(kdst + r * d.ks[3] * E::BYTES) = x;
            *reinterpret_cast<u32x4 *>(vdst + r * d.vs[3] * E::BYTES) = y;
            b.add(x);
        }
    if (!pv.bounds) return;
    char *at = bounds_at(d, pv, layer, id, head);
    store_joined<BF16>(b, sh, groups, chunks, group, c, active, d.D * E::BYTES, false, [&](int place) { return at + place * 16; });
}

// grid P
template <int RUN>
__global__ void __launch_bounds__(PICK_NT)
pick_rows_kernel(PageDims d, PageView pv, EvictDims ed)
{
    __shared__ PickShared sh;
    const int p = blockIdx.x, s = seq_of_problem(d, p), layer = layer_of_problem(d, p), head = head_of_problem(d, p), tid = threadIdx.x;
    const int capacity = d.max_pages << d.shift;
    uint32_t own[RUN];
#pragma unroll
    for (int j = 0; j < RUN; j += KEY_ROWS) {                  // before the length is known: whatever lies behind it is not looked at
        const int r = min(tid * RUN + j, capacity - KEY_ROWS), id = page_at(d, pv.table, s, r >> d.shift);
        const f32x4 w = *reinterpret_cast<const f32x4 *>(ed.weights + weight_at(d, layer, max(id, 0), head) + (r & (d.page - 1)));
#pragma unroll
        for (int i = 0; i < KEY_ROWS; ++i) own[j + i] = id < 0 ? NO_ROW : row_key(w[i]);
    }
    const int n = rows_of(d, pv.lengths, s);
    int32_t *list = ed.rows_out + (int64_t)p * ed.n_keep;
    if (n <= ed.n_keep) {
        for (uint32_t i = tid; i < (uint32_t)ed.n_keep; i += PICK_NT) list[i] = (int)i < n ? (int)i : -1;
        return;
    }
    pick<RUN>(sh, own, nullptr, n, ed.n_keep, ed.n_first, ed.n_last, [&](int at, int i) __attribute__((always_inline)) { list[at] = i; });
}

int64_t row_stride(const PageDims &d) { return (int64_t)d.max_pages << d.shift; }

}  // namespace

size_t evict_ws_bytes(const PageDims &d) { return align256((size_t)d.P * row_stride(d) * 4); }

hipError_t launch_evict(const PageDims &d, const PageView &pv, const EvictDims &ed, void *ws, hipStream_t st)
{
    const int64_t rows = row_stride(d), pages = evict_pages(d, ed.n_keep), run = (rows + PICK_NT - 1) / PICK_NT;
    const int chunks = d.D * elt_bytes(d) / 16;
    if (run <= 16) {                                           // keys per thread
        hipLaunchKernelGGL(run <= 4 ? pick_rows_kernel<4> : run <= 8 ? pick_rows_kernel<8> : pick_rows_kernel<16>, dim3(d.P), dim3(PICK_NT), 0, st, d, pv, ed);
    } else {
        uint32_t *keys = static_cast<uint32_t *>(ws);
        if (rows > ed.n_keep) {                                // otherwise every row stays
            const int64_t most = (rows + NT * KEY_ROWS - 1) / (NT * KEY_ROWS), parts = std::min<int64_t>(most, (KEY_WGS * d.cus + d.P - 1) / d.P);
            hipLaunchKernelGGL(row_keys_kernel, dim3((unsigned)parts, d.P), dim3(NT), 0, st, d, pv, ed.weights, keys, rows);
        }
        PageDims as_rows = d;                                  // pages of one row
        as_rows.page = 1;
        as_rows.shift = 0;
        as_rows.max_pages = (int32_t)rows;
        const hipError_t picked = launch_pick(as_rows, pv, ed.n_keep, ed.n_first, ed.n_last, keys, (int32_t)rows, ed.rows_out, st);
        if (picked != hipSuccess) return picked;
    }
    hipLaunchKernelGGL(d.dtype == SABLOCK_BF16 ? evict_kernel<true> : evict_kernel<false>, dim3((unsigned)pages, d.P), dim3(NT), 0, st, d, pv, ed, chunks);
    return hipGetLastError();
}

}  // namespace sablock
