// Decode-time attention of one new token per sequence over a paged cache (Sec. 2.1 Eq. 1 for a single query position), over all
// of a sequence's pages or over listed ones.
//
//   decode_paged_kernel   Work is counted in steps of 32 or 16 rows.  A short problem (a sequence's KV head in a layer) is one
//       workgroup's, which finishes it; the first n_seq * n_layers * Hkv workgroups see to those, and write zeros where there is no row.  The
//       steps of the long ones are dealt out in even runs to as many workgroups as reside at a time (see Places): the lengths,
//       which only the device knows, do not matter.  A run is a piece of one problem, or pieces of several; a problem inside
//       one run is finished there, of another's piece (reference, denominator, numerators) go to the workspace, at most two
//       per workgroup.
//   decode_paged_merge_kernel   joins the pieces of each problem.  Not launched where no sequence has room to be long.
//
// A wavefront does a step alone, on matrix instructions of 16 x 16 whose 16 columns are the query heads of the KV head (G <= 16,
// the rest zeros): S^T = K Q^T, then out^T += V^T P^T.  Both products take K and V as they lie in memory, without LDS:
//   - K as A operand has a row per lane (lane & 15) and consecutive elements in it: 16-byte loads, four lanes per row.  The order in
//     which the inner dimension is summed is free, so it is that of the loads.
//   - The result has a head per lane and four rows in it, which is how P^T as B operand wants its inner dimension, the rows; bf16
//     takes eight rows there: the A rows of two products are dealt out so that a lane's results are rows 8 (lane >> 4) + 0 .. 7.
//   - V^T as A operand wants an element of V per lane and those rows in it.  A lane loads D / 16 consecutive elements of each of its
//     rows, 16 lanes a whole row; element e of the lanes is the e-th product's operand, fp32 as it is, bf16 after one
//     v_perm_b32 for two rows.  Product e then gives the elements D / 16 (lane & 15) + e.
// Everything about a head, logits, reference, denominator and numerators, is in the lanes of its column: no exchange but a
// maximum over four lanes where a reference moves.  References are set AHEAD (log2 domain) above the largest logit so far and move when
// a logit passes them.  bf16 probabilities enter the second product in three parts of 8 bits (each part but the first 2^-28 of the
// whole too large, so that none is zero): the result is as good as in fp32 (rounded to bf16 they would be off by
// 2^-9), and the matrix pipe has the time.
//
// What bounds it: HBM.  4 x 8 heads x 131 072 rows of 128 bf16 elements (2.15 GB, four query heads or eight): 325-340 us, 6.3-6.6 TB/s,
// what the dense cache's kernel reaches over the same rows (330 us); every byte fetched once; the matrix pipe is busy 8 % of
// the time, the vector pipe 14 %.  Few rows: the chain of dependent loads (length, table, rows), and that of the second kernel, 9.85 us
// in all (8 heads x 1 056 rows); what does not depend on the rows is kept short, the code too, which comes cold from memory (with
// the dealing in 64 bits 0.5 more).  A wavefront holds one step's K and one step's V in flight, the next one's as soon as the products
// have taken their operands; a third workgroup per compute unit, spilling, was slower (375 us), ordinary loads in place of non-temporal ones
// as well (378).
#include "sablock_internal.h"

#include <cfloat>
#include <type_traits>

namespace sablock {
namespace {

constexpr int NW = 4, NT = NW * 64;
constexpr float AHEAD = 8.f;
constexpr float PART_LEAST = 0x1p-28f;         // a part of a probability that would be zero times an infinite value would be no number
constexpr int SPARE = 4;
constexpr int LEAST_STEPS = 4;                 // of a workgroup's run: one per wavefront

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
template <int N> struct Words;                 // N dwords of a row that begin on any dword
template <> struct Words<1> { typedef uint32_t T __attribute__((aligned(4))); };
template <> struct Words<2> { typedef uint32_t T __attribute__((ext_vector_type(2), aligned(4))); };
template <> struct Words<3> { typedef uint32_t T __attribute__((ext_vector_type(3), aligned(4))); };
template <> struct Words<4> { typedef uint32_t T __attribute__((ext_vector_type(4), aligned(4))); };

// N dwords from p into w; what is read once is non-temporal
template <int N>
__device__ __forceinline__ void load_words(uint32_t *w, const char *p)
{
    if constexpr (N > 4) {
        load_words<4>(w, p);
        load_words<N - 4>(w + 4, p + 16);
    } else if constexpr (N == 1) {
        w[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(p));
    } else {
        const auto v = __builtin_nontemporal_load(reinterpret_cast<const typename Words<N>::T *>(p));
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = v[i];
    }
}

// Rows of a step.  bf16 takes 32, but 16 of rows of more than 256 bytes, so that what is in flight leaves room for a second workgroup on
// the compute unit (heads of 256, 4 x 65 536 rows: 399 -> 382 us), and 16 of rows of more than 128 bytes where every problem is one
// workgroup's: a third one fits, and there the latencies of many short ones count (heads of 128: 1 024 problems of up to
// 256 rows 23.7 -> 20.6 us, 64 of 512 rows 12.3 -> 11.0; heads of 64, 64 problems of 512 rows: 7.3 -> 8.3; shared, 4 x 131 072 rows: 345 -> 349).
constexpr int step_rows(bool bf16, int D, bool alone) { return bf16 && D <= 128 && !(alone && D > 64) ? 32 : 16; }

struct DecodePagedArgs {
    PageDims d;
    PageView pv;
    const char *q;
    const int32_t *list;
    int n_listed;
    float qscale;                // log2(e) / sqrt(D)
    int workgroups;              // that share the long problems' steps
    int limit;                   // steps of the longest problem that a workgroup takes alone
    float *out;                  // [n_seq][n_layers][Hq][D]
    float *weights;              // pieces [2 * workgroups][G][2]: reference (log2 domain), denominator
    float *sums;                 // pieces [2 * workgroups][G][D]
};

// steps of a problem of sequence s
template <int STEP>
__device__ __forceinline__ int steps_of(const DecodePagedArgs &a, int s)
{
    const int len = rows_of(a.d, a.pv.lengths, s);
    int rows = len;
    if (a.list) {
        const int pages = (len + a.d.page - 1) >> a.d.shift;
        rows = min(a.n_listed, pages) << a.d.shift;
    }
    return (rows + STEP - 1) / STEP;
}
// the same of a problem whose steps are shared, 0 of one that is not
template <int STEP>
__device__ __forceinline__ int shared_steps_of(const DecodePagedArgs &a, int s)
{
    const int n = steps_of<STEP>(a, s);
    return n > a.limit ? n : 0;
}

// a number that is the same in all lanes, for the scalar registers: what comes from memory or another lane is not known to be
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// the value of one lane, the same one for all
__device__ __forceinline__ int of_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ int quotient(int x, int n) { return (int)((uint32_t)x / (uint32_t)n); }            // neither negative

// How the long problems' steps are dealt out: in runs that are cut at the problems' ends, one per workgroup, where the workgroups are
// enough for them, or would be with runs of up to SPARE steps more; else in equal runs of the steps of all, one problem's behind the other's,
// so that a workgroup may have pieces of several problems (a piece's chain of loads costs it as much as SPARE steps: 8 heads x 700 rows
// 12.7 us in even runs, 10.7 cut at the ends; x 4 001 14.1 and 12.5).  A
// wavefront's view: each lane has the sums up to its share of the sequences.  All problems' steps fit 32 bits (the launch sees to it).
template <int STEP>
struct Places {
    const DecodePagedArgs &a;
    int lane, share, heads;                    // sequences per lane, problems per sequence
    int steps;                                 // of the lane's sequence, where it has one
    bool whole;                                // a piece per workgroup
    int run;                                   // steps of a workgroup, at most
    int upto, total;                           // units (pieces, or steps) of one problem of each sequence up to the lane's last, of all problems
    __device__ Places(const DecodePagedArgs &args, int l) : a(args), lane(l) {}
    __device__ int units_of(int steps) const { return whole ? quotient(steps + run - 1, run) : steps; }
    __device__ int last() const { return a.d.n_seq > 1 ? of_lane(upto, 63) : upto; }
    __device__ void deal()
    {
        heads = a.d.n_layers * a.d.Hkv;
        share = (a.d.n_seq + 63) / 64;
        int longs = 0;
        steps = 0;
        if (a.d.n_seq == 1) {
            upto = steps = uniform(shared_steps_of<STEP>(a, 0));
            longs = steps > 0;
        } else {
#pragma unroll 4
            for (int i = 0; i < share; ++i) {                  // loads without a branch, several at a time
                const int s = lane * share + i, n = shared_steps_of<STEP>(a, min(s, a.d.n_seq - 1));
                steps += s < a.d.n_seq ? n : 0;
                longs += s < a.d.n_seq && n > 0;
            }
            upto = sum_upto_lane(steps);
            longs = of_lane(sum_upto_lane(longs), 63);
        }
        total = last() * heads;
        const int evenly = upto, all = total, problems = longs * heads;
        run = max(LEAST_STEPS, quotient(total + a.workgroups - 1, a.workgroups));
        const int even = run;
        if (cut()) return;
        if (problems < a.workgroups) {                         // a piece more of each problem, and the workgroups are enough
            run = max(run, quotient(all + a.workgroups - problems - 1, a.workgroups - problems));
            if (run <= even + SPARE && cut()) return;
        }
        whole = false;
        run = even;
        upto = evenly;
        total = all;
    }
    // units are pieces of up to `run` steps, if there are no more than workgroups
    __device__ bool cut()
    {
        whole = true;
        int own = 0;
        if (share == 1) own = units_of(steps);
        else
            for (int i = 0; i < share; ++i)
                if (lane * share + i < a.d.n_seq) own += units_of(shared_steps_of<STEP>(a, lane * share + i));
        upto = a.d.n_seq > 1 ? sum_upto_lane(own) : own;
        total = last() * heads;
        return total <= a.workgroups;
    }
    // the sequence that unit x of all lies in (x < total), the units of one problem of those before it, and the units and steps of its own
    __device__ void find(int x, int &seq, int &before, int &units, int &n) const
    {
        if (a.d.n_seq == 1) { seq = 0; before = 0; units = upto; n = steps; return; }
        const int first = uniform(__ffsll((unsigned long long)__ballot(upto * heads > x)) - 1), at = first > 0 ? of_lane(upto, first - 1) : 0;
        if (share == 1) {
            seq = first;
            before = at;
            units = of_lane(upto, first) - at;
            n = of_lane(steps, first);
            return;
        }
        const int s = first * share + lane, own_steps = lane < share && s < a.d.n_seq ? shared_steps_of<STEP>(a, s) : 0;
        const int own = units_of(own_steps), inner = sum_upto_lane(own) + at, j = uniform(__ffsll((unsigned long long)__ballot(inner * heads > x)) - 1);
        seq = first * share + j;
        units = of_lane(own, j);
        n = of_lane(own_steps, j);
        before = of_lane(inner, j) - units;
    }
    // units of one problem of the sequences before the given one
    __device__ int before(int seq) const
    {
        const int first = uniform(quotient(seq, share));
        int sum = first > 0 ? of_lane(upto, first - 1) : 0;
        for (int s = first * share; s < seq; ++s) sum += units_of(shared_steps_of<STEP>(a, s));
        return sum;
    }
};

__device__ __forceinline__ float over_quarters(float x, bool take_max)        // lanes l, l ^ 16, l ^ 32, l ^ 48
{
    float y = __shfl_xor(x, 16);
    x = take_max ? fmaxf(x, y) : x + y;
    y = __shfl_xor(x, 32);
    return take_max ? fmaxf(x, y) : x + y;
}

// EP: elements of a row per lane in the second product, D / 16.  SHARED: some problems may be long; else there is nothing but a workgroup per
// problem (whose registers let a third one reside, heads of 128).
template <bool BF16, int EP, int STEP, bool SHARED>
__global__ void __launch_bounds__(NT)
decode_paged_kernel(DecodePagedArgs a)
{
    constexpr int D = EP * 16, ELT = BF16 ? 2 : 4, R = STEP / 4;            // R: rows per lane in the second product
    constexpr int KT = STEP / 16;                              // products of 16 rows per step
    constexpr int KC = D * ELT / 64;                           // 16-byte pieces of a row per lane in the first product
    constexpr int VW = EP * ELT / 4;                           // dwords of a row per lane in the second
    constexpr int KEEP = D / 4 + 2;                            // registers of a lane that wavefronts join
    __shared__ float sh[(NW - 1) * KEEP * 64];
    const PageDims &d = a.d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, c = lane >> 4;
    // a lane's rows of a step: of K as operand (bf16: and that row + 4), of the results and of V from `row` on
    const int krow = KT == 2 ? (m >> 2) * 8 + (m & 3) : m, row = R * c;
    const int64_t kstep = d.ks[3] * ELT, vstep = d.vs[3] * ELT;

    // a piece: steps off .. off + count of the n of problem p
    auto piece = [&](int p, int s, int off, int count, int n) __attribute__((always_inline)) {
        const int layer = layer_of_problem(d, p), head = head_of_problem(d, p);
        // not made uniform: with the length in a scalar register the compiler's order of the loop is 2 % slower
        const int len = rows_of(d, a.pv.lengths, s), pages = (len + d.page - 1) >> d.shift;
        const int entries = a.list ? min(a.n_listed, pages) : pages;
        const int64_t qrow = (((int64_t)s * d.n_layers + layer) * d.Hq + head * d.G) * D;

        u32x4 q[KC];
#pragma unroll
        for (int j = 0; j < KC; ++j)
            q[j] = m < d.G ? *reinterpret_cast<const u32x4 *>(a.q + (qrow + m * D) * ELT + j * 64 + c * 16) : u32x4{0, 0, 0, 0};
        float ref = -FLT_MAX, den = 0.f;
        f32x4 acc[EP];
#pragma unroll
        for (int e = 0; e < EP; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};

        const int from = off + (int)((int64_t)count * wave / NW), to = off + (int)((int64_t)count * (wave + 1) / NW);
        // the page and the rows of it that count, of 64 entries at a time, one per lane
        int ids = 0, held = 0, base = -1 << 30;
        const char *kat = nullptr, *vat = nullptr;
        int limit = 0;                                         // of this lane's rows of the step, so many count (from the first on)
        bool whole = false;                                    // all rows of the step count
        auto locate = [&](int st) {
            const int r0 = st * STEP, e0 = r0 >> d.shift;
            if (e0 - base >= 64) {
                base = e0;
                const int e = e0 + lane;
                int at = e;
                if (a.list && e < entries) at = a.list[(int64_t)p * a.n_listed + e];
                ids = held = 0;
                if (e < entries && (uint32_t)at < (uint32_t)pages) {
                    const int id = page_at(d, a.pv.table, s, at);
                    if (id >= 0) {
                        ids = id;
                        held = min(d.page, len - (at << d.shift));
                    }
                }
            }
            const int at = e0 - base, in_page = r0 & (d.page - 1);
            int idk = __builtin_amdgcn_readlane(ids, at), idv = idk, n_held = __builtin_amdgcn_readlane(held, at);
            int rk = in_page + krow, rv = in_page + row;
            whole = in_page + STEP <= n_held;
            if (KT == 2 && d.shift == 4) {                      // two pages; a lane's rows lie in one of them
                const int id1 = __builtin_amdgcn_readlane(ids, at + 1), held1 = __builtin_amdgcn_readlane(held, at + 1);
                whole = n_held == 16 && held1 == 16;
                idk = krow < 16 ? idk : id1;
                idv = row < 16 ? idv : id1;
                n_held = row < 16 ? n_held : held1;
                rk &= 15;
                rv &= 15;
            }
            limit = n_held - rv;
            kat = a.pv.k + (layer * d.ks[0] + idk * d.ks[1] + head * d.ks[2]) * ELT + rk * kstep + c * 16;
            vat = a.pv.v + (layer * d.vs[0] + idv * d.vs[1] + head * d.vs[2]) * ELT + rv * vstep + m * EP * ELT;
        };
        u32x4 k[KT][KC];
        uint32_t v[R][VW];
        auto load_k = [&]() {
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int j = 0; j < KC; ++j)
                    k[t][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kat + t * 4 * kstep + j * 64));
        };
        auto load_v = [&]() {
#pragma unroll
            for (int i = 0; i < R; ++i) load_words<VW>(v[i], vat + i * vstep);
        };
        if (from < to) {
            locate(from);
            load_k();
            load_v();
        }
        // `more`: another step follows, whose loads are issued here.  Known to the compiler: behind a branch it could not count
        // the loads in flight, and would wait for all of them.
        auto step = [&](int st, auto more) __attribute__((always_inline)) {
            float z[R];
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                f32x4 r{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < KC; ++j) {
                    if constexpr (BF16) {
                        r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][j]), __builtin_bit_cast(bf16x8, q[j]), r, 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            r = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][j][e]), __uint_as_float(q[j][e]), r, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) z[4 * t + i] = r[i] * a.qscale;
            }
            // The products' results are read here, before any branch: the compiler puts the wait states between a product and the
            // first read of its result, but where a branch came in between it was found to leave some out, and old values were read.
#pragma unroll
            for (int i = 0; i < R; ++i) asm volatile("" : "+v"(z[i]));
            const bool now_whole = whole;
            const int now_limit = limit;
            if constexpr (more.value) {
                locate(st + 1);
                load_k();
            }
            if (!now_whole) {
#pragma unroll
                for (int i = 0; i < R; ++i)
                    if (i >= now_limit) {
                        z[i] = -INFINITY;
#pragma unroll
                        for (int w = 0; w < VW; ++w) v[i][w] = 0;             // zero times what lies there may be no number
                    }
            }
            float most = z[0];
#pragma unroll
            for (int i = 1; i < R; ++i) most = fmaxf(most, z[i]);
            if (__ballot(most > ref) != 0ull) {
                const float top = over_quarters(most, true), to_ref = top > ref ? top + AHEAD : ref;
                const float f = __builtin_amdgcn_exp2f(ref - to_ref);
                ref = to_ref;
                den *= f;
#pragma unroll
                for (int e = 0; e < EP; ++e) acc[e] *= f;
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                z[i] = __builtin_amdgcn_exp2f(z[i] - ref);
                den += z[i];
            }
            if constexpr (BF16) {
                typedef uint32_t Operand __attribute__((ext_vector_type(R / 2)));
                Operand part[3];
#pragma unroll
                for (int i = 0; i < R / 2; ++i) {
                    float lo = z[2 * i], hi = z[2 * i + 1];
#pragma unroll
                    for (int t = 0; t < 3; ++t) {
                        part[t][i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
                        lo = fmaf(z[2 * i], PART_LEAST, lo - __uint_as_float(__float_as_uint(lo) & 0xffff0000u));
                        hi = fmaf(z[2 * i + 1], PART_LEAST, hi - __uint_as_float(__float_as_uint(hi) & 0xffff0000u));
                    }
                }
#pragma unroll
                for (int e = 0; e < EP; ++e) {
                    Operand o;
#pragma unroll
                    for (int i = 0; i < R / 2; ++i)
                        o[i] = __builtin_amdgcn_perm(v[2 * i + 1][e / 2], v[2 * i][e / 2], e % 2 ? 0x07060302 : 0x05040100);
#pragma unroll
                    for (int t = 2; t >= 0; --t) {
                        if constexpr (R == 8)
                            acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, o), __builtin_bit_cast(bf16x8, part[t]), acc[e], 0, 0, 0);
                        else
                            acc[e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, o), __builtin_bit_cast(s16x4, part[t]), acc[e], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int e = 0; e < EP; ++e)
                        acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][e]), z[i], acc[e], 0, 0, 0);
            }
            if constexpr (more.value) load_v();
        };
        if (from < to) {
            for (int st = from; st + 1 < to; ++st) step(st, std::true_type{});
            step(to - 1, std::false_type{});
        }
        den = over_quarters(den, false);

        // the wavefronts' shares, lane by lane; the first one joins them
        __syncthreads();                                       // of the piece before
        if (wave > 0) {
            float *o = sh + (wave - 1) * KEEP * 64 + lane;
            o[0] = ref;
            o[64] = den;
#pragma unroll
            for (int e = 0; e < EP; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[(2 + 4 * e + i) * 64] = acc[e][i];
        }
        __syncthreads();
        if (wave == 0 && m < d.G) {                            // elements EP (4 c + i) + e of head m
            float w[NW], top = ref;
#pragma unroll
            for (int u = 1; u < NW; ++u) { w[u] = sh[(u - 1) * KEEP * 64 + lane]; top = fmaxf(top, w[u]); }
            w[0] = __builtin_amdgcn_exp2f(ref - top);
            den *= w[0];
#pragma unroll
            for (int u = 1; u < NW; ++u) {
                w[u] = __builtin_amdgcn_exp2f(w[u] - top);
                den += sh[((u - 1) * KEEP + 1) * 64 + lane] * w[u];
            }
            float *o;
            float f = 1.f;
            if (count == n) {                                  // the whole problem
                o = a.out + qrow + m * D;
                f = den == 0.f ? 0.f : 1.f / den;
            } else {
                const int64_t slot = 2 * (int64_t)(blockIdx.x - d.P) + (off == 0);
                o = a.sums + (slot * d.G + m) * D;
                if (c == 0) {
                    a.weights[(slot * d.G + m) * 2] = top;
                    a.weights[(slot * d.G + m) * 2 + 1] = den;
                }
            }
#pragma unroll
            for (int u = 0; u < NW; ++u) w[u] *= f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int e = 0; e < EP; ++e) {
                    float t = acc[e][i] * w[0];
#pragma unroll
                    for (int u = 1; u < NW; ++u) t = fmaf(sh[((u - 1) * KEEP + 2 + 4 * e + i) * 64 + lane], w[u], t);
                    o[EP * (4 * c + i) + e] = t;
                }
                asm volatile("" ::: "memory");                 // a quarter at a time: all of the others' sums do not fit the registers
            }
        }
    };
    if constexpr (!SHARED) {
        const int s = seq_of_problem(d, blockIdx.x), n = uniform(steps_of<STEP>(a, s));
        piece(blockIdx.x, s, 0, n, n);
        return;
    }
    // one call of the above, whatever the workgroup's part is: its code is long, and comes cold from memory
    const int me = (int)blockIdx.x - d.P;                      // the first ones see to short problems
    Places<STEP> places(a, lane);
    int p = blockIdx.x, s = 0, off = 0, count = 0, n = 0;
    int x = 0, to = 0, seq_from = 0, seq_to = 0, units = 0;    // seq_from, seq_to: all units of sequence s
    if (me < 0) {
        s = seq_of_problem(d, p);
        n = count = uniform(steps_of<STEP>(a, s));
        if (n > a.limit) return;
    } else {
        places.deal();
        const int share = places.whole ? 1 : places.run;
        if (me > quotient(places.total, share)) return;        // and so no overflow below
        x = me * share;
        to = min(x + share, places.total);
        if (x >= to) return;
    }
    for (;;) {
        if (me >= 0) {
            if (x >= seq_to) {
                int before;
                places.find(x, s, before, units, n);
                seq_from = before * places.heads;
                seq_to = seq_from + units * places.heads;
            }
            const int problem = uniform(quotient(x - seq_from, units)), unit = uniform(x - seq_from - problem * units);
            off = places.whole ? unit * places.run : unit;
            count = uniform(min(n - off, places.whole ? places.run : to - x));
            p = s * places.heads + problem;
            x += places.whole ? 1 : count;
        }
        piece(p, s, off, count, n);
        if (x >= to) break;
    }
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float out4 __attribute__((ext_vector_type(4), aligned(4)));             // the caller's, on any fp32 number's place
template <int M> __device__ __forceinline__ float over_lanes(float x, bool take_max)
{
    if constexpr (M < 64) {
        const float y = xor_lane<M>(x);
        return over_lanes<2 * M>(take_max ? fmaxf(x, y) : x + y, take_max);
    } else return x;
}

// grid (G, problems) of the long ones: the pieces' weights first, then their weighted sum, four elements per thread, the pieces dealt out to groups of threads
constexpr int MERGE_T = 256, MAX_PIECES = 1024, EARLY = 2;
template <int STEP>
__global__ void __launch_bounds__(MERGE_T)
decode_paged_merge_kernel(DecodePagedArgs a)
{
    __shared__ float w_sh[MERGE_T / 64][MAX_PIECES];           // every wavefront forms all weights, no barrier: 8 heads x 1 056 rows 10.3 -> 9.85 us in all
    __shared__ f32x4 sum[MERGE_T];
    const PageDims &d = a.d;
    const int g = blockIdx.x, p = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
    float *w = w_sh[tid >> 6];
    const int seq = seq_of_problem(d, p), n = shared_steps_of<STEP>(a, seq);
    if (n == 0) return;                                        // a workgroup's alone
    float *out = a.out + ((((int64_t)seq * d.n_layers + layer_of_problem(d, p)) * d.Hq) + head_of_problem(d, p) * d.G + g) * d.D;
    Places<STEP> places(a, lane);
    places.deal();
    const int units = places.units_of(n), at = places.before(seq) * places.heads + (p - seq * places.heads) * units;
    const int first = places.whole ? at : quotient(at, places.run);
    const int pieces = places.whole ? units : quotient(at + n - 1, places.run) - first + 1;
    if (pieces == 1) return;                                   // finished where it was computed
    auto slot = [&](int i) { return (int64_t)(2 * (first + i) + (i == 0)) * d.G + g; };
    const int per = d.D / 4, groups = MERGE_T / per, group = tid / per, c = tid - group * per;
    // the first of the numerators are on their way while the weights are formed
    auto part = [&](int i) { return *reinterpret_cast<const f32x4 *>(a.sums + slot(min(i, pieces - 1)) * d.D + 4 * c); };
    f32x4 early[EARLY];
#pragma unroll
    for (int j = 0; j < EARLY; ++j) early[j] = part(group + j * groups);
    auto weight = [&](int i) { return *reinterpret_cast<const f32x2 *>(a.weights + slot(min(i, pieces - 1)) * 2); };
    f32x2 own = weight(lane);                                  // reference, denominator
    if (lane >= pieces) own = f32x2{-FLT_MAX, 0.f};
    float m = own[0];
    for (int i = lane + 64; i < pieces; i += 64) m = fmaxf(m, weight(i)[0]);
    m = over_lanes<1>(m, true);
    float den = 0.f;
    for (int i = lane; i < pieces; i += 64) {
        if (i > lane) own = weight(i);
        w[i] = __builtin_amdgcn_exp2f(own[0] - m);
        den += own[1] * w[i];
    }
    den = over_lanes<1>(den, false);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");     // w: other lanes' stores from here on
    f32x4 t{0.f, 0.f, 0.f, 0.f};
    if (group < groups) {
#pragma unroll
        for (int j = 0; j < EARLY; ++j)
            if (group + j * groups < pieces) t += early[j] * w[group + j * groups];
#pragma unroll 4
        for (int i = group + EARLY * groups; i < pieces; i += groups) t += part(i) * w[i];
    }
    sum[tid] = t;
    __syncthreads();
    if (group > 0) return;
    for (int i = 1; i < groups; ++i) t += sum[i * per + c];
    *reinterpret_cast<out4 *>(out + 4 * c) = den == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : t / den;
}

// Workgroups per compute unit that the registers leave room for.  The long problems are dealt out to just as many: with two of three
// 64 sequences of up to 8 192 rows took 218 us in place of 184.
int resident(const PageDims &d)
{
    return d.D <= 64 ? 3 : d.dtype == SABLOCK_BF16 || d.D <= 160 ? 2 : 1;
}
int workgroups_of(const PageDims &d) { return std::min(d.cus * resident(d), MAX_PIECES - 1); }
// Rows of the longest problem that a workgroup takes alone: 256 KB of K and V, or 512 KB where the problems fill the compute units by
// themselves.  Alone against dealt out, rows of 256 bytes, 4 query heads: 8 problems of 512 rows 9.2 and 10.4 us, of 1 024 14.0 and
// 11.0; 64 of 512 12.2 and 12.8, of 1 024 20.9 and 15.9; 256 of 1 024 26.5 and 32.0; lengths spread up to the given ones:
// 1 024 problems of 256 22.5 and 50.4, of 1 024 57.7 and 81.2.  With 1 MB the longest are waited for: 256 problems of up to
// 4 096 76.8 us, with 512 KB 63.4.
int rows_alone(const PageDims &d) { return (d.P >= d.cus ? 1 << 19 : 1 << 18) / (2 * d.D * elt_bytes(d)); }

}  // namespace

bool decode_paged_supported(const PageDims &d) { return d.G <= 16 && d.D % (d.dtype == SABLOCK_F32 ? 16 : 32) == 0; }

size_t decode_paged_ws_bytes(const PageDims &d)
{
    const size_t rows = 2 * (size_t)workgroups_of(d) * d.G;
    return align256(rows * 8) + align256(rows * d.D * 4);
}

hipError_t launch_decode_paged(const PageDims &d, const void *q, const PageView &pv, const int32_t *list, int32_t n_listed, float *out,
                               void *ws, hipStream_t st)
{
    DecodePagedArgs a;
    a.d = d;
    a.pv = pv;
    a.q = static_cast<const char *>(q);
    a.list = list;
    a.n_listed = n_listed;
    a.qscale = (float)(1.4426950408889634 / sqrt((double)d.D));
    a.out = out;
    const int64_t capacity = (int64_t)(list ? std::min(n_listed, d.max_pages) : d.max_pages) * d.page;
    // no problem can be longer; or tables with room for so many rows that 32 bits do not count all steps, with a workgroup's run to spare
    const bool bf = d.dtype == SABLOCK_BF16, alone = capacity <= rows_alone(d) || d.P * (capacity / 16 + 1) >= 1 << 30;
    const int workgroups = workgroups_of(d), step = step_rows(bf, d.D, alone);
    a.limit = (rows_alone(d) + step - 1) / step;
    a.workgroups = alone ? 0 : workgroups;
    a.weights = static_cast<float *>(ws);
    a.sums = reinterpret_cast<float *>(static_cast<char *>(ws) + align256(2 * (size_t)workgroups * d.G * 8));
    using Kern = void (*)(DecodePagedArgs);
    Kern fn = nullptr;
#define SABLOCK_PAGED(BV, EV)                                                                                             \
    if (bf == BV && d.D == EV * 16)                                                                                       \
        fn = alone ? decode_paged_kernel<BV, EV, step_rows(BV, EV * 16, true), false> : decode_paged_kernel<BV, EV, step_rows(BV, EV * 16, false), true>;
#define SABLOCK_PAGED_F(EV) SABLOCK_PAGED(false, EV)
#define SABLOCK_PAGED_B(EV) SABLOCK_PAGED(true, EV) SABLOCK_PAGED(false, EV)
    SABLOCK_PAGED_F(1) SABLOCK_PAGED_B(2) SABLOCK_PAGED_F(3) SABLOCK_PAGED_B(4) SABLOCK_PAGED_F(5) SABLOCK_PAGED_B(6) SABLOCK_PAGED_F(7) SABLOCK_PAGED_B(8)
    SABLOCK_PAGED_F(9) SABLOCK_PAGED_B(10) SABLOCK_PAGED_F(11) SABLOCK_PAGED_B(12) SABLOCK_PAGED_F(13) SABLOCK_PAGED_B(14) SABLOCK_PAGED_F(15) SABLOCK_PAGED_B(16)
#undef SABLOCK_PAGED_B
#undef SABLOCK_PAGED_F
#undef SABLOCK_PAGED
    if (!fn) return hipErrorInvalidValue;
    hipLaunchKernelGGL(fn, dim3(a.workgroups + d.P), dim3(NT), 0, st, a);
    if (a.workgroups) hipLaunchKernelGGL(step == 32 ? decode_paged_merge_kernel<32> : decode_paged_merge_kernel<16>, dim3(d.G, d.P), dim3(MERGE_T), 0, st, a);
    return hipGetLastError();
}

}  // namespace sablock
