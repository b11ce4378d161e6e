// Decode attention of a batch whose sequences have their first pages in common: those are read once for all of them.
//
//   decode_paged_kernel (paged_decode.h)   sees to the sequences' own rows, and its first workgroups to the prefixes.  The columns of a prefix are the
//       queries of all its sequences and of the KV head's query heads, side by side without a gap; its rows are cut into pieces.  A workgroup takes a
//       block of columns over a piece of the rows and leaves references, denominators and numerators in the workspace.  Pieces are dealt out by
//       every workgroup for itself: the prefixes, which only the device knows, are few.
//   join_kernel      joins the pieces of a sequence's prefix and those of its own rows, or what a workgroup had finished of these.
//
// A sequence takes part in its prefix if all the prefix's rows are its own; one that ends before reads its rows by itself, so that no row of
// the prefix has to be masked for one column and not for another.
//
// What bounds it: with many columns the matrix products.  64 sequences x 32 query heads over 32 768 common rows and up to 2 048 of their own (8 heads of 128 bf16
// elements, 405 MB, 35 GFLOP, twice that with probabilities in three parts): 113-117 us where a large product's rate would take 59 and the reads 62;
// the start takes 13 us and the pieces' sums are 17 MB to write and read again, 13 us of it their joining.  The common rows alone 107 us; products run at
// 690 TFLOP/s over the kernel, at 957 over 131 072 common rows (287 us), and a large product's at 1 204.  Few columns: the chain of begins, lengths, table
// and rows, and that of the second launch: 8 sequences x 2 048 common rows 15.0 us in a graph (12.8 and 4.6), the counting in 64 bits 1 more.  The same
// chains make the call slower than sablock_decode_paged, which finds common rows in the caches, where these are few: 8 sequences with 256 rows of their
// own behind 512 common rows 13.8 us against 11.9, behind 2 048 14.6 against 17.7, 64 sequences behind 2 048 40 against 57, behind 32 768 105 against 859.
// On the way, 64 x 32 768 and 8 x 2 048: in three launches, a wavefront's tiles fed from memory 238 and 28.9; an XCD's blocks of columns over the same
// rows 184; K and V in LDS 160; the probabilities' parts by dot products 157; one launch for prefixes and own rows, the joins as one 122 and 18.1;
// pieces over all XCDs however few 115.  Products of a step between the next one's vector instructions: 123 in place of 115, not taken.
#include "paged_decode.h"

namespace sablock {
namespace {

struct PrefixView { const int32_t *begin, *pages; int n; };    // device: [n + 1], [n]

// Sequences of prefix i, and its pages: none where a single sequence has it
struct Prefix { int first, count, pages; };
__device__ __forceinline__ Prefix prefix_at(const PageDims &d, const PrefixView &v, int i)
{
    const int from = min(max(v.begin[i], 0), d.n_seq), to = min(max(v.begin[i + 1], 0), d.n_seq);
    return Prefix{from, max(to - from, 0), to - from > 1 ? min(max(v.pages[i], 0), d.max_pages) : 0};
}
// the prefix that sequence s may have: the last one that begins at it or before, or the first
__device__ __forceinline__ int prefix_of(const PrefixView &v, int s)
{
    int lo = 0, hi = v.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (v.begin[mid] <= s) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct PrefixArgs : DecodePagedArgs {
    PrefixView prefixes;
    float *stats;                // [P][G][2] of the sequences' own rows: reference (log2 domain), 1 / denominator
    uint32_t inv_group;          // ceil(2^32 / G)
    int prefix_workgroups;       // that see to the prefixes, a multiple of XCDS
    int slots;                   // pieces that the workspace has room for
    float *piece_weights;        // [slots][columns][2]: reference, denominator
    float *piece_sums;           // [slots][columns][D]
    static constexpr bool STATS = true, SKIP = true;
    // pages in front of the own rows of sequence s
    __device__ __forceinline__ int skipped(int s, int rows) const
    {
        const Prefix x = prefix_at(d, prefixes, prefix_of(prefixes, s));
        return s >= x.first && s < x.first + x.count && rows >> d.shift >= x.pages ? x.pages : 0;
    }
};

constexpr int XCDS = 8;
constexpr int TILE = 16;                       // columns of a matrix product

// Prefixes that do not follow each other may have any number of pieces.  Of each so many are counted, no more than the workspace has room for: 32 bits then
// hold the sums of 4 096 prefixes (229 374 places at most, with 65 536 compute units), which never descend
__host__ __device__ inline int counted_pieces(int all, int slots) { return all < slots ? all : slots; }
// whether pieces at, at + blocks, .. of a block of columns have places in the workspace
__host__ __device__ inline bool have_places(int64_t at, int pieces, int blocks, int slots) { return at >= 0 && at + (int64_t)(pieces - 1) * blocks < slots; }

// How the prefixes' rows are cut: pieces of `run` steps at most, as many as there are workgroups if those are enough.  A wavefront's view, a
// prefix per lane, 64 of them at a time.  32 bits count all steps of prefixes that follow each other (the call's limits see to it).  Of others the sum may pass
// them, and is good enough for a `run`, the same one everywhere.
template <int STEP, int COLUMNS>
struct Cut {
    const PrefixArgs &a;
    int lane, run, heads, total;                               // total: pieces of all
    Prefix own;                                                // of the first 64, the lane's
    __device__ Cut(const PrefixArgs &args, int l) : a(args), lane(l), heads(args.d.n_layers * args.d.Hkv)
    {
        own = load(lane);
        uint32_t steps = 0, blocks = 0;
        for (int base = 0; base < a.prefixes.n; base += 64) {
            const Prefix x = at(base);
            const uint32_t b = x.pages ? (uint32_t)heads * blocks_of(x) : 0;
            steps += b * steps_of_pages(x.pages);
            blocks += b;
        }
        steps = of_lane(sum_upto_lane(steps), 63);
        blocks = of_lane(sum_upto_lane(blocks), 63);
        const uint32_t all = a.prefix_workgroups, shares = blocks < all ? all - blocks : all;
        run = (int)min(max((uint32_t)LEAST_STEPS, (steps + shares - 1) / shares), 1u << 27);            // no table has room for more
        total = before(a.prefixes.n);
    }
    __device__ Prefix load(int i) const { return i < a.prefixes.n ? prefix_at(a.d, a.prefixes, i) : Prefix{0, 0, 0}; }
    __device__ Prefix at(int base) const { return base == 0 ? own : load(base + lane); }               // a lane's of 64
    __device__ Prefix get(int i) const                         // the same for all
    {
        return i < 64 ? Prefix{of_lane(own.first, i), of_lane(own.count, i), of_lane(own.pages, i)} : prefix_at(a.d, a.prefixes, i);
    }
    __device__ int all_of(const Prefix &x) const { return x.pages ? counted_pieces(heads * blocks_of(x) * pieces_of(x), a.slots) : 0; }
    __device__ int blocks_of(const Prefix &x) const { return (x.count * a.d.G + COLUMNS - 1) / COLUMNS; }
    __device__ int steps_of_pages(int pages) const { return ((pages << a.d.shift) + STEP - 1) / STEP; }
    __device__ int pieces_of(const Prefix &x) const { return x.pages ? (steps_of_pages(x.pages) + run - 1) / run : 0; }
    // the prefix that piece x of all lies in, and the pieces in front of it
    __device__ int find(int x, int &before) const
    {
        before = 0;
        for (int base = 0; base < a.prefixes.n; base += 64) {
            const int n = all_of(at(base)), upto = sum_upto_lane(n) + before;
            const unsigned long long behind = __ballot(upto > x);
            if (behind) {
                const int l = uniform(__ffsll(behind) - 1);
                before = of_lane(upto, l) - of_lane(n, l);
                return base + l;
            }
            before = of_lane(upto, 63);
        }
        return -1;
    }
    // pieces of the prefixes in front of prefix i
    __device__ int before(int i) const
    {
        int sum = 0;
        for (int base = 0; base < i; base += 64) sum += of_lane(sum_upto_lane(base + lane < i ? all_of(at(base)) : 0), 63);
        return sum;
    }
    // f(piece) for the workgroup's pieces.  Those that follow each other are an XCD's, which workgroups go round: blocks of columns over the same rows
    // find each other's rows in its L2
    template <typename F> __device__ __forceinline__ void each_piece(F &&f) const
    {
        const int n = min(total, a.slots), share = (n + XCDS - 1) / XCDS, from = blockIdx.x % XCDS * share, to = min(n, from + share);
        for (int x = from + (int)blockIdx.x / XCDS; x < to; x += a.prefix_workgroups / XCDS) f(x);
    }
};

// the first of a prefix's sequences that takes part in it: the others' rows of the table may not have its pages
__device__ __forceinline__ int first_member(const PrefixArgs &a, const Prefix &x, int lane)
{
    for (int at = 0; at < x.count; at += 64) {
        const bool member = at + lane < x.count && rows_of(a.d, a.pv.lengths, min(x.first + at + lane, a.d.n_seq - 1)) >> a.d.shift >= x.pages;
        const unsigned long long members = __ballot(member);
        if (members) return uniform(at + __ffsll(members) - 1);
    }
    return x.count;
}

// What a step of either kernel makes of its logits: a tile's references, denominators and probabilities in parts
template <int CT, int EP, int R>
struct Columns {
    float ref[CT], den[CT];
    f32x4 acc[CT][EP];
    __device__ void clear()
    {
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            ref[t] = -FLT_MAX;
            den[t] = 0.f;
#pragma unroll
            for (int e = 0; e < EP; ++e) acc[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    static __device__ __forceinline__ void largest(const float (&z)[CT][R], float (&most)[CT])
    {
#pragma unroll
        for (int u = 0; u < CT; ++u) {
            most[u] = z[u][0];
#pragma unroll
            for (int r = 1; r < R; ++r) most[u] = fmaxf(most[u], z[u][r]);
        }
    }
    // logits z, the largest of a lane given, become probabilities; references move where a logit passes them.  SCALE: they are still to be multiplied by `scale`
    template <bool SCALE> __device__ __forceinline__ void take(float (&z)[CT][R], float (&most)[CT], float scale)
    {
        bool moves = false;
#pragma unroll
        for (int u = 0; u < CT; ++u) {
            if constexpr (SCALE) most[u] *= scale;
            moves |= most[u] > ref[u];
        }
        if (__ballot(moves) != 0ull) {
#pragma unroll
            for (int u = 0; u < CT; ++u) {
                const float top = over_quarters(most[u], true), to_ref = top > ref[u] ? top + AHEAD : ref[u];
                const float f = __builtin_amdgcn_exp2f(ref[u] - to_ref);
                ref[u] = to_ref;
                den[u] *= f;
#pragma unroll
                for (int e = 0; e < EP; ++e) acc[u][e] *= f;
            }
        }
#pragma unroll
        for (int u = 0; u < CT; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                z[u][r] = __builtin_amdgcn_exp2f(SCALE ? fmaf(z[u][r], scale, -ref[u]) : z[u][r] - ref[u]);
                den[u] += z[u][r];
            }
    }
    // Probabilities as three bf16 numbers each, 24 bits; none but the first is ever zero, as zero times an infinite value would be no number.  A part is
    // the upper half of what is left, which the next difference (of one element: the other's factor is zero) leaves
    typedef uint32_t Operand __attribute__((ext_vector_type(R / 2)));
    static __device__ __forceinline__ void split(const float (&z)[CT][R], Operand (&part)[CT][3])
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef short s16x2 __attribute__((ext_vector_type(2)));
        // (-1, 0) and (0, -1), in registers: as a constant of the instruction the first one was taken for another pair
        uint32_t of_x = 0x0000bf80u, of_y = 0xbf800000u;
        asm("" : "+s"(of_x), "+s"(of_y));
        const bf16x2 first = __builtin_bit_cast(bf16x2, of_x), second = __builtin_bit_cast(bf16x2, of_y);
        const s16x2 least = {0x0d00, 0x0d00};                  // 2^-101
#pragma unroll
        for (int u = 0; u < CT; ++u)
#pragma unroll
            for (int r = 0; r < R / 2; ++r) {
                float x = z[u][2 * r], y = z[u][2 * r + 1];
#pragma unroll
                for (int t = 0; t < 3; ++t) {
                    const uint32_t top = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302);
                    part[u][t][r] = t ? __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, top), least)) : top;
                    if (t == 2) break;
                    x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, top), first, x, false);
                    y = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, top), second, y, false);
                }
            }
    }
    // element e of V's rows (dwords of two elements) as operand
    static __device__ __forceinline__ Operand operand(const uint32_t (&v)[R][(EP + 1) / 2], int e)
    {
        Operand o;
#pragma unroll
        for (int r = 0; r < R / 2; ++r) o[r] = __builtin_amdgcn_perm(v[2 * r + 1][e / 2], v[2 * r][e / 2], e % 2 ? 0x07060302 : 0x05040100);
        return o;
    }
    __device__ __forceinline__ void product(const Operand &o, const Operand &part, int e, int u)
    {
        if constexpr (R == 8)
            acc[u][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, o), __builtin_bit_cast(bf16x8, part), acc[u][e], 0, 0, 0);
        else
            acc[u][e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, o), __builtin_bit_cast(s16x4, part), acc[u][e], 0, 0, 0);
    }
    // out^T += V^T P^T, products into one accumulator far from each other: the next one waits for the last one's result
    __device__ __forceinline__ void multiply(const Operand (&o)[EP], const Operand (&part)[CT][3])
    {
#pragma unroll
        for (int t = 2; t >= 0; --t)
#pragma unroll
            for (int e = 0; e < EP; ++e)
#pragma unroll
                for (int u = 0; u < CT; ++u) product(o[e], part[u][t], e, u);
    }
};

// CT: tiles of 16 columns of a workgroup, which every wavefront has; the steps of a piece are shared among the wavefronts.  A step is that of
// decode_paged_kernel, with the operands of K and V used for all tiles.
template <bool BF16, int EP, int STEP, int CT>
__device__ __forceinline__ void narrow_prefixes(const PrefixArgs &a, float *sh)
{
    constexpr int D = EP * 16, ELT = BF16 ? 2 : 4, R = STEP / 4, KT = STEP / 16, KC = D * ELT / 64, VW = EP * ELT / 4, KEEP = D / 4 + 2;
    constexpr int COLUMNS = CT * TILE;
    const PageDims &d = a.d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, c = lane >> 4;
    const int krow = KT == 2 ? (m >> 2) * 8 + (m & 3) : m, row = R * c;
    const int64_t kstep = d.ks[3] * ELT, vstep = d.vs[3] * ELT;
    const Cut<STEP, COLUMNS> cut(a, lane);
    cut.each_piece([&](int x) __attribute__((always_inline)) {
        int before;
        const Prefix prefix = cut.get(cut.find(x, before));
        const int blocks = cut.blocks_of(prefix), pieces = cut.pieces_of(prefix), n = cut.steps_of_pages(prefix.pages);
        const int part = uniform(quotient(x - before, blocks)), column0 = uniform(x - before - part * blocks) * COLUMNS;
        const int problem = uniform(quotient(part, pieces)), j = part - problem * pieces;
        const int layer = uniform(quotient(problem, d.Hkv)), head = problem - layer * d.Hkv;
        const int off = j * cut.run, count = min(cut.run, n - off), from = off + (int)((int64_t)count * wave / NW), to = off + (int)((int64_t)count * (wave + 1) / NW);
        // pages of 64 places at a time, one per lane; the first ones of the first sequence, in case that it takes part
        int base = from * STEP >> d.shift, ids = base + lane < prefix.pages ? page_at(d, a.pv.table, prefix.first, base + lane) : -1;
        const int columns = prefix.count * d.G, s = prefix.first + first_member(a, prefix, lane);     // the table's row that is read
        if (s >= prefix.first + prefix.count) return;
        if (s > prefix.first) base = -1 << 30;

        u32x4 q[CT][KC];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const int col = column0 + t * TILE + m, at = sablock::quotient(min(col, columns - 1), a.inv_group), g = min(col, columns - 1) - at * d.G;
            const int64_t qrow = (((int64_t)(prefix.first + at) * d.n_layers + layer) * d.Hq + head * d.G + g) * D;
#pragma unroll
            for (int e = 0; e < KC; ++e) q[t][e] = *reinterpret_cast<const u32x4 *>(a.q + qrow * ELT + e * 64 + c * 16);
        }
        Columns<CT, EP, R> own;
        own.clear();
        const char *kat = nullptr, *vat = nullptr;
        bool whole = false, there = false;                     // all rows of the step exist; this lane's results' rows do
        auto locate = [&](int st) {
            const int r0 = st * STEP, e0 = r0 >> d.shift;
            if (e0 - base >= 64) {
                base = e0;
                ids = e0 + lane < prefix.pages ? page_at(d, a.pv.table, s, e0 + lane) : -1;
            }
            const int at = e0 - base, in_page = r0 & (d.page - 1);
            int idk = __builtin_amdgcn_readlane(ids, at), idv = idk;
            int rk = in_page + krow, rv = in_page + row;
            whole = there = idk >= 0;
            if (KT == 2 && d.shift == 4) {                     // two pages; a lane's rows lie in one of them
                const int id1 = at < 63 ? __builtin_amdgcn_readlane(ids, at + 1) : -1;
                whole = idk >= 0 && id1 >= 0;
                idk = krow < 16 ? idk : id1;
                idv = row < 16 ? idv : id1;
                there = idv >= 0;
                rk &= 15;
                rv &= 15;
            }
            kat = a.pv.k + (layer * d.ks[0] + max(idk, 0) * d.ks[1] + head * d.ks[2]) * ELT + rk * kstep + c * 16;
            vat = a.pv.v + (layer * d.vs[0] + max(idv, 0) * d.vs[1] + head * d.vs[2]) * ELT + rv * vstep + m * EP * ELT;
        };
        u32x4 k[KT][KC];
        uint32_t v[R][VW];
        auto load_k = [&]() {
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int e = 0; e < KC; ++e) k[t][e] = *reinterpret_cast<const u32x4 *>(kat + t * 4 * kstep + e * 64);
        };
        auto load_v = [&]() {
#pragma unroll
            for (int r = 0; r < R; ++r) load_words<VW>(v[r], vat + r * vstep);
        };
        if (from < to) {
            locate(from);
            load_k();
            load_v();
        }
        auto step = [&](int st, auto more) __attribute__((always_inline)) {
            float z[CT][R];
#pragma unroll
            for (int u = 0; u < CT; ++u) {
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    f32x4 r{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < KC; ++e) {
                        if constexpr (BF16) {
                            r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][e]), __builtin_bit_cast(bf16x8, q[u][e]), r, 0, 0, 0);
                        } else {
#pragma unroll
                            for (int w = 0; w < 4; ++w)
                                r = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][e][w]), __uint_as_float(q[u][e][w]), r, 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int w = 0; w < 4; ++w) z[u][4 * t + w] = r[w] * a.qscale;
                }
                // read before any branch, see decode_paged_kernel
#pragma unroll
                for (int r = 0; r < R; ++r) asm volatile("" : "+v"(z[u][r]));
            }
            const bool now_whole = whole, now_there = there;
            if constexpr (more.value) {
                locate(st + 1);
                load_k();
            }
            if (!now_whole) {
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (!now_there) {
#pragma unroll
                        for (int u = 0; u < CT; ++u) z[u][r] = -INFINITY;
#pragma unroll
                        for (int w = 0; w < VW; ++w) v[r][w] = 0;
                    }
            }
            float most[CT];
            own.largest(z, most);
            own.template take<false>(z, most, 1.f);
            if constexpr (BF16) {
                typename Columns<CT, EP, R>::Operand p_part[CT][3];
                own.split(z, p_part);
#pragma unroll
                for (int e = 0; e < EP; ++e) {
                    const auto o = own.operand(v, e);
#pragma unroll
                    for (int u = 0; u < CT; ++u)
#pragma unroll
                        for (int t = 2; t >= 0; --t) own.product(o, p_part[u][t], e, u);
                }
            } else {
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int e = 0; e < EP; ++e)
#pragma unroll
                        for (int u = 0; u < CT; ++u)
                            own.acc[u][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[r][e]), z[u][r], own.acc[u][e], 0, 0, 0);
            }
            if constexpr (more.value) load_v();
        };
        if (from < to) {
            for (int st = from; st + 1 < to; ++st) step(st, std::true_type{});
            step(to - 1, std::false_type{});
        }
        // the wavefronts' shares, lane by lane and tile by tile; the first one joins them
#pragma unroll
        for (int u = 0; u < CT; ++u) {
            own.den[u] = over_quarters(own.den[u], false);
            __syncthreads();                                   // of the tile before
            if (wave > 0) {
                float *o = sh + (wave - 1) * KEEP * 64 + lane;
                o[0] = own.ref[u];
                o[64] = own.den[u];
#pragma unroll
                for (int e = 0; e < EP; ++e)
#pragma unroll
                    for (int w = 0; w < 4; ++w) o[(2 + 4 * e + w) * 64] = own.acc[u][e][w];
            }
            __syncthreads();
            const int col = u * TILE + m;
            if (wave == 0 && column0 + col < columns) {        // elements EP (4 c + w) + e of the column
                float w[NW], top = own.ref[u];
#pragma unroll
                for (int t = 1; t < NW; ++t) { w[t] = sh[(t - 1) * KEEP * 64 + lane]; top = fmaxf(top, w[t]); }
                w[0] = __builtin_amdgcn_exp2f(own.ref[u] - top);
                float sum = own.den[u] * w[0];
#pragma unroll
                for (int t = 1; t < NW; ++t) {
                    w[t] = __builtin_amdgcn_exp2f(w[t] - top);
                    sum += sh[((t - 1) * KEEP + 1) * 64 + lane] * w[t];
                }
                const int64_t slot = (int64_t)x * COLUMNS + col;
                float *o = a.piece_sums + slot * D;
                if (c == 0) *reinterpret_cast<f32x2 *>(a.piece_weights + slot * 2) = f32x2{top, sum};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
#pragma unroll
                    for (int e = 0; e < EP; ++e) {
                        float t = own.acc[u][e][r] * w[0];
#pragma unroll
                        for (int y = 1; y < NW; ++y) t = fmaf(sh[((y - 1) * KEEP + 2 + 4 * e + r) * 64 + lane], w[y], t);
                        o[EP * (4 * c + r) + e] = t;
                    }
                    asm volatile("" ::: "memory");             // a quarter at a time: all of the others' sums do not fit the registers
                }
            }
        }
    });
}

typedef __attribute__((address_space(3))) const void *lds_ptr;
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(lds_ptr)p; }
// 16 bytes per lane from base + offset to consecutive places of LDS; waited for by wait_for_pieces
__device__ __forceinline__ void piece_to_lds(uint32_t offset, const char *base, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(to) : "memory", "m0");
}
template <int BEHIND> __device__ __forceinline__ void wait_for_pieces() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(BEHIND) : "memory"); }
template <int N> __device__ __forceinline__ void row_of_lds(uint32_t (&w)[N], const char *p)  // on a multiple of its size, or of 4 bytes
{
    if constexpr (N == 4 || N == 2) {
        typedef uint32_t T __attribute__((ext_vector_type(N)));
        const T x = *reinterpret_cast<const T *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = x[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
    }
}
// all LDS traffic of this wavefront done, then the workgroup barrier (loads to LDS stay in flight)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The same for prefixes with many columns, bf16: a wavefront has columns of its own, 32 of the workgroup's 128 (or,
// heads of more than 128 elements, 16 of 64), and all wavefronts do every step, from K and V in LDS.  Steps come there four (two) at a time, each
// wavefront seeing to a quarter of the pieces of 1 KiB; a piece's rows lie in one page.  One barrier per step: everybody's pieces of this step have landed, and the last step's place is free.
// A row of K in LDS has its 16-byte chunks in the order of place(): the 16 rows of an operand, (m >> 2) * 8 + (m & 3) apart from 4, come from different banks.
constexpr int wide_tiles(int D) { return D <= 128 ? 2 : 1; }
constexpr int wide_columns(int D) { return NW * wide_tiles(D) * TILE; }
constexpr int wide_stages(int D) { return D <= 128 ? 4 : 2; }
template <int EP> __device__ __forceinline__ int place(int chunk, int row)
{
    return chunk ^ (EP % 8 == 0 ? (row >> 3) * 4 + (row & 3) : EP % 8 == 4 ? (row >> 3) * 2 + (row >> 1 & 1) : row >> 3);
}

constexpr int wide_bytes(int D) { return wide_stages(D) * 2 * 32 * D * 2; }
template <int EP>
__device__ __forceinline__ void wide_prefixes(const PrefixArgs &a, char *lds)
{
    constexpr int D = EP * 16, STEP = 32, R = 8, KT = 2, CT = wide_tiles(D), KC = D / 32, VW = EP / 2, WIDE = wide_columns(D), STAGES = wide_stages(D);
    constexpr int ROW = D * 2, CHUNKS = D / 8, PIECES = D / 16, OWN = (PIECES + NW - 1) / NW, KV = STEP * ROW;
    static_assert(wide_bytes(D) == STAGES * 2 * KV);
    const PageDims &d = a.d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, c = lane >> 4;
    const int64_t kstep = d.ks[3] * 2, vstep = d.vs[3] * 2;
    // this lane's part of its wavefront's pieces
    uint32_t k_offset[OWN], v_offset[OWN];
    int piece[OWN];
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        piece[o] = min(wave * OWN + o, PIECES - 1);
        const int at = piece[o] * 64 + lane, r = at / CHUNKS, pos = at - r * CHUNKS, in_page = d.shift == 4 ? r & 15 : r;
        k_offset[o] = (uint32_t)(in_page * (int)kstep + place<EP>(pos, r) * 16);
        v_offset[o] = (uint32_t)(in_page * (int)vstep + pos * 16);
    }
    const int krow = (m >> 2) * 8 + (m & 3);                   // and that row + 4, whose chunks have the same order
    uint32_t k_at[KC];
#pragma unroll
    for (int e = 0; e < KC; ++e) k_at[e] = krow * ROW + place<EP>(4 * e + c, krow) * 16;
    const uint32_t v_at = R * c * ROW + m * (EP < 16 ? EP * 2 : 16);

    const Cut<STEP, WIDE> cut(a, lane);
    cut.each_piece([&](int x) __attribute__((always_inline)) {
        int before;
        const Prefix prefix = cut.get(cut.find(x, before));
        const int blocks = cut.blocks_of(prefix), pieces = cut.pieces_of(prefix), n = cut.steps_of_pages(prefix.pages);
        const int part = uniform(quotient(x - before, blocks)), column0 = uniform(x - before - part * blocks) * WIDE + wave * CT * TILE;
        const int problem = uniform(quotient(part, pieces)), j = part - problem * pieces;
        const int layer = uniform(quotient(problem, d.Hkv)), head = problem - layer * d.Hkv;
        const int columns = prefix.count * d.G, s = prefix.first + first_member(a, prefix, lane);
        if (s >= prefix.first + prefix.count) return;
        const int off = uniform(j * cut.run), count = uniform(min(cut.run, n - off));
        const bool active = column0 < columns;

        lds_barrier();                                         // the piece before has been read
        int ids = -1, base = -1 << 30;                         // pages of 64 places at a time, one per lane
        uint32_t there = 0;                                    // two bits a step, the newest lowest: whether its first and its last 16 rows exist
        const char *k_head = a.pv.k + (layer * d.ks[0] + head * d.ks[2]) * 2, *v_head = a.pv.v + (layer * d.vs[0] + head * d.vs[2]) * 2;
        auto issue = [&](int st, int stage) {
            const int r0 = st * STEP, e0 = r0 >> d.shift;
            if (e0 - base >= 64) {
                base = e0;
                ids = e0 + lane < prefix.pages ? page_at(d, a.pv.table, s, e0 + lane) : -1;
            }
            const int in_page = r0 & (d.page - 1), id0 = of_lane(ids, e0 - base);
            const int id1 = d.shift > 4 ? id0 : e0 - base < 63 ? of_lane(ids, e0 - base + 1) : -1;
            there = there << 2 | (id0 >= 0 ? 1u : 0u) | (id1 >= 0 ? 2u : 0u);
            const uint32_t to = uniform((int)lds_address(lds) + stage * 2 * KV);
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                const int64_t id = max(2 * piece[o] >= PIECES ? id1 : id0, 0);
                piece_to_lds(k_offset[o], k_head + (id * d.ks[1] + in_page * d.ks[3]) * 2, to + piece[o] * 1024);
                piece_to_lds(v_offset[o], v_head + (id * d.vs[1] + in_page * d.vs[3]) * 2, to + KV + piece[o] * 1024);
            }
        };
        u32x4 q[CT][KC];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const int col = min(column0 + t * TILE + m, columns - 1), at = sablock::quotient(col, a.inv_group), g = col - at * d.G;
            const int64_t qrow = (((int64_t)(prefix.first + at) * d.n_layers + layer) * d.Hq + head * d.G + g) * D;
#pragma unroll
            for (int e = 0; e < KC; ++e) q[t][e] = *reinterpret_cast<const u32x4 *>(a.q + qrow * 2 + e * 64 + c * 16);
        }
        // here, in front of the loads that the compiler does not count: it would wait for these, and all of those, in every step
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int e = 0; e < KC; ++e) asm volatile("" : "+v"(q[t][e]));
        Columns<CT, EP, R> own;
        own.clear();
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t) issue(off + min(t, count - 1), t);
        for (int st = 0, stage = 0; st < count; ++st) {
            wait_for_pieces<(STAGES - 2) * 2 * OWN>();
            lds_barrier();
            issue(off + min(st + STAGES - 1, count - 1), (stage + STAGES - 1) % STAGES);
            const char *kt = lds + stage * 2 * KV, *vt = kt + KV;
            stage = (stage + 1) % STAGES;
            if (!active) continue;
            float z[CT][R];
            {
                u32x4 k[KT][KC];
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int e = 0; e < KC; ++e) k[t][e] = *reinterpret_cast<const u32x4 *>(kt + k_at[e] + t * 4 * ROW);
                f32x4 r[CT][KT];
#pragma unroll
                for (int e = 0; e < KC; ++e)
#pragma unroll
                    for (int u = 0; u < CT; ++u)
#pragma unroll
                        for (int t = 0; t < KT; ++t)
                            r[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][e]), __builtin_bit_cast(bf16x8, q[u][e]),
                                                                             e ? r[u][t] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int u = 0; u < CT; ++u)
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int w = 0; w < 4; ++w) z[u][4 * t + w] = r[u][t][w];
            }
            // all results are read before any branch, see decode_paged_kernel
            float most[CT];
            own.largest(z, most);
#pragma unroll
            for (int u = 0; u < CT; ++u) asm volatile("" : "+v"(most[u]));
            uint32_t v[R][VW];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if constexpr (EP < 16) {
                    row_of_lds(v[r], vt + v_at + r * ROW);
                } else {                                       // eight elements of either half: side by side the lanes' 32 bytes would lie in half of the banks
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const u32x4 x = *reinterpret_cast<const u32x4 *>(vt + v_at + r * ROW + y * ROW / 2);
#pragma unroll
                        for (int w = 0; w < 4; ++w) v[r][4 * y + w] = x[w];
                    }
                }
            }
            const uint32_t now = there >> 2 * (STAGES - 1) & 3;
            if (now != 3 && !(now >> (c >> 1) & 1)) {
#pragma unroll
                for (int u = 0; u < CT; ++u) {
                    most[u] = -INFINITY;
#pragma unroll
                    for (int r = 0; r < R; ++r) z[u][r] = -INFINITY;
                }
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int w = 0; w < VW; ++w) v[r][w] = 0;
            }
            own.template take<true>(z, most, a.qscale);
            typename Columns<CT, EP, R>::Operand p_part[CT][3], o[EP];
            own.split(z, p_part);
#pragma unroll
            for (int e = 0; e < EP; ++e) o[e] = own.operand(v, e);
            own.multiply(o, p_part);
        }
        wait_for_pieces<0>();                                  // those that came again for the last steps: LDS may be another workgroup's soon
        if (!active) return;
#pragma unroll
        for (int u = 0; u < CT; ++u) {
            own.den[u] = over_quarters(own.den[u], false);
            const int col = column0 + u * TILE + m;
            if (col >= columns) continue;
            // elements EP (4 c + w) + e of the column; EP = 16: 8 (4 c + w) + e of either half
            const int64_t slot = (int64_t)x * WIDE + wave * CT * TILE + u * TILE + m;
            if (c == 0) *reinterpret_cast<f32x2 *>(a.piece_weights + slot * 2) = f32x2{own.ref[u], own.den[u]};
            constexpr int RUN = EP < 16 ? EP : 8;
            float *o = a.piece_sums + slot * D + RUN * 4 * c;
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int e = 0; e < EP; ++e) o[e / RUN * (D / 2) + RUN * w + e % RUN] = own.acc[u][e][w];
        }
    });
}

constexpr int prefix_tiles(bool bf16, int D) { return D <= (bf16 ? 128 : 64) ? 2 : 1; }

// The arguments by what the first workgroups do
template <bool BF16, int EP, bool MANY> struct PrefixPart : PrefixArgs {
    static constexpr int FLOATS = MANY ? wide_bytes(EP * 16) / 4 : 0;          // of LDS
    __device__ __forceinline__ void prefix_part(float *sh) const
    {
        if constexpr (MANY) wide_prefixes<EP>(*this, reinterpret_cast<char *>(sh));
        else narrow_prefixes<BF16, EP, step_rows(BF16, EP * 16, false), prefix_tiles(BF16, EP * 16)>(*this, sh);
    }
};

constexpr int JOIN_EARLY = 4;
// grid (G, problems).  STEP: of the own rows, CUT: of the prefixes
template <int STEP, int CUT, int COLUMNS>
__global__ void __launch_bounds__(MERGE_T)
join_kernel(PrefixArgs a)
{
    __shared__ f32x4 sum[MERGE_T];
    const PageDims &d = a.d;
    const int g = blockIdx.x, p = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
    const int s = seq_of_problem(d, p), skip = a.skipped(s, rows_of(d, a.pv.lengths, s)), n = shared_steps_of<STEP>(a, s);
    if (skip == 0 && n == 0) return;                           // finished
    // Entries: the prefix's pieces, then those of the own rows, or what they gave
    int pieces = 0, own_pieces = 1;
    int64_t first = 0, by = 0, own_first = -1;                 // rows of weights and sums; own_first < 0: finished
    if (skip) {
        const int i = uniform(prefix_of(a.prefixes, s));
        const Cut<CUT, COLUMNS> cut(a, lane);
        const Prefix prefix = cut.get(i);
        const int blocks = cut.blocks_of(prefix), column = (s - prefix.first) * d.G + g, block = column / COLUMNS;
        pieces = cut.pieces_of(prefix);
        const int64_t at = cut.before(i) + (int64_t)(p - s * cut.heads) * pieces * blocks + block;
        if (!have_places(at, pieces, blocks, a.slots)) pieces = 0;             // prefixes that do not follow each other: the own rows alone
        first = at * COLUMNS + column - block * COLUMNS;
        by = (int64_t)blocks * COLUMNS;
    }
    if (n) {
        Places<STEP, PrefixArgs> places(a, lane);
        places.deal();
        const int units = places.units_of(n), at = places.before(s) * places.heads + (p - s * places.heads) * units;
        const int from = places.whole ? at : quotient(at, places.run), count = places.whole ? units : quotient(at + n - 1, places.run) - from + 1;
        if (count > 1) {
            own_first = from;
            own_pieces = count;
        }
    }
    if (pieces == 0 && own_first < 0) return;                  // finished
    struct Entry { f32x2 weight; const float *sums; };         // reference, denominator; numerators
    float *out = a.out + (((int64_t)s * d.n_layers + layer_of_problem(d, p)) * d.Hq + head_of_problem(d, p) * d.G + g) * d.D;
    auto entry = [&](int j) {
        if (j < pieces) return Entry{*reinterpret_cast<const f32x2 *>(a.piece_weights + (first + j * by) * 2), a.piece_sums + (first + j * by) * d.D};
        if (own_first >= 0) {
            const int64_t slot = (2 * (own_first + j - pieces) + (j == pieces)) * d.G + g;
            return Entry{*reinterpret_cast<const f32x2 *>(a.weights + slot * 2), a.sums + slot * d.D};
        }
        const f32x2 x = *reinterpret_cast<const f32x2 *>(a.stats + ((int64_t)p * d.G + g) * 2);
        return Entry{f32x2{x[0], x[1] == 0.f ? 0.f : 1.f / x[1]}, out};
    };
    const int entries = pieces + own_pieces, per = d.D / 4, groups = MERGE_T / per, group = tid / per, c = tid - group * per;
    // the first of the numerators are on their way while the weights are formed
    f32x4 early[JOIN_EARLY], t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < JOIN_EARLY; ++e) early[e] = *reinterpret_cast<const out4 *>(entry(min(group + e * groups, entries - 1)).sums + 4 * c);
    const f32x2 mine = entry(min(lane, entries - 1)).weight;
    float m = mine[0], den = 0.f;
    for (int j = lane + 64; j < entries; j += 64) m = fmaxf(m, entry(j).weight[0]);
    m = over_lanes<1>(m, true);
    for (int j = lane; j < entries; j += 64) {
        const f32x2 w = j == lane ? mine : entry(j).weight;
        den += w[1] * __builtin_amdgcn_exp2f(w[0] - m);
    }
    den = over_lanes<1>(den, false);
    auto add = [&](int j, const f32x4 &x) {
        const f32x2 e = entry(j).weight;
        const bool finished = j >= pieces && own_first < 0;    // what is finished is divided by its denominator
        const float w = __builtin_amdgcn_exp2f(e[0] - m) * (finished ? e[1] : 1.f);
        if (!finished || w != 0.f) t += x * w;
    };
    if (group < groups) {
#pragma unroll
        for (int e = 0; e < JOIN_EARLY; ++e)
            if (group + e * groups < entries) add(group + e * groups, early[e]);
        for (int j = group + JOIN_EARLY * groups; j < entries; j += groups) add(j, *reinterpret_cast<const out4 *>(entry(j).sums + 4 * c));
    }
    sum[tid] = t;
    __syncthreads();
    if (group > 0) return;
    for (int j = 1; j < groups; ++j) t += sum[j * per + c];
    *reinterpret_cast<out4 *>(out + 4 * c) = den == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : t / den;
}

// Prefixes have more than 64 columns on average, 16 where heads have more than 128 elements, and the rows of a step lie within reach of 31 bits.  Wide
// against narrow, 68 columns and 128: 2 048 rows 20.1 and 21.5 us, 23.8 and 25.8; 8 192 rows 26.2 and 29.4, 30.3 and 34.0; 32 768 rows 57.5 and 56.7, 59.3 and 66.0.  64 columns, 32 768 rows: narrow 45.5.
// Heads of 256, 16 columns and 64: 2 048 rows 16.8 and 18.6 us, 24.4 and 26.2; 8 192 rows 26.1 and 27.9, 33.9 and 44.7; 32 768 rows 56.8 and 57.3, 68.4 and 132; 256
// columns 215 and 561.
int prefixes_wide(const PageDims &d)           // so many prefixes at most
{
    const int64_t reach = 31 * 2 * std::max(d.ks[3], d.vs[3]);
    return d.dtype == SABLOCK_BF16 && reach + 512 < (int64_t)1 << 31 ? (d.n_seq * d.G - 1) / (d.D <= 128 ? 64 : 16) : 0;
}
bool prefix_wide(const PageDims &d, int n_prefixes) { return n_prefixes <= prefixes_wide(d); }
int prefix_columns(const PageDims &d, int n_prefixes) { return prefix_wide(d, n_prefixes) ? wide_columns(d.D) : prefix_tiles(d.dtype == SABLOCK_BF16, d.D) * TILE; }
// A wide workgroup for every compute unit, beside one of the own rows' (two: 139 us in place of 122 for 64 x 32 768 and own rows, the common rows alone 101
// in place of 107), and two narrow ones
int prefix_workgroups(const PageDims &d, int n_prefixes) { return (d.cus * (prefix_wide(d, n_prefixes) ? 1 : 2) + XCDS - 1) / XCDS * XCDS; }
// pieces at most: one more than its share for every workgroup, and one for every block of columns, of which the last ones of prefixes of two sequences
// or more may be short
int prefix_slots(const PageDims &d, int n_prefixes)
{
    const int64_t blocks = ((int64_t)d.n_seq * d.G) / prefix_columns(d, n_prefixes) + std::min(n_prefixes, d.n_seq / 2);
    return (int)(prefix_workgroups(d, n_prefixes) + (int64_t)d.n_layers * d.Hkv * blocks);
}
size_t stats_bytes(const PageDims &d) { return align256((size_t)d.P * d.G * 8); }
size_t weights_bytes(const PageDims &d, int n_prefixes) { return align256((size_t)prefix_slots(d, n_prefixes) * prefix_columns(d, n_prefixes) * 8); }
size_t sums_bytes(const PageDims &d, int n_prefixes) { return align256((size_t)prefix_slots(d, n_prefixes) * prefix_columns(d, n_prefixes) * d.D * 4); }

}  // namespace

size_t decode_prefix_ws_need(const PageDims &d, int32_t n_prefixes)
{
    return decode_ws_bytes_of(d) + stats_bytes(d) + weights_bytes(d, n_prefixes) + sums_bytes(d, n_prefixes);
}
// It grows with the prefixes but for one step down, from blocks of many columns to blocks of few: 64 sequences of 8 x 4 heads of 128, 3 prefixes 21.8 MB, 4 12.3
size_t decode_prefix_ws_bytes(const PageDims &d, int32_t n_prefixes)
{
    const int wide = std::min(n_prefixes, prefixes_wide(d));
    return std::max(decode_prefix_ws_need(d, n_prefixes), wide ? decode_prefix_ws_need(d, wide) : 0);
}

// 32 bits count all steps, as they do not where a table has room for more
bool decode_prefix_supported(const PageDims &d) { return decode_paged_supported(d) && d.P * (((int64_t)d.max_pages << d.shift) / 16 + 1) < 1 << 30; }

hipError_t launch_decode_prefix(const PageDims &d, const void *q, const PageView &pv, const int32_t *begin, const int32_t *pages, int32_t n_prefixes,
                                float *out, void *ws, hipStream_t st)
{
    PrefixArgs a;
    fill_args(a, d, q, pv, nullptr, 0, out, ws);
    a.prefixes = PrefixView{begin, pages, n_prefixes};
    a.inv_group = inverse_of((uint32_t)d.G);
    a.prefix_workgroups = prefix_workgroups(d, n_prefixes);
    a.slots = prefix_slots(d, n_prefixes);
    char *at = static_cast<char *>(ws) + decode_ws_bytes_of(d);
    a.stats = reinterpret_cast<float *>(at);
    at += stats_bytes(d);
    a.piece_weights = reinterpret_cast<float *>(at);
    a.piece_sums = reinterpret_cast<float *>(at + weights_bytes(d, n_prefixes));
    const bool bf = d.dtype == SABLOCK_BF16, wide = prefix_wide(d, n_prefixes);
    const int step = step_rows(bf, d.D, false);
    a.workgroups = workgroups_of(d);
    a.limit = (rows_alone(d) + step - 1) / step;
    const dim3 grid(a.prefix_workgroups + d.P + a.workgroups);
    using Join = void (*)(PrefixArgs);
    const Join join = wide ? (d.D <= 128 ? join_kernel<32, 32, wide_columns(128)> : join_kernel<16, 32, wide_columns(256)>)
                    : prefix_tiles(bf, d.D) == 1 ? join_kernel<16, 16, TILE> : step == 32 ? join_kernel<32, 32, 2 * TILE> : join_kernel<16, 16, 2 * TILE>;
#define SABLOCK_PREFIX(BV, EV, WV)                                                                                                            \
    if (bf == BV && d.D == EV * 16 && wide == WV)                                                                                             \
        hipLaunchKernelGGL((decode_paged_kernel<BV, EV, step_rows(BV, EV * 16, false), true, PrefixPart<BV, EV, WV>>), grid, dim3(NT), 0, st, \
                           PrefixPart<BV, EV, WV>{a});
#define SABLOCK_PREFIX_F(EV) SABLOCK_PREFIX(false, EV, false)
#define SABLOCK_PREFIX_B(EV) SABLOCK_PREFIX(true, EV, true) SABLOCK_PREFIX(true, EV, false) SABLOCK_PREFIX_F(EV)
    SABLOCK_PREFIX_F(1) SABLOCK_PREFIX_B(2) SABLOCK_PREFIX_F(3) SABLOCK_PREFIX_B(4) SABLOCK_PREFIX_F(5) SABLOCK_PREFIX_B(6) SABLOCK_PREFIX_F(7) SABLOCK_PREFIX_B(8)
    SABLOCK_PREFIX_F(9) SABLOCK_PREFIX_B(10) SABLOCK_PREFIX_F(11) SABLOCK_PREFIX_B(12) SABLOCK_PREFIX_F(13) SABLOCK_PREFIX_B(14) SABLOCK_PREFIX_F(15) SABLOCK_PREFIX_B(16)
#undef SABLOCK_PREFIX_B
#undef SABLOCK_PREFIX_F
#undef SABLOCK_PREFIX
    hipLaunchKernelGGL(join, dim3(d.G, d.P), dim3(MERGE_T), 0, st, a);
    return hipGetLastError();
}

}  // namespace sablock
