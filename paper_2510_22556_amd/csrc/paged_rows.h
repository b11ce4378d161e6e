// What the paged cache's writers share: elements of a row in 16-byte pieces, and the page bounds, the least and the largest value of
// every element of K over a page's rows, taken on order-preserving whole numbers (a packed 16-bit minimum serves two bf16 elements) and
// joined over the rows of a workgroup through LDS.
#pragma once

#include "sablock_internal.h"

namespace sablock {
namespace {

constexpr int NT = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr double TURN = 0.15915494309189535, TURN_REST = -9.839338337591243e-18;                // 1 / (2 pi), and what fp64 leaves of it

template <bool BF16> struct Elem;
template <> struct Elem<true> {
    static constexpr int N = 8, BYTES = 2;                     // per 16 bytes, of one
    // signed whole numbers in the order of the values; its own inverse
    static __device__ uint32_t ordered(uint32_t w)
    {
        const s16x2 x = __builtin_bit_cast(s16x2, w);
        return __builtin_bit_cast(uint32_t, x ^ ((x >> 15) & (short)0x7fff));
    }
    static __device__ uint32_t lower(uint32_t a, uint32_t b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
    }
    static __device__ uint32_t upper(uint32_t a, uint32_t b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
    }
    static constexpr uint32_t LEAST = 0x80008000u, MOST = 0x7fff7fffu;
    static __device__ float get(const u32x4 &v, int e) { return __uint_as_float((e & 1) ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
    static __device__ u32x4 pack(const float (&x)[8])          // rounded to nearest, ties to even
    {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
        return o;
    }
    // cosine and sine of position * freq.  The fraction of a turn, sine and cosine in fp32: off by 2^-22, which rows of 8 bits do not show
    static __device__ float2 turn(double position, float freq)
    {
        const double turns = position * ((double)freq * TURN);
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        return make_float2(cs, sn);
    }
};
template <> struct Elem<false> {
    static constexpr int N = 4, BYTES = 4;
    static __device__ uint32_t ordered(uint32_t w) { return w ^ ((uint32_t)((int32_t)w >> 31) & 0x7fffffffu); }
    static __device__ uint32_t lower(uint32_t a, uint32_t b) { return (uint32_t)min((int32_t)a, (int32_t)b); }
    static __device__ uint32_t upper(uint32_t a, uint32_t b) { return (uint32_t)max((int32_t)a, (int32_t)b); }
    static constexpr uint32_t LEAST = 0x80000000u, MOST = 0x7fffffffu;
    static __device__ float get(const u32x4 &v, int e) { return __uint_as_float(v[e]); }
    static __device__ u32x4 pack(const float (&x)[4])
    {
        return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
    // The angle as the fp64 number that it is, its fraction of a turn to 2^-53 of one however many there are, less the nearest quarter.  What is left, at
    // most pi / 4, as the sum h + l of two fp32 numbers; sine and cosine by the first terms of their series (the next are below 2^-32 of them), with
    // what l and the roundings of the large terms leave out put back: off by 0.75 and 0.6 units in the last place at most, on average by as much as fp64
    // rounded once.  (In fp64 throughout, the registers would leave room for a workgroup less.)
    static __device__ float2 turn(double position, float freq)
    {
        const double angle = position * (double)freq, part = fma(angle, TURN_REST, fma(angle, TURN, -rint(angle * TURN)));
        const double quarters = rint(4.0 * part), r = (part - 0.25 * quarters) * 6.283185307179586;
        const float h = (float)r, l = (float)(r - (double)h), z = h * h, zl = fmaf(h, h, -z) + 2.f * h * l;
        float sn = fmaf(z, -1.f / 39916800, 1.f / 362880), cs = fmaf(z, -1.f / 3628800, 1.f / 40320);
        sn = fmaf(z, sn, -1.f / 5040);
        cs = fmaf(z, cs, -1.f / 720);
        sn = fmaf(z, sn, 1.f / 120);
        cs = fmaf(z, cs, 1.f / 24);
        sn = fmaf(z, sn, -1.f / 6);
        const float most = fmaf(z, -0.5f, 1.f), rest = (1.f - most) - 0.5f * z;
        const float s = h + fmaf(h * z, sn, l * most), c = most + (fmaf(zl, -0.5f, rest) + z * z * cs);
        const int q = (int)quarters & 3;                       // the pair turned by a quarter: (c, s) -> (-s, c)
        const float x = q & 1 ? s : c, y = q & 1 ? c : s;
        return make_float2(q == 1 || q == 2 ? -x : x, q & 2 ? -y : y);
    }
};

template <bool BF16> struct Bounds {                           // of the elements of one 16-byte chunk, as ordered whole numbers
    using E = Elem<BF16>;
    u32x4 lo, hi;
    __device__ void clear()
    {
        lo = u32x4{E::MOST, E::MOST, E::MOST, E::MOST};
        hi = u32x4{E::LEAST, E::LEAST, E::LEAST, E::LEAST};
    }
    __device__ void add(const u32x4 &v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = E::ordered(v[i]);
            lo[i] = E::lower(lo[i], x);
            hi[i] = E::upper(hi[i], x);
        }
    }
    __device__ void merge_stored(const u32x4 &l, const u32x4 &h)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = E::lower(lo[i], E::ordered(l[i]));
            hi[i] = E::upper(hi[i], E::ordered(h[i]));
        }
    }
    __device__ void store(char *b, int row_bytes) const
    {
        u32x4 l, h;
#pragma unroll
        for (int i = 0; i < 4; ++i) { l[i] = E::ordered(lo[i]); h[i] = E::ordered(hi[i]); }
        *reinterpret_cast<u32x4 *>(b) = l;
        *reinterpret_cast<u32x4 *>(b + row_bytes) = h;
    }
};

// Bounds of a workgroup's chunks over its row groups, sh[group][place], written where at(place) says (nullptr: nowhere), joined with what is
// there if `extend`.  A thread joins one dword of one place: consecutive lanes, consecutive banks.
template <bool BF16, typename At>
__device__ void store_joined(const Bounds<BF16> &b, uint32_t *sh, int groups, int places, int group, int place, bool active, int row_bytes, bool extend, At &&at)
{
    using E = Elem<BF16>;
    __syncthreads();
    if (active) {
        u32x4 *o = reinterpret_cast<u32x4 *>(sh) + (group * places + place) * 2;
        o[0] = b.lo;
        o[1] = b.hi;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < places * 8; i += NT) {
        const int w = i & 7;
        char *dst = at(i >> 3);
        if (!dst) continue;
        uint32_t x = sh[i];
        auto join = [&](uint32_t y) { x = w < 4 ? E::lower(x, y) : E::upper(x, y); };
#pragma unroll 4
        for (int g = 1; g < groups; ++g) join(sh[g * places * 8 + i]);
        uint32_t *word = reinterpret_cast<uint32_t *>(dst + (w < 4 ? 0 : row_bytes)) + (w & 3);
        if (extend) join(E::ordered(*word));
        *word = E::ordered(x);
    }
}

__device__ __forceinline__ char *bounds_at(const PageDims &d, const PageView &v, int32_t layer, int32_t id, int32_t head)
{
    return v.bounds + (((int64_t)layer * d.n_pages + id) * d.Hkv + head) * 2 * d.D * elt_bytes(d);
}

}  // namespace
}  // namespace sablock
