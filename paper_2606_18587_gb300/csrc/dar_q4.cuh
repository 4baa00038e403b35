// dar_q4.cuh -- bottleneck vectors held in 4 bits: the groups, their codes and
// scales, and where a page keeps them.
//
// 16 consecutive entries of a vector (the 8 of a d_down of 8) are a group:
//   a = max |x|,  s = a / 7 rounded to 5 significant bits,  code = x / s rounded, in [-7, 7].
// Five bits of s and three of a code make a value code * s of at most 8 significant
// bits: every stored value is a bf16 number, so that reading back is exact, and
// quantising what was read back gives the same codes (7 s / 7 is s).  The maximum
// keeps the code 7 whichever way s was rounded: a / s lies in 7 (1 +- 2^-5).
//
// A page of one KV head is kBlock bytes for every 16 entries (8): codes of the keys,
// codes of the values, 64 scales of the keys, 64 of the values (bf16).  Codes lie
// where the lanes of a warp want them as operands of mma.sync (dar_q4_decode.cu), all
// 64 tokens of a group with one load of 16 bytes (8) a lane.  A word is eight codes, in
// slots 0 to 3 of either half: slot r is bits 4 r .. 4 r + 3, code + 8.  fp16 numbers are
// linear in their lowest 11 bits, so that slots 0 and 1 are (code + 8) 2^-24 and 2^-20 where
// they lie, and slots 2 and 3 shifted right by 8: an AND each and a shift make four operand
// registers.  The products take the offset back.
//   row      r of a page is token 4 i + 2 c + o of 16 t ..: t = r / 16, i = r / 4 mod 4, c = r / 2 mod 2, o = r mod 2
//   keys     lane (g, u) = 4 g + u has rows with 2 t + o = g: word i, slots c and 2 + c, are
//            entries 4 u, 4 u + 1 and 4 u + 2, 4 u + 3 in the two halves
//   values   lane (g, t): word i, slots 2 c and 2 c + 1, are entries e = 4 (g / 2) + g mod 2 and e + 2 in half o
//   scales   of row r at (2 t + o) * 8 + 2 i + c
// With 8 entries, two rows' words are one: word i / 2, slots 2 (i mod 2) + c, are entries
// 2 u, 2 u + 1 of a key in the two halves, or entry g of a value in half o.
// So four consecutive tokens (eight) share eight words of keys and eight of values: a unit,
// which one thread writes where few tokens come; pages are written and read by warps.
#pragma once

#include "dar_common.cuh"
#include "dar_sm100.cuh"

namespace dar {
namespace q4 {

template <int DD>
struct Fmt {
    static constexpr int kGroup = DD < 16 ? DD : 16;   // entries that share a scale
    static constexpr int kGroups = DD / kGroup;        // of a vector
    static constexpr int kCodes = kPage * kGroup / 2;  // bytes of codes of a page's keys (values) of a group
    static constexpr int kScales = 2 * kCodes;         // offset of the keys' scales; the values' are kPage * 2 behind
    static constexpr int kBlock = 2 * kCodes + 4 * kPage;
    static constexpr int kBytes = kGroups * kBlock;    // of a page of one KV head
    static constexpr int kUnit = kGroup == 16 ? 4 : 8; // rows that share words
};

// Bits of a quotient rounded to a scale: 5 significant bits, nearest even; 7 s is finite in bf16.
__device__ __forceinline__ float round_scale(uint32_t u)
{
    u = (u + 0x3ffffu + ((u >> 19) & 1u)) & ~0x7ffffu;
    return fminf(__uint_as_float(u), 0x1.2p125f);
}

// The scale of a group whose largest magnitude has the bits `a` (of NaN and infinity the group is NaN).
__device__ __forceinline__ float group_scale(uint32_t a)
{
    if (a >= 0x7f800000u)
        return __uint_as_float(0x7fc00000u);
    return round_scale(__float_as_uint(__fdiv_rn(__uint_as_float(a), 7.0f)));
}

// The same of a bf16 number without a division.  a has 8 significant bits: where a / 7 does not lie halfway between two
// scales, it lies 2^-12 of itself away at least, so that the product's rounding error goes with the bits below 2^-13.
// (Subnormal quotients have fewer bits: from 2^-100 down it is a division.)
__device__ __forceinline__ float group_scale_bf16(uint32_t a)
{
    if (a - 0x0d800000u >= 0x7f800000u - 0x0d800000u)
        return group_scale(a);
    const uint32_t u = __float_as_uint(__uint_as_float(a) * (1.0f / 7.0f));
    return round_scale((u + 0x200u) & ~0x3ffu);
}

// x / s of two entries, rounded, plus 8 in either half.  The quotient is a product with 1 / s; exact: on bf16
// numbers, whose quotients lie 2^-11 away from halves at least where they are no halves, its error goes with a rounding
// to 2^-13.  Else by division (rounded to 24 bits it is on the same side of a half as the quotient).
__device__ __forceinline__ uint32_t codes_bf16(float x, float y, float inv)
{
    constexpr float kGrid = 1536.f, kInt = 8388616.f;  // 1.5 * 2^10, 2^23 + 8
    const float a = fmaf(x, inv, kGrid) - kGrid + kInt, b = fmaf(y, inv, kGrid) - kGrid + kInt;
    return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410);
}
__device__ __forceinline__ uint32_t code_of(float x, float s)
{
    return s > 0.f ? (uint32_t)((int)fminf(fmaxf(rintf(__fdiv_rn(x, s)), -7.f), 7.f) + 8) : 8u;
}

// The same for s from 2^-126 on, with inv close to 1 / s (1 ulp): the product lies 2^-20 from the quotient at most, and
// where that could be on the other side of a half there is a division.
__device__ __forceinline__ uint32_t code_near(float x, float s, float inv)
{
    const float q = x * inv, r = rintf(q);
    return fabsf(q - r) <= 0.5f - 0x1p-16f ? (uint32_t)((int)r + 8) : code_of(x, s);
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Where slot r of half h of a word is.
__host__ __device__ constexpr int slot_shift(int r, int h) { return 16 * h + 4 * r; }

// Word j (of 8) of a unit: the row in the unit and the entry that slot r of half h holds.
template <int GS, bool VALUES>
__host__ __device__ constexpr int word_row(int j, int r, int h)
{
    return GS == 16 ? (VALUES ? 2 * (r >> 1) + h : (j >> 2) + 2 * (r & 1)) : VALUES ? 2 * r + h : (j >> 2) + 2 * r;
}
template <int GS, bool VALUES>
__host__ __device__ constexpr int word_entry(int j, int r, int h)
{
    return VALUES ? (GS == 16 ? 4 * (j >> 1) + (j & 1) + 2 * (r & 1) : j) : GS == 16 ? 4 * (j & 3) + 2 * (r >> 1) + h : 2 * (j & 3) + h;
}
// Its offset in the block's keys (values); row0: the unit's first row.
template <int GS, bool VALUES>
__device__ __forceinline__ int word_offset(int row0, int j)
{
    const int t = row0 >> 4, lane = VALUES ? j * 4 + t : (2 * t + (j >> 2)) * 4 + (j & 3);
    return GS == 16 ? lane * 16 + ((row0 >> 2) & 3) * 4 : lane * 8 + ((row0 >> 3) & 1) * 4;
}
__device__ __forceinline__ int scale_index(int row)
{
    return (2 * (row >> 4) + (row & 1)) * 8 + 2 * ((row >> 2) & 3) + ((row >> 1) & 1);
}

template <int GS, bool VALUES>
__device__ __forceinline__ uint16_t *scales_of(unsigned char *block)
{
    return reinterpret_cast<uint16_t *>(block + kPage * GS + (VALUES ? 2 * kPage : 0));
}

// The values that a row of a block stands for.
template <int GS, bool VALUES>
__device__ __forceinline__ void read_row(const unsigned char *block, int row, float (&x)[GS])
{
    constexpr int U = GS == 16 ? 4 : 8;
    const int row0 = row & ~(U - 1), k = row - row0;
    const float s = __uint_as_float((uint32_t)scales_of<GS, VALUES>(const_cast<unsigned char *>(block))[scale_index(row)] << 16);
    const unsigned char *at = block + (VALUES ? kPage * GS / 2 : 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (!VALUES && (j >> 2) != (row & 1))
            continue;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(at + word_offset<GS, VALUES>(row0, j));
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (word_row<GS, VALUES>(j, r, h) == k)
                    x[word_entry<GS, VALUES>(j, r, h)] = (float)((int)((w >> slot_shift(r, h)) & 15u) - 8) * s;
    }
}

// ------------------------------------------------------------------ pages, by warps
//
// Lane (g, u) has entries 4 u .. 4 u + 3 (of 8: 2 u, 2 u + 1) of rows with 2 t + o = g.  As pairs (two codes in the
// form of a word's slot 0) they are the slots of its words of keys, and transposed those of its words of values.

// A pair's codes as numbers (2^23 + code + 8 less 2^23 + 8).
__device__ __forceinline__ void pair_numbers(uint32_t x, float &a, float &b)
{
    a = __uint_as_float((x & 15u) | 0x4b000000u) - 8388616.f;
    b = __uint_as_float((x >> 16) | 0x4b000000u) - 8388616.f;
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ int lane_row(int g, int i, int c) { return 16 * (g >> 1) + 4 * i + 2 * c + (g & 1); }

// Entries of a lane's rows as they come from memory: pairs of T.
template <typename T, int GS>
struct Raw;
template <int GS>
struct Raw<bf16, GS> {
    static constexpr int N = GS / 8;  // pairs
    uint32_t w[N];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            w[i] = 0u;
    }
    __device__ __forceinline__ void load(const bf16 *p)
    {
        if constexpr (N == 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x, w[1] = v.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        }
    }
    // The pairs' codes, and the group's scale in 16 bits; all lanes.
    __device__ __forceinline__ uint32_t codes(uint32_t (&x)[N]) const
    {
        uint32_t m = w[0] & 0x7fff7fffu;
        if constexpr (N == 2)
            m = __vmaxu2(m, w[N - 1] & 0x7fff7fffu);
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const uint32_t a = max(m << 16, m & 0xffff0000u);
        const float s = group_scale_bf16(a);
        if (a - 0x0d800000u < 0x7f800000u - 0x0d800000u) {
            float inv;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
#pragma unroll
            for (int i = 0; i < N; ++i)
                x[i] = codes_bf16(bf16lo(w[i]), bf16hi(w[i]), inv);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                x[i] = code_of(bf16lo(w[i]), s) | code_of(bf16hi(w[i]), s) << 16;
        }
        return __float_as_uint(s) >> 16;
    }
    static __device__ __forceinline__ void store(bf16 *p, const uint32_t (&x)[N], float s)
    {
        uint32_t y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float a, b;
            pair_numbers(x[i], a, b);
            y[i] = sm100::cvt_bf16x2(a * s, b * s);
        }
        if constexpr (N == 2)
            *reinterpret_cast<uint2 *>(p) = make_uint2(y[0], y[N - 1]);
        else
            *reinterpret_cast<uint32_t *>(p) = y[0];
    }
};
template <int GS>
struct Raw<float, GS> {
    static constexpr int N = GS / 8;
    float w[2 * N];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 2 * N; ++i)
            w[i] = 0.f;
    }
    __device__ __forceinline__ void load(const float *p)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 v = reinterpret_cast<const float2 *>(p)[i];
            w[2 * i] = v.x, w[2 * i + 1] = v.y;
        }
    }
    __device__ __forceinline__ uint32_t codes(uint32_t (&x)[N]) const
    {
        uint32_t a = 0u;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i)
            a = max(a, magnitude(w[i]));
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
        const float s = group_scale(a);
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s >= 0x1p-126f ? s : __uint_as_float(0x7fc00000u)));
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = code_near(w[2 * i], s, inv) | code_near(w[2 * i + 1], s, inv) << 16;
        return __float_as_uint(s) >> 16;
    }
    static __device__ __forceinline__ void store(float *p, const uint32_t (&x)[N], float s)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float a, b;
            pair_numbers(x[i], a, b);
            reinterpret_cast<float2 *>(p)[i] = make_float2(a * s, b * s);
        }
    }
};

// bf16: the maxima of a page's 64 groups, whose quarter of each lane u of (g, u) reduces, end with lane u having those of
// rows i = u: three exchanges, and two scales a lane instead of eight, each four times.  False where one of them is
// infinite, NaN or tiny (the rows' own path then).  sc[0]: the scales of the lane's two rows, inv: 1 / them.
template <typename T, int GS>
__device__ __forceinline__ bool even_page(const Raw<T, GS> (&raw)[4][2], int lane, uint32_t (&sc)[4], float (&inv)[2])
{
    if constexpr (sizeof(T) != 2) {
        return false;
    } else {
        constexpr int N = GS / 8;
        uint32_t m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t x[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                x[c] = raw[i][c].w[0] & 0x7fff7fffu;
                if constexpr (N == 2)
                    x[c] = __vmaxu2(x[c], raw[i][c].w[N - 1] & 0x7fff7fffu);
            }
            m[i] = __vmaxu2(__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[0], x[1], 0x7632));
        }
        const bool u0 = lane & 1, u1 = lane & 2;
        const uint32_t a = __vmaxu2(u0 ? m[1] : m[0], __shfl_xor_sync(0xffffffffu, u0 ? m[0] : m[1], 1));
        const uint32_t b = __vmaxu2(u0 ? m[3] : m[2], __shfl_xor_sync(0xffffffffu, u0 ? m[2] : m[3], 1));
        const uint32_t r = __vmaxu2(u1 ? b : a, __shfl_xor_sync(0xffffffffu, u1 ? a : b, 2));
        const uint32_t top[2] = {r << 16, r & 0xffff0000u};
        bool fine = true;
        float s[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            fine &= top[c] == 0u || top[c] - 0x0d800000u < 0x7f800000u - 0x0d800000u;
            s[c] = round_scale((__float_as_uint(__uint_as_float(top[c]) * (1.0f / 7.0f)) + 0x200u) & ~0x3ffu);
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv[c]) : "f"(s[c]));
            inv[c] = s[c] > 0.f ? inv[c] : 0.f;
        }
        sc[0] = __byte_perm(__float_as_uint(s[0]), __float_as_uint(s[1]), 0x7632);
        return __all_sync(0xffffffffu, fine);
    }
}
template <typename T, int GS>
__device__ __forceinline__ void even_codes(const Raw<T, GS> (&raw)[2], int from, const float (&inv)[2], uint32_t (&x)[2][GS / 8])
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float v = __shfl_sync(0xffffffffu, inv[c], from);
#pragma unroll
            for (int k = 0; k < GS / 8; ++k)
                x[c][k] = codes_bf16(bf16lo(raw[c].w[k]), bf16hi(raw[c].w[k]), v);
        }
    }
}

// Writes the bits `mask` of a word of codes.  Sequences that list a page together write rows of the same word at the same
// time, each those that it has: two atomic operations on its own bits lose nobody's (bits of a row that two of them have
// come out alike in any order, since both write the same).
__device__ __forceinline__ void put_word(uint32_t *p, uint32_t x, uint32_t mask)
{
    if (mask == ~0u) {
        *p = x;
    } else if (mask) {
        atomicAnd(p, x | ~mask);
        atomicOr(p, x & mask);
    }
}

// Quantises rows [first, end) of a page into a block; row r's entries are at vec + r * stride.
template <typename T, int GS, bool VALUES>
__device__ __forceinline__ void write_page(unsigned char *block, const T *vec, int stride, int first, int end, int lane)
{
    constexpr int N = GS / 8;
    const int g = lane >> 2, u = lane & 3;
    Raw<T, GS> raw[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int r = lane_row(g, i, c);
            raw[i][c].zero();
            if (r >= first && r < end)
                raw[i][c].load(vec + (size_t)r * stride + u * 2 * N);
        }
    uint32_t w[4], sc[4];
    float inv[2];
    const bool even = even_page<T, GS>(raw, lane, sc, inv);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t x[2][N];
        if (even) {
            even_codes<T, GS>(raw[i], (lane & ~3) + i, inv, x);
        } else {
            const uint32_t s0 = raw[i][0].codes(x[0]), s1 = raw[i][1].codes(x[1]);
            sc[i] = s0 | s1 << 16;
        }
        if constexpr (VALUES) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int k = 0; k < N; ++k)
                    x[c][k] = transpose8(x[c][k]);
        }
        if constexpr (GS == 16) {  // slots: keys c + 2 k, values 2 c + k
            const uint32_t y1 = VALUES ? x[0][N - 1] : x[1][0], y2 = VALUES ? x[1][0] : x[0][N - 1];
            w[i] = x[0][0] | y1 << 4 | y2 << 8 | x[1][N - 1] << 12;
        } else {
            const uint32_t y = x[0][0] | x[1][0] << 4;
            w[i] = i % 2 ? w[i - i % 2] | y << 8 : y;
        }
    }
    constexpr int kCodes = kPage * GS / 2;
    unsigned char *at = block + (VALUES ? kCodes : 0) + lane * GS;
    uint16_t *scales = scales_of<GS, VALUES>(block) + g * 8;
    if (first <= 0 && end >= kPage) {
        if constexpr (GS == 16)
            *reinterpret_cast<uint4 *>(at) = make_uint4(w[0], w[1], w[2], w[3]);
        else
            *reinterpret_cast<uint2 *>(at) = make_uint2(w[1], w[3]);
        if (even)
            reinterpret_cast<uint32_t *>(scales)[u] = sc[0];
        else if (u == 0)
            *reinterpret_cast<uint4 *>(scales) = make_uint4(sc[0], sc[1], sc[2], sc[3]);
        return;
    }
    uint32_t *words = reinterpret_cast<uint32_t *>(at);
#pragma unroll
    for (int i = 0; i < (GS == 16 ? 4 : 2); ++i) {
        const int row0 = VALUES ? 16 * u : 16 * (g >> 1);
        uint32_t mask = 0u;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = row0 + (GS == 16 ? 4 : 8) * i + word_row<GS, VALUES>(VALUES ? 0 : 4 * (g & 1), r, h);
                mask |= row >= first && row < end ? 15u << slot_shift(r, h) : 0u;
            }
        put_word(words + i, w[GS == 16 ? i : 2 * i + 1], mask);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int r = lane_row(g, i, c);
            if (u == (even ? i : 0) && r >= first && r < end)
                scales[2 * i + c] = (uint16_t)((even ? sc[0] : sc[i]) >> (16 * c));
        }
}

// Reads rows [first, end) of a block back.
template <typename T, int GS, bool VALUES>
__device__ __forceinline__ void read_page(const unsigned char *block, T *vec, int stride, int first, int end, int lane)
{
    constexpr int N = GS / 8, kCodes = kPage * GS / 2;
    const int g = lane >> 2, u = lane & 3;
    const unsigned char *at = block + (VALUES ? kCodes : 0) + lane * GS;
    uint32_t w[4];
    if constexpr (GS == 16) {
        const uint4 v = *reinterpret_cast<const uint4 *>(at);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
        const uint2 v = *reinterpret_cast<const uint2 *>(at);
        w[0] = v.x, w[1] = v.x >> 8, w[2] = v.y, w[3] = v.y >> 8;
    }
    const uint4 v = *reinterpret_cast<const uint4 *>(scales_of<GS, VALUES>(const_cast<unsigned char *>(block)) + g * 8);
    const uint32_t sc[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t x[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int r = GS == 16 ? (VALUES ? 2 * c + k : c + 2 * k) : c;
                x[k] = (w[i] >> (4 * r)) & 0x000f000fu;
                if constexpr (VALUES)
                    x[k] = transpose8(x[k]);
            }
            const int row = lane_row(g, i, c);
            if (row >= first && row < end)
                Raw<T, GS>::store(vec + (size_t)row * stride + u * 2 * N, x, c ? bf16hi(sc[i]) : bf16lo(sc[i]));
        }
}

}  // namespace q4
}  // namespace dar
