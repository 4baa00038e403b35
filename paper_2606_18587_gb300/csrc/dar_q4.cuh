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
// where the lanes of a warp want them as operands of mma.sync (dar_q4_decode.cu),
// lane 4 g + t with one 16-byte load for all 64 tokens of a group:
//   keys    lane (g, t) holds entries 4 t .. 4 t + 3 of tokens 8 g .. 8 g + 7, a word for
//           two consecutive tokens: the even one's codes as sign and magnitude in bits 7
//           and 0-2 of each byte, the odd one's in the same places of the word turned
//           right by four bits.  As an e4m3 number such a byte is code * 2^-9.
//   values  lane (g, t) holds entries g and g + 8 of tokens 16 t .. 16 t + 15 as code + 8:
//           tokens 16 t + 2 i + {0, 1} and 16 t + 8 + 2 i + {0, 1} are bytes 0 to 3 of
//           word i, entry g the low half of a byte.  (Of a d_down of 8, a byte is two
//           tokens' entry g.)
// Two consecutive tokens from an even row on share words, so one thread writes both.
#pragma once

#include "dar_common.cuh"

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
};

// The scale of a group whose largest magnitude has the bits `a` (of NaN and infinity the group is NaN).
__device__ __forceinline__ float group_scale(uint32_t a)
{
    if (a >= 0x7f800000u)
        return __uint_as_float(0x7fc00000u);
    uint32_t u = __float_as_uint(__fdiv_rn(__uint_as_float(a), 7.0f));
    u = (u + 0x3ffffu + ((u >> 19) & 1u)) & ~0x7ffffu;     // nearest even at 5 significant bits
    return fminf(__uint_as_float(u), 0x1.2p125f);          // 7 s is finite in bf16
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Codes of a group of GS entries; returns its scale.
template <int GS>
__device__ __forceinline__ float quantise(const float (&x)[GS], int (&code)[GS])
{
    uint32_t a = 0u;
#pragma unroll
    for (int i = 0; i < GS; ++i)
        a = max(a, magnitude(x[i]));
    const float s = group_scale(a);
#pragma unroll
    for (int i = 0; i < GS; ++i)
        code[i] = s > 0.f ? (int)fminf(fmaxf(rintf(__fdiv_rn(x[i], s)), -7.f), 7.f) : 0;
    return s;
}

// Offsets within a block: the word of a token pair's four key entries from 4 t on, and the 16-bit unit (8 bits where a
// group has 8 entries) of the pair's value entries gg (and gg + 8).  r: row of the pair's first token, even.
template <int GS>
__device__ __forceinline__ int key_word(int r, int t)
{
    return (r >> 3) * (4 * GS) + t * 16 + ((r >> 1) & 3) * 4;
}
template <int GS>
__device__ __forceinline__ int value_unit(int r, int gg)
{
    const int t = r >> 4, h = (r >> 3) & 1, i = (r >> 1) & 3;
    return GS == 16 ? (gg * 4 + t) * 16 + i * 4 + 2 * h : (gg * 4 + t) * 8 + (i >> 1) * 4 + 2 * h + (i & 1);
}

// Writes the keys' (VALUES: the values') codes and scales of rows r and r + 1 (r even) into a block; `has`: bit 0 for
// row r, bit 1 for row r + 1.  The other one's codes stay.
template <int GS, bool VALUES>
__device__ __forceinline__ void write_pair(unsigned char *block, int r, unsigned has, const int (&c0)[GS],
                                           const int (&c1)[GS], float s0, float s1)
{
    constexpr int kCodes = kPage * GS / 2;
    unsigned char *at = block + (VALUES ? kCodes : 0);
    if constexpr (!VALUES) {
#pragma unroll
        for (int t = 0; t < GS / 4; ++t) {
            uint32_t x0 = 0u, x1 = 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int p = c0[4 * t + e], q = c1[4 * t + e];
                x0 |= ((uint32_t)abs(p) | (p < 0 ? 0x80u : 0u)) << (8 * e);
                x1 |= ((uint32_t)abs(q) | (q < 0 ? 0x80u : 0u)) << (8 * e);
            }
            uint32_t *w = reinterpret_cast<uint32_t *>(at + key_word<GS>(r, t));
            const uint32_t x = x0 | __funnelshift_l(x1, x1, 4);
            if (has == 3u)
                *w = x;
            else if (has == 1u)
                *w = (*w & ~0x87878787u) | x0;
            else
                *w = (*w & 0x87878787u) | __funnelshift_l(x1, x1, 4);
        }
    } else if constexpr (GS == 16) {
#pragma unroll
        for (int gg = 0; gg < 8; ++gg) {
            const uint32_t x0 = (c0[gg] + 8) | (c0[gg + 8] + 8) << 4, x1 = (c1[gg] + 8) | (c1[gg + 8] + 8) << 4;
            unsigned char *u = at + value_unit<16>(r, gg);
            if (has == 3u)
                *reinterpret_cast<uint16_t *>(u) = (uint16_t)(x0 | x1 << 8);
            else
                u[has == 1u ? 0 : 1] = (unsigned char)(has == 1u ? x0 : x1);
        }
    } else {
#pragma unroll
        for (int gg = 0; gg < 8; ++gg) {
            const uint32_t x0 = c0[gg] + 8, x1 = (c1[gg] + 8) << 4;
            unsigned char *u = at + value_unit<8>(r, gg);
            *u = (unsigned char)(has == 3u ? x0 | x1 : has == 1u ? (*u & 0xf0u) | x0 : (*u & 0x0fu) | x1);
        }
    }
    uint16_t *sc = reinterpret_cast<uint16_t *>(block + 2 * kCodes + (VALUES ? 2 * kPage : 0)) + r;
    const uint32_t b0 = __float_as_uint(s0) >> 16, b1 = __float_as_uint(s1) >> 16;  // (a scale is a bf16 number)
    if (has == 3u)
        *reinterpret_cast<uint32_t *>(sc) = b0 | b1 << 16;
    else if (has == 1u)
        sc[0] = (uint16_t)b0;
    else
        sc[1] = (uint16_t)b1;
}

// The values that rows r and r + 1 (r even) of a block stand for.
template <int GS, bool VALUES>
__device__ __forceinline__ void read_pair(const unsigned char *block, int r, float (&x0)[GS], float (&x1)[GS])
{
    constexpr int kCodes = kPage * GS / 2;
    const unsigned char *at = block + (VALUES ? kCodes : 0);
    const uint32_t sc = *reinterpret_cast<const uint32_t *>(block + 2 * kCodes + (VALUES ? 2 * kPage : 0) + 2 * r);
    const float s0 = bf16lo(sc), s1 = bf16hi(sc);
    if constexpr (!VALUES) {
#pragma unroll
        for (int t = 0; t < GS / 4; ++t) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(at + key_word<GS>(r, t));
            const uint32_t v = __funnelshift_r(w, w, 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y0 = (float)((w >> (8 * e)) & 7u) * s0, y1 = (float)((v >> (8 * e)) & 7u) * s1;
                x0[4 * t + e] = (w >> (8 * e)) & 0x80u ? -y0 : y0;
                x1[4 * t + e] = (v >> (8 * e)) & 0x80u ? -y1 : y1;
            }
        }
    } else {
#pragma unroll
        for (int gg = 0; gg < 8; ++gg) {
            const unsigned char *p = at + value_unit<GS>(r, gg);
            if constexpr (GS == 16) {
                const uint32_t u = *reinterpret_cast<const uint16_t *>(p);
                x0[gg] = (float)((int)(u & 15u) - 8) * s0;
                x0[gg + 8] = (float)((int)(u >> 4 & 15u) - 8) * s0;
                x1[gg] = (float)((int)(u >> 8 & 15u) - 8) * s1;
                x1[gg + 8] = (float)((int)(u >> 12) - 8) * s1;
            } else {
                x0[gg] = (float)((int)(*p & 15u) - 8) * s0;
                x1[gg] = (float)((int)(*p >> 4) - 8) * s1;
            }
        }
    }
}

}  // namespace q4
}  // namespace dar
