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
// slots 0 to 3 of either half: turned right by 4 r bits it has slot r's two codes as sign
// and magnitude in bits 15, 0-2 and 31, 16-18, which are the fp16 numbers code * 2^-24:
// an instruction to turn and one to mask make an operand register.
//   row      r of a page is token 4 i + 2 c + o of 16 t ..: t = r / 16, i = r / 4 mod 4, c = r / 2 mod 2, o = r mod 2
//   keys     lane (g, u) = 4 g + u has rows with 2 t + o = g: word i, slots c and 2 + c, are
//            entries 4 u, 4 u + 1 and 4 u + 2, 4 u + 3 in the two halves
//   values   lane (g, t): word i, slots 2 c and 2 c + 1, are entries g and g + 8 in half o
//   scales   of row r at (2 t + o) * 8 + 2 i + c
// With 8 entries, two rows' words are one: word i / 2, slots 2 (i mod 2) + c, are entries
// 2 u, 2 u + 1 of a key in the two halves, or entry g of a value in half o.
// So four consecutive tokens (eight) share eight words of keys and eight of values, and
// one thread writes either (a unit).
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
    static constexpr int kUnit = kGroup == 16 ? 4 : 8; // rows that share words
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

// Slot r of half h of a word: where a code's magnitude and its sign are.
__host__ __device__ constexpr int slot_shift(int r, int h) { return 16 * h + 4 * r; }
__host__ __device__ constexpr int slot_sign(int r, int h) { return (15 + 16 * h + 4 * r) % 32; }
__host__ __device__ constexpr uint32_t slot_mask(int r, int h) { return 7u << slot_shift(r, h) | 1u << slot_sign(r, h); }

// Word j (of 8) of a unit: the row in the unit and the entry that slot r of half h holds.
template <int GS, bool VALUES>
__host__ __device__ constexpr int word_row(int j, int r, int h)
{
    return GS == 16 ? (VALUES ? 2 * (r >> 1) + h : (j >> 2) + 2 * (r & 1)) : VALUES ? 2 * r + h : (j >> 2) + 2 * r;
}
template <int GS, bool VALUES>
__host__ __device__ constexpr int word_entry(int j, int r, int h)
{
    return VALUES ? j + (GS == 16 ? 8 * (r & 1) : 0) : GS == 16 ? 4 * (j & 3) + 2 * (r >> 1) + h : 2 * (j & 3) + h;
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

// A unit on its way into a block: eight words of its keys or values.
template <int GS, bool VALUES>
struct UnitWords {
    static constexpr int kRows = GS == 16 ? 4 : 8;
    uint32_t w[8];
    __device__ __forceinline__ UnitWords()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            w[j] = 0u;
    }
    // Row k (a constant) of the unit; returns its scale.
    __device__ __forceinline__ float add(const float (&x)[GS], int k)
    {
        uint32_t a = 0u;
#pragma unroll
        for (int i = 0; i < GS; ++i)
            a = max(a, magnitude(x[i]));
        const float s = group_scale(a);
        uint32_t code[GS];  // magnitude, sign at bit 31
#pragma unroll
        for (int i = 0; i < GS; ++i) {
            const float q = s > 0.f ? fminf(rintf(__fdiv_rn(fabsf(x[i]), s)), 7.f) : 0.f;
            code[i] = (uint32_t)q | (q > 0.f ? __float_as_uint(x[i]) & 0x80000000u : 0u);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (word_row<GS, VALUES>(j, r, h) == k) {
                        const uint32_t c = code[word_entry<GS, VALUES>(j, r, h)];
                        w[j] |= (c & 7u) << slot_shift(r, h) | (c >> 31) << slot_sign(r, h);
                    }
        return s;
    }
    // Rows of which `has` has no bit keep their codes.
    __device__ __forceinline__ void store(unsigned char *block, int row0, unsigned has) const
    {
        unsigned char *at = block + (VALUES ? kPage * GS / 2 : 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t *p = reinterpret_cast<uint32_t *>(at + word_offset<GS, VALUES>(row0, j));
            uint32_t x = w[j];
            if (has != (1u << kRows) - 1u) {
                uint32_t mask = 0u;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        mask |= has >> word_row<GS, VALUES>(j, r, h) & 1u ? slot_mask(r, h) : 0u;
                x = (*p & ~mask) | (x & mask);
            }
            *p = x;
        }
    }
};

template <int GS, bool VALUES>
__device__ __forceinline__ uint16_t *scales_of(unsigned char *block)
{
    return reinterpret_cast<uint16_t *>(block + kPage * GS + (VALUES ? 2 * kPage : 0));
}

// Quantises rows row0 .. (a unit's; row(k, x) fetches row k of it) into a block.
template <int GS, bool VALUES, typename Row>
__device__ __forceinline__ void write_unit(unsigned char *block, int row0, unsigned has, const Row &row)
{
    UnitWords<GS, VALUES> u;
    uint16_t *scales = scales_of<GS, VALUES>(block);
#pragma unroll
    for (int k = 0; k < UnitWords<GS, VALUES>::kRows; ++k)
        if (has >> k & 1u) {
            float x[GS];
            row(k, x);
            scales[scale_index(row0 + k)] = (uint16_t)(__float_as_uint(u.add(x, k)) >> 16);  // (a bf16 number)
        }
    u.store(block, row0, has);
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
                if (word_row<GS, VALUES>(j, r, h) == k) {
                    const float y = (float)((w >> slot_shift(r, h)) & 7u) * s;
                    x[word_entry<GS, VALUES>(j, r, h)] = w >> slot_sign(r, h) & 1u ? -y : y;
                }
    }
}

// All rows of a unit; put(k, x) takes row k.
template <int GS, bool VALUES, typename Put>
__device__ __forceinline__ void read_unit(const unsigned char *block, int row0, const Put &put)
{
    constexpr int U = GS == 16 ? 4 : 8;
    const unsigned char *at = block + (VALUES ? kPage * GS / 2 : 0);
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        w[j] = *reinterpret_cast<const uint32_t *>(at + word_offset<GS, VALUES>(row0, j));
    const uint16_t *scales = scales_of<GS, VALUES>(const_cast<unsigned char *>(block));
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const float s = __uint_as_float((uint32_t)scales[scale_index(row0 + k)] << 16);
        float x[GS];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (word_row<GS, VALUES>(j, r, h) == k) {
                        const float y = (float)((w[j] >> slot_shift(r, h)) & 7u) * s;
                        x[word_entry<GS, VALUES>(j, r, h)] = w[j] >> slot_sign(r, h) & 1u ? -y : y;
                    }
        put(k, x);
    }
}

}  // namespace q4
}  // namespace dar
