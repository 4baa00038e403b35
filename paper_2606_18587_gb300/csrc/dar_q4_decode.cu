// dar_q4_decode.cu -- one decode step over a cache whose pages hold 4 bits an entry
// (dar_q4.cuh): Eq. 3-4 for the query at position L_b - 1, with the ring in the
// storage type.  With a stored key code_k s_k and q~ = q Uk^T, a distant token's
// score is sum over groups of s_k (q~_group . code_k), and the sums that Uv lifts
// are sum_j (p_j s_v,j) code_v,j: scales multiply scores and weights, one per group,
// and the products take the codes themselves.
//
// Two kernels on the caller's stream, the second launched programmatically:
//
//  attend  The work is a line of units (sequence, KV head, up to kRows query heads):
//          the ring in runs of kRun tokens, then the pages.  Every warp of the grid has
//          an equal share of the line by cost, and leaves one partial result (m, l,
//          acc) per query head for each unit that its share cuts; unit u's cut by
//          share k has the slot u + k.  The shares of a unit's first and last stage leave
//          their numbers for the joining kernel.  Lengths are read on the device.
//  join    a block per output row joins its partial results by log-sum-exp and lifts the
//          bottleneck sum once by Uv.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_q4.cuh"
#include "dar_sm100.cuh"

namespace dar {
namespace q4 {

using namespace sm100;

constexpr int kRows = 8;         // query heads of a unit at most
constexpr int kRun = 16;         // ring tokens of a stage
constexpr int kWarps = 8;        // of a CTA (CUDA cores)
// Of a CTA (tensor cores), and stages in flight of each: as many warps as registers allow.
template <int DD>
__host__ __device__ constexpr int mma_warps() { return DD <= 16 ? 16 : 12; }
template <int DD>
__host__ __device__ constexpr int mma_slots() { return DD <= 16 ? 2 : 3; }
constexpr int kSlot = 5120;      // bytes of a stage at most
constexpr int kMaxShares = 2560; // the workspace holds partial results of this many warps
constexpr int kCostUnit = 8;     // cost of a unit's set-up (its place on the line is before the stages)
constexpr int kCostRun = 8;      // of kRun ring tokens
template <int DD>
__host__ __device__ constexpr int cost_page() { return DD == 8 ? 4 : 5 * DD / 16; }

template <int DD>
__host__ __device__ constexpr int rec_floats() { return 4 + kHeadDim + DD; }

struct Args {
    Q4DecodeArgs c;
    int2 *span;  // [units] first and last share of every unit
    float *rec;  // [units + shares][rows of a unit][rec_floats]
    int G, RT, RU;  // query heads per KV head, units per (sequence, KV head), rows of a unit at most
    int shares;
};

// ------------------------------------------------------------------ the line

struct Tables {  // in shared memory, B entries each, and the total
    int *L, *start, *total;
};

__device__ __forceinline__ Tables tables_at(int *p, int B) { return Tables{p, p + B, p + 2 * B}; }

__device__ __forceinline__ int runs_of(int L, int w) { return (min(L, w) + kRun - 1) / kRun; }
__device__ __forceinline__ int pages_of(int L, int w) { return L > w ? (L - w + kPage - 1) / kPage : 0; }

template <int DD>
__device__ __forceinline__ int unit_length(int L, int w)
{
    return L > 0 ? kCostUnit + runs_of(L, w) * kCostRun + pages_of(L, w) * cost_page<DD>() : 0;
}

// Lengths and the places of the sequences' units on the line, the same in every CTA.
template <int DD>
__device__ void build_tables(const Args &a, const Tables &t)
{
    const int tid = threadIdx.x, lane = tid & 31;
    for (int b = tid; b < a.c.B; b += blockDim.x) {
        int L = a.c.seq_lens[b];
        if (L < 0 || (long long)L > (long long)a.c.maxp * kPage + a.c.w) {
            if (blockIdx.x == 0)
                report(a.c.status, DAR_ERR_CAPACITY);
            L = 0;
        }
        t.L[b] = L;
    }
    __syncthreads();
    if (tid < 32) {
        int run = 0;
        for (int b0 = 0; b0 < a.c.B; b0 += 32) {
            const int b = b0 + lane, v = b < a.c.B ? a.c.Hkv * a.RT * unit_length<DD>(t.L[b], a.c.w) : 0;
            int x = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o)
                    x += y;
            }
            if (b < a.c.B)
                t.start[b] = run + x - v;
            run += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0)
            *t.total = run;
    }
    __syncthreads();
}

// A share's cut of a unit: its stages [st0, st1), runs of the ring first and then pages.
struct Cut {
    int b, g, rt, rows;
    int unit, slot;
    int L, nwin, nrun;  // tokens, those in the ring, its runs
    int st0, st1;
    bool first, last;   // the unit's first, last stage is in the cut
};

// The cuts of share k, in order.
struct Walk {
    int p, hi, k;
    template <int DD>
    static __device__ __forceinline__ int shares(const Args &a, const Tables &t)
    {
        // a share holds a whole stage at least, so every share between a unit's first and last has one of it
        constexpr int most = kCostRun > cost_page<DD>() ? kCostRun : cost_page<DD>();
        return max(1, min(a.shares, *t.total / most));
    }
    template <int DD>
    __device__ __forceinline__ void begin(const Args &a, const Tables &t, int share)
    {
        const int n = shares<DD>(a, t);
        k = share;
        p = k < n ? (int)((long long)*t.total * k / n) : 0;
        hi = k < n ? (int)((long long)*t.total * (k + 1) / n) : 0;
    }
    template <int DD>
    __device__ __forceinline__ bool next(const Args &a, const Tables &t, Cut &c)
    {
        while (p < hi) {
            int lo = 0, up = a.c.B - 1;  // the last sequence that starts at or before p (empty ones share a start)
            while (lo < up) {
                const int mid = (lo + up + 1) >> 1;
                if (t.start[mid] <= p)
                    lo = mid;
                else
                    up = mid - 1;
            }
            c.b = lo;
            c.L = t.L[lo];
            c.nwin = min(c.L, a.c.w);
            c.nrun = runs_of(c.L, a.c.w);
            const int pages = pages_of(c.L, a.c.w), len = unit_length<DD>(c.L, a.c.w);
            const int u = (p - t.start[lo]) / len, from = p - t.start[lo] - u * len;
            const int to = min(len, from + hi - p);
            c.g = u / a.RT;
            c.rt = u % a.RT;
            c.rows = min(kRows, a.G - c.rt * kRows);
            c.unit = lo * a.c.Hkv * a.RT + u;
            c.slot = c.unit + k;
            auto stage = [&](int at) {  // the first stage whose place is at or behind `at`
                const int x = at - kCostUnit, y = x - c.nrun * kCostRun;
                if (x <= 0)
                    return 0;
                return y <= 0 ? (x + kCostRun - 1) / kCostRun
                              : c.nrun + min(pages, (y + cost_page<DD>() - 1) / cost_page<DD>());
            };
            c.st0 = stage(from);
            c.st1 = to == len ? c.nrun + pages : stage(to);
            c.first = c.st0 == 0;
            c.last = c.st1 == c.nrun + pages;
            p += to - from;
            if (c.st0 < c.st1)
                return true;
        }
        return false;
    }
};

__device__ __forceinline__ void leave_span(const Args &a, const Cut &c, int share)
{
    if (c.first)
        a.span[c.unit].x = share;
    if (c.last)
        a.span[c.unit].y = share;
}

// ------------------------------------------------------------------ attend, CUDA cores
//
// A warp takes two tokens a lane for the scores; for the sums a lane has an entry (of 64
// tokens' weights, through shared memory).
struct LaneSmem {
    float q[kRows][kHeadDim], qt[kRows][kHeadDim];
    float p[kRows][kPage], x[kPage][16];
    float sv[kPage];
};

template <typename T, int DD>
__device__ __forceinline__ void attend_lanes(const Args &a, const Tables &t, LaneSmem &s)
{
    using F = Fmt<DD>;
    constexpr int GS = F::kGroup, NB = F::kGroups, HALVES = 32 / GS;  // lanes that share an entry
    const int lane = threadIdx.x & 31, share = blockIdx.x * kWarps + (threadIdx.x >> 5);
    Walk walk;
    walk.begin<DD>(a, t, share);
    for (Cut c; walk.next<DD>(a, t, c);) {
        if (lane == 0)
            leave_span(a, c, share);
        __syncwarp();
        const size_t row0 = (size_t)c.b * a.c.Hq + c.g * a.G + c.rt * kRows;
        for (int i = lane; i < kRows * kHeadDim; i += 32) {
            const int r = i / kHeadDim;
            s.q[r][i % kHeadDim] =
                r < c.rows ? to_f32(static_cast<const T *>(a.c.q)[(row0 + r) * kHeadDim + i % kHeadDim]) : 0.f;
        }
        __syncwarp();
        for (int i = lane; i < kRows * DD; i += 32) {
            const int r = i / DD, e = i % DD;
            float x[4] = {0.f, 0.f, 0.f, 0.f};
            if (r < c.rows) {
                const float4 *u = reinterpret_cast<const float4 *>(a.c.Uk + ((size_t)c.g * DD + e) * kHeadDim);
                const float4 *q = reinterpret_cast<const float4 *>(s.q[r]);
#pragma unroll 4
                for (int k = 0; k < kHeadDim / 4; ++k) {
                    const float4 uu = __ldg(u + k), qq = q[k];
                    x[0] = fmaf(uu.x, qq.x, x[0]);
                    x[1] = fmaf(uu.y, qq.y, x[1]);
                    x[2] = fmaf(uu.z, qq.z, x[2]);
                    x[3] = fmaf(uu.w, qq.w, x[3]);
                }
            }
            s.qt[r][e] = (x[0] + x[1]) + (x[2] + x[3]);
        }
        __syncwarp();
        float m[kRows], l[kRows], ol[kRows][2], od[kRows][NB];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            m[r] = -INFINITY;
            l[r] = ol[r][0] = ol[r][1] = 0.f;
#pragma unroll
            for (int i = 0; i < NB; ++i)
                od[r][i] = 0.f;
        }
        // weights of up to two tokens a lane (scores y0 of tokens 2 lane and y1 of 2 lane + 1, -inf: none)
        auto weigh = [&](int r, float y0, float y1) {
            float top = fmaxf(y0, y1);
#pragma unroll
            for (int o = 16; o; o >>= 1)
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float mn = fmaxf(m[r], top), base = mn == -INFINITY ? 0.f : mn, f = exp2f(m[r] - base);
            const float p0 = exp2f(y0 - base), p1 = exp2f(y1 - base);
            m[r] = mn;
            l[r] = l[r] * f + (p0 + p1);
            ol[r][0] *= f;
            ol[r][1] *= f;
#pragma unroll
            for (int i = 0; i < NB; ++i)
                od[r][i] *= f;
            s.p[r][2 * lane] = p0;
            s.p[r][2 * lane + 1] = p1;
        };
        for (int st = c.st0; st < c.st1; ++st) {
            if (st < c.nrun) {
                const int t0 = st * kRun, n = min(kRun, c.nwin - t0);
                const size_t ring = (((size_t)c.b * a.c.Hkv + c.g) * a.c.w + t0) * kHeadDim;
                const T *k = static_cast<const T *>(a.c.win_k) + ring, *v = static_cast<const T *>(a.c.win_v) + ring;
                float y[kRows][2];
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    y[r][0] = y[r][1] = -INFINITY;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int tok = 2 * lane + e;
                    if (tok >= n)
                        continue;
                    float x[kRows] = {};
                    constexpr int E = Granule<T>::kElems;
#pragma unroll 2
                    for (int i = 0; i < kHeadDim / E; ++i) {
                        float kk[E];
                        unpack(reinterpret_cast<const uint4 *>(k + tok * kHeadDim)[i], kk, T());
#pragma unroll
                        for (int r = 0; r < kRows; ++r)
#pragma unroll
                            for (int j = 0; j < E; ++j)
                                x[r] = fmaf(s.q[r][i * E + j], kk[j], x[r]);
                    }
#pragma unroll
                    for (int r = 0; r < kRows; ++r)
                        y[r][e] = x[r] * a.c.c2;
                }
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    weigh(r, y[r][0], y[r][1]);
                __syncwarp();
                for (int tok = 0; tok < n; ++tok) {
                    const float v0 = to_f32(v[tok * kHeadDim + lane]), v1 = to_f32(v[tok * kHeadDim + 32 + lane]);
#pragma unroll
                    for (int r = 0; r < kRows; ++r) {
                        const float p = s.p[r][tok];
                        ol[r][0] = fmaf(p, v0, ol[r][0]);
                        ol[r][1] = fmaf(p, v1, ol[r][1]);
                    }
                }
                __syncwarp();
                continue;
            }
            const int lp = st - c.nrun, n = min(kPage, c.L - c.nwin - lp * kPage);
            const int id = a.c.block_table[(size_t)c.b * a.c.maxp + lp];
            if (id < 0 || id >= a.c.num_pages) {
                if (lane == 0)
                    report(a.c.status, DAR_ERR_CAPACITY);
                continue;
            }
            const unsigned char *page =
                static_cast<const unsigned char *>(a.c.pool) + ((size_t)id * a.c.Hkv + c.g) * F::kBytes;
            float y[kRows][2] = {};
#pragma unroll 1
            for (int i = 0; i < NB; ++i) {
                float x0[GS], x1[GS];
                read_row<GS, false>(page + i * F::kBlock, 2 * lane, x0);
                read_row<GS, false>(page + i * F::kBlock, 2 * lane + 1, x1);
#pragma unroll
                for (int r = 0; r < kRows; ++r)
#pragma unroll
                    for (int e = 0; e < GS; ++e) {
                        const float q = s.qt[r][i * GS + e];
                        y[r][0] = fmaf(q, x0[e], y[r][0]);
                        y[r][1] = fmaf(q, x1[e], y[r][1]);
                    }
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                weigh(r, 2 * lane < n ? y[r][0] * a.c.c2 : -INFINITY, 2 * lane + 1 < n ? y[r][1] * a.c.c2 : -INFINITY);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                float x0[GS], x1[GS];
                read_row<GS, true>(page + i * F::kBlock, 2 * lane, x0);
                read_row<GS, true>(page + i * F::kBlock, 2 * lane + 1, x1);
                __syncwarp();
#pragma unroll
                for (int e = 0; e < GS; ++e) {  // rows behind the last token may hold anything
                    s.x[2 * lane][e] = 2 * lane < n ? x0[e] : 0.f;
                    s.x[2 * lane + 1][e] = 2 * lane + 1 < n ? x1[e] : 0.f;
                }
                __syncwarp();
                for (int tok = lane / GS; tok < kPage; tok += HALVES) {
                    const float v = s.x[tok][lane % GS];
#pragma unroll
                    for (int r = 0; r < kRows; ++r)
                        od[r][i] = fmaf(s.p[r][tok], v, od[r][i]);
                }
            }
            __syncwarp();
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
#pragma unroll
            for (int o = 16; o; o >>= 1)
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int o = 16; o >= GS; o >>= 1)
                    od[r][i] += __shfl_xor_sync(0xffffffffu, od[r][i], o);
            if (r >= c.rows)
                continue;
            float *rec = a.rec + ((size_t)c.slot * a.RU + r) * rec_floats<DD>();
            if (lane == 0) {
                rec[0] = m[r];
                rec[1] = l[r];
            }
            rec[4 + lane] = ol[r][0];
            rec[4 + 32 + lane] = ol[r][1];
            if (lane < GS)
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    rec[4 + kHeadDim + i * GS + lane] = od[r][i];
        }
    }
}

constexpr size_t lanes_smem(int B) { return kWarps * sizeof(LaneSmem) + (2 * (size_t)B + 1) * 4; }

template <typename T, int DD>
__global__ void __launch_bounds__(kWarps * 32) attend_kernel(Args a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const Tables t = tables_at(reinterpret_cast<int *>(smem + kWarps * sizeof(LaneSmem)), a.c.B);
    grid_dep_launch();
    build_tables<DD>(a, t);
    attend_lanes<T, DD>(a, t, reinterpret_cast<LaneSmem *>(smem)[threadIdx.x >> 5]);
}

// ------------------------------------------------------------------ attend, tensor cores
//
// Up to 8 query heads lie on the N side of mma.sync products (m16n8k16, fp16) with 16 tokens
// on the M side (a tcgen05 tile has 128 rows: most calls have 1 to 8 heads per KV head).
// Column 2 t of a product belongs to head t and column 2 t + 1 to head t + 4, so lane (g, t) =
// 4 g + t has the scores, weights, references and sums of heads t and t + 4 (CT = 2); with CT = 1
// of head t alone, and the other column takes what is said below.
//
//  codes    fp16 subnormals as they lie (dar_q4.cuh): five instructions for the eight of a word of
//           keys, seven for one of values.  (Conversions of offset codes take 13: an AND and an OR each,
//           since an instruction has one immediate, and the offset subtracted; e4m3 operands are
//           converted by twice as many: mma.sync has no products of them here.)
//  scores   q~, brought to [2^14, 2^15) by a power of two, is two fp16 terms (2^-22 of it).  CT = 1:
//           the second one is the other column's.  CT = 2: a product of its own.  A d_down of 8:
//           the two halves of a product's 16 entries.  The sum starts from
//           minus 8 times theirs.  Rows with c = 1 are in slots 1 and 3: their scores are 16 times as large.
//  weights  p s_v as fp16 (2^-11) relative to a reference of the row that keeps the largest at
//           2^8 when it is set and below 2^15 always; it is raised by a vote.  (bf16 operands need two
//           terms for the same error, twice the conversions and transpositions.)

struct Soft {  // of one head of a lane
    float bias, l;  // minus the reference; the lane's share of the sum of weights
};

__device__ __forceinline__ void mma_f16_acc(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma_f16_c(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1,
                                          const float (&c)[4])
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

__device__ __forceinline__ uint32_t cvt_f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Two values as two fp16 terms each, all but 2^-22 of them; the terms are added to their sums.
__device__ __forceinline__ void split_f16(float x, float y, uint32_t &hi, uint32_t &lo, float (&sums)[2])
{
    hi = cvt_f16x2(x, y);
    float a, b, c, d;
    asm("{.reg .b16 p, q; mov.b32 {p, q}, %2; cvt.f32.f16 %0, p; cvt.f32.f16 %1, q;}" : "=f"(a), "=f"(b) : "r"(hi));
    lo = cvt_f16x2(x - a, y - b);
    asm("{.reg .b16 p, q; mov.b32 {p, q}, %2; cvt.f32.f16 %0, p; cvt.f32.f16 %1, q;}" : "=f"(c), "=f"(d) : "r"(lo));
    sums[0] += a + b;
    sums[1] += c + d;
}

// Slots 0 to 3 of a word of keys (slots 1 and 3 times 16) and of values as operand registers.
__device__ __forceinline__ void keys_of(uint32_t w, uint32_t (&c)[4])
{
    c[0] = w & 0x000f000fu;
    c[1] = w & 0x00f000f0u;
    c[2] = (w >> 8) & 0x000f000fu;
    c[3] = (w >> 8) & 0x00f000f0u;
}
__device__ __forceinline__ void values_of(uint32_t w, uint32_t (&c)[4])
{
#pragma unroll
    for (int r = 0; r < 4; ++r)
        c[r] = __funnelshift_r(w, w, 4 * r) & 0x80078007u;
}

// Two fp32 values as three bf16 terms each: all but 2^-24 of them.
__device__ __forceinline__ void split3(float x, float y, uint32_t (&t)[3])
{
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        t[i] = cvt_bf16x2(x, y);
        x -= bf16lo(t[i]);
        y -= bf16hi(t[i]);
    }
}

// 0xffff in the halves whose key (key, key + 1) is below n.
__device__ __forceinline__ uint32_t key_mask(int key, int n)
{
    return (key < n ? 0xffffu : 0u) | (key + 1 < n ? 0xffff0000u : 0u);
}

// What a warp fills its slots with, ahead of what it computes.
template <int DD>
struct Filler {
    static constexpr int kSlots = mma_slots<DD>();
    static constexpr int kPages = Fmt<DD>::kBytes > kSlot / 4 ? kSlot / Fmt<DD>::kBytes : 4;  // of a stage
    Walk walk;
    Cut c;
    int st;          // next stage of the cut
    int ids0, ids;   // block-table entries ids0 .. ids0 + 31 of its sequence, one per lane
    int filled;
    bool more;

    __device__ __forceinline__ void begin(const Args &a, const Tables &t, int share)
    {
        walk.begin<DD>(a, t, share);
        filled = 0;
        next_cut(a, t);
    }
    __device__ __forceinline__ void next_cut(const Args &a, const Tables &t)
    {
        more = walk.next<DD>(a, t, c);
        st = c.st0;
        ids0 = -1;
    }
    // Starts the copies of the next stage.
    __device__ __forceinline__ void fill(const Args &a, const Tables &t, const CUtensorMap &wk, const CUtensorMap &wv,
                                         unsigned char *slots, uint64_t *full, uint64_t policy, int lane)
    {
        if (!more)
            return;
        unsigned char *dst = slots + filled % kSlots * kSlot;
        uint64_t *bar = full + filled % kSlots;
        ++filled;
        if (st < c.nrun) {
            if (lane == 0) {
                mbar_expect_tx(bar, 2 * kRun * kHeadDim * 2);
                const int y = (c.b * a.c.Hkv + c.g) * a.c.w + st * kRun;
                tma_load_2d_hint(smem_u32(dst), &wk, 0, y, bar, policy);
                tma_load_2d_hint(smem_u32(dst + kRun * kHeadDim * 2), &wv, 0, y, bar, policy);
            }
            ++st;
        } else {
            const int lp = st - c.nrun, n = min(kPages, c.st1 - st);
            if (ids0 < 0 || lp + n > ids0 + 32) {
                ids0 = lp;
                ids = lp + lane < a.c.maxp ? __ldg(a.c.block_table + (size_t)c.b * a.c.maxp + lp + lane) : -1;
            }
            const int id = __shfl_sync(0xffffffffu, ids, (lp - ids0 + lane) & 31);
            const bool mine = lane < n, good = mine && id >= 0 && id < a.c.num_pages;
            const unsigned pages = __popc(__ballot_sync(0xffffffffu, good));
            if (lane == 0)
                mbar_expect_tx(bar, pages * Fmt<DD>::kBytes);
            __syncwarp();
            if (good)
                bulk_g2s_hint(dst + lane * Fmt<DD>::kBytes,
                              static_cast<const unsigned char *>(a.c.pool) + ((size_t)id * a.c.Hkv + c.g) * Fmt<DD>::kBytes,
                              Fmt<DD>::kBytes, bar, policy);
            else if (mine)
                report(a.c.status, DAR_ERR_CAPACITY);
            st += n;
        }
        if (st >= c.st1)
            next_cut(a, t);
    }
};

// What a warp has of a cut's query heads, and its sums.
template <int DD, int CT>
struct Heads {
    static constexpr int GS = Fmt<DD>::kGroup, NB = Fmt<DD>::kGroups;
    static constexpr int TB = GS == 16 && CT == 2 ? 2 : 1;  // score products of a group
    static constexpr int OD = CT == 1 ? 2 : 1;    // sums of a group (see page_step)
    uint32_t q[4][2];        // ring: queries as B operands
    uint32_t qt[NB][TB][2];  // pages: q~ as B operands, two fp16 terms
    float from[NB][4];       // what a score's sum starts from
    float cq[CT];            // scale of a score: c2, the power of two taken out of q~, and the codes' 2^24
    Soft ring[CT], page[CT];
    float ol[kHeadDim / 16][4], od[NB][OD][4];

    // Queries of a cut, and q~^T = Uk q^T with Uk in three bf16 terms (products exact but for 2^-24).
    __device__ __forceinline__ void begin(const Args &a, const Cut &c, int lane)
    {
        const int i0 = lane >> 2, c0 = lane & 3;
        const int head = (i0 >> 1) + 4 * (i0 & 1);  // of column i0
        const uint32_t *qp = static_cast<const uint32_t *>(a.c.q) +
                             ((size_t)c.b * a.c.Hq + c.g * a.G + c.rt * kRows + head) * (kHeadDim / 2) + c0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            q[e / 2][e % 2] = head < c.rows ? __ldg(qp + 4 * e) : 0u;
        float x[NB][4];  // entries 16 j + i0 (+ 8) of heads c0, c0 + 4: [0] i0 c0, [1] i0 c0 + 4, [2], [3] i0 + 8
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const float *u = a.c.Uk + ((size_t)c.g * DD + 16 * j + i0) * kHeadDim + 2 * c0;
            float z[3][4] = {};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t t[4][3];
#pragma unroll
                for (int y = 0; y < 4; ++y) {  // entries i0, i0 + 8 and inputs 2 c, 2 c + 8
                    float2 v = make_float2(0.f, 0.f);
                    if (GS == 16 || y % 2 == 0)
                        v = __ldg(reinterpret_cast<const float2 *>(u + (y & 1) * 8 * kHeadDim + 16 * e + 8 * (y >> 1)));
                    split3(v.x, v.y, t[y]);
                }
#pragma unroll
                for (int y = 0; y < 3; ++y) {
                    const uint32_t ua[4] = {t[0][y], t[1][y], t[2][y], t[3][y]};
                    mma_bf16_acc(z[y], ua, q[e][0], q[e][1]);
                }
            }
#pragma unroll
            for (int y = 0; y < 4; ++y)
                x[j][y] = z[0][y] + (z[1][y] + z[2][y]);
        }
        // the largest entry of each head, and the power of two that brings it to [2^14, 2^15)
        float up[CT];
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            uint32_t top = 0u;
#pragma unroll
            for (int j = 0; j < NB; ++j)
                top = max(top, max(magnitude(x[j][k]), magnitude(x[j][2 + k])));
#pragma unroll
            for (int o = 4; o < 32; o <<= 1)
                top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const int e = max((int)(top >> 23) - 127, -100);
            up[k] = __uint_as_float((uint32_t)(127 + 14 - e) << 23);  // e <= 127: 2^-113 at least
            // infinite or NaN: so are all scores
            cq[k] = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u)
                                       : a.c.c2 * __uint_as_float((uint32_t)(127 + e) << 23) * 1024.f;
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                x[j][k] *= up[k];
                x[j][2 + k] *= up[k];
            }
        }
        // column i0 of a score product wants consecutive entries of its head, i0 / 2 (+ 4 in odd columns): four
        // from 4 c0 on, or of a d_down of 8 two from 2 c0 on
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            constexpr int NE = GS == 16 ? 4 : 2;
            float y[NE];
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const int from = ((NE * c0 + e) & 7) * 4 + (i0 >> 1);
                float z[CT];
#pragma unroll
                for (int k = 0; k < CT; ++k) {
                    z[k] = __shfl_sync(0xffffffffu, x[j][k], from);
                    if constexpr (GS == 16) {
                        const float hi = __shfl_sync(0xffffffffu, x[j][2 + k], from);
                        z[k] = c0 < 2 ? z[k] : hi;
                    }
                }
                y[e] = CT == 2 && (i0 & 1) ? z[CT - 1] : z[0];  // (with CT = 1 the odd columns are not used)
            }
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < NE / 2; ++e) {
                uint32_t hi, lo;
                float sums[2] = {0.f, 0.f};
                split_f16(y[2 * e], y[2 * e + 1], hi, lo, sums);
                if constexpr (GS == 8) {
                    qt[j][0][0] = hi;
                    qt[j][0][1] = lo;
                } else if constexpr (CT == 2) {
                    qt[j][0][e] = hi;
                    qt[j][TB - 1][e] = lo;
                } else {
                    qt[j][0][e] = i0 & 1 ? lo : hi;
                }
                sum += CT == 2 || GS == 8 ? sums[0] + sums[1] : i0 & 1 ? sums[1] : sums[0];
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                from[j][k] = -0x1p-21f * __shfl_sync(0xffffffffu, sum, (2 * c0 + k) * 4);  // 8 * 2^-24
                from[j][2 + k] = 16.f * from[j][k];
            }
        }
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            ring[k].bias = page[k].bias = INFINITY;
            ring[k].l = page[k].l = 0.f;
        }
#pragma unroll
        for (int e = 0; e < kHeadDim / 16; ++e)
            ol[e][0] = ol[e][1] = ol[e][2] = ol[e][3] = 0.f;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int o = 0; o < OD; ++o)
                od[j][o][0] = od[j][o][1] = od[j][o][2] = od[j][o][3] = 0.f;
    }

    // A run of n ring tokens at `tile`: 16 rows of keys, then of values, 128-byte swizzle.
    __device__ __forceinline__ void ring_step(uint32_t tile, int n, float c2, int lane)
    {
        const int i0 = lane >> 2, c0 = lane & 3, mat = lane >> 3, r = lane & 7;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        const uint32_t krow = tile + (r + 8 * (mat & 1)) * 128;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t k[4];
            ldsm_x4(krow + (((2 * e + (mat >> 1)) ^ r) << 4), k);
            mma_bf16_acc(s, k, q[e][0], q[e][1]);
        }
        uint32_t w0[2], w1[2];  // weights as two bf16 terms: tokens i0, and i0 + 8
        float p[2][2] = {};
        bool up = false;
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            s[k] = i0 < n ? s[k] * c2 : -INFINITY;
            s[2 + k] = i0 + 8 < n ? s[2 + k] * c2 : -INFINITY;
            up |= fmaxf(s[k], s[2 + k]) > -ring[k].bias;
        }
        if (__any_sync(0xffffffffu, up)) {
#pragma unroll
            for (int k = 0; k < CT; ++k) {
                float top = fmaxf(s[k], s[2 + k]);
#pragma unroll
                for (int o = 4; o < 32; o <<= 1)
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float was = -ring[k].bias, now = fmaxf(top, was), f = now == -INFINITY ? 1.f : ex2_approx(was - now);
                ring[k].bias = -now;
                ring[k].l *= f;
#pragma unroll
                for (int e = 0; e < kHeadDim / 16; ++e) {
                    ol[e][k] *= f;
                    ol[e][2 + k] *= f;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            const float bias = ring[k].bias == INFINITY ? 0.f : ring[k].bias;
            p[0][k] = ex2_approx(s[k] + bias);
            p[1][k] = ex2_approx(s[2 + k] + bias);
            ring[k].l += p[0][k] + p[1][k];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // hi cut off, so that both terms have the weight's sign; 2^-22 of it keeps lo from 0, where an infinite
            // value would become NaN
            constexpr float kUp = 1.f + 0x1p-22f;
            const uint32_t x = __float_as_uint(p[h][0]), y = __float_as_uint(p[h][1]);
            uint32_t &hi = h ? w1[0] : w0[0], &lo = h ? w1[1] : w0[1];
            hi = transpose8(__byte_perm(x, y, 0x7632));
            lo = transpose8(cvt_bf16x2(fmaf(p[h][0], kUp, -__uint_as_float(x & 0xffff0000u)),
                                       fmaf(p[h][1], kUp, -__uint_as_float(y & 0xffff0000u))));
        }
        const uint32_t m0 = key_mask(2 * c0, n), m1 = key_mask(2 * c0 + 8, n);  // 0 * NaN is NaN
        const uint32_t vrow = tile + kRun * kHeadDim * 2 + (r + 8 * (mat >> 1)) * 128;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t v[4];
            ldsm_x4_t(vrow + (((2 * e + (mat & 1)) ^ r) << 4), v);
            const uint32_t vm[4] = {v[0] & m0, v[1] & m0, v[2] & m1, v[3] & m1};
            mma_bf16_acc(ol[e], vm, w0[0], w1[0]);
            mma_bf16_acc(ol[e], vm, w0[1], w1[1]);
        }
    }

    // The lane's words of a page's keys or values: four, or of a d_down of 8 two, each twice.
    static __device__ __forceinline__ void load_words(const unsigned char *at, int lane, uint32_t (&w)[4])
    {
        if constexpr (GS == 16) {
            const uint4 v = *reinterpret_cast<const uint4 *>(at + lane * 16);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2 *>(at + lane * 8);
            w[0] = w[1] = v.x, w[2] = w[3] = v.y;
        }
    }

    // A page of n tokens; lane (g, t) has the scores of rows 16 (g / 2) + 4 i + 2 c + g mod 2.  Products of weights: with
    // CT = 2 a column has 8 tokens' weights of head t or t + 4.  With CT = 1 column 2 t has those of rows with c = 0 and
    // column 2 t + 1 those with c = 1, which one transposition brings; products with the codes of c = 0 are right in the
    // even columns and products with those of c = 1 in the odd ones, so each has sums of its own, whose other columns are
    // not used.
    __device__ __forceinline__ void page_step(const unsigned char *at, int n, int lane)
    {
        using F = Fmt<DD>;
        const int i0 = lane >> 2, c0 = lane & 3;
        // pairs: two tokens (c = 0, 1) of a head, or two heads of a token; pair i, or pairs 2 i, 2 i + 1
        constexpr int NP = 4 * CT;
        float y[NP][2];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const unsigned char *block = at + j * F::kBlock;
            const uint4 sw = *reinterpret_cast<const uint4 *>(block + F::kScales + i0 * 16);
            const uint32_t sc[4] = {sw.x, sw.y, sw.z, sw.w};
            uint32_t w[4];
            load_words(block, lane, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t c[4];
                keys_of(w[i], c);
                if constexpr (GS == 8) {  // both halves of the product's 16 entries are the key's 8
                    c[0] = i % 2 ? c[2] : c[0];
                    c[1] = i % 2 ? c[3] : c[1];
                    c[2] = c[0];
                    c[3] = c[1];
                }
                float d[4];
                mma_f16_c(d, c, qt[j][0][0], qt[j][0][1], from[j]);
                if constexpr (TB == 2)
                    mma_f16_acc(d, c, qt[j][TB - 1][0], qt[j][TB - 1][1]);
                const float s0 = bf16lo(sc[i]), s1 = bf16hi(sc[i]);
                if constexpr (CT == 1) {
                    const float x0 = GS == 16 ? d[0] + d[1] : d[0], x1 = GS == 16 ? d[2] + d[3] : d[2];
                    y[i][0] = j ? fmaf(x0, s0, y[i][0]) : x0 * s0;
                    y[i][1] = j ? fmaf(x1, s1, y[i][1]) : x1 * s1;
                } else {
                    float(&u)[2] = y[2 * i], (&v)[2] = y[(2 * i + 1) % NP];
                    if (j == 0) {
                        mul2(u[0], u[1], d[0], d[1], s0, s0);
                        mul2(v[0], v[1], d[2], d[3], s1, s1);
                    } else {
                        ffma2(u[0], u[1], d[0], d[1], s0, s0, u[0], u[1]);
                        ffma2(v[0], v[1], d[2], d[3], s1, s1, v[0], v[1]);
                    }
                }
            }
        }
        uint32_t vs[NB][4];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const uint4 v = *reinterpret_cast<const uint4 *>(at + j * F::kBlock + F::kScales + 2 * kPage + i0 * 16);
            vs[j][0] = v.x, vs[j][1] = v.y, vs[j][2] = v.z, vs[j][3] = v.w;
        }
        if (n < kPage) {  // rows behind the last token may hold anything
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int tok = 16 * (i0 >> 1) + 4 * i + (i0 & 1);  // and tok + 2
                const uint32_t m = (tok < n ? 0xffffu : 0u) | (tok + 2 < n ? 0xffff0000u : 0u);
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    vs[j][i] &= m;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if constexpr (CT == 1) {
                        y[i][e] = tok + 2 * e < n ? y[i][e] : -INFINITY;
                    } else {
                        y[2 * i][e] = tok < n ? y[2 * i][e] : -INFINITY;
                        y[(2 * i + 1) % NP][e] = tok + 2 < n ? y[(2 * i + 1) % NP][e] : -INFINITY;
                    }
                }
            }
        }
        // the largest scales of the tokens' groups
        uint32_t vm[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vm[i] = vs[0][i];
#pragma unroll
            for (int j = 1; j < NB; ++j)
                asm("max.bf16x2 %0, %0, %1;" : "+r"(vm[i]) : "r"(vs[j][i]));
        }
        constexpr float kFar = 32768.f, kFarSum = 0x1p90f;
        float p[NP][2], pw[NP][2], l[2];  // weights, and times vm
        // a pair's scales
        auto scales = [](uint32_t s, int k, float &s0, float &s1) {
            s0 = CT == 1 || k % 2 == 0 ? bf16lo(s) : bf16hi(s);
            s1 = CT == 1 || k % 2 != 0 ? bf16hi(s) : bf16lo(s);
        };
        // scale of a pair's scores: slots of c = 1 are 16 times as large
        auto scale = [&](int k, int e) {
            const float s = cq[CT == 2 ? e : 0];
            return (CT == 1 ? e : k % 2) ? s * 0.0625f : s;
        };
        auto weigh = [&]() {  // returns whether something got far above the reference
            float top = 0.f;
            l[0] = l[1] = 0.f;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                float x0, x1, s0, s1;
                ffma2(x0, x1, y[k][0], y[k][1], scale(k, 0), scale(k, 1), page[0].bias, page[CT - 1].bias);
                p[k][0] = ex2_approx(x0);
                p[k][1] = ex2_approx(x1);
                add2(l[0], l[1], l[0], l[1], p[k][0], p[k][1]);
                scales(vm[k / CT], k, s0, s1);
                mul2(pw[k][0], pw[k][1], p[k][0], p[k][1], s0, s1);
                top = max3(top, pw[k][0], pw[k][1]);
            }
            return fmaxf(l[0], l[1]) > kFarSum || top > kFar;
        };
        if (__any_sync(0xffffffffu, weigh())) {
#pragma unroll
            for (int k = 0; k < CT; ++k) {
                float top = -INFINITY;  // of p s_v, and of 2^-64 p
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (CT == 2 && e != k)
                            continue;
                        float s[2];
                        scales(vm[i / CT], i, s[0], s[1]);
                        top = fmaxf(top, fmaf(y[i][e], scale(i, e), __log2f(fmaxf(0x1p-64f, s[e]))));
                    }
#pragma unroll
                for (int o = 4; o < 32; o <<= 1)
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float was = -page[k].bias, now = fmaxf(was, top - 8.f);
                const float f = now == -INFINITY ? 1.f : ex2_approx(was - now);
                page[k].bias = -now;
                page[k].l *= f;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    od[j][0][k] *= f;
                    od[j][0][2 + k] *= f;
                    if constexpr (CT == 1) {
                        od[j][OD - 1][1] *= f;
                        od[j][OD - 1][3] *= f;
                    }
                }
            }
            weigh();
        }
        if constexpr (CT == 1) {
            page[0].l += l[0] + l[1];
        } else {
            page[0].l += l[0];
            page[CT - 1].l += l[1];
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            uint32_t w[4];
            load_words(at + j * F::kBlock + F::kCodes, lane, w);
            uint32_t b[NP];
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                float s0, s1, w0 = pw[k][0], w1 = pw[k][1];
                if constexpr (NB > 1) {
                    scales(vs[j][k / CT], k, s0, s1);
                    mul2(w0, w1, p[k][0], p[k][1], s0, s1);
                }
                b[k] = transpose8(cvt_f16x2(w0, w1));
            }
            uint32_t v[4][4];  // both entries of the rows of word i with c = 0, and with c = 1
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (GS == 16) {
                    values_of(w[i], v[i]);
                } else if (i % 2 == 0) {
                    uint32_t c[4];
                    values_of(w[i], c);
                    v[i][0] = c[0], v[i][2] = c[1], v[i + 1][0] = c[2], v[i + 1][2] = c[3];
                    v[i][1] = v[i][3] = v[i + 1][1] = v[i + 1][3] = 0u;
                }
            }
            if constexpr (CT == 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mma_f16_acc(od[j][0], v[i], b[2 * i], b[(2 * i + 1) % NP]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const uint32_t even[4] = {v[i][0], v[i][1], v[i + 1][0], v[i + 1][1]};
                    const uint32_t odd[4] = {v[i][2], v[i][3], v[i + 1][2], v[i + 1][3]};
                    mma_f16_acc(od[j][0], even, b[i], b[i + 1]);
                    mma_f16_acc(od[j][OD - 1], odd, b[i], b[i + 1]);
                }
            }
        }
    }

    // The partial result of the cut.
    __device__ __forceinline__ void leave(const Args &a, const Cut &c, int lane)
    {
        const int i0 = lane >> 2, c0 = lane & 3;
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            float lr = ring[k].l, lp = page[k].l;
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                lr += __shfl_xor_sync(0xffffffffu, lr, o);
                lp += __shfl_xor_sync(0xffffffffu, lp, o);
            }
            const int head = c0 + 4 * k;
            if (head >= c.rows)
                continue;
            const float m = fmaxf(-ring[k].bias, -page[k].bias), base = m == -INFINITY ? 0.f : m;
            const float fr = ex2_approx(-ring[k].bias - base), fp = ex2_approx(-page[k].bias - base);
            float *rec = a.rec + ((size_t)c.slot * a.RU + head) * rec_floats<DD>();
            if (i0 == 0) {
                rec[0] = m;
                rec[1] = lr * fr + lp * fp;
            }
#pragma unroll
            for (int e = 0; e < kHeadDim / 16; ++e) {
                rec[4 + 16 * e + i0] = ol[e][k] * fr;
                rec[4 + 16 * e + 8 + i0] = ol[e][2 + k] * fr;
            }
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                float x = od[j][0][k], y = od[j][0][2 + k];
                if constexpr (CT == 1) {
                    x += od[j][OD - 1][1];
                    y += od[j][OD - 1][3];
                }
                const int e = GS == 16 ? 16 * j + 4 * (i0 >> 1) + (i0 & 1) : i0;
                rec[4 + kHeadDim + e] = x * (fp * 0x1p24f);  // (the codes were 2^-24 of themselves)
                if (GS == 16)
                    rec[4 + kHeadDim + e + 2] = y * (fp * 0x1p24f);
            }
        }
    }
};

template <int DD>
constexpr size_t mma_smem(int B)
{
    return 1024 + (size_t)mma_warps<DD>() * mma_slots<DD>() * (kSlot + 8) + 16 + (2 * (size_t)B + 1) * 4;
}

template <int DD, int CT>
__global__ void __launch_bounds__(mma_warps<DD>() * 32, 1)
    attend_mma_kernel(const __grid_constant__ CUtensorMap wk, const __grid_constant__ CUtensorMap wv, const Args a)
{
    constexpr int kMmaWarps = mma_warps<DD>(), kSlots = mma_slots<DD>();
    extern __shared__ unsigned char raw[];
    unsigned char *base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);  // the swizzle's atoms
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, share = blockIdx.x * kMmaWarps + warp;
    unsigned char *slots = base + warp * kSlots * kSlot;
    uint64_t *bars = reinterpret_cast<uint64_t *>(base + kMmaWarps * kSlots * kSlot), *full = bars + warp * kSlots;
    volatile int *gave_up = reinterpret_cast<volatile int *>(bars + kMmaWarps * kSlots);
    const Tables t = tables_at(reinterpret_cast<int *>(bars + kMmaWarps * kSlots + 2), a.c.B);
    grid_dep_launch();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMmaWarps * kSlots; ++i)
            mbar_init(bars + i, 1);
        *gave_up = 0;
        mbar_init_fence();
    }
    build_tables<DD>(a, t);  // its barriers also publish the mbarriers
    const uint64_t once = l2_evict_first_policy();  // the cache is read once
    Filler<DD> fill;
    fill.begin(a, t, share);
#pragma unroll 1
    for (int i = 0; i < kSlots; ++i)
        fill.fill(a, t, wk, wv, slots, full, once, lane);
    Walk walk;
    walk.begin<DD>(a, t, share);
    int n = 0;  // stages taken
    bool alive = true;
    for (Cut c; alive && walk.next<DD>(a, t, c);) {
        if (lane == 0)
            leave_span(a, c, share);
        Heads<DD, CT> h;
        h.begin(a, c, lane);
        for (int st = c.st0; st < c.st1; ++n) {
            const int s = n % kSlots;
            if (!mbar_wait_warp(full + s, (unsigned)((n / kSlots) & 1), gave_up)) {
                alive = false;
                break;
            }
            const unsigned char *slot = slots + s * kSlot;
            if (st < c.nrun) {
                h.ring_step(smem_u32(slot), min(kRun, c.nwin - st * kRun), a.c.c2, lane);
                ++st;
            } else {
                const int pages = min(Filler<DD>::kPages, c.st1 - st);
                for (int i = 0; i < pages; ++i)
                    h.page_step(slot + i * Fmt<DD>::kBytes, min(kPage, c.L - c.nwin - (st - c.nrun + i) * kPage), lane);
                st += pages;
            }
            __syncwarp();  // the slot is read
            fill.fill(a, t, wk, wv, slots, full, once, lane);
        }
        if (alive)
            h.leave(a, c, lane);
    }
    if (!alive) {
        // a wait gave up: the copies in flight land (again a bounded wait) before the warp leaves
        if (lane == 0)
            report(a.c.status, DAR_ERR_DEVICE);
        for (int i = n; i < fill.filled; ++i)
            mbar_wait(full + i % kSlots, (unsigned)((i / kSlots) & 1), nullptr);
    }
}

// ------------------------------------------------------------------ join

// Block i writes output row i: the warps take its partial results in turn, and are joined.
template <typename T, int DD, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) join_kernel(Args a)
{
    constexpr int ND = (DD + 31) / 32, N = 2 + ND;
    __shared__ float part[WARPS][2 + 32 * N], sum[kHeadDim + DD];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x, b = row / a.c.Hq, h = row % a.c.Hq, g = h / a.G, j = h % a.G;
    grid_dep_wait();
    const int L = a.c.seq_lens[b];
    if (L <= 0 || (long long)L > (long long)a.c.maxp * kPage + a.c.w) {  // empty, or refused
        for (int i = threadIdx.x; i < kHeadDim; i += WARPS * 32)
            static_cast<T *>(a.c.out)[(size_t)row * kHeadDim + i] = from_f32<T>(0.f);
        return;
    }
    const int unit = (b * a.c.Hkv + g) * a.RT + j / kRows;
    const int2 span = a.span[unit];
    const int k0 = min(max(span.x, 0), kMaxShares - 1), k1 = min(max(span.y, k0), kMaxShares - 1);
    float m = -INFINITY, l = 0.f, x[N] = {};
    const size_t stride = (size_t)a.RU * rec_floats<DD>();
    const float *rec = a.rec + ((size_t)(unit + k0) * a.RU + j % kRows) * rec_floats<DD>();
    for (int i = warp; i <= k1 - k0; i += WARPS) {
        const float *p = rec + i * stride;
        const float mo = p[0], lo = p[1], mn = fmaxf(m, mo), base = mn == -INFINITY ? 0.f : mn;
        const float f = ex2_approx(m - base), fo = ex2_approx(mo - base);
        m = mn;
        l = l * f + lo * fo;
        x[0] = x[0] * f + p[4 + lane] * fo;
        x[1] = x[1] * f + p[36 + lane] * fo;
#pragma unroll
        for (int e = 0; e < ND; ++e)
            if (32 * e + lane < DD)
                x[2 + e] = x[2 + e] * f + p[4 + kHeadDim + 32 * e + lane] * fo;
    }
    if (lane == 0) {
        part[warp][0] = m;
        part[warp][1] = l;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        part[warp][2 + 32 * e + lane] = x[e];
    __syncthreads();
    float top = -INFINITY, f[WARPS], all = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i)
        top = fmaxf(top, part[i][0]);
    if (top == -INFINITY)
        top = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        f[i] = ex2_approx(part[i][0] - top);
        all = fmaf(part[i][1], f[i], all);
    }
    for (int i = threadIdx.x; i < kHeadDim + DD; i += WARPS * 32) {
        float y = 0.f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k)
            y = fmaf(f[k], part[k][2 + i], y);
        sum[i] = y;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kHeadDim; i += WARPS * 32) {
        float o = sum[i];
#pragma unroll
        for (int e = 0; e < DD; ++e)
            o = fmaf(sum[kHeadDim + e], __ldg(a.c.Uv + ((size_t)g * DD + e) * kHeadDim + i), o);
        static_cast<T *>(a.c.out)[(size_t)row * kHeadDim + i] = from_f32<T>(o / all);
    }
}

// ------------------------------------------------------------------ launch

static size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

struct Layout {
    size_t span, rec, total;
    int RT, RU;
};

static Layout layout(int B, int Hq, int Hkv, int dd)
{
    Layout y;
    const int G = Hq / Hkv;
    y.RU = std::min(G, kRows);
    y.RT = (G + kRows - 1) / kRows;
    const size_t units = (size_t)B * Hkv * y.RT;
    y.span = 0;
    y.rec = up256(units * sizeof(int2));
    y.total = y.rec + up256((units + kMaxShares) * y.RU * (4 + kHeadDim + dd) * sizeof(float));
    return y;
}

template <typename T, int DD>
static cudaError_t launch(const Q4DecodeArgs &c, void *workspace, cudaStream_t s)
{
    const Layout y = layout(c.B, c.Hq, c.Hkv, DD);
    char *ws = static_cast<char *>(workspace);
    Args a;
    a.c = c;
    a.span = reinterpret_cast<int2 *>(ws + y.span);
    a.rec = reinterpret_cast<float *>(ws + y.rec);
    a.G = c.Hq / c.Hkv;
    a.RT = y.RT;
    a.RU = y.RU;
    static PerDeviceOnce once;
    int sms = 0;
    cudaError_t e = per_device_once(
        once,
        [&](int d) {
            cudaError_t e2 = cudaDeviceGetAttribute(&once.value[d], cudaDevAttrMultiProcessorCount, d);
            if constexpr (sizeof(T) == 2) {
                if (e2 == cudaSuccess)
                    e2 = cudaFuncSetAttribute(attend_mma_kernel<DD, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)mma_smem<DD>(DAR_DECODE_MAX_BATCH));
                if (e2 == cudaSuccess)
                    e2 = cudaFuncSetAttribute(attend_mma_kernel<DD, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)mma_smem<DD>(DAR_DECODE_MAX_BATCH));
            } else if (e2 == cudaSuccess) {
                e2 = cudaFuncSetAttribute(attend_kernel<T, DD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                          (int)lanes_smem(DAR_DECODE_MAX_BATCH));
            }
            return e2;
        },
        &sms);
    if (e != cudaSuccess)
        return e;
    if constexpr (sizeof(T) == 2) {
        CUtensorMap wk, wv;
        const unsigned long long rows = (unsigned long long)c.B * c.Hkv * c.w;
        if (!make_tma_2d_bf16(&wk, c.win_k, rows, kHeadDim, kRun) || !make_tma_2d_bf16(&wv, c.win_v, rows, kHeadDim, kRun))
            return cudaErrorInvalidValue;
        constexpr int warps = mma_warps<DD>();
        const int grid = std::min(sms, kMaxShares / warps);
        a.shares = grid * warps;
        if (y.RU <= 4)
            attend_mma_kernel<DD, 1><<<grid, warps * 32, mma_smem<DD>(c.B), s>>>(wk, wv, a);
        else
            attend_mma_kernel<DD, 2><<<grid, warps * 32, mma_smem<DD>(c.B), s>>>(wk, wv, a);
    } else {
        const int grid = std::min(sms, kMaxShares / kWarps);
        a.shares = grid * kWarps;
        attend_kernel<T, DD><<<grid, kWarps * 32, lanes_smem(c.B), s>>>(a);
    }
    e = cudaGetLastError();
    if (e != cudaSuccess)
        return e;
    cudaLaunchAttribute pdl[1];
    pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    pdl[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = s;
    cfg.attrs = pdl;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)(c.B * c.Hq));
    cfg.blockDim = dim3(4 * 32);
    return cudaLaunchKernelEx(&cfg, join_kernel<T, DD, 4>, a);
}

template <typename T>
static cudaError_t launch_t(int dd, const Q4DecodeArgs &a, void *workspace, cudaStream_t s)
{
    switch (dd) {
    case 8: return launch<T, 8>(a, workspace, s);
    case 16: return launch<T, 16>(a, workspace, s);
    case 32: return launch<T, 32>(a, workspace, s);
    case 64: return launch<T, 64>(a, workspace, s);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace q4

size_t q4_decode_workspace_bytes(int B, int Hq, int Hkv, int dd) { return q4::layout(B, Hq, Hkv, dd).total; }

// Upper bound of the line's length: every sequence at capacity.
double q4_decode_line_bound(int B, int Hq, int Hkv, int dd, int w, int maxp)
{
    const int page = dd == 8 ? q4::cost_page<8>() : q4::cost_page<16>() * (dd / 16);
    const double unit = q4::kCostUnit + ((double)w / q4::kRun + 1) * q4::kCostRun + ((double)maxp + 1) * page;
    return (double)B * Hkv * ((Hq / Hkv + q4::kRows - 1) / q4::kRows) * unit;
}

cudaError_t launch_decode_q4(dar_dtype dt, int dd, const Q4DecodeArgs &a, void *workspace, cudaStream_t s)
{
    if (a.B == 0)
        return cudaSuccess;
    return dt == DAR_F32 ? q4::launch_t<float>(dd, a, workspace, s) : q4::launch_t<bf16>(dd, a, workspace, s);
}

}  // namespace dar
