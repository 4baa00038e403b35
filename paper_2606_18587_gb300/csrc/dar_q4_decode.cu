// dar_q4_decode.cu -- one decode step over a cache whose pages hold 4 bits an entry
// (dar_q4.cuh): Eq. 3-4 for the query at position L_b - 1, with the ring in the
// storage type.  With a stored key code_k s_k and q~ = q Uk^T, a distant token's
// score is sum over groups of s_k (q~_group . code_k), and the sums that Uv lifts
// are sum_j (p_j s_v,j) code_v,j: scales multiply scores and weights, one per group,
// and the products take the codes themselves.
//
// Two or three kernels on the caller's stream, the later ones launched programmatically:
//
//  prep    (bf16, tensor cores) q~ of every unit as operands; in a step of few tokens by further blocks
//          of the append's kernel.  (Made by every warp for itself it delays the first page by 3 us, and one
//          sequence of 901 tokens takes 9.0 us in a graph instead of 8.3.)
//  attend  The work is a line of units (sequence, KV head, up to kRows query heads):
//          the ring in runs of kRun tokens, then the pages.  Every warp of the grid has
//          an equal share of the line by cost, and leaves one partial result per query
//          head for each unit that its share cuts: (m, l, acc) of its ring tokens and of
//          its pages, each by its own reference; unit u's cut by share k has the slot u + k.  The
//          shares of a unit's first and last stage leave their numbers for the joining kernel.
//          Lengths are read on the device.
//  join    a block per output row joins its partial results by log-sum-exp and lifts the
//          bottleneck sum once by Uv.
#include <algorithm>
#include <type_traits>

#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_q4.cuh"
#include "dar_q4_append.cuh"
#include "dar_sm100.cuh"

namespace dar {
namespace q4 {

using namespace sm100;

constexpr int kRows = 8;         // query heads of a unit at most
constexpr int kRun = 16;         // ring tokens of a stage
constexpr int kWarps = 8;        // of a CTA (CUDA cores)
// Of a CTA (tensor cores), and stages in flight of each: as many warps as registers allow (18 or 20 spill, and 12 or 14 of
// narrow vectors, or three stages, are as fast within 3 %).
template <int DD>
__host__ __device__ constexpr int mma_warps() { return DD <= 16 ? 16 : 12; }
template <int DD>
__host__ __device__ constexpr int mma_slots() { return DD <= 16 ? 2 : 3; }
// Registers of a thread: without spills (eight heads: 30 bytes at most), and for one or two heads of narrow vectors such that blocks of the first kernel
// fit beside on an SM (else half the blocks start 1 us later; with four heads the spills cost more: 46.9 and 48.7 us).
template <int DD, int NH>
__host__ __device__ constexpr int mma_registers() { return DD > 16 ? 168 : NH < 4 ? 112 : 128; }
constexpr int kSlot = 5120;      // bytes of a stage at most
constexpr int kMaxShares = 2560; // the workspace holds partial results of this many warps
// Costs on the line, in fifths of a page of 16 entries: of a unit's set-up (its place is before the stages), of kRun ring
// tokens.  Measured, runs at 8, 12 and 16: 17.4, 17.7 and 18.0 us (32 sequences, 12 heads, w = 128, 4096 tokens); 48.6, 48.8
// and 50.2 (64 of 1024 to 32768, 32 heads over 8 KV heads, w = 256); 44.4, 42.4 and 43.2 (the same with 8 heads).  Set-up
// at 8 and 20, runs at 8: 17.4 and 17.3, 48.6 and 47.7.
constexpr int kCostUnit = 20;
constexpr int kCostRun = 10;
template <int DD>
__host__ __device__ constexpr int cost_page() { return DD == 8 ? 4 : 5 * DD / 16; }

template <int DD>
__host__ __device__ constexpr int rec_floats() { return 4 + kHeadDim + DD; }

struct Args {
    Q4DecodeArgs c;
    int2 *span;  // [units] first and last share of every unit; -1: it has no tokens
    uint32_t *prep;  // of every unit, what the first kernel makes of its queries (Pages)
    bool front;      // the kernel before is the step's first one: it appends too
    float *rec;  // [units + shares][rows of a unit][rec_floats]: m, l of the ring, m, l of the pages, acc[64], acc[d_down]
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

// Of a unit at the cache's capacity.
template <int DD>
static long long unit_capacity(int w, int maxp)
{
    return kCostUnit + ((long long)w + kRun - 1) / kRun * kCostRun + (long long)maxp * cost_page<DD>();
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
        if (L == 0 && blockIdx.x == 0)  // empty, or refused: the output is 0
            for (int u = 0; u < a.c.Hkv * a.RT; ++u)
                a.span[b * a.c.Hkv * a.RT + u].x = -1;
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
// tokens' weights, through shared memory).  R: 1, 2, 4 or 8 rows, the unit's at least (fp32, 4 sequences of up to
// 1501 tokens, three heads a KV head: 16.0 us, 18.7 with 8).  What is left is latency: q~ of every cut, and
// shuffles and expf that wait on one another.
template <int R>
struct LaneSmem {
    float q[R][kHeadDim], qt[R][kHeadDim];
    float p[R][kPage], x[kPage][16];
};

template <typename T, int DD, int R>
__device__ __forceinline__ void attend_lanes(const Args &a, const Tables &t, LaneSmem<R> &s)
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
        for (int i = lane; i < R * kHeadDim; i += 32) {
            const int r = i / kHeadDim;
            s.q[r][i % kHeadDim] =
                r < c.rows ? to_f32(static_cast<const T *>(a.c.q)[(row0 + r) * kHeadDim + i % kHeadDim]) : 0.f;
        }
        __syncwarp();
        for (int i = lane; i < R * DD; i += 32) {
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
        float m[R], l[R], ol[R][2], od[R][NB];
#pragma unroll
        for (int r = 0; r < R; ++r) {
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
                float y[R][2];
#pragma unroll
                for (int r = 0; r < R; ++r)
                    y[r][0] = y[r][1] = -INFINITY;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int tok = 2 * lane + e;
                    if (tok >= n)
                        continue;
                    float x[R] = {};
                    constexpr int E = Granule<T>::kElems;
#pragma unroll 2
                    for (int i = 0; i < kHeadDim / E; ++i) {
                        float kk[E];
                        unpack(reinterpret_cast<const uint4 *>(k + tok * kHeadDim)[i], kk, T());
#pragma unroll
                        for (int r = 0; r < R; ++r)
#pragma unroll
                            for (int j = 0; j < E; ++j)
                                x[r] = fmaf(s.q[r][i * E + j], kk[j], x[r]);
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        y[r][e] = x[r] * a.c.c2;
                }
#pragma unroll
                for (int r = 0; r < R; ++r)
                    weigh(r, y[r][0], y[r][1]);
                __syncwarp();
                for (int tok = 0; tok < n; ++tok) {
                    const float v0 = to_f32(v[tok * kHeadDim + lane]), v1 = to_f32(v[tok * kHeadDim + 32 + lane]);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
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
            float y[R][2] = {};
#pragma unroll 1
            for (int i = 0; i < NB; ++i) {
                float x0[GS], x1[GS];
                read_row<GS, false>(page + i * F::kBlock, 2 * lane, x0);
                read_row<GS, false>(page + i * F::kBlock, 2 * lane + 1, x1);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int e = 0; e < GS; ++e) {
                        const float q = s.qt[r][i * GS + e];
                        y[r][0] = fmaf(q, x0[e], y[r][0]);
                        y[r][1] = fmaf(q, x1[e], y[r][1]);
                    }
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
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
                    for (int r = 0; r < R; ++r)
                        od[r][i] = fmaf(s.p[r][tok], v, od[r][i]);
                }
            }
            __syncwarp();
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
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
            if (lane == 0)  // one reference for both
                *reinterpret_cast<float4 *>(rec) = make_float4(m[r], l[r], m[r], 0.f);
            rec[4 + lane] = ol[r][0];
            rec[4 + 32 + lane] = ol[r][1];
            if (lane < GS)
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    rec[4 + kHeadDim + i * GS + lane] = od[r][i];
        }
    }
}

template <int R>
constexpr size_t lanes_smem(int B) { return kWarps * sizeof(LaneSmem<R>) + (2 * (size_t)B + 1) * 4; }

template <typename T, int DD, int R>
__global__ void __launch_bounds__(kWarps * 32) attend_kernel(Args a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const Tables t = tables_at(reinterpret_cast<int *>(smem + kWarps * sizeof(LaneSmem<R>)), a.c.B);
    grid_dep_launch();
    build_tables<DD>(a, t);
    attend_lanes<T, DD, R>(a, t, reinterpret_cast<LaneSmem<R> *>(smem)[threadIdx.x >> 5]);
}

// ------------------------------------------------------------------ attend, tensor cores
//
// Up to 8 query heads lie on the N side of mma.sync products (m16n8k16, fp16) with 16 tokens
// on the M side (a tcgen05 tile has 128 rows: most calls have 1 to 8 heads per KV head).
// Column 2 t of a product belongs to head t and column 2 t + 1 to head t + 4, so lane (g, t) =
// 4 g + t has the scores, weights, references and sums of heads t and t + 4 (CT = 2); with CT = 1
// of head t alone, and the other column takes what is said below.
//
//  codes    fp16 subnormals as they lie (dar_q4.cuh), five instructions for the eight of a word.  (Their
//           values take 13: an AND and an OR each, since an instruction has one immediate, and the
//           offset subtracted; e4m3 operands are converted by twice as many: mma.sync has no products
//           of them here; sign and magnitude, which needs no offset, takes seven.)
//  scores   q~, brought to [2^14, 2^15) by a power of two, is two fp16 terms (2^-22 of it).  CT = 1:
//           the second one is the other column's.  CT = 2: a product of its own.  A d_down of 8:
//           the two halves of a product's 16 entries.  The sum starts from
//           minus 8 times theirs.  Rows with c = 1 are in slots 1 and 3: their scores are 16 times as large.
//  weights  p s_v as fp16 (2^-11) relative to a reference of the row, one for all groups, that keeps the
//           largest at 2^8 when it is set: half a step of the smallest fp16 numbers is 2^-33 of that one, and
//           what lies 2^-22 below it has fewer bits (a group of much smaller values too).  It is raised where a
//           weight overflows, which shows in the sums of a stage: the stage is done again, page by page with the
//           weights looked at first.  (bf16 operands need two terms for the same error, twice the conversions
//           and transpositions; a reference of each group, a multiplication for each weight.)
//  sums     of a stage start from 0, and beside them those of the weights times the offset, which come
//           from a product with constant rows; what joins the other stages' is the difference (at
//           256 tokens the offset's part is some 100 times the rest's 2^-24).
// What bounds it: a page of 64 tokens (1280 bytes) of four heads is 175 instructions of a warp, some 74 of them in the
// integer pipe at two cycles each; all SMs at the clock of a measurement could take 152 x 4 pages in 148 cycles, 10 TB/s, but
// issue is 62 % and that pipe 48 % (latency between dependent products is what four warps a quarter do not hide).  64
// sequences of 1024 to 32768 tokens (206 MB): 47 us, 4.4 TB/s; one, two, eight heads a KV head: 42, 44, 63; the copies
// alone, nothing computed: 44 us.  d_down 64, 339 MB: 62 us, 5.5 TB/s.  Before: on CUDA cores 518 us; e4m3 operands
// 65; sign and magnitude 54.

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

// Slots 0 to 3 of a word of codes as operand registers (slots 1 and 3 times 16).
__device__ __forceinline__ void codes_of(uint32_t w, uint32_t (&c)[4])
{
    c[0] = w & 0x000f000fu;
    c[1] = w & 0x00f000f0u;
    c[2] = (w >> 8) & 0x000f000fu;
    c[3] = (w >> 8) & 0x00f000f0u;
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

// Pages of a stage: 1, 2 or 4.
template <int DD>
__host__ __device__ constexpr int stage_pages() { return Fmt<DD>::kBytes > kSlot / 4 ? kSlot / Fmt<DD>::kBytes : 4; }

__device__ __forceinline__ void cp_async16_hint(uint32_t dst, const void *src, uint64_t policy)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}

// What a warp fills its slots with, ahead of what it computes: a run of the ring, or pages.  By 16-byte copies of its
// lanes, a group of them a stage.  (A bulk copy takes the SM's copy engine some 36 cycles, whatever its size: at 768 to
// 1280 bytes a page that is as long as HBM takes for them.)
template <int DD>
struct Filler {
    static constexpr int S = mma_slots<DD>(), P = stage_pages<DD>(), kBytes = Fmt<DD>::kBytes;
    Walk walk;
    const int32_t *table;       // block table of the cut's sequence
    const unsigned char *heads; // page 0 of the cut's KV head, this lane's part
    int ring, nwin;             // row of the ring's first token, tokens in it
    int st, st1, nrun;          // next stage, end of the cut, runs of the ring
    int ids, later, at;         // 32 entries of the table, one per lane, of which the next stage's are at .., and the next 32
    int slot;                   // to be filled next
    bool more;

    __device__ __forceinline__ void begin(const Args &a, const Tables &t, int share)
    {
        walk.begin<DD>(a, t, share);
        slot = 0;
        next_cut(a, t);
    }
    __device__ __forceinline__ void next_cut(const Args &a, const Tables &t)
    {
        Cut c;
        more = walk.next<DD>(a, t, c);
        if (!more)
            return;
        st = c.st0;
        st1 = c.st1;
        nrun = c.nrun;
        nwin = c.nwin;
        table = a.c.block_table + (size_t)c.b * a.c.maxp;
        load_ids(a, max(0, st - nrun));
        heads = static_cast<const unsigned char *>(a.c.pool) + (size_t)c.g * kBytes + (threadIdx.x & 31) * 16;
        ring = (c.b * a.c.Hkv + c.g) * a.c.w;
    }
    // Entries from page lp on; they are there by the time a stage wants them.
    __device__ __forceinline__ void load_ids(const Args &a, int lp)
    {
        const int i = lp + (threadIdx.x & 31);
        ids = i < a.c.maxp ? __ldg(table + i) : -1;
        later = i + 32 < a.c.maxp ? __ldg(table + i + 32) : -1;
        at = 0;
    }
    // Starts the copies of the next stage, as one group (of none when there is no more).
    __device__ __forceinline__ void fill(const Args &a, const Tables &t, uint32_t slots, int lane)
    {
        if (more) {
            const uint64_t once = l2_evict_first_policy();  // the cache is read once
            const uint32_t dst = slots + slot * kSlot;
            if (st < nrun) {  // 16 rows of 128 bytes, 16-byte piece c of row r at c ^ (r mod 8)
                const int n = min(kRun, nwin - st * kRun), r0 = lane >> 3, c = lane & 7;
                const size_t from = ((size_t)ring + st * kRun + r0) * (kHeadDim * 2) + c * 16;
                const unsigned char *k = static_cast<const unsigned char *>(a.c.win_k) + from;
                const unsigned char *v = static_cast<const unsigned char *>(a.c.win_v) + from;
#pragma unroll
                for (int i = 0; i < kRun / 4; ++i) {
                    const int r = r0 + 4 * i;
                    const uint32_t to = dst + r * 128 + ((c ^ (r & 7)) << 4);
                    if (r < n) {
                        cp_async16_hint(to, k + i * 4 * 128, once);
                        cp_async16_hint(to + kRun * 128, v + i * 4 * 128, once);
                    }
                }
                ++st;
            } else {
                const int lp = st - nrun, n = min(P, st1 - st);
                if (at >= 32) {
                    ids = later;
                    later = lp + 32 + lane < a.c.maxp ? __ldg(table + lp + 32 + lane) : -1;
                    at = 0;
                }
                const uint32_t to = dst + lane * 16;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    if (i >= n)
                        break;
                    const int id = __shfl_sync(0xffffffffu, ids, at + i);
                    if ((unsigned)id < (unsigned)a.c.num_pages) {
                        const unsigned char *page = heads + (size_t)id * (unsigned)(a.c.Hkv * kBytes);
#pragma unroll
                        for (int k = 0; k < kBytes; k += 512)
                            if (k + 512 <= kBytes || lane * 16 < kBytes - k)
                                cp_async16_hint(to + i * kBytes + k, page + k, once);
                    } else if (lane == 0) {
                        report(a.c.status, DAR_ERR_CAPACITY);
                    }
                }
                st += n;
                at += n;
            }
            slot = slot + 1 < S ? slot + 1 : 0;
            if (st >= st1)
                next_cut(a, t);
        }
        cp_async_commit();
    }
};

// The queries of a cut as B operands: column i0 = lane / 4 is head (i0 / 2) mod NH + 4 (i0 mod 2).
template <int NH>
__device__ __forceinline__ void queries_of(const Args &a, const Cut &c, int lane, uint32_t (&q)[4][2])
{
    const int i0 = lane >> 2, c0 = lane & 3, head = (i0 >> 1) % NH + 4 * (i0 & 1);
    const uint32_t *qp = static_cast<const uint32_t *>(a.c.q) +
                         ((size_t)c.b * a.c.Hq + c.g * a.G + c.rt * kRows + head) * (kHeadDim / 2) + c0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        q[e / 2][e % 2] = head < c.rows ? __ldg(qp + 4 * e) : 0u;
}

// A cut without ring tokens (at 0) or pages (at 2) says so: nothing else of that part is read.
template <int DD>
__device__ __forceinline__ void leave_none(const Args &a, const Cut &c, int at, int lane)
{
    if (lane < c.rows)
        *reinterpret_cast<float2 *>(a.rec + ((size_t)c.slot * a.RU + lane) * rec_floats<DD>() + at) =
            make_float2(-INFINITY, 0.f);
}

// A cut's ring tokens.
template <int CT, int NH>
struct Ring {
    Soft ring[CT];
    float ol[kHeadDim / 16][4];
    __device__ __forceinline__ Ring()
    {
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            ring[k].bias = INFINITY;
            ring[k].l = 0.f;
        }
#pragma unroll
        for (int e = 0; e < kHeadDim / 16; ++e)
            ol[e][0] = ol[e][1] = ol[e][2] = ol[e][3] = 0.f;
    }

    // A run of n ring tokens at `tile`: 16 rows of keys, then of values, 128-byte swizzle.
    __device__ __forceinline__ void step(const uint32_t (&q)[4][2], uint32_t tile, int n, float c2, int lane)
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

    __device__ __forceinline__ void leave(const Args &a, const Cut &c, int stride, int lane)
    {
        const int i0 = lane >> 2, c0 = lane & 3;
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            float l = ring[k].l;
#pragma unroll
            for (int o = 4; o < 32; o <<= 1)
                l += __shfl_xor_sync(0xffffffffu, l, o);
            const int head = c0 + 4 * k;
            if (head >= c.rows || c0 >= NH)  // (with fewer than four heads the other columns are copies)
                continue;
            float *rec = a.rec + ((size_t)c.slot * a.RU + head) * stride;
            if (i0 == 0)
                *reinterpret_cast<float2 *>(rec) = make_float2(-ring[k].bias, l);
#pragma unroll
            for (int e = 0; e < kHeadDim / 16; ++e) {
                rec[4 + 16 * e + i0] = ol[e][k];
                rec[4 + 16 * e + 8 + i0] = ol[e][2 + k];
            }
        }
    }
};

// A cut's pages: what a warp has of its query heads, and the sums.
//
// NH heads (1, 2 or 4; CT = 2: 8) share the columns of a product out: with one head, columns 2 x, 2 x + 1 belong to words
// x of its lanes, and the products of the four words go into one result, each with an operand that is zero in the
// others' columns.  So a lane has two scores of a page, not eight of which the lanes t have the same: 139 instructions a
// page instead of 175 (64 sequences as above with one head: 45.1 us and 49).  In general word i = x ND + d goes to columns of x in result d.
template <int DD, int CT, int NH>
struct Pages {
    static constexpr int GS = Fmt<DD>::kGroup, NB = Fmt<DD>::kGroups;
    static constexpr int ND = NH, NW = 4 / NH;              // results of a page's scores, words in one
    static constexpr int TB = GS == 16 && CT == 2 ? 2 : 1;  // score products of a group
    static_assert(CT == 1 || NH == 4, "eight heads fill the columns");
    uint32_t qt[NB][TB][2];  // q~ as B operands, two fp16 terms
    uint32_t mine[NW][2];    // all ones where the lane's column belongs to words x ND .., and is even (0) or odd (1)
    float from[NB][4];       // what a score's sum starts from
    float cq[CT];            // scale of a score: c2, the power of two taken out of q~, and the codes' 2^24
    Soft page[CT];
    float od[NB][2 * CT];    // times 2^-24, entries e of the heads and then e + 2 (see Sums)

    // Words of a lane that the first kernel leaves of a unit, [unit][word][lane]: of its groups, and the factors.
    static constexpr int kGroupWords = TB * 2 + 2, kWords = NB * kGroupWords + CT;
    template <typename F>
    __device__ __forceinline__ void each_word(const F &f)
    {
        int i = 0;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
#pragma unroll
            for (int k = 0; k < TB; ++k) {
                f(i++, qt[j][k][0]);
                f(i++, qt[j][k][1]);
            }
            f(i++, from[j][0]);
            f(i++, from[j][1]);
        }
#pragma unroll
        for (int k = 0; k < CT; ++k)
            f(i++, cq[k]);
    }
    // As group j of n.
    __device__ __forceinline__ void save(const Args &a, int unit, int j, int n, int lane)
    {
        static_assert(NB == 1, "a group");
        uint32_t *p = a.prep + (size_t)unit * (n * kGroupWords + CT) * 32 + lane;
        each_word([&](int i, auto &x) {
            const int at = i < kGroupWords ? j * kGroupWords + i : n * kGroupWords + (i - kGroupWords);
            if (i < kGroupWords || j == 0)
                p[at * 32] = *reinterpret_cast<const uint32_t *>(&x);
        });
    }
    __device__ __forceinline__ void load(const Args &a, int unit, int lane)
    {
        const uint32_t *p = a.prep + (size_t)unit * kWords * 32 + lane;
        each_word([&](int i, auto &x) { *reinterpret_cast<uint32_t *>(&x) = p[i * 32]; });
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            from[j][2] = 16.f * from[j][0];
            from[j][3] = 16.f * from[j][1];
        }
#pragma unroll
        for (int x = 0; x < NW; ++x)
#pragma unroll
            for (int c = 0; c < 2; ++c)
                mine[x][c] = (lane >> 3) / NH == x && ((lane >> 2) & 1) == c ? ~0u : 0u;
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            page[k].bias = INFINITY;
            page[k].l = 0.f;
        }
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int o = 0; o < 2 * CT; ++o)
                od[j][o] = 0.f;
    }

    // q~^T = Uk q^T of a group's rows uk, with Uk in three bf16 terms (products exact but for 2^-24).  most: takes the
    // largest magnitudes of the group's entries to those of all groups'.
    template <typename F>
    __device__ __forceinline__ void make(const Args &a, const float *uk, const uint32_t (&q)[4][2], int lane, const F &most)
    {
        static_assert(NB == 1, "a group");
        const int i0 = lane >> 2, c0 = lane & 3;
        float x[NB][4];  // entries 16 j + i0 (+ 8) of heads c0 mod NH, and + 4: [0] i0 c0, [1] i0 c0 + 4, [2], [3] i0 + 8
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const float *u = uk + i0 * kHeadDim + 2 * c0;
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
        uint32_t tops[CT];
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            tops[k] = max(magnitude(x[0][k]), magnitude(x[0][2 + k]));
#pragma unroll
            for (int o = 4; o < 32; o <<= 1)
                tops[k] = max(tops[k], __shfl_xor_sync(0xffffffffu, tops[k], o));
        }
        most(tops);
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            const uint32_t top = tops[k];
            const int e = max((int)(top >> 23) - 127, -100);
            up[k] = __uint_as_float((uint32_t)(127 + 14 - e) << 23);  // e <= 127: 2^-113 at least
            // infinite or NaN: so are all scores.  Not 0: no token's score is minus infinity before it is multiplied.  Nor
            // infinite: the scores of keys of zero stay 0
            cq[k] = top >= 0x7f800000u
                        ? __uint_as_float(0x7fc00000u)
                        : fminf(fmaxf(a.c.c2 * __uint_as_float((uint32_t)(127 + e) << 23) * 1024.f, 0x1p-120f), 0x1p126f);
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
            for (int k = 0; k < 2; ++k)
                from[j][k] = -0x1p-21f * __shfl_sync(0xffffffffu, sum, (2 * c0 + k) * 4);  // 8 * 2^-24
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

    // Lane (g, t) has the scores of rows 16 (g / 2) + 4 i + 2 c + g mod 2, i = (t / NH) ND + d, in pairs: two tokens (c =
    // 0, 1) of a head (pair d), or with CT = 2 two heads of a token (pairs 2 d, 2 d + 1).
    static constexpr int NP = ND * CT;
    struct Scores {
        float y[NP][2];
    };
    // The lane's words of 64 scales.
    static __device__ __forceinline__ void load_scales(const unsigned char *at, int lane, uint32_t (&s)[ND])
    {
        at += (lane >> 2) * 16 + (lane & 3) / NH * (4 * ND);
        if constexpr (ND == 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(at);
            s[0] = v.x, s[1] = v.y, s[2 % ND] = v.z, s[3 % ND] = v.w;
        } else if constexpr (ND == 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(at);
            s[0] = v.x, s[1 % ND] = v.y;
        } else {
            s[0] = *reinterpret_cast<const uint32_t *>(at);
        }
    }
    __device__ __forceinline__ void scores(const unsigned char *at, int lane, Scores &z) const
    {
        using F = Fmt<DD>;
        float(&y)[NP][2] = z.y;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const unsigned char *block = at + j * F::kBlock;
            uint32_t w[4], sc[ND];
            load_scales(block + F::kScales, lane, sc);
            load_words(block, lane, w);
            float r[ND][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t c[4];
                codes_of(w[i], c);
                if constexpr (GS == 8) {  // both halves of the product's 16 entries are the key's 8
                    c[0] = i % 2 ? c[2] : c[0];
                    c[1] = i % 2 ? c[3] : c[1];
                    c[2] = c[0];
                    c[3] = c[1];
                }
                float(&d)[4] = r[i % ND];
                const uint32_t m = mine[i / ND][0] | mine[i / ND][1];
                if (i < ND)
                    mma_f16_c(d, c, NW == 1 ? qt[j][0][0] : qt[j][0][0] & m, NW == 1 ? qt[j][0][1] : qt[j][0][1] & m, from[j]);
                else
                    mma_f16_acc(d, c, qt[j][0][0] & m, qt[j][0][1] & m);
                if constexpr (TB == 2)
                    mma_f16_acc(d, c, qt[j][TB - 1][0], qt[j][TB - 1][1]);
            }
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                const float s0 = bf16lo(sc[i]), s1 = bf16hi(sc[i]);
                const float(&d)[4] = r[i];
                if constexpr (CT == 1) {
                    const float x0 = GS == 16 ? d[0] + d[1] : d[0], x1 = GS == 16 ? d[2] + d[3] : d[2];
                    y[i][0] = j ? fmaf(x0, s0, y[i][0]) : x0 * s0;
                    y[i][1] = j ? fmaf(x1, s1, y[i][1]) : x1 * s1;
                } else {
                    float(&u)[2] = y[2 * i % NP], (&v)[2] = y[(2 * i + 1) % NP];
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
    }
    // Factor of a pair's scores: slots of c = 1 are 16 times as large.
    __device__ __forceinline__ float factor(int k, int e) const
    {
        const float s = cq[CT == 2 ? e : 0];
        return (CT == 1 ? e : k % 2) ? s * 0.0625f : s;
    }
    // Weights of a page relative to the references, and their sums.
    __device__ __forceinline__ void weigh(const Scores &z, float (&p)[NP][2], float (&l)[2]) const
    {
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            float x0, x1;
            ffma2(x0, x1, z.y[k][0], z.y[k][1], factor(k, 0), factor(k, 1), page[0].bias, page[CT - 1].bias);
            p[k][0] = ex2_approx(x0);
            p[k][1] = ex2_approx(x1);
            add2(l[0], l[1], l[0], l[1], p[k][0], p[k][1]);
        }
    }
    // A pair's scales.
    static __device__ __forceinline__ void scales(uint32_t s, int k, float &s0, float &s1)
    {
        s0 = CT == 1 || k % 2 == 0 ? bf16lo(s) : bf16hi(s);
        s1 = CT == 1 || k % 2 != 0 ? bf16hi(s) : bf16lo(s);
    }
    // Sums of some pages, of codes + 8; off: of 8 (both times 2^-24, entries e + 2 times 2^-20).  With CT = 2 a column has
    // 8 tokens' weights of head t or t + 4.  With CT = 1 column 2 t has those of rows with c = 0 and column 2 t + 1 those
    // with c = 1, which one transposition brings; products with the codes of c = 0 are right in the even columns and
    // products with those of c = 1 in the odd ones, so each has sums of its own, whose other columns are not used.  With
    // fewer than four heads a word's weights are in its columns alone, and masks leave the rest 0.
    struct Sums {
        static constexpr int OD = NH == 4 && CT == 1 ? 2 : 1;
        float x[NB][OD][4], off[NB][4];
        __device__ __forceinline__ Sums()
        {
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
#pragma unroll
                    for (int o = 0; o < OD; ++o)
                        x[j][o][e] = 0.f;
                    off[j][e] = 0.f;
                }
        }
        // keep: rows that count (bits as in a word of scales)
        template <bool MASK>
        __device__ __forceinline__ void add(const unsigned char *at, int lane, const float (&p)[NP][2],
                                            const uint32_t (&keep)[ND], const uint32_t (&mine)[NW][2])
        {
            using F = Fmt<DD>;
            constexpr uint32_t kOff0 = 0x80088008u, kOff1 = 0x80808080u;  // -8 in slots 0 and 1
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                uint32_t w[4], s[ND], b[NP];
                load_words(at + j * F::kBlock + F::kCodes, lane, w);
                load_scales(at + j * F::kBlock + F::kScales + 2 * kPage, lane, s);
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    float s0, s1, w0, w1;
                    scales(MASK ? s[k / CT] & keep[k / CT] : s[k / CT], k, s0, s1);
                    mul2(w0, w1, p[k][0], p[k][1], s0, s1);
                    b[k] = transpose8(cvt_f16x2(w0, w1));
                }
                uint32_t v[4][4];  // both entries of the rows of word i with c = 0, and with c = 1
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (GS == 16) {
                        codes_of(w[i], v[i]);
                    } else {
                        v[i][0] = (i % 2 ? w[i] >> 8 : w[i]) & 0x000f000fu;
                        v[i][2] = (i % 2 ? w[i] >> 12 : w[i] >> 4) & 0x000f000fu;
                        v[i][1] = v[i][3] = 0u;
                    }
                }
                const uint32_t off8[4] = {kOff0, GS == 16 ? kOff1 : 0u, kOff0, GS == 16 ? kOff1 : 0u};
#pragma unroll
                for (int k = 0; k < NP; k += 2)
                    mma_f16_acc(off[j], off8, b[k], k + 1 < NP ? b[(k + 1) % NP] : 0u);
                if constexpr (CT == 2) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mma_f16_acc(x[j][0], v[i], b[2 * i % NP], b[(2 * i + 1) % NP]);
                } else if constexpr (NH == 4) {
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const uint32_t even[4] = {v[i][0], v[i][1], v[i + 1][0], v[i + 1][1]};
                        const uint32_t odd[4] = {v[i][2], v[i][3], v[i + 1][2], v[i + 1][3]};
                        mma_f16_acc(x[j][0], even, b[i % NP], b[(i + 1) % NP]);
                        mma_f16_acc(x[j][OD - 1], odd, b[i % NP], b[(i + 1) % NP]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mma_f16_acc(x[j][0], v[i], b[i % ND] & mine[i / ND][0], b[i % ND] & mine[i / ND][1]);
                }
            }
        }
        // Entry e (k = 0) or e + 2 (k = 1) of head h of the lane.
        __device__ __forceinline__ float value(int j, int k, int h) const
        {
            if constexpr (CT == 2)
                return x[j][0][2 * k + h] + off[j][2 * k + h];
            else
                return (x[j][0][2 * k] + off[j][2 * k]) + (x[j][OD - 1][2 * k + 1] + off[j][2 * k + 1]);  // both columns
        }
    };
    __device__ __forceinline__ void join(const Sums &s, const float (&l)[2])
    {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int h = 0; h < CT; ++h) {
                od[j][h] += s.value(j, 0, h);
                if constexpr (GS == 16)
                    od[j][CT + h] = fmaf(0.0625f, s.value(j, 1, h), od[j][CT + h]);
            }
        page[0].l += CT == 1 ? l[0] + l[1] : l[0];
        if constexpr (CT == 2)
            page[CT - 1].l += l[1];
    }

    // n whole pages.  False if a weight was too large for its operand (or a sum for what comes of it): nothing is added then.
    __device__ __forceinline__ bool pages_step(const unsigned char *at, int n, int lane)
    {
        Sums s;
        float l[2] = {0.f, 0.f};
        const uint32_t all[ND] = {};
        auto one = [&](const unsigned char *page) {
            Scores z;
            float p[NP][2];
            scores(page, lane, z);
            weigh(z, p, l);
            s.template add<false>(page, lane, p, all, mine);
        };
        if (n == stage_pages<DD>()) {  // (unrolled it is 175 instructions a page instead of 187)
#pragma unroll
            for (int i = 0; i < stage_pages<DD>(); ++i)
                one(at + i * Fmt<DD>::kBytes);
        } else {
#pragma unroll 1
            for (int i = 0; i < n; ++i)
                one(at + i * Fmt<DD>::kBytes);
        }
        // an infinite weight makes its column infinite or NaN
        bool fine = fmaxf(l[0], l[1]) < 0x1p100f;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int h = 0; h < CT; ++h)
                fine &= fabsf(s.off[j][h]) < INFINITY && (CT == 2 || fabsf(s.off[j][1]) < INFINITY);
        if (!__all_sync(0xffffffffu, fine))
            return false;
        join(s, l);
        return true;
    }

    // A page of n tokens, whose weights are looked at first.
    __device__ __forceinline__ void page_step(const unsigned char *at, int n, int lane)
    {
        Scores z;
        scores(at, lane, z);
        uint32_t keep[ND], vm[ND];  // rows that count, and the largest scales of their groups
#pragma unroll
        for (int i = 0; i < ND; ++i) {  // rows behind the last token may hold anything
            const int tok = 16 * (lane >> 3) + 4 * ((lane & 3) / NH * ND + i) + ((lane >> 2) & 1);  // and tok + 2
            keep[i] = (tok < n ? 0xffffu : 0u) | (tok + 2 < n ? 0xffff0000u : 0u);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if constexpr (CT == 1) {
                    z.y[i][e] = tok + 2 * e < n ? z.y[i][e] : -INFINITY;
                } else {
                    z.y[2 * i % NP][e] = tok < n ? z.y[2 * i % NP][e] : -INFINITY;
                    z.y[(2 * i + 1) % NP][e] = tok + 2 < n ? z.y[(2 * i + 1) % NP][e] : -INFINITY;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            uint32_t s[ND];
            load_scales(at + j * Fmt<DD>::kBlock + Fmt<DD>::kScales + 2 * kPage, lane, s);
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                if (j == 0)
                    vm[i] = s[i] & keep[i];
                else
                    asm("max.bf16x2 %0, %0, %1;" : "+r"(vm[i]) : "r"(s[i] & keep[i]));
            }
        }
        constexpr float kFar = 32768.f, kFarSum = 0x1p96f;
        float p[NP][2], l[2] = {0.f, 0.f}, top = 0.f;
        weigh(z, p, l);
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            float s0, s1;
            scales(vm[k / CT], k, s0, s1);
            top = max3(top, p[k][0] * s0, p[k][1] * s1);
        }
        // Without a reference yet the weights of rows that count are infinite and the others' NaN, and so is each of a lane's
        // sums (top may miss it: an infinite weight times a scale of 0): what is not known to be small asks for one.
        if (__any_sync(0xffffffffu, !(l[0] <= kFarSum && l[1] <= kFarSum && top <= kFar))) {
#pragma unroll
            for (int k = 0; k < CT; ++k) {
                top = -INFINITY;  // of p s_v, and of 2^-80 p
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (CT == 2 && e != k)
                            continue;
                        float s[2];
                        scales(vm[i / CT], i, s[0], s[1]);
                        top = fmaxf(top, fmaf(z.y[i][e], factor(i, e), __log2f(fmaxf(0x1p-80f, s[e]))));
                    }
#pragma unroll
                for (int o = NH; o < 32; o <<= 1)  // all lanes of the head
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float was = -page[k].bias, now = fmaxf(was, top - 8.f);
                const float f = now == -INFINITY ? 1.f : ex2_approx(was - now);
                page[k].bias = -now;
                page[k].l *= f;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    od[j][k] *= f;
                    od[j][CT + k] *= f;
                }
            }
            l[0] = l[1] = 0.f;
            weigh(z, p, l);
        }
        Sums s;
        s.template add<true>(at, lane, p, keep, mine);
        join(s, l);
    }

    __device__ __forceinline__ void leave(const Args &a, const Cut &c, int lane)
    {
        const int i0 = lane >> 2, c0 = lane & 3;
        if constexpr (NH < 4) {  // lanes t of a head have different words' columns
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int o = NH; o < 4; o <<= 1)
                        od[j][k] += __shfl_xor_sync(0xffffffffu, od[j][k], o);
        }
#pragma unroll
        for (int k = 0; k < CT; ++k) {
            float l = page[k].l;
#pragma unroll
            for (int o = NH; o < 32; o <<= 1)
                l += __shfl_xor_sync(0xffffffffu, l, o);
            const int head = c0 + 4 * k;
            if (head >= c.rows || c0 >= NH)
                continue;
            float *rec = a.rec + ((size_t)c.slot * a.RU + head) * rec_floats<DD>();
            if (i0 == 0)
                *reinterpret_cast<float2 *>(rec + 2) = make_float2(-page[k].bias, l);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int e = GS == 16 ? 16 * j + 4 * (i0 >> 1) + (i0 & 1) : i0;
                rec[4 + kHeadDim + e] = od[j][k] * 0x1p24f;  // (the codes were 2^-24 of themselves)
                if (GS == 16)
                    rec[4 + kHeadDim + e + 2] = od[j][CT + k] * 0x1p24f;
            }
        }
    }
};

// q~ of the units from `first` on, a warp for each group of 16 entries, as the next kernel's lanes want it; all threads of
// a block of WARPS warps.  (A warp for all four groups of 64 entries takes 5 us, during which it keeps attending blocks off
// its SM.)
template <int DD, int CT, int NH, int WARPS>
__device__ __forceinline__ void prep_units(const Args &a, int first, int units)
{
    constexpr int NB = Fmt<DD>::kGroups;
    using Group = Pages<(DD < 16 ? DD : 16), CT, NH>;
    __shared__ uint32_t tops[WARPS][CT][4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = warp % NB;
    const int unit = min(first + warp / NB, units - 1);  // (the last one once more)
    Cut c;
    c.b = unit / (a.c.Hkv * a.RT);
    c.g = unit / a.RT % a.c.Hkv;
    c.rt = unit % a.RT;
    c.rows = min(kRows, a.G - c.rt * kRows);
    uint32_t q[4][2];
    queries_of<NH>(a, c, lane, q);
    Group h;
    h.make(a, a.c.Uk + ((size_t)c.g * DD + 16 * j) * kHeadDim, q, lane, [&](uint32_t (&top)[CT]) {
        if constexpr (NB > 1) {
#pragma unroll
            for (int k = 0; k < CT; ++k)
                if (lane < 4)
                    tops[warp][k][lane] = top[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < CT; ++k)
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    top[k] = max(top[k], tops[warp - j + i][k][lane & 3]);
        }
    });
    if (first + warp / NB < units)
        h.save(a, unit, j, NB, lane);
}

// 4, 8 and 16 warps a block: 16.6, 17.1 and 17.8 us for 32 sequences of 12 heads; the large calls within 2 %.
constexpr int kPrepWarps = 4;
template <int DD, int WARPS>
static int prep_blocks(int units)
{
    constexpr int per = WARPS / Fmt<DD>::kGroups;
    return (units + per - 1) / per;
}

template <int DD, int CT, int NH>
__global__ void __launch_bounds__(kPrepWarps * 32) prep_kernel(const Args a, int units)
{
    grid_dep_launch();
    prep_units<DD, CT, NH, kPrepWarps>(a, (int)blockIdx.x * (kPrepWarps / Fmt<DD>::kGroups), units);
}

// The first kernel of a step of few tokens: the append's blocks, and the same.
template <int DD, int CT, int NH>
__global__ void __launch_bounds__(kFewThreads) front_kernel(AppendArgs ap, const Args a, int units)
{
    constexpr int kPer = kFewThreads / 32;
    grid_dep_launch();
    if ((int)blockIdx.x < ap.B)
        append_few<bf16, DD>(ap);
    else
        prep_units<DD, CT, NH, kPer>(a, ((int)blockIdx.x - ap.B) * (kPer / Fmt<DD>::kGroups), units);
}

template <int DD>
constexpr size_t mma_smem(int B)
{
    return 128 + (size_t)mma_warps<DD>() * mma_slots<DD>() * kSlot + (2 * (size_t)B + 1) * 4;
}

template <int DD, int CT, int NH>
__global__ void __maxnreg__((mma_registers<DD, NH>())) attend_mma_kernel(const Args a)
{
    constexpr int W = mma_warps<DD>(), S = mma_slots<DD>();
    extern __shared__ unsigned char raw[];
    unsigned char *slots = raw + ((128u - (smem_u32(raw) & 127u)) & 127u);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Tables t = tables_at(reinterpret_cast<int *>(slots + W * S * kSlot), a.c.B);
    grid_dep_launch();
    // the lengths, tables and pages may be read at once, unless the kernel before appends to them
    bool waited = false;
    if (a.front) {
        grid_dep_wait();
        waited = true;
    }
    build_tables<DD>(a, t);
    slots += warp * S * kSlot;
    const uint32_t slots_s = smem_u32(slots);
    const int share = blockIdx.x * W + warp;
    Filler<DD> ahead;
    ahead.begin(a, t, share);
#pragma unroll 1
    for (int i = 0; i < S; ++i)
        ahead.fill(a, t, slots_s, lane);
    Walk walk;
    walk.begin<DD>(a, t, share);
    int s = 0;  // slot of the next stage
    auto take = [&]() {
        cp_async_wait<S - 1>();
        __syncwarp();  // the stage's copies by all lanes have landed
        return s * kSlot;
    };
    auto give = [&]() {
        __syncwarp();  // the slot is read
        s = s + 1 < S ? s + 1 : 0;
        ahead.fill(a, t, slots_s, lane);
    };
    for (Cut c; walk.next<DD>(a, t, c);) {
        if (lane == 0)
            leave_span(a, c, share);
        int st = c.st0;
        if (st < c.nrun) {
            uint32_t q[4][2];
            queries_of<NH>(a, c, lane, q);
            Ring<CT, NH> r;
            for (; st < min(c.st1, c.nrun); ++st) {
                r.step(q, slots_s + take(), min(kRun, c.nwin - st * kRun), a.c.c2, lane);
                give();
            }
            r.leave(a, c, rec_floats<DD>(), lane);
        } else {
            leave_none<DD>(a, c, 0, lane);
        }
        if (st == c.st1) {
            leave_none<DD>(a, c, 2, lane);
            continue;
        }
        if (!waited) {  // for the first kernel
            grid_dep_wait();
            waited = true;
        }
        Pages<DD, CT, NH> h;
        h.load(a, c.unit, lane);
        int left = c.L - c.nwin - (st - c.nrun) * kPage;  // tokens of the unit from here on
        bool first = true;
        for (int pages = c.st1 - st; pages > 0; pages -= stage_pages<DD>()) {
            const unsigned char *slot = slots + take();
            const int m = min(stage_pages<DD>(), pages), whole = min(m, left / kPage);
            // the cut's first page sets the references
            int done = first ? 0 : h.pages_step(slot, whole, lane) ? whole : 0;
            for (; done < m; ++done) {
                h.page_step(slot + done * Fmt<DD>::kBytes, min(kPage, left - done * kPage), lane);
                if (first && done + 1 < whole && h.pages_step(slot + (done + 1) * Fmt<DD>::kBytes, whole - done - 1, lane))
                    done = whole - 1;
                first = false;
            }
            left -= m * kPage;
            give();
        }
        h.leave(a, c, lane);
    }
    if (!waited)
        grid_dep_wait();  // this kernel ends after the first one
}

// ------------------------------------------------------------------ join

// Block i writes output row i: the warps take its partial results in turn, U of them in flight together, and are
// joined.
template <typename T, int DD, int WARPS, int U>
__global__ void __launch_bounds__(WARPS * 32) join_kernel(Args a)
{
    constexpr int ND = (DD + 31) / 32, N = 2 + ND;
    __shared__ float part[WARPS][2 + 32 * N], sum[kHeadDim + DD];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x, b = row / a.c.Hq, h = row % a.c.Hq, g = h / a.G, j = h % a.G;
    // the lift's columns are the caller's: no kernel that may still run writes them
    float uv[DD >= 32 ? 1 : DD];
    if constexpr (DD < 32) {
        if (threadIdx.x < kHeadDim)
#pragma unroll
            for (int e = 0; e < DD; ++e)
                uv[e] = __ldg(a.c.Uv + ((size_t)g * DD + e) * kHeadDim + threadIdx.x);
    }
    grid_dep_wait();
    const int unit = (b * a.c.Hkv + g) * a.RT + j / kRows;
    const int2 span = a.span[unit];
    if (span.x < 0) {
        for (int i = threadIdx.x; i < kHeadDim; i += WARPS * 32)
            static_cast<T *>(a.c.out)[(size_t)row * kHeadDim + i] = from_f32<T>(0.f);
        return;
    }
    const int k0 = min(max(span.x, 0), kMaxShares - 1), k1 = min(max(span.y, k0), kMaxShares - 1), parts = k1 - k0 + 1;
    float m = -INFINITY, l = 0.f, x[N] = {};
    const size_t stride = (size_t)a.RU * rec_floats<DD>();
    const float *rec = a.rec + ((size_t)(unit + k0) * a.RU + j % kRows) * rec_floats<DD>();
    for (int i0 = warp; i0 < parts; i0 += WARPS * U) {
        float4 ml[U];
        float o[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * WARPS;
            ml[u] = make_float4(-INFINITY, 0.f, -INFINITY, 0.f);
            if (i < parts)
                ml[u] = *reinterpret_cast<const float4 *>(rec + i * stride);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float *p = rec + (i0 + u * WARPS) * stride + 4 + lane;
            const bool ring = ml[u].x != -INFINITY, pages = ml[u].z != -INFINITY;
            o[u][0] = ring ? p[0] : 0.f;
            o[u][1] = ring ? p[32] : 0.f;
#pragma unroll
            for (int e = 0; e < ND; ++e)
                o[u][2 + e] = pages && 32 * e + lane < DD ? p[kHeadDim + 32 * e] : 0.f;
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u)
            top = max3(top, ml[u].x, ml[u].z);
        const float base = top == -INFINITY ? 0.f : top, f = ex2_approx(m - base);
        m = top;
        l *= f;
#pragma unroll
        for (int e = 0; e < N; ++e)
            x[e] *= f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float fr = ex2_approx(ml[u].x - base), fp = ex2_approx(ml[u].z - base);
            l += ml[u].y * fr + ml[u].w * fp;
            x[0] = fmaf(o[u][0], fr, x[0]);
            x[1] = fmaf(o[u][1], fr, x[1]);
#pragma unroll
            for (int e = 0; e < ND; ++e)
                x[2 + e] = fmaf(o[u][2 + e], fp, x[2 + e]);
        }
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
    if (threadIdx.x >= kHeadDim)
        return;
    float o = sum[threadIdx.x];
#pragma unroll
    for (int e = 0; e < DD; ++e) {
        if constexpr (DD < 32)
            o = fmaf(sum[kHeadDim + e], uv[e], o);
        else
            o = fmaf(sum[kHeadDim + e], __ldg(a.c.Uv + ((size_t)g * DD + e) * kHeadDim + threadIdx.x), o);
    }
    static_cast<T *>(a.c.out)[(size_t)row * kHeadDim + threadIdx.x] = from_f32<T>(o / all);
}

// ------------------------------------------------------------------ launch

static size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

struct Layout {
    size_t span, prep, rec, total;
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
    y.prep = up256(units * sizeof(int2));
    // (words of a lane: two or four of q~ and two of its sum a group, and two factors at most)
    y.rec = y.prep + up256(units * ((size_t)std::max(1, dd / 16) * (y.RU > 4 ? 6 : 4) + 2) * 32 * sizeof(uint32_t));
    y.total = y.rec + up256((units + kMaxShares) * y.RU * (4 + kHeadDim + dd) * sizeof(float));
    return y;
}

// ap: the append of few tokens that comes first, or nullptr.
template <typename T, int DD>
static cudaError_t launch(const Q4DecodeArgs &c, const AppendArgs *ap, void *workspace, cudaStream_t s)
{
    const Layout y = layout(c.B, c.Hq, c.Hkv, DD);
    char *ws = static_cast<char *>(workspace);
    Args a;
    a.c = c;
    a.span = reinterpret_cast<int2 *>(ws + y.span);
    a.prep = reinterpret_cast<uint32_t *>(ws + y.prep);
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
                for (const auto k : {front_kernel<DD, 1, 1>, front_kernel<DD, 1, 2>, front_kernel<DD, 1, 4>,
                                     front_kernel<DD, 2, 4>})
                    if (e2 == cudaSuccess)
                        e2 = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewStageBytes);
                // with another split of an SM's L1 and shared memory the attending blocks would wait for it to run empty
                for (const auto k : {prep_kernel<DD, 1, 1>, prep_kernel<DD, 1, 2>, prep_kernel<DD, 1, 4>, prep_kernel<DD, 2, 4>})
                    if (e2 == cudaSuccess)
                        e2 = cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout,
                                                  cudaSharedmemCarveoutMaxShared);
                for (const auto k : {join_kernel<T, DD, 16, 4>, join_kernel<T, DD, 8, 4>, join_kernel<T, DD, 4, 4>,
                                     join_kernel<T, DD, 2, 4>})
                    if (e2 == cudaSuccess)
                        e2 = cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout,
                                                  cudaSharedmemCarveoutMaxShared);
                for (const auto k : {attend_mma_kernel<DD, 1, 1>, attend_mma_kernel<DD, 1, 2>, attend_mma_kernel<DD, 1, 4>,
                                     attend_mma_kernel<DD, 2, 4>})
                    if (e2 == cudaSuccess)
                        e2 = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                  (int)mma_smem<DD>(DAR_DECODE_MAX_BATCH));
            } else {
                for (const auto k : {attend_kernel<T, DD, 1>, attend_kernel<T, DD, 2>, attend_kernel<T, DD, 4>,
                                     attend_kernel<T, DD, 8>})
                    if (e2 == cudaSuccess)
                        e2 = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                  (int)lanes_smem<8>(DAR_DECODE_MAX_BATCH));
            }
            return e2;
        },
        &sms);
    if (e != cudaSuccess)
        return e;
    cudaLaunchAttribute pdl[1];
    pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    pdl[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = s;
    cfg.attrs = pdl;
    cfg.numAttrs = 1;
    if constexpr (sizeof(T) == 2) {
        constexpr int warps = mma_warps<DD>();
        const int grid = std::min(sms, kMaxShares / warps), units = c.B * c.Hkv * y.RT;
        a.shares = grid * warps;
        const auto prep = y.RU == 1 ? prep_kernel<DD, 1, 1> : y.RU == 2 ? prep_kernel<DD, 1, 2>
                          : y.RU <= 4 ? prep_kernel<DD, 1, 4> : prep_kernel<DD, 2, 4>;
        const auto attend = y.RU == 1 ? attend_mma_kernel<DD, 1, 1> : y.RU == 2 ? attend_mma_kernel<DD, 1, 2>
                            : y.RU <= 4 ? attend_mma_kernel<DD, 1, 4> : attend_mma_kernel<DD, 2, 4>;
        a.front = ap != nullptr;
        if (ap) {
            const auto front = y.RU == 1 ? front_kernel<DD, 1, 1> : y.RU == 2 ? front_kernel<DD, 1, 2>
                               : y.RU <= 4 ? front_kernel<DD, 1, 4> : front_kernel<DD, 2, 4>;
            front<<<ap->B + prep_blocks<DD, kFewThreads / 32>(units), kFewThreads, few_smem<T>(ap->Hkv), s>>>(*ap, a, units);
            e = cudaGetLastError();
        } else {
            prep<<<prep_blocks<DD, kPrepWarps>(units), kPrepWarps * 32, 0, s>>>(a, units);
            e = cudaGetLastError();
        }
        if (e != cudaSuccess)
            return e;
        cfg.gridDim = dim3(grid);
        cfg.blockDim = dim3(warps * 32);
        cfg.dynamicSmemBytes = mma_smem<DD>(c.B);
        e = cudaLaunchKernelEx(&cfg, attend, a);
    } else {
        const int grid = std::min(sms, kMaxShares / kWarps);
        a.shares = grid * kWarps;
        const auto attend = y.RU == 1 ? attend_kernel<T, DD, 1> : y.RU == 2 ? attend_kernel<T, DD, 2>
                            : y.RU <= 4 ? attend_kernel<T, DD, 4> : attend_kernel<T, DD, 8>;
        const size_t smem = y.RU == 1 ? lanes_smem<1>(c.B) : y.RU == 2 ? lanes_smem<2>(c.B)
                            : y.RU <= 4 ? lanes_smem<4>(c.B) : lanes_smem<8>(c.B);
        attend<<<grid, kWarps * 32, smem, s>>>(a);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess)
        return e;
    cfg.dynamicSmemBytes = 0;
    // Few rows may have a partial result of every share each, and many rows few: 2, 4 and 16 warps a row take 17.2, 29 and
    // 44 us with 8 rows of 131072 tokens, 27.2, 27.0 and 33.1 with 1024 of 4096, and 77, 87 and 174 with 16384 of 2048.
    // Of few rows as many as take all that a sequence of the cache's capacity can have in one go: 4, 8 and 16 take 8.3,
    // 8.5 and 9.0 with 901 tokens, 9.4, 8.8 and 9.5 with 2000, and 10.4, 9.9 and 9.7 with 4000.  (By capacity, since
    // lengths are on the device: 901 tokens in a cache with room for 4096 or more take 8.8 to 9.0.)
    constexpr int least = kCostRun > cost_page<DD>() ? kCostRun : cost_page<DD>();  // of a share
    const int rows = c.B * c.Hq;
    const long long parts = unit_capacity<DD>(c.w, c.maxp) / least + 1;
    const int warps = rows >= 1024 ? 2 : rows >= 192 || parts <= 20 ? 4 : parts <= 36 ? 8 : 16;
    cfg.gridDim = dim3((unsigned)rows);
    cfg.blockDim = dim3(warps * 32);
    if (warps == 16)
        return cudaLaunchKernelEx(&cfg, join_kernel<T, DD, 16, 4>, a);
    if (warps == 8)
        return cudaLaunchKernelEx(&cfg, join_kernel<T, DD, 8, 4>, a);
    if (warps == 4)
        return cudaLaunchKernelEx(&cfg, join_kernel<T, DD, 4, 4>, a);
    return cudaLaunchKernelEx(&cfg, join_kernel<T, DD, 2, 4>, a);
}

template <typename T>
static cudaError_t launch_t(int dd, const Q4DecodeArgs &a, const AppendArgs *ap, void *workspace, cudaStream_t s)
{
    switch (dd) {
    case 8: return launch<T, 8>(a, ap, workspace, s);
    case 16: return launch<T, 16>(a, ap, workspace, s);
    case 32: return launch<T, 32>(a, ap, workspace, s);
    case 64: return launch<T, 64>(a, ap, workspace, s);
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
    return dt == DAR_F32 ? q4::launch_t<float>(dd, a, nullptr, workspace, s)
                         : q4::launch_t<bf16>(dd, a, nullptr, workspace, s);
}

cudaError_t launch_step_q4(dar_dtype dt, int dd, const AppendArgs &ap, const Q4DecodeArgs &a, void *workspace,
                           cudaStream_t s)
{
    if (a.B == 0)
        return cudaSuccess;
    if (dt == DAR_BF16 && q4::append_is_few<bf16>(ap, dd))
        return q4::launch_t<bf16>(dd, a, &ap, workspace, s);
    const cudaError_t e = launch_append_q4(dt, dd, ap, s);
    return e != cudaSuccess ? e : launch_decode_q4(dt, dd, a, workspace, s);
}

}  // namespace dar
