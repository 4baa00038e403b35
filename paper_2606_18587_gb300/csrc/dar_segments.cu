// dar_segments.cu -- two decode steps over the mixed-dimension cache that
// dar_decode.cu does not cover (Eq. 3-4 for the query at position L_b - 1):
//
//  shared   the sequences of a group list the same first P pages.  The softmax of
//           a row over prefix, rest and window is one softmax, so the three can be
//           computed apart and joined by their maxima and sums:
//             o = (sum_local p v + (sum_prefix p v^D + sum_rest p v^D) Uv) / sum p.
//           The prefix part has the same keys for every row of the group: it is a
//           product of all members' queries with one set of keys, read once.
//  scored   every token's attention weight, summed over the query heads of its KV
//           head, is added to a running total.  A weight needs the row's final
//           maximum and sum, so the scores are kept (4 bytes per query head and
//           token) and turned into weights by the second kernel.
//
// Two kernels on the caller's stream, the second launched programmatically:
//
//  segments  The work is a line of stages, cut evenly among the CTAs.  A stage is
//            8 KB of keys and 8 KB of values: 64 lines of 128 bytes each, whatever
//            the type and width.  A unit is a run of stages with the same rows:
//              prefix unit   (group, KV head, up to R rows): the group's prefix;
//                            rows are (member, head) pairs;
//              private unit  (sequence, KV head, up to R rows): the ring, then the
//                            pages behind the prefix.
//            A CTA's cut of a unit leaves one partial result (m, l, acc) per row and
//            key warp.  Units are laid end to end with lengths by their cost, so unit u's
//            cut by CTA k has the slot u + k; the CTAs of a unit's first and last stage
//            leave their numbers for the joining kernel.  (A line for each kind, of which
//            every CTA has a share, takes two set-ups per CTA: 4 to 11 us more in all three
//            batches of 32 and 64 sequences.)
//            Every CTA builds the same tables from the lengths and groups.  One warp
//            fills a ring of shared-memory slots by TMA; four warps consume them,
//            RW of them on different rows and 4 / RW on different keys of a stage.
//  join      a block per row joins its partial results by log-sum-exp and lifts the
//            bottleneck sum once by Uv.  Scored: other blocks turn the kept scores into
//            weights, p = 2^(s - m) / l, and add them.
//
// Bound: HBM for the rings, the private pages, the weights and the kept scores (6.4 TB/s
// while a CTA streams); a prefix that many rows share by its scores (see cut_prefix).
// Measured, calls in a graph: 64 sequences behind 32512 shared tokens, 32 query and 8 KV
// heads, 39 us; 64 sequences behind four prompts 34.4 us (97.5 MB); a scored step of 64
// sequences of 1024 to 32768 tokens 154 us (658 MB).
#include <cuda.h>

#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_sm100.cuh"

namespace dar {
namespace seg {

using namespace sm100;

constexpr int kLines = 64;               // 128-byte lines of keys (and of values) in a stage
constexpr int kHalf = kLines * 128;      // bytes of keys in a stage
constexpr int kSlot = 2 * kHalf;
constexpr int kStages = 4;
constexpr int kWarps = 4;                // consumer warps
constexpr int kThreads = (kWarps + 1) * 32;
constexpr int kSmemPerSm = 228 * 1024;  // of which a CTA's share is its own and 1 KB
constexpr int kMaxCtas = 480;            // the workspace holds partial results of this many CTAs
constexpr int kCostPrivate = 4;          // cost of a private stage
constexpr int kCostUnit = 2;             // cost of a unit's set-up (its place on the line is before the stages)

// Rows a warp takes (a tensor-core tile; registers in fp32), and rows of a unit at most.
template <typename T>
__host__ __device__ constexpr int rpw() { return sizeof(T) == 2 ? 16 : 4; }
template <typename T>
__host__ __device__ constexpr int unit_rows() { return kWarps * rpw<T>(); }

// Rows of a tile of nr rows go to RW warps; the other warps split the keys.
template <typename T>
__host__ __device__ inline int row_warps(int nr) { return nr <= rpw<T>() ? 1 : nr <= 2 * rpw<T>() ? 2 : 4; }

// Cost of a prefix stage for nr rows, in quarters of a private stage.  (bf16, three CTAs on an SM: about 2000
// cycles a private stage where HBM feeds it and 1400 where other CTAs are busy with a prefix, 4030 a prefix
// stage of 64 rows.  fp32, by the row warps: 11.8, 23.2, 33.9 and 46.1 us a thousand stages of 4, 8, 12 and 16 rows
// on the whole GPU, whatever d_down.)
template <typename T>
__host__ __device__ inline int prefix_cost(int nr)
{
    const int c = sizeof(T) == 2 ? (nr + 7) / 8 : (nr + rpw<T>() - 1) / rpw<T>() * 4;
    return c < kCostPrivate ? kCostPrivate : c;
}
constexpr int kCostMax = 16;  // the largest

template <typename T>
__host__ __device__ constexpr int ring_tokens() { return kHalf / (kHeadDim * (int)sizeof(T)); }
template <typename T, int DD>
__host__ __device__ constexpr int page_tokens() { return kHalf / (DD * (int)sizeof(T)); }

// What the joining kernel has to know: of a sequence, and which CTAs have the first and the last cut of a unit.
struct PlanSeq {
    int L;      // tokens
    int xunit;  // index of its group's first prefix unit
    int xrt;    // row tiles of the group (0: not in a group)
    int row0;   // the sequence's first row among the group's rows of a KV head
    int xrows;  // rows of the group per KV head
    int pad[3];
};

struct Args {
    const void *q;
    void *out;
    const int32_t *block_table, *seq_lens, *group, *prefix_pages;
    int32_t *status;
    const float *Uk, *Uv;
    PlanSeq *plan;         // [B]
    int2 *span_p, *span_x; // of every private and every prefix unit
    float *rec_p, *rec_x;  // partial results of private and prefix units
    float *scores;         // [B][Hq][score_stride] scores, unscaled, or nullptr
    float *weights;        // [B][Hkv][slots], or nullptr
    long long slots, score_stride;  // positions of a sequence at capacity, and rounded up to whole 16 bytes
    int B, Hq, Hkv, G, w, maxp, num_pages, ngroups;
    int RP, RTP;  // rows of a private unit at most, row tiles of a (sequence, KV head)
    float c2;     // scale * log2(e)
    float decay;
};

template <int DD>
__host__ __device__ constexpr int rec_p_floats() { return 4 + kHeadDim + DD; }
template <int DD>
__host__ __device__ constexpr int rec_x_floats() { return 4 + DD; }

// Length of a unit of n stages on the line: its set-up, then the stages.
__host__ __device__ inline int unit_length(int n, int cost) { return n ? kCostUnit + n * cost : 0; }

// ------------------------------------------------------------------ tables

struct Tables {  // in shared memory; B or ngroups entries each
    int *L, *grp, *rank, *start, *members;
    int *gP, *gcnt, *gmoff, *gxst, *gxu;
    int *tot;  // lengths of the prefix and of the private units, the largest cost of a stage
};

__host__ __device__ inline int table_ints(int B, int ngroups) { return 5 * B + 5 * ngroups + 4; }

__device__ __forceinline__ Tables table_ptrs(int *p, int B, int ng)
{
    Tables t;
    t.L = p;
    t.grp = t.L + B;
    t.rank = t.grp + B;
    t.start = t.rank + B;
    t.members = t.start + B;
    t.gP = t.members + B;
    t.gcnt = t.gP + ng;
    t.gmoff = t.gcnt + ng;
    t.gxst = t.gmoff + ng;
    t.gxu = t.gxst + ng;
    t.tot = t.gxu + ng;
    return t;
}

__device__ __forceinline__ int distant(int L, int w) { return L > w ? L - w : 0; }

template <typename T, int DD>
__device__ __forceinline__ int private_stages(int L, int w, int P)
{
    constexpr int TW = ring_tokens<T>(), TP = page_tokens<T, DD>();
    const int nwin = min(L, w);
    return (nwin + TW - 1) / TW + (L - nwin - P * kPage + TP - 1) / TP;
}
template <typename T, int DD>
__device__ __forceinline__ int prefix_stages(int P)
{
    constexpr int TP = page_tokens<T, DD>();
    return (P * kPage + TP - 1) / TP;
}

// The sum of v over the lanes before this one.
__device__ __forceinline__ int warp_before(int v, int lane)
{
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o)
            x += y;
    }
    return x - v;
}

// The tables of the line of units, the same in every CTA.  A sequence belongs to its group if all
// of the group's shared pages are distant for it; a group of one is none.
template <typename T, int DD>
__device__ void build_tables(const Args &a, const Tables &t, bool first_cta)
{
    constexpr int kR = unit_rows<T>();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, ng = a.ngroups;
    for (int i = tid; i < ng; i += kThreads) {
        int P = a.prefix_pages[i];
        if (P < 0 || P > a.maxp) {
            if (first_cta)
                report(a.status, DAR_ERR_CAPACITY);
            P = 0;
        }
        t.gP[i] = P;
        t.gcnt[i] = 0;
    }
    for (int b = tid; b < a.B; b += kThreads) {
        int L = a.seq_lens[b];
        if (L < 0 || (long long)L > (long long)a.maxp * kPage + a.w) {
            if (first_cta)
                report(a.status, DAR_ERR_CAPACITY);
            L = 0;
        }
        int g = ng ? a.group[b] : -1;
        if (g < -1 || g >= ng) {
            if (first_cta)
                report(a.status, DAR_ERR_INVALID_ARG);
            g = -1;
        }
        t.L[b] = L;
        t.grp[b] = g;
    }
    __syncthreads();
    if (ng) {
        if (warp == 0) {  // members are numbered in the order of their sequences
            for (int b0 = 0; b0 < a.B; b0 += 32) {
                const int b = b0 + lane;
                int g = b < a.B ? t.grp[b] : -1;
                if (g >= 0 && (t.gP[g] == 0 || distant(t.L[b], a.w) < t.gP[g] * kPage))
                    t.grp[b] = g = -1;
                const unsigned same = __match_any_sync(0xffffffffu, g);
                const int before = __popc(same & ((1u << lane) - 1u));
                const int base = g >= 0 ? t.gcnt[g] : 0;
                __syncwarp();
                if (g >= 0) {
                    t.rank[b] = base + before;
                    if (before == 0)
                        t.gcnt[g] = base + __popc(same);
                }
                __syncwarp();
            }
        }
        __syncthreads();
    }
    // exclusive sums: one warp over the sequences' private units, one over the groups' prefix units
    if (warp == 0) {
        int run = 0;
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int b = b0 + lane;
            int v = 0;
            if (b < a.B) {
                const int g = t.grp[b], P = g >= 0 && t.gcnt[g] >= 2 ? t.gP[g] : 0;
                v = a.Hkv * a.RTP * unit_length(private_stages<T, DD>(t.L[b], a.w, P), kCostPrivate);
            }
            const int x = run + warp_before(v, lane);
            if (b < a.B)
                t.start[b] = x;
            run = __shfl_sync(0xffffffffu, x + v, 31);
        }
        if (lane == 0)
            t.tot[1] = run;
    } else if (warp == 1) {
        int members = 0, units = 0, cost = 0, most = kCostPrivate;
        for (int i0 = 0; i0 < ng; i0 += 32) {
            const int i = i0 + lane;
            int cnt = 0, u = 0, v = 0;
            if (i < ng && t.gcnt[i] >= 2) {
                cnt = t.gcnt[i];
                const int rows = cnt * a.G;
                u = a.Hkv * ((rows + kR - 1) / kR);
                const int c = prefix_cost<T>(min(rows, kR));
                most = max(most, c);
                v = u * unit_length(prefix_stages<T, DD>(t.gP[i]), c);
            }
            const int m0 = warp_before(cnt, lane), u0 = warp_before(u, lane), v0 = warp_before(v, lane);
            if (i < ng) {
                t.gmoff[i] = members + m0;
                t.gxu[i] = units + u0;
                t.gxst[i] = cost + v0;
            }
            members += __shfl_sync(0xffffffffu, m0 + cnt, 31);
            units += __shfl_sync(0xffffffffu, u0 + u, 31);
            cost += __shfl_sync(0xffffffffu, v0 + v, 31);
        }
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) {
            t.tot[0] = cost;
            t.tot[2] = most;
        }
    }
    __syncthreads();
    for (int b = tid; b < a.B; b += kThreads) {
        const int g = t.grp[b];
        if (g >= 0) {
            if (t.gcnt[g] < 2)
                t.grp[b] = -1;
            else
                t.members[t.gmoff[g] + t.rank[b]] = b;
        }
        t.start[b] += t.tot[0];
    }
    __syncthreads();
}

// A CTA's cut of a unit.
struct Cut {
    int b;            // sequence whose block table is read
    int g;            // KV head
    int grp;          // group of a prefix unit, or -1
    int rt;           // row tile
    int rows;         // rows of this tile
    int RW;           // warps on different rows (the others split the keys)
    int unit;         // index among the units of its kind
    int slot;         // slot of the partial results
    bool first, last; // the unit's first, last stage is in the cut
    int st0, st1;     // stages [st0, st1) of the unit
    int nwin;         // ring tokens (0 in a prefix unit)
    int tok0, tok1;   // distant tokens [tok0, tok1) of the whole unit
    int nsw;          // ring stages of the whole unit
};

// The cut that begins at place p of the line; *next = where the unit ends.  False when the rest of
// the unit holds no stage that starts at or after p.
template <typename T, int DD>
__device__ bool find_cut(const Args &a, const Tables &t, int p, int hi, int cta, Cut &c, int &next)
{
    constexpr int kR = unit_rows<T>();
    int start, cost, nst, unit;
    if (p < t.tot[0]) {
        int lo = 0, up = a.ngroups - 1;  // the last group that starts at or before p (empty ones share a start)
        while (lo < up) {
            const int mid = (lo + up + 1) >> 1;
            if (t.gxst[mid] <= p)
                lo = mid;
            else
                up = mid - 1;
        }
        const int i = lo, rows = t.gcnt[i] * a.G, rts = (rows + kR - 1) / kR;
        cost = prefix_cost<T>(min(rows, kR));
        nst = prefix_stages<T, DD>(t.gP[i]);
        const int len = unit_length(nst, cost), u = (p - t.gxst[i]) / len;
        start = t.gxst[i] + u * len;
        unit = t.gxu[i] + u;
        c.grp = i;
        c.g = u / rts;
        c.rt = u % rts;
        c.rows = min(kR, rows - c.rt * kR);
        c.RW = row_warps<T>(c.rows);
        c.b = t.members[t.gmoff[i]];
        c.nwin = c.nsw = 0;
        c.tok0 = 0;
        c.tok1 = t.gP[i] * kPage;
    } else {
        int lo = 0, up = a.B - 1;
        while (lo < up) {
            const int mid = (lo + up + 1) >> 1;
            if (t.start[mid] <= p)
                lo = mid;
            else
                up = mid - 1;
        }
        const int b = lo, P = t.grp[b] >= 0 ? t.gP[t.grp[b]] : 0;
        cost = kCostPrivate;
        nst = private_stages<T, DD>(t.L[b], a.w, P);
        const int len = unit_length(nst, cost), u = (p - t.start[b]) / len;
        start = t.start[b] + u * len;
        unit = b * a.Hkv * a.RTP + u;
        c.grp = -1;
        c.b = b;
        c.g = u / a.RTP;
        c.rt = u % a.RTP;
        c.rows = min(a.RP, a.G - c.rt * kR);
        c.RW = row_warps<T>(a.RP);
        c.nwin = min(t.L[b], a.w);
        c.nsw = (c.nwin + ring_tokens<T>() - 1) / ring_tokens<T>();
        c.tok0 = P * kPage;
        c.tok1 = t.L[b] - c.nwin;
    }
    c.unit = unit;
    c.slot = unit + cta;
    next = start + unit_length(nst, cost);
    const int first = start + kCostUnit;  // place of stage 0
    c.st0 = p <= first ? 0 : (p - first + cost - 1) / cost;
    c.st1 = hi <= first ? 0 : min(nst, (hi - first + cost - 1) / cost);
    c.first = c.st0 == 0;
    c.last = c.st1 == nst;
    return c.st0 < c.st1;
}

// The cuts of this CTA.
struct Walk {
    int p, hi;
    // CTAs that share the line: a share holds a whole stage at least, so every CTA between a unit's first and
    // last has one of it.
    static __device__ __forceinline__ int ctas(const Tables &t)
    {
        return max(1, min((int)gridDim.x, (t.tot[0] + t.tot[1]) / t.tot[2]));
    }
    __device__ __forceinline__ Walk(const Tables &t)
    {
        const int total = t.tot[0] + t.tot[1], n = ctas(t), k = blockIdx.x;
        p = k < n ? (int)((long long)total * k / n) : 0;
        hi = k < n ? (int)((long long)total * (k + 1) / n) : 0;
    }
    template <typename T, int DD>
    __device__ __forceinline__ bool next(const Args &a, const Tables &t, Cut &c)
    {
        while (p < hi) {
            int after;
            const bool some = find_cut<T, DD>(a, t, p, hi, blockIdx.x, c, after);
            p = after;
            if (some)
                return true;
        }
        return false;
    }
};

// Query row `row` of a cut: its (sequence, head).
template <int kR>
__device__ __forceinline__ void row_of(const Args &a, const Tables &t, const Cut &c, int row, int &b, int &h)
{
    if (c.grp < 0) {
        b = c.b;
        h = c.g * a.G + c.rt * kR + row;
    } else {
        const int i = c.rt * kR + row;
        b = t.members[t.gmoff[c.grp] + i / a.G];
        h = c.g * a.G + i % a.G;
    }
}

__device__ __forceinline__ void prefetch_l1(const void *p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p)); }

// Byte of a tile whose 128-byte lines are swizzled in 16-byte chunks.
__device__ __forceinline__ int swz(int byte)
{
    return byte ^ (((byte >> 7) & 7) << 4);
}

__device__ __forceinline__ void load8(const unsigned char *tile, int byte, float (&x)[8], float)
{
    const float4 u = *reinterpret_cast<const float4 *>(tile + swz(byte));
    const float4 v = *reinterpret_cast<const float4 *>(tile + swz(byte + 16));
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
}
__device__ __forceinline__ void load8(const unsigned char *tile, int byte, float (&x)[8], bf16)
{
    unpack(*reinterpret_cast<const uint4 *>(tile + swz(byte)), x, bf16());
}

// Running softmax of a warp's rows over the tokens of its lanes: ROW / 8 lanes share a token, each
// with 8 of its entries; every group of lanes has its own maximum and sum until finish().
constexpr int kRPW = rpw<float>();

template <int ROW>
struct Running {
    static constexpr int LPT = ROW / 8, TPI = 32 / LPT;
    float m[kRPW], l[kRPW], acc[kRPW][8];
    __device__ void clear()
    {
#pragma unroll
        for (int r = 0; r < kRPW; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                acc[r][e] = 0.f;
        }
    }
    __device__ void finish()
    {
#pragma unroll
        for (int off = LPT; off < 32; off <<= 1)
#pragma unroll
            for (int r = 0; r < kRPW; ++r) {
                const float mo = __shfl_xor_sync(0xffffffffu, m[r], off);
                const float lo = __shfl_xor_sync(0xffffffffu, l[r], off);
                const float mn = fmaxf(m[r], mo);
                const float fa = mn == -INFINITY ? 1.f : exp2f(m[r] - mn), fb = mn == -INFINITY ? 1.f : exp2f(mo - mn);
                l[r] = l[r] * fa + lo * fb;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    acc[r][e] = acc[r][e] * fa + __shfl_xor_sync(0xffffffffu, acc[r][e], off) * fb;
                m[r] = mn;
            }
    }
};

// ntok tokens of a stage; this warp takes those of its key share (kw of kws).  score(r, tok, s): what
// becomes of the score of a valid token.
template <typename T, int ROW, typename Score>
__device__ __forceinline__ void lane_stage(const unsigned char *tile, int ntok, int kw, int kws,
                                           const float (&q)[kRPW][8], float c2, Running<ROW> &s, int lane, Score score)
{
    constexpr int LPT = Running<ROW>::LPT, TPI = Running<ROW>::TPI;
    const int grp = lane / LPT, sub = lane % LPT;
    for (int t0 = kw * TPI; t0 < ntok; t0 += kws * TPI) {
        const int t = t0 + grp;
        const bool valid = t < ntok;
        const int byte = (t * ROW + sub * 8) * (int)sizeof(T);
        float k[8], v[8];
        load8(tile, byte, k, T());
        load8(tile + kHalf, byte, v, T());
        float x[kRPW];
#pragma unroll
        for (int r = 0; r < kRPW; ++r) {
            x[r] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[r] = fmaf(q[r][e], k[e], x[r]);
        }
#pragma unroll
        for (int off = 1; off < LPT; off <<= 1)
#pragma unroll
            for (int r = 0; r < kRPW; ++r)
                x[r] += __shfl_xor_sync(0xffffffffu, x[r], off);
        if (!valid) {  // whatever the slot holds there must not reach a sum
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = 0.f;
        }
#pragma unroll
        for (int r = 0; r < kRPW; ++r) {
            const float y = valid ? x[r] * c2 : -INFINITY;
            if (valid && sub == 0)
                score(r, t, x[r]);
            const float mn = fmaxf(s.m[r], y);
            const float base = mn == -INFINITY ? 0.f : mn;
            const float f = exp2f(s.m[r] - base), p = exp2f(y - base);
            s.m[r] = mn;
            s.l[r] = s.l[r] * f + p;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s.acc[r][e] = fmaf(p, v[e], s.acc[r][e] * f);
        }
    }
}

// ------------------------------------------------------------------ segments

// Shared memory: the slots (1024-byte aligned, as the swizzle wants), fp32 query rows, barriers, tables.
constexpr int kQBytes = 2 * unit_rows<float>() * kHeadDim * 4;  // fp32
template <typename T>
inline size_t segments_smem(int B, int ngroups)
{
    return 1024 + (size_t)kStages * kSlot + (sizeof(T) == 4 ? kQBytes : 0) + (size_t)table_ints(B, ngroups) * 4 +
           2 * kStages * 8 + 16;
}

// Scores kept for the joining kernel are among what leaves L2 last (the cache's bytes, which stream past them,
// what leaves first), and the joining kernel lets go of them: the step of the 1B shape, whose 140 MB of scores are
// more than L2, 181 us without and 175 with, 20 of either the setting back of the totals between two calls.
__device__ __forceinline__ void keep_score(float *p, float x, uint64_t policy)
{
    asm volatile("st.global.L2::cache_hint.f32 [%0], %1, %2;" ::"l"(p), "f"(x), "l"(policy) : "memory");
}
__device__ __forceinline__ void keep_scores(float *p, float x, float y, uint64_t policy)
{
    asm volatile("st.global.L2::cache_hint.v2.f32 [%0], {%1, %2}, %3;" ::"l"(p), "f"(x), "f"(y), "l"(policy) : "memory");
}
__device__ __forceinline__ float take_score(const float *p, uint64_t policy)
{
    float x;
    asm volatile("ld.global.L2::cache_hint.f32 %0, [%1], %2;" : "=f"(x) : "l"(p), "l"(policy));
    return x;
}
__device__ __forceinline__ uint64_t l2_evict_last_policy()
{
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}

// ---- the four warps that consume the stages, fp32: CUDA cores
template <typename T, int DD, bool SCORED>
__device__ __forceinline__ void consume_lanes(const Args &a, const Tables &t, const unsigned char *slots, float *qs,
                                              uint64_t *full, uint64_t *empty, volatile int *gave_up)
{
    constexpr int TW = ring_tokens<T>(), TP = page_tokens<T, DD>(), kR = unit_rows<T>();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int n = 0;
    bool alive = true;
    Walk walk(t);
    float *qt = qs + kR * kHeadDim;  // [kR][64] query rows, then [kR][DD] absorbed rows
    const uint64_t last = SCORED ? l2_evict_last_policy() : 0;
    for (Cut c; walk.next<T, DD>(a, t, c);) {
        asm volatile("bar.sync 1, 128;" ::: "memory");  // the rows of the cut before are read
        for (int i = tid; i < kR * kHeadDim; i += kWarps * 32) {
            const int row = i / kHeadDim;
            float x = 0.f;
            if (row < c.rows) {
                int b, h;
                row_of<kR>(a, t, c, row, b, h);
                x = to_f32(static_cast<const T *>(a.q)[((size_t)b * a.Hq + h) * kHeadDim + i % kHeadDim]);
            }
            qs[i] = x;
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        for (int i = tid; i < kR * DD; i += kWarps * 32) {
            const int row = i / DD, e = i % DD;
            const float4 *u = reinterpret_cast<const float4 *>(a.Uk + ((size_t)c.g * DD + e) * kHeadDim);
            const float4 *x = reinterpret_cast<const float4 *>(qs + row * kHeadDim);
            float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
            if (row < c.rows) {
#pragma unroll
                for (int k = 0; k < kHeadDim / 4; ++k) {
                    const float4 uu = __ldg(u + k), xx = x[k];
                    s0 = fmaf(uu.x, xx.x, s0);
                    s1 = fmaf(uu.y, xx.y, s1);
                    s2 = fmaf(uu.z, xx.z, s2);
                    s3 = fmaf(uu.w, xx.w, s3);
                }
            }
            qt[i] = (s0 + s1) + (s2 + s3);
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        const int RW = c.RW, KW = kWarps / RW, rw = warp % RW, kw = warp / RW;
        const int r0 = rw * kRPW;
        Running<kHeadDim> sl;
        Running<DD> sd;
        sl.clear();
        sd.clear();
        float ql[kRPW][8], qd[kRPW][8];
#pragma unroll
        for (int r = 0; r < kRPW; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ql[r][e] = qs[(r0 + r) * kHeadDim + (lane % 8) * 8 + e];
                qd[r][e] = qt[(r0 + r) * DD + (lane % (DD / 8)) * 8 + e];
            }
        float *srow = nullptr;  // scores of the warp's first row
        if constexpr (SCORED)
            srow = a.scores + ((size_t)c.b * a.Hq + c.g * a.G + c.rt * kR + r0) * a.score_stride;
        const int L = c.tok1 + c.nwin;
        for (int st = c.st0; st < c.st1; ++st, ++n) {
            const int s = n % kStages;
            // a warp that gave up computes nothing more, but still meets the others at the barriers
            if (!alive || !mbar_wait_warp(&full[s], (unsigned)((n / kStages) & 1), gave_up)) {
                if (alive && lane == 0)
                    report(a.status, DAR_ERR_DEVICE);
                alive = false;
                continue;
            }
            const unsigned char *tile = slots + s * kSlot;
            if (st < c.nsw) {
                const int t0 = st * TW;
                lane_stage<T, kHeadDim>(tile, min(TW, c.nwin - t0), kw, KW, ql, a.c2, sl, lane,
                                        [&](int r, int tok, float y) {
                                            if constexpr (SCORED) {
                                                // the position that a ring slot holds
                                                const int slot = t0 + tok, pos = (L - 1) - ((L - 1 - slot) % a.w);
                                                if (r0 + r < c.rows)
                                                    keep_score(srow + (size_t)r * a.score_stride + pos, y, last);
                                            }
                                        });
            } else {
                const int t0 = c.tok0 + (st - c.nsw) * TP;
                lane_stage<T, DD>(tile, min(TP, c.tok1 - t0), kw, KW, qd, a.c2, sd, lane,
                                  [&](int r, int tok, float y) {
                                      if constexpr (SCORED) {
                                          if (r0 + r < c.rows)
                                              keep_score(srow + (size_t)r * a.score_stride + t0 + tok, y, last);
                                      }
                                  });
            }
            __syncwarp();
            if (lane == 0)
                mbar_arrive(&empty[s]);
        }
        sl.finish();
        sd.finish();
#pragma unroll
        for (int r = 0; r < kRPW; ++r) {
            if (r0 + r >= c.rows)
                continue;
            const float m = fmaxf(sl.m[r], sd.m[r]);
            const float base = m == -INFINITY ? 0.f : m;
            const float fl = exp2f(sl.m[r] - base), fd = exp2f(sd.m[r] - base);
            float *rec;
            if (c.grp < 0) {
                rec = a.rec_p + ((size_t)c.slot * (KW * a.RP) + kw * a.RP + r0 + r) * rec_p_floats<DD>();
                if (lane < 8)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        rec[4 + lane * 8 + e] = sl.acc[r][e] * fl;
                if (lane < DD / 8)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        rec[4 + kHeadDim + lane * 8 + e] = sd.acc[r][e] * fd;
            } else {
                rec = a.rec_x + ((size_t)c.slot * kR + kw * (RW * kRPW) + r0 + r) * rec_x_floats<DD>();
                if (lane < DD / 8)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        rec[4 + lane * 8 + e] = sd.acc[r][e] * fd;
            }
            if (lane == 0) {
                rec[0] = m;
                rec[1] = sl.l[r] * fl + sd.l[r] * fd;
            }
        }
    }
}

// ---- the same, bf16: tensor cores (mma.sync m16n8k16; a tile has few rows in most calls, and tcgen05
// products of 128 rows would be mostly padding).
//
// Two forms.  cut16: a warp holds 16 rows, which are the M side of the scores (A = queries, B = keys);
// lane 4 i + c holds rows i and i + 8 and columns 2 c, 2 c + 1 of every 8-column tile.  cut8: a warp holds
// up to 8 rows, which are the N side (A = keys, B = queries), so that a product has no idle rows; lane
// 4 i + c holds keys i and i + 8 of a block of 16 and rows 2 c, 2 c + 1, and the weights become a B
// operand by two 8 x 8 transpositions.  Rows up to 8 in a private unit take cut8 (half the products,
// exponentials and accumulators of cut16).

// Two fp32 values as NT bf16 terms each: x = t0 + t1 (+ t2) but for 2^-16 (2^-24) of it.
template <int NT>
__device__ __forceinline__ void split2(float x, float y, uint32_t (&t)[NT])
{
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        t[i] = cvt_bf16x2(x, y);
        x -= bf16lo(t[i]);
        y -= bf16hi(t[i]);
    }
}

__device__ __forceinline__ void ldsm_x2_t(uint32_t saddr, uint32_t (&r)[2])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(saddr));
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// d = a * b where `first`, else d += a * b.
__device__ __forceinline__ void mma_first(bool first, float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (first) {
        const float z[4] = {0.f, 0.f, 0.f, 0.f};
        mma_bf16_c(d, a, b0, b1, z);
    } else {
        mma_bf16_acc(d, a, b0, b1);
    }
}

// 0xffff in the halves whose key (key, key + 1) is below ntok.
__device__ __forceinline__ uint32_t key_mask(int key, int ntok)
{
    return (key < ntok ? 0xffffu : 0u) | (key + 1 < ntok ? 0xffff0000u : 0u);
}

// Shared-memory address of a lane's row in an ldmatrix: block i (16 keys) of the step at `base`, 16-entry
// piece e.  `lane0` is the lane's swizzled place in block 0, piece 0; steps start on 1024-byte boundaries,
// so the swizzle of later blocks and pieces differs by constants (see swz).
template <int ROW>
__device__ __forceinline__ uint32_t frag(uint32_t base, uint32_t lane0, int i, int e)
{
    const uint32_t flip = ROW == 8 ? (uint32_t)(i & 3) << 5 : ROW == 16 ? (uint32_t)(i & 1) << 6 : (uint32_t)e << 5;
    return base + (uint32_t)(i * 16 * ROW * 2) + (lane0 ^ flip);
}

struct Soft {
    float ms[2];     // running maximum of the lane's two rows
    float l[2][2];   // its share of their sums: of either row twice (cut16), or of both rows twice (cut8)
    float bias[2];         // minus the maxima, 0 before the first
    __device__ void clear()
    {
        ms[0] = ms[1] = -INFINITY;
        bias[0] = bias[1] = 0.f;
        l[0][0] = l[0][1] = l[1][0] = l[1][1] = 0.f;
    }
};

// Scores into weights relative to the reference of their row, and their sums.  BYKEY: the layout of cut8, s[i] =
// (key, row 0), (key, row 1), (key + 8, row 0), (key + 8, row 1); else that of cut16, rows 0 0 1 1.
template <int TILES, bool BYKEY>
__device__ __forceinline__ void weigh(float (&s)[TILES][4], float c2, Soft &f)
{
    // pairs of scores that lie in consecutive registers: two rows of a key, or two keys of a row
    const float b0 = f.bias[0], b1 = f.bias[1];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        float x0, x1, y0, y1;
        ffma2(x0, x1, s[i][0], s[i][1], c2, c2, b0, BYKEY ? b1 : b0);
        ffma2(y0, y1, s[i][2], s[i][3], c2, c2, BYKEY ? b0 : b1, b1);
        s[i][0] = ex2_approx(x0);
        s[i][1] = ex2_approx(x1);
        s[i][2] = ex2_approx(y0);
        s[i][3] = ex2_approx(y1);
        add2(f.l[0][0], f.l[0][1], f.l[0][0], f.l[0][1], s[i][0], s[i][1]);
        add2(f.l[1][0], f.l[1][1], f.l[1][0], f.l[1][1], s[i][2], s[i][3]);
    }
}

// The same relative to the running maximum of the row, which the step may raise.
// rescale(f0, f1): what was summed against the old maxima.
template <int TILES, bool BYKEY, typename Rescale>
__device__ __forceinline__ void soft_step(float (&s)[TILES][4], float c2, Soft &f, const Rescale &rescale)
{
    constexpr int P1 = BYKEY ? 2 : 1, Q0 = BYKEY ? 1 : 2;  // the first row's second score, the second row's first
    float m0 = s[0][0], m1 = s[0][Q0];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        m0 = max3(m0, s[i][0], s[i][P1]);
        m1 = max3(m1, s[i][Q0], s[i][3]);
    }
    m0 *= c2;
    m1 *= c2;
    if (__any_sync(0xffffffffu, m0 > f.ms[0] || m1 > f.ms[1])) {
#pragma unroll
        for (int o = BYKEY ? 4 : 1; o < (BYKEY ? 32 : 4); o <<= 1) {
            m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, o));
            m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, o));
        }
        m0 = fmaxf(f.ms[0], m0);
        m1 = fmaxf(f.ms[1], m1);
        const float r0 = m0 == -INFINITY ? 1.f : ex2_approx(f.ms[0] - m0);
        const float r1 = m1 == -INFINITY ? 1.f : ex2_approx(f.ms[1] - m1);
        f.l[0][0] *= r0;
        f.l[0][1] *= BYKEY ? r1 : r0;
        f.l[1][0] *= BYKEY ? r0 : r1;
        f.l[1][1] *= r1;
        rescale(r0, r1);
        f.ms[0] = m0;
        f.ms[1] = m1;
        f.bias[0] = m0 == -INFINITY ? 0.f : -m0;
        f.bias[1] = m1 == -INFINITY ? 0.f : -m1;
    }
    weigh<TILES, BYKEY>(s, c2, f);
}

// Lane's place of an ldmatrix.x4 whose matrices are ordered keys first (0-7 and 8-15, then the next 8
// entries) or entries first.  ROW 8: a row is one 16-byte chunk, so the matrices are four times 8 keys.
template <int ROW, bool KEYS_FIRST>
__device__ __forceinline__ uint32_t lane_place(int lane)
{
    const int mat = lane >> 3, r = lane & 7;
    if (ROW == 8)
        return (uint32_t)swz((8 * mat + r) * 16);
    const int key = 8 * (KEYS_FIRST ? mat & 1 : mat >> 1) + r, half = KEYS_FIRST ? mat >> 1 : mat & 1;
    return (uint32_t)swz(key * ROW * 2 + 16 * half);
}

// Scores of NB blocks of 16 keys, rows on the M side.  qa: KS products of 16 entries each; a key's entries
// repeat every ROW.
template <int ROW, int KS, int NB>
__device__ __forceinline__ void scores16(uint32_t base, const uint32_t (&qa)[KS][4], float (&s)[2 * NB][4], int lane)
{
    const uint32_t lk = lane_place<ROW, false>(lane);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        if constexpr (ROW == 8) {  // both halves of the product's 16 entries are the key's 8
            if (i % 2 == 0) {
                uint32_t k[4];
                ldsm_x4(frag<ROW>(base, lk, i, 0), k);
#pragma unroll
                for (int x = 0; x < KS; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma_first(x == 0, s[2 * i + j], qa[x], k[j], k[j]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < ROW / 16; ++e) {
                uint32_t k[4];
                ldsm_x4(frag<ROW>(base, lk, i, e), k);
#pragma unroll
                for (int x = e; x < KS; x += ROW / 16) {
                    mma_first(x == 0, s[2 * i], qa[x], k[0], k[1]);
                    mma_first(x == 0, s[2 * i + 1], qa[x], k[2], k[3]);
                }
            }
        }
    }
}

// Two weights as WT bf16 terms.  One: rounded, 2^-8.  Two: x = t0 + t1 but for 2^-15, t0 cut off so that both have
// x's sign, and 2^-22 of x added so that t1 is never 0: an infinite value keeps its sign (t0 inf + t1 inf), where a
// zero or a negative remainder would make it NaN.
template <int WT>
__device__ __forceinline__ void weight_terms(float x, float y, uint32_t (&t)[WT])
{
    if constexpr (WT == 1) {
        t[0] = cvt_bf16x2(x, y);
    } else {
        constexpr float kUp = 1.f + 0x1p-22f;
        const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
        t[0] = __byte_perm(a, b, 0x7632);
        t[1] = cvt_bf16x2(fmaf(x, kUp, -__uint_as_float(a & 0xffff0000u)), fmaf(y, kUp, -__uint_as_float(b & 0xffff0000u)));
    }
}

// The weights of 16 keys as WT A operands (see Shape).
template <int WT>
__device__ __forceinline__ void weights16(const float (&s0)[4], const float (&s1)[4], uint32_t (&p)[WT][4])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t t0[WT], t1[WT];
        weight_terms<WT>(s0[2 * h], s0[2 * h + 1], t0);
        weight_terms<WT>(s1[2 * h], s1[2 * h + 1], t1);
#pragma unroll
        for (int y = 0; y < WT; ++y) {
            p[y][h] = t0[y];
            p[y][2 + h] = t1[y];
        }
    }
}

// Value sums of the same keys with weights s, of which WT bf16 terms are operands.  Keys from ntok on (counted from
// the step) do not count.
template <int ROW, int NB, bool MASK, int WT>
__device__ __forceinline__ void sums16(uint32_t base, int ntok, const float (&s)[2 * NB][4], float (&acc)[ROW / 8][4],
                                       int lane)
{
    const uint32_t lv = lane_place<ROW, true>(lane);
    const int c0 = lane & 3;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        uint32_t p[WT][4];
        weights16<WT>(s[2 * i], s[2 * i + 1], p);
        uint32_t mk0 = ~0u, mk1 = ~0u;  // bytes behind the last key must not reach a sum: 0 * NaN is NaN
        if constexpr (MASK) {
            mk0 = key_mask(16 * i + 2 * c0, ntok);
            mk1 = key_mask(16 * i + 8 + 2 * c0, ntok);
        }
        if constexpr (ROW == 8) {
            if (i % 2 == 0) {
                uint32_t v[4];
                ldsm_x4_t(frag<ROW>(base + kHalf, lv, i, 0), v);
                uint32_t p2[WT][4];
                weights16<WT>(s[2 * i + 2], s[2 * i + 3], p2);
                uint32_t mk2 = ~0u, mk3 = ~0u;
                if constexpr (MASK) {
                    mk2 = key_mask(16 * i + 16 + 2 * c0, ntok);
                    mk3 = key_mask(16 * i + 24 + 2 * c0, ntok);
                }
#pragma unroll
                for (int y = 0; y < WT; ++y) {
                    mma_bf16_acc(acc[0], p[y], v[0] & mk0, v[1] & mk1);
                    mma_bf16_acc(acc[0], p2[y], v[2] & mk2, v[3] & mk3);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < ROW / 16; ++e) {
                uint32_t v[4];
                ldsm_x4_t(frag<ROW>(base + kHalf, lv, i, e), v);
#pragma unroll
                for (int y = 0; y < WT; ++y) {
                    mma_bf16_acc(acc[2 * e], p[y], v[0] & mk0, v[1] & mk1);
                    mma_bf16_acc(acc[2 * e + 1], p[y], v[2] & mk0, v[3] & mk1);
                }
            }
        }
    }
}

// Both, with the softmax between them.
template <int ROW, int KS, int NB, bool MASK, int WT, typename Keep, typename Rescale>
__device__ __forceinline__ void step16(uint32_t base, int ntok, const uint32_t (&qa)[KS][4], float c2,
                                       float (&acc)[ROW / 8][4], Soft &f, int lane, const Keep &keep,
                                       const Rescale &rescale)
{
    const int c0 = lane & 3;
    float s[2 * NB][4];
    scores16<ROW, KS, NB>(base, qa, s, lane);
    if constexpr (MASK) {
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (8 * i + 2 * c0 + (e & 1) >= ntok)
                    s[i][e] = -INFINITY;
    }
    keep(s, !MASK);
    soft_step<2 * NB, false>(s, c2, f, rescale);
    sums16<ROW, NB, MASK, WT>(base, ntok, s, acc, lane);
}

// The weights of 16 keys as WT B operands.
template <int WT>
__device__ __forceinline__ void weights8(const float (&s)[4], uint32_t (&p)[WT][2])
{
    uint32_t t0[WT], t1[WT];
    weight_terms<WT>(s[0], s[1], t0);
    weight_terms<WT>(s[2], s[3], t1);
#pragma unroll
    for (int y = 0; y < WT; ++y) {
        p[y][0] = transpose8(t0[y]);
        p[y][1] = transpose8(t1[y]);
    }
}

// The same with up to 8 rows on the N side.  qb: B operands; acc: [16 entries][8 rows] tiles.
template <int ROW, int KS, int NB, bool MASK, int WT, typename Keep, typename Rescale>
__device__ __forceinline__ void step8(uint32_t base, int ntok, const uint32_t (&qb)[KS][2], float c2,
                                      float (&acc)[(ROW + 15) / 16][4], Soft &f, int lane, const Keep &keep,
                                      const Rescale &rescale)
{
    const uint32_t lk = lane_place<ROW, true>(lane), lv = lane_place<ROW, false>(lane);
    const int i0 = lane >> 2, c0 = lane & 3;
    float s[NB][4];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        if constexpr (ROW == 8) {
            if (i % 2 == 0) {
                uint32_t k[4];
                ldsm_x4(frag<ROW>(base, lk, i, 0), k);
                const uint32_t ka[4] = {k[0], k[1], k[0], k[1]}, kb[4] = {k[2], k[3], k[2], k[3]};
#pragma unroll
                for (int x = 0; x < KS; ++x) {
                    mma_first(x == 0, s[i], ka, qb[x][0], qb[x][1]);
                    mma_first(x == 0, s[i + 1], kb, qb[x][0], qb[x][1]);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < ROW / 16; ++e) {
                uint32_t k[4];
                ldsm_x4(frag<ROW>(base, lk, i, e), k);
#pragma unroll
                for (int x = e; x < KS; x += ROW / 16)
                    mma_first(x == 0, s[i], k, qb[x][0], qb[x][1]);
            }
        }
    }
    if constexpr (MASK) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (16 * i + i0 + 8 * (e >> 1) >= ntok)
                    s[i][e] = -INFINITY;
    }
    keep(s, !MASK);
    soft_step<NB, true>(s, c2, f, rescale);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        uint32_t p[WT][2];
        weights8<WT>(s[i], p);
        uint32_t mk0 = ~0u, mk1 = ~0u;
        if constexpr (MASK) {
            mk0 = key_mask(16 * i + 2 * c0, ntok);
            mk1 = key_mask(16 * i + 8 + 2 * c0, ntok);
        }
        if constexpr (ROW == 8) {
            if (i % 2 == 0) {
                uint32_t v[4], mk2 = ~0u, mk3 = ~0u;
                ldsm_x4_t(frag<ROW>(base + kHalf, lv, i, 0), v);
                if constexpr (MASK) {
                    mk2 = key_mask(16 * i + 16 + 2 * c0, ntok);
                    mk3 = key_mask(16 * i + 24 + 2 * c0, ntok);
                }
                const uint32_t va[4] = {v[0] & mk0, 0u, v[1] & mk1, 0u}, vb[4] = {v[2] & mk2, 0u, v[3] & mk3, 0u};
                uint32_t p2[WT][2];
                weights8<WT>(s[i + 1], p2);
#pragma unroll
                for (int y = 0; y < WT; ++y) {
                    mma_bf16_acc(acc[0], va, p[y][0], p[y][1]);
                    mma_bf16_acc(acc[0], vb, p2[y][0], p2[y][1]);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < ROW / 16; ++e) {
                uint32_t v[4];
                ldsm_x4_t(frag<ROW>(base + kHalf, lv, i, e), v);
                const uint32_t vm[4] = {v[0] & mk0, v[1] & mk0, v[2] & mk1, v[3] & mk1};
#pragma unroll
                for (int y = 0; y < WT; ++y)
                    mma_bf16_acc(acc[e], vm, p[y][0], p[y][1]);
            }
        }
    }
}

// What a consumer warp carries from cut to cut.
struct Consumer {
    const Args &a;
    const Tables &t;
    const unsigned char *slots;
    uint64_t *full, *empty;
    volatile int *gave_up;
    int taken, given;  // stages
    bool alive;        // false once a wait gave up: nothing more is computed
    // The next stage's slot, or nullptr.
    __device__ __forceinline__ const unsigned char *take(int lane)
    {
        const int s = taken % kStages;
        if (!alive || !mbar_wait_warp(&full[s], (unsigned)((taken / kStages) & 1), gave_up)) {
            if (alive && lane == 0)
                report(a.status, DAR_ERR_DEVICE);
            alive = false;
            ++taken;
            ++given;
            return nullptr;
        }
        ++taken;
        return slots + s * kSlot;
    }
    __device__ __forceinline__ void give(int lane)
    {
        __syncwarp();
        if (lane == 0)
            mbar_arrive(&empty[given % kStages]);
        ++given;
    }
};

// Steps of a page stage (of 16 * NBP keys) and of a ring stage, products of a global score, and the bf16 terms of q~
// (NT) and of the weights in the value sums (WT).  FINE: three leave 2^-24 of q~ and two 2^-15 of a weight, so that
// nothing shows beside the output's own rounding; where dar_attn_decode has fp32 weights and q~ (one query head a
// slice at d_down 16, and d_down 8), and in scored steps, whose weights are results.  Elsewhere dar_attn_decode rounds
// q~ and the weights to one term; here q~ has two and the weights one (2^-8), which a second one would make exact at
// 39 -> 50 us for 64 sequences behind 32512 shared tokens and 33.7 -> 40 behind four prompts (four heads per KV head).
// FINE costs 16.0 -> 17.3 us for 32 samples of a prompt of 4000 tokens, 12 heads, and 29.8 -> 34.7 us for 64 sequences
// behind 16256 shared tokens, 16 heads; scored steps, bound by HBM, 28.6 -> 29.2 us and 155.6 -> 154.
template <int DD, bool FINE>
struct Shape {
    static constexpr int TW = ring_tokens<bf16>(), TP = page_tokens<bf16, DD>();
    static constexpr int NT = FINE ? 3 : 2, WT = FINE ? 2 : 1;
    static constexpr int KS = DD == 8 ? (NT + 1) / 2 : NT * DD / 16;
    static constexpr int NBP = TP / kWarps >= 64 ? 4 : TP / kWarps / 16, NBW = TW / kWarps / 16;
};

// A row of a cut, as an index into [B][Hq] (-1: none).
template <int kR>
__device__ __forceinline__ long long row_index(const Args &a, const Tables &t, const Cut &c, int row)
{
    if (row >= c.rows)
        return -1;
    int b, h;
    row_of<kR>(a, t, c, row, b, h);
    return (long long)b * a.Hq + h;
}

// The queries of rows r0 and r1 (indices into [B][Hq], -1: none) as A operands.
__device__ __forceinline__ void queries16(const Args &a, long long r0, long long r1, int c0, uint32_t (&qa)[4][4])
{
    const uint32_t *q = static_cast<const uint32_t *>(a.q) + c0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {  // entries 8 e + 2 c, + 1 of either row
        qa[e / 2][e % 2 * 2] = r0 >= 0 ? __ldg(q + r0 * (kHeadDim / 2) + 4 * e) : 0u;
        qa[e / 2][e % 2 * 2 + 1] = r1 >= 0 ? __ldg(q + r1 * (kHeadDim / 2) + 4 * e) : 0u;
    }
}

// q~ = q Uk^T of the same rows as A operands, its NT terms one after the other.  Uk is taken in three bf16
// terms, so that the products are fp32 ones but for 2^-24.
template <int DD, int NT, int KS>
__device__ __forceinline__ void absorbed16(const Args &a, int g, const uint32_t (&qa)[4][4], int lane,
                                           uint32_t (&qt)[KS][4])
{
    const float *u = a.Uk + ((size_t)g * DD + (lane >> 2)) * kHeadDim + 2 * (lane & 3);
    uint32_t prev[NT][2];  // terms of the tile of 8 entries before
#pragma unroll
    for (int j = 0; j < DD / 8; ++j) {
        float x[3][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 u0 = __ldg(reinterpret_cast<const float2 *>(u + j * 8 * kHeadDim + 16 * e));
            const float2 u1 = __ldg(reinterpret_cast<const float2 *>(u + j * 8 * kHeadDim + 16 * e + 8));
            uint32_t t0[3], t1[3];
            split2<3>(u0.x, u0.y, t0);
            split2<3>(u1.x, u1.y, t1);
#pragma unroll
            for (int y = 0; y < 3; ++y)
                mma_first(e == 0, x[y], qa[e], t0[y], t1[y]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[0][i] += x[1][i] + x[2][i];
        uint32_t lo8[NT], hi8[NT];  // terms of rows i and i + 8
        split2<NT>(x[0][0], x[0][1], lo8);
        split2<NT>(x[0][2], x[0][3], hi8);
        if constexpr (DD == 8) {  // two terms are the two halves of a product's 16 entries
#pragma unroll
            for (int y = 0; y < KS; ++y) {
                qt[y][0] = lo8[2 * y];
                qt[y][1] = hi8[2 * y];
                qt[y][2] = 2 * y + 1 < NT ? lo8[2 * y + 1 < NT ? 2 * y + 1 : 0] : 0u;
                qt[y][3] = 2 * y + 1 < NT ? hi8[2 * y + 1 < NT ? 2 * y + 1 : 0] : 0u;
            }
        } else if (j % 2 == 0) {
#pragma unroll
            for (int y = 0; y < NT; ++y) {
                prev[y][0] = lo8[y];
                prev[y][1] = hi8[y];
            }
        } else {
#pragma unroll
            for (int y = 0; y < NT; ++y) {  // term y of entries 16 (j / 2) ..: product y * DD / 16 + j / 2
                uint32_t *o = qt[y * (DD / 16) + j / 2];
                o[0] = prev[y][0];
                o[1] = prev[y][1];
                o[2] = lo8[y];
                o[3] = hi8[y];
            }
        }
    }
}

// A cut of a private unit.
template <int DD, bool SCORED, bool FINE>
__device__ __forceinline__ void cut16(Consumer &w, const Cut &c)
{
    using S = Shape<DD, FINE>;
    constexpr int TW = S::TW, TP = S::TP, NT = S::NT, KS = S::KS, NBP = S::NBP, NBW = S::NBW, kR = unit_rows<bf16>();
    constexpr int NL = kHeadDim / 8;
    const Args &a = w.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i0 = lane >> 2, c0 = lane & 3;
    const int RW = c.RW, KW = kWarps / RW, rw = warp % RW, kw = warp / RW;
    const int r0 = rw * 16 + i0, r1 = r0 + 8;  // this lane's rows
    uint32_t qa[4][4], qt[KS][4];
    queries16(a, row_index<kR>(a, w.t, c, r0), row_index<kR>(a, w.t, c, r1), c0, qa);
    absorbed16<DD, NT>(a, c.g, qa, lane, qt);
    float ol[NL][4], od[DD / 8][4];
    Soft f;
    f.clear();
#pragma unroll
    for (int j = 0; j < NL; ++j)
        ol[j][0] = ol[j][1] = ol[j][2] = ol[j][3] = 0.f;
#pragma unroll
    for (int j = 0; j < DD / 8; ++j)
        od[j][0] = od[j][1] = od[j][2] = od[j][3] = 0.f;
    const bool ring = c.st0 < c.nsw;  // the cut holds ring stages
    auto rescale = [&](float f0, float f1) {
        if (ring)
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                ol[j][0] *= f0;
                ol[j][1] *= f0;
                ol[j][2] *= f1;
                ol[j][3] *= f1;
            }
#pragma unroll
        for (int j = 0; j < DD / 8; ++j) {
            od[j][0] *= f0;
            od[j][1] *= f0;
            od[j][2] *= f1;
            od[j][3] *= f1;
        }
    };
    float *s0 = nullptr, *s1 = nullptr;  // scores of the lane's rows
    if constexpr (SCORED) {
        float *x = a.scores + ((size_t)c.b * a.Hq + c.g * a.G + c.rt * kR) * a.score_stride;
        s0 = r0 < c.rows ? x + (size_t)r0 * a.score_stride : nullptr;
        s1 = r1 < c.rows ? x + (size_t)r1 * a.score_stride : nullptr;
    }
    const int L = c.tok1 + c.nwin;
    const uint64_t last = SCORED ? l2_evict_last_policy() : 0;
    int st = c.st0;
    for (; st < min(c.st1, c.nsw); ++st) {
        const unsigned char *slot = w.take(lane);
        if (!slot)
            continue;
        const uint32_t tile = smem_u32(slot);
        const int t0 = st * TW, ntok = min(TW, c.nwin - t0);
        for (int k = kw * (TW / KW); k < min(ntok, (kw + 1) * (TW / KW)); k += 16 * NBW) {
            auto keep = [&](const float (&x)[2 * NBW][4], bool) {
                if constexpr (SCORED) {
#pragma unroll
                    for (int i = 0; i < 2 * NBW; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int kk = k + 8 * i + 2 * c0 + e;
                            if (kk >= ntok)
                                continue;
                            const int pos = (L - 1) - ((L - 1 - (t0 + kk)) % a.w);  // held by ring slot t0 + kk
                            if (s0)
                                keep_score(s0 + pos, x[i][e], last);
                            if (s1)
                                keep_score(s1 + pos, x[i][2 + e], last);
                        }
                }
            };
            const uint32_t base = tile + k * kHeadDim * 2;
            if (k + 16 * NBW <= ntok)
                step16<kHeadDim, 4, NBW, false, S::WT>(base, ntok - k, qa, a.c2, ol, f, lane, keep, rescale);
            else
                step16<kHeadDim, 4, NBW, true, S::WT>(base, ntok - k, qa, a.c2, ol, f, lane, keep, rescale);
        }
        w.give(lane);
    }
    for (; st < c.st1; ++st) {
        const unsigned char *slot = w.take(lane);
        if (!slot)
            continue;
        const uint32_t tile = smem_u32(slot);
        const int t0 = c.tok0 + (st - c.nsw) * TP, ntok = min(TP, c.tok1 - t0);
        for (int k = kw * (TP / KW); k < min(ntok, (kw + 1) * (TP / KW)); k += 16 * NBP) {
            auto keep = [&](const float (&x)[2 * NBP][4], bool) {
                if constexpr (SCORED) {
#pragma unroll
                    for (int i = 0; i < 2 * NBP; ++i) {
                        const int kk = k + 8 * i + 2 * c0;
                        auto put = [&](float *row, float x0, float x1) {
                            if (kk + 1 < ntok)
                                keep_scores(row + t0 + kk, x0, x1, last);
                            else if (kk < ntok)  // the next position is the ring's
                                keep_score(row + t0 + kk, x0, last);
                        };
                        if (s0)
                            put(s0, x[i][0], x[i][1]);
                        if (s1)
                            put(s1, x[i][2], x[i][3]);
                    }
                }
            };
            const uint32_t base = tile + k * DD * 2;
            if (k + 16 * NBP <= ntok)
                step16<DD, KS, NBP, false, S::WT>(base, ntok - k, qt, a.c2, od, f, lane, keep, rescale);
            else
                step16<DD, KS, NBP, true, S::WT>(base, ntok - k, qt, a.c2, od, f, lane, keep, rescale);
        }
        w.give(lane);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        float l = f.l[y][0] + f.l[y][1];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        const int row = y ? r1 : r0;
        if (row >= c.rows)
            continue;
        float *rec = a.rec_p + ((size_t)c.slot * (KW * a.RP) + kw * a.RP + row) * rec_p_floats<DD>();
#pragma unroll
        for (int j = 0; j < NL; ++j)
            *reinterpret_cast<float2 *>(rec + 4 + 8 * j + 2 * c0) = make_float2(ol[j][2 * y], ol[j][2 * y + 1]);
#pragma unroll
        for (int j = 0; j < DD / 8; ++j)
            *reinterpret_cast<float2 *>(rec + 4 + kHeadDim + 8 * j + 2 * c0) =
                make_float2(od[j][2 * y], od[j][2 * y + 1]);
        if (c0 == 0)
            *reinterpret_cast<float2 *>(rec) = make_float2(f.ms[y], l);
    }
}

// A cut of a prefix unit.  Bound: of a block of 16 x 16 scores the products take 48 cycles of an SM's quarter and
// the rest of its instructions (8 exponentials, 4 conversions, 8 paired sums and products, 4 maxima) some 37,
// which do not overlap: a loop of nothing else takes 85, without the maxima 71 (this kernel 84; 90 with them).
// (Two tiles of 16 rows a warp, which share what is loaded of a key: as many cycles a score, and units twice as
// large to deal out.  The scores of the next step started before this one's are exponentiated: 5850 cycles a
// stage instead of 4450.  Four CTAs an SM: as many cycles a score.)
template <int DD, bool FINE>
__device__ __forceinline__ void cut_prefix(Consumer &w, const Cut &c)
{
    using S = Shape<DD, FINE>;
    constexpr int TP = S::TP, KS = S::KS, NB = S::NBP, kR = unit_rows<bf16>();
    const Args &a = w.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = lane & 3;
    const int RW = c.RW, KW = kWarps / RW, rw = warp % RW, kw = warp / RW, r0 = rw * 16 + (lane >> 2);
    uint32_t qt[KS][4];
    {
        uint32_t qa[4][4];
        queries16(a, row_index<kR>(a, w.t, c, r0), row_index<kR>(a, w.t, c, r0 + 8), c0, qa);
        absorbed16<DD, S::NT>(a, c.g, qa, lane, qt);
    }
    float od[DD / 8][4];
    Soft f;
    f.clear();
#pragma unroll
    for (int j = 0; j < DD / 8; ++j)
        od[j][0] = od[j][1] = od[j][2] = od[j][3] = 0.f;
    auto rescale = [&](float f0, float f1) {
#pragma unroll
        for (int j = 0; j < DD / 8; ++j) {
            od[j][0] *= f0;
            od[j][1] *= f0;
            od[j][2] *= f1;
            od[j][3] *= f1;
        }
    };
    // Once every row has seen a finite score, weights are taken relative to the maximum so far without looking
    // for a new one: they and their sums are as exact far above 1, and only sums beyond kFar (an overflow's too)
    // have the step done again with its maximum.  A row's weights sum to 8 kFar at most (four lanes' two sums), so
    // value sums are finite for values up to 2^104.  (64 sequences behind 32512 shared tokens: 39.3 us at scores of
    // standard deviation 1 to 4, 41.9 at 12, where a tenth of the steps is done again.)
    constexpr float kFar = 1048576.f;
    bool settled = false;
    for (int st = c.st0; st < c.st1; ++st) {
        const unsigned char *slot = w.take(lane);
        if (!slot)
            continue;
        const int k0 = kw * (TP / KW), k1 = min(c.tok1 - (c.tok0 + st * TP), k0 + TP / KW);
        uint32_t base = smem_u32(slot) + k0 * DD * 2;
        for (int k = k0; k < k1; k += 16 * NB, base += 16 * NB * DD * 2) {  // whole pages, and so whole steps
            float s[2 * NB][4];
            scores16<DD, KS, NB>(base, qt, s, lane);
            const float l00 = f.l[0][0], l01 = f.l[0][1], l10 = f.l[1][0], l11 = f.l[1][1];
            bool far = !settled;
            if (settled) {
                weigh<2 * NB, false>(s, a.c2, f);
                far = fmaxf(fmaxf(f.l[0][0], f.l[0][1]), fmaxf(f.l[1][0], f.l[1][1])) > kFar;
            }
            if (__any_sync(0xffffffffu, far)) {
                if (settled) {
                    f.l[0][0] = l00, f.l[0][1] = l01, f.l[1][0] = l10, f.l[1][1] = l11;
                    scores16<DD, KS, NB>(base, qt, s, lane);
                }
                soft_step<2 * NB, false>(s, a.c2, f, rescale);
                settled = __all_sync(0xffffffffu, f.ms[0] > -INFINITY && f.ms[1] > -INFINITY);
            }
            sums16<DD, NB, false, S::WT>(base, 16 * NB, s, od, lane);
        }
        w.give(lane);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        float l = f.l[y][0] + f.l[y][1];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        const int row = r0 + 8 * y;
        if (row >= c.rows)
            continue;
        float *rec = a.rec_x + ((size_t)c.slot * kR + kw * (RW * 16) + row) * rec_x_floats<DD>();
#pragma unroll
        for (int j = 0; j < DD / 8; ++j)
            *reinterpret_cast<float2 *>(rec + 4 + 8 * j + 2 * c0) = make_float2(od[j][2 * y], od[j][2 * y + 1]);
        if (c0 == 0)
            *reinterpret_cast<float2 *>(rec) = make_float2(f.ms[y], l);
    }
}

// A private unit's cut of up to 8 rows; the four warps share its keys.
template <int DD, bool SCORED, bool FINE>
__device__ __forceinline__ void cut8(Consumer &w, const Cut &c)
{
    using S = Shape<DD, FINE>;
    constexpr int TW = S::TW, TP = S::TP, NT = S::NT, KS = S::KS, NBP = S::NBP, NBW = S::NBW, kR = unit_rows<bf16>();
    constexpr int ND = (DD + 15) / 16;
    const Args &a = w.a;
    const int lane = threadIdx.x & 31, kw = threadIdx.x >> 5, i0 = lane >> 2, c0 = lane & 3;
    // B operands: row i0, entries 8 e + 2 c, + 1
    uint32_t qb[4][2], qt[KS][2];
    {
        const long long row = row_index<kR>(a, w.t, c, i0);
        const uint32_t *q = static_cast<const uint32_t *>(a.q) + row * (kHeadDim / 2) + c0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            qb[e / 2][e % 2] = row >= 0 ? __ldg(q + 4 * e) : 0u;
    }
    // q~^T = Uk q^T, 16 entries at a time, as in absorbed16; its terms turned into B operands
#pragma unroll
    for (int j = 0; j < ND; ++j) {
        const float *u = a.Uk + ((size_t)c.g * DD + 16 * j + i0) * kHeadDim + 2 * c0;
        float z[3][4], x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t t[4][3];
#pragma unroll
            for (int y = 0; y < 4; ++y) {  // entries i0, i0 + 8 and inputs 2 c, 2 c + 8
                float2 v = make_float2(0.f, 0.f);
                if (DD >= 16 || y % 2 == 0)
                    v = __ldg(reinterpret_cast<const float2 *>(u + (y & 1) * 8 * kHeadDim + 16 * e + 8 * (y >> 1)));
                split2<3>(v.x, v.y, t[y]);
            }
#pragma unroll
            for (int y = 0; y < 3; ++y) {
                const uint32_t ua[4] = {t[0][y], t[1][y], t[2][y], t[3][y]};
                mma_first(e == 0, z[y], ua, qb[e][0], qb[e][1]);
            }
        }
#pragma unroll
        for (int y = 0; y < 4; ++y)
            x[y] = z[0][y] + (z[1][y] + z[2][y]);
        uint32_t lo8[NT], hi8[NT];  // terms of entries i0 and i0 + 8, rows 2 c, 2 c + 1
        split2<NT>(x[0], x[1], lo8);
        split2<NT>(x[2], x[3], hi8);
        if constexpr (DD == 8) {
#pragma unroll
            for (int y = 0; y < KS; ++y) {
                qt[y][0] = transpose8(lo8[2 * y]);
                qt[y][1] = 2 * y + 1 < NT ? transpose8(lo8[2 * y + 1 < NT ? 2 * y + 1 : 0]) : 0u;
            }
        } else {
#pragma unroll
            for (int y = 0; y < NT; ++y) {
                qt[y * ND + j][0] = transpose8(lo8[y]);
                qt[y * ND + j][1] = transpose8(hi8[y]);
            }
        }
    }
    float ol[kHeadDim / 16][4], od[ND][4];
    Soft f;
    f.clear();
#pragma unroll
    for (int j = 0; j < kHeadDim / 16; ++j)
        ol[j][0] = ol[j][1] = ol[j][2] = ol[j][3] = 0.f;
#pragma unroll
    for (int j = 0; j < ND; ++j)
        od[j][0] = od[j][1] = od[j][2] = od[j][3] = 0.f;
    auto rescale = [&](float f0, float f1) {
#pragma unroll
        for (int j = 0; j < kHeadDim / 16; ++j) {
            ol[j][0] *= f0;
            ol[j][1] *= f1;
            ol[j][2] *= f0;
            ol[j][3] *= f1;
        }
#pragma unroll
        for (int j = 0; j < ND; ++j) {
            od[j][0] *= f0;
            od[j][1] *= f1;
            od[j][2] *= f0;
            od[j][3] *= f1;
        }
    };
    float *s0 = nullptr, *s1 = nullptr;  // scores of the lane's rows 2 c, 2 c + 1
    if constexpr (SCORED) {
        float *x = a.scores + ((size_t)c.b * a.Hq + c.g * a.G) * a.score_stride;
        s0 = 2 * c0 < c.rows ? x + (size_t)(2 * c0) * a.score_stride : nullptr;
        s1 = 2 * c0 + 1 < c.rows ? x + (size_t)(2 * c0 + 1) * a.score_stride : nullptr;
    }
    const int L = c.tok1 + c.nwin;
    const uint64_t last = SCORED ? l2_evict_last_policy() : 0;
    int st = c.st0;
    for (; st < min(c.st1, c.nsw); ++st) {
        const unsigned char *slot = w.take(lane);
        if (!slot)
            continue;
        const int k = kw * (TW / kWarps), t0 = st * TW, ntok = min(TW, c.nwin - t0) - k;
        auto keep = [&](const float (&x)[NBW][4], bool) {
            if constexpr (SCORED) {
#pragma unroll
                for (int i = 0; i < NBW; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int kk = 16 * i + 8 * e + i0;
                        if (kk >= ntok)
                            continue;
                        const int pos = (L - 1) - ((L - 1 - (t0 + k + kk)) % a.w);  // held by that ring slot
                        if (s0)
                            keep_score(s0 + pos, x[i][2 * e], last);
                        if (s1)
                            keep_score(s1 + pos, x[i][2 * e + 1], last);
                    }
            }
        };
        const uint32_t base = smem_u32(slot) + k * kHeadDim * 2;
        if (16 * NBW <= ntok)
            step8<kHeadDim, 4, NBW, false, S::WT>(base, ntok, qb, a.c2, ol, f, lane, keep, rescale);
        else if (ntok > 0)
            step8<kHeadDim, 4, NBW, true, S::WT>(base, ntok, qb, a.c2, ol, f, lane, keep, rescale);
        w.give(lane);
    }
    for (; st < c.st1; ++st) {
        const unsigned char *slot = w.take(lane);
        if (!slot)
            continue;
        const int t0 = c.tok0 + (st - c.nsw) * TP, nstage = min(TP, c.tok1 - t0);
#pragma unroll 1
        for (int k = kw * (TP / kWarps); k < (kw + 1) * (TP / kWarps); k += 16 * NBP) {
            const int ntok = nstage - k;
            auto keep = [&](const float (&x)[NBP][4], bool whole) {
                if constexpr (SCORED) {
#pragma unroll
                    for (int i = 0; i < NBP; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int kk = 16 * i + 8 * e + i0;
                            if (whole || kk < ntok) {
                                if (s0)
                                    keep_score(s0 + t0 + k + kk, x[i][2 * e], last);
                                if (s1)
                                    keep_score(s1 + t0 + k + kk, x[i][2 * e + 1], last);
                            }
                        }
                }
            };
            const uint32_t base = smem_u32(slot) + k * DD * 2;
            if (16 * NBP <= ntok)
                step8<DD, KS, NBP, false, S::WT>(base, ntok, qt, a.c2, od, f, lane, keep, rescale);
            else if (ntok > 0)
                step8<DD, KS, NBP, true, S::WT>(base, ntok, qt, a.c2, od, f, lane, keep, rescale);
        }
        w.give(lane);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        float l = f.l[0][y] + f.l[1][y];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
            l += __shfl_xor_sync(0xffffffffu, l, o);
        const int row = 2 * c0 + y;
        if (row >= c.rows)
            continue;
        float *rec = a.rec_p + ((size_t)c.slot * (kWarps * a.RP) + kw * a.RP + row) * rec_p_floats<DD>();
#pragma unroll
        for (int j = 0; j < kHeadDim / 16; ++j) {
            rec[4 + 16 * j + i0] = ol[j][y];
            rec[4 + 16 * j + 8 + i0] = ol[j][2 + y];
        }
#pragma unroll
        for (int j = 0; j < ND; ++j) {
            rec[4 + kHeadDim + 16 * j + i0] = od[j][y];
            if (DD >= 16)
                rec[4 + kHeadDim + 16 * j + 8 + i0] = od[j][2 + y];
        }
        if (i0 == 0)
            *reinterpret_cast<float2 *>(rec) = make_float2(f.ms[y], l);
    }
}

// SMALL: private units have at most 8 rows.  FINE: see Shape.
template <int DD, bool SCORED, bool SMALL, bool FINE>
__device__ __forceinline__ void consume_mma(const Args &a, const Tables &t, const unsigned char *slots, uint64_t *full,
                                            uint64_t *empty, volatile int *gave_up)
{
    Consumer w{a, t, slots, full, empty, gave_up, 0, 0, true};
    Walk walk(t);
    for (Cut c; walk.next<bf16, DD>(a, t, c);) {
        if (!SCORED && c.grp >= 0) {
            cut_prefix<DD, FINE>(w, c);
        } else if constexpr (SMALL) {
            cut8<DD, SCORED, FINE>(w, c);
        } else {
            cut16<DD, SCORED, FINE>(w, c);
        }
    }
}

template <typename T, int DD, bool SCORED, bool SMALL, bool FINE>
__global__ void __launch_bounds__(kThreads, SMALL ? 3 : 1) segments_kernel(const __grid_constant__ CUtensorMap m_wk,
                                                            const __grid_constant__ CUtensorMap m_wv,
                                                            const __grid_constant__ CUtensorMap m_pk,
                                                            const __grid_constant__ CUtensorMap m_pv, Args a)
{
    constexpr int TW = ring_tokens<T>(), TP = page_tokens<T, DD>();
    constexpr int PL = kPage * DD * (int)sizeof(T) / 128;  // lines of a head's page
    constexpr int BOX = PL < kLines ? PL : kLines;         // lines of one copy
    constexpr int WL = kHeadDim * (int)sizeof(T) / 128;    // lines of a ring row
    extern __shared__ unsigned char raw[];
    unsigned char *slots = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    unsigned char *rows_at = slots + kStages * kSlot;  // fp32: query rows
    uint64_t *full = reinterpret_cast<uint64_t *>(rows_at + (sizeof(T) == 4 ? kQBytes : 0));
    uint64_t *empty = full + kStages;
    int *ints = reinterpret_cast<int *>(empty + kStages);
    volatile int *gave_up = ints;
    const Tables t = table_ptrs(ints + 1, a.B, a.ngroups);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], kWarps);
        }
        *gave_up = 0;
        mbar_init_fence();
    }
    build_tables<T, DD>(a, t, blockIdx.x == 0);  // its barriers also publish the mbarriers
    if (blockIdx.x == 0) {
        for (int b = tid; b < a.B; b += kThreads) {
            PlanSeq s{};
            const int g = t.grp[b];
            s.L = t.L[b];
            if (g >= 0) {
                s.xrows = t.gcnt[g] * a.G;
                s.xrt = (s.xrows + unit_rows<T>() - 1) / unit_rows<T>();
                s.xunit = t.gxu[g];
                s.row0 = t.rank[b] * a.G;
            }
            a.plan[b] = s;
        }
    }
    if (warp == kWarps) {
        // ---- one warp fills the slots
        // a sequence's own bytes are read once: they leave L2 first, not the scores, records and prefixes
        const uint64_t once = l2_evict_first_policy();
        int n = 0;
        bool alive = true;
        Walk walk(t);
        for (Cut c; alive && walk.next<T, DD>(a, t, c);) {
            if (lane == 0) {
                int2 *span = (c.grp < 0 ? a.span_p : a.span_x) + c.unit;
                if (c.first)
                    span->x = blockIdx.x;
                if (c.last)
                    span->y = blockIdx.x;
            }
            // what the consumers will want first, while they are at the cut before
            for (int i = lane; i < DD * 2; i += 32)
                prefetch_l1(a.Uk + ((size_t)c.g * DD * 2 + i) * (kHeadDim / 2));
            for (int i = lane; i < c.rows; i += 32) {
                int b, h;
                row_of<unit_rows<T>()>(a, t, c, i, b, h);
                prefetch_l1(static_cast<const T *>(a.q) + ((size_t)b * a.Hq + h) * kHeadDim);
            }
            const int32_t *table = a.block_table + (size_t)c.b * a.maxp;
            const int ring0 = (c.b * a.Hkv + c.g) * a.w;
            int ids0 = -1, ids = -1;  // block-table entries ids0 .. ids0 + 31, one per lane
            for (int st = c.st0; st < c.st1; ++st, ++n) {
                const int s = n % kStages;
                if (n >= kStages && !mbar_wait_warp(&empty[s], (unsigned)((n / kStages - 1) & 1), gave_up)) {
                    alive = false;
                    break;
                }
                unsigned char *dst = slots + s * kSlot;
                if (st < c.nsw) {
                    if (lane == 0) {
                        mbar_expect_tx(&full[s], kSlot);
                        const int y = (ring0 + st * TW) * WL;
                        tma_load_2d_hint(smem_u32(dst), &m_wk, 0, y, &full[s], once);
                        tma_load_2d_hint(smem_u32(dst + kHalf), &m_wv, 0, y, &full[s], once);
                    }
                    continue;
                }
                const int tok = c.tok0 + (st - c.nsw) * TP;
                const int end = min(c.tok1, tok + TP);
                const int pg0 = tok / kPage, pg1 = (end + kPage - 1) / kPage;
                if (ids0 < 0 || pg1 > ids0 + 32 || pg0 < ids0) {
                    ids0 = pg0;
                    ids = ids0 + lane < a.maxp ? __ldg(table + ids0 + lane) : -1;
                }
                unsigned bytes = 0;
                for (int pg = pg0; pg < pg1; ++pg) {
                    const int id = __shfl_sync(0xffffffffu, ids, pg - ids0);
                    bytes += id >= 0 && id < a.num_pages ? 2u * BOX * 128u : 0u;
                }
                if (lane == 0)
                    mbar_expect_tx(&full[s], bytes);
                for (int pg = pg0; pg < pg1; ++pg) {
                    const int id = __shfl_sync(0xffffffffu, ids, pg - ids0);
                    if (lane != 0)
                        continue;
                    if (id < 0 || id >= a.num_pages) {
                        report(a.status, DAR_ERR_CAPACITY);
                        continue;
                    }
                    const int y = (id * a.Hkv + c.g) * PL + (tok % kPage) * PL / kPage;
                    const int off = (pg - pg0) * BOX * 128;
                    if (c.grp < 0) {
                        tma_load_2d_hint(smem_u32(dst + off), &m_pk, 0, y, &full[s], once);
                        tma_load_2d_hint(smem_u32(dst + kHalf + off), &m_pv, 0, y, &full[s], once);
                    } else {  // the group's other row tiles read them too
                        tma_load_2d(dst + off, &m_pk, 0, y, &full[s]);
                        tma_load_2d(dst + kHalf + off, &m_pv, 0, y, &full[s]);
                    }
                }
            }
        }
        if (!alive) {
            // a wait gave up: the copies in flight land (again a bounded wait) before the block leaves
            if (lane == 0)
                report(a.status, DAR_ERR_DEVICE);
            for (int r = max(0, n - kStages); r < n; ++r)
                mbar_wait(&full[r % kStages], (unsigned)((r / kStages) & 1), nullptr);
        }
        return;
    }

    // ---- four warps consume them
    if constexpr (sizeof(T) == 2)
        consume_mma<DD, SCORED, SMALL, FINE>(a, t, slots, full, empty, gave_up);
    else
        consume_lanes<T, DD, SCORED>(a, t, slots, reinterpret_cast<float *>(rows_at), full, empty, gave_up);
}

// ------------------------------------------------------------------ join

// Where the partial results of a row are: result i of n, those of a CTA's 2^lg key warps one after the other.
struct Parts {
    const float *base;
    int n, lg;
    size_t far, near;  // from one CTA's to the next one's, from one key warp's to the next one's
    __device__ __forceinline__ const float *at(int i) const
    {
        return base + (size_t)(i >> lg) * far + (size_t)(i & ((1 << lg) - 1)) * near;
    }
};

// The CTAs of a unit (in range whatever a kernel that gave up has left).
__device__ __forceinline__ void span_of(const int2 *span, int &k0, int &k1)
{
    const int2 s = *span;
    k0 = min(max(s.x, 0), kMaxCtas - 1);
    k1 = min(max(s.y, k0), kMaxCtas - 1);
}

// log2 of the key warps beside RW row warps
__device__ __forceinline__ int key_warps_lg(int RW) { return RW == 1 ? 2 : RW == 2 ? 1 : 0; }

template <typename T, int DD>
__device__ __forceinline__ Parts private_parts(const Args &a, int b, int g, int j)
{
    constexpr int kR = unit_rows<T>();
    Parts r;
    const int rt = j / kR, row = j % kR;
    const size_t u = ((size_t)b * a.Hkv + g) * a.RTP + rt;
    int k0, k1;
    span_of(a.span_p + u, k0, k1);
    r.lg = key_warps_lg(row_warps<T>(a.RP));
    r.near = (size_t)a.RP * rec_p_floats<DD>();
    r.far = r.near << r.lg;
    r.n = (k1 - k0 + 1) << r.lg;
    r.base = a.rec_p + (u + k0) * r.far + (size_t)row * rec_p_floats<DD>();
    return r;
}

template <typename T, int DD>
__device__ __forceinline__ Parts prefix_parts(const Args &a, const PlanSeq &s, int g, int j)
{
    constexpr int kR = unit_rows<T>();
    Parts r{nullptr, 0, 0, 0, 0};
    if (s.xrt == 0)
        return r;
    const int i = s.row0 + j, rt = i / kR, row = i % kR, RW = row_warps<T>(min(kR, s.xrows - rt * kR));
    const size_t u = s.xunit + g * s.xrt + rt;
    int k0, k1;
    span_of(a.span_x + u, k0, k1);
    r.lg = key_warps_lg(RW);
    r.near = (size_t)(RW * rpw<T>()) * rec_x_floats<DD>();
    r.far = (size_t)kR * rec_x_floats<DD>();
    r.n = (k1 - k0 + 1) << r.lg;
    r.base = a.rec_x + (u + k0) * r.far + (size_t)row * rec_x_floats<DD>();
    return r;
}

constexpr int kJoinPer = 8;        // tokens of a thread at a time
constexpr int kJoinTokens = 2048;  // tokens whose weights a block updates

// The entries lane, lane + 32 (and so on) of a run of partial results, joined on the way: NLOC and ND
// registers of the full-width and of the bottleneck sum.
template <int NLOC, int DD>
struct Joined {
    static constexpr int ND = (DD + 31) / 32, N = NLOC + ND;
    float m, l, x[N];
    __device__ void clear()
    {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = 0.f;
    }
    // parts first, first + step, .., U of them in flight together; LOC: they hold full-width sums before the others
    template <bool LOC, int U>
    __device__ void add(const Parts &r, int first, int step, int lane)
    {
        for (int i0 = first; i0 < r.n; i0 += U * step) {
            float mo[U], lo[U], o[U][N];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * step;
                mo[u] = -INFINITY;
                lo[u] = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    o[u][e] = 0.f;
                if (i >= r.n)
                    continue;
                const float *p = r.at(i);
                const float2 ml = *reinterpret_cast<const float2 *>(p);
                mo[u] = ml.x;
                lo[u] = ml.y;
                if (LOC)
#pragma unroll
                    for (int e = 0; e < NLOC; ++e)
                        o[u][e] = p[4 + 32 * e + lane];
                const float *d = p + 4 + (LOC ? kHeadDim : 0);
#pragma unroll
                for (int e = 0; e < ND; ++e)
                    if (32 * e + lane < DD)
                        o[u][NLOC + e] = d[32 * e + lane];
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < U; ++u)
                top = fmaxf(top, mo[u]);
            const float base = top == -INFINITY ? 0.f : top, f = ex2_approx(m - base);
            m = top;
            l *= f;
#pragma unroll
            for (int e = 0; e < N; ++e)
                x[e] *= f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float fo = ex2_approx(mo[u] - base);
                l = fmaf(lo[u], fo, l);
#pragma unroll
                for (int e = 0; e < N; ++e)
                    x[e] = fmaf(o[u][e], fo, x[e]);
            }
        }
    }
};

// Blocks 0 .. B * Hq - 1 write one output row each: the warps take the row's partial results in turn, are
// joined, and the bottleneck sum is lifted.  Scored: the other blocks update the weights of kJoinTokens
// tokens of a (sequence, KV head) each.
template <typename T, int DD, bool SCORED, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) join_kernel(Args a, int chunks)
{
    constexpr int kJoinThreads = WARPS * 32, U = WARPS > 4 ? 8 : 4;
    constexpr int NLOC = kHeadDim / 32;
    using J = Joined<NLOC, DD>;
    __shared__ float part[WARPS][2 + 32 * J::N], sum[kHeadDim + DD];
    extern __shared__ float stat[];  // SCORED: [G][2] m and 1 / l
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rows = a.B * a.Hq;
    if (!SCORED || (int)blockIdx.x < rows) {
        const int row = blockIdx.x, b = row / a.Hq, h = row % a.Hq, g = h / a.G, j = h % a.G;
        // the lift's columns are the caller's: nothing on the stream before writes them any more
        float uv[DD >= 32 ? 1 : DD];
        if constexpr (DD < 32) {
            if (threadIdx.x < kHeadDim)
#pragma unroll
                for (int e = 0; e < DD; ++e)
                    uv[e] = __ldg(a.Uv + ((size_t)g * DD + e) * kHeadDim + threadIdx.x);
        }
        grid_dep_wait();
        const PlanSeq s = a.plan[b];
        J x;
        x.clear();
        if (s.L > 0) {
            x.template add<true, U>(private_parts<T, DD>(a, b, g, j), warp, WARPS, lane);
            if constexpr (!SCORED)
                x.template add<false, U>(prefix_parts<T, DD>(a, s, g, j), warp, WARPS, lane);
        }
        float *p = part[warp];
        if (lane == 0) {
            p[0] = x.m;
            p[1] = x.l;
        }
#pragma unroll
        for (int e = 0; e < J::N; ++e)
            p[2 + 32 * e + lane] = x.x[e];
        __syncthreads();
        float m = -INFINITY, f[WARPS], l = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i)
            m = fmaxf(m, part[i][0]);
        if (m == -INFINITY)
            m = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            f[i] = ex2_approx(part[i][0] - m);
            l = fmaf(part[i][1], f[i], l);
        }
        for (int t = threadIdx.x; t < kHeadDim + DD; t += kJoinThreads) {
            float y = 0.f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i)
                y = fmaf(f[i], part[i][2 + t], y);
            sum[t] = y;
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
                o = fmaf(sum[kHeadDim + e], __ldg(a.Uv + ((size_t)g * DD + e) * kHeadDim + threadIdx.x), o);
        }
        static_cast<T *>(a.out)[(size_t)row * kHeadDim + threadIdx.x] = from_f32<T>(s.L == 0 ? 0.f : o / l);
        return;
    }
    if constexpr (SCORED) {
        // the last chunks first: their scores were kept last and are the likeliest to be in L2 still
        const int heads = a.B * a.Hkv, i = (int)blockIdx.x - rows, bg = i % heads, chunk = chunks - 1 - i / heads;
        const int b = bg / a.Hkv, g = bg % a.Hkv;
        grid_dep_wait();
        const int L = a.plan[b].L;
        if ((long long)chunk * kJoinTokens >= L)
            return;
        for (int j = warp; j < a.G; j += WARPS) {  // the row's maximum and sum
            const Parts r = private_parts<T, DD>(a, b, g, j);
            float m = -INFINITY, l = 0.f;
            for (int i = lane; i < r.n; i += 32) {
                const float2 v = *reinterpret_cast<const float2 *>(r.at(i));
                const float mn = fmaxf(m, v.x), base = mn == -INFINITY ? 0.f : mn;
                l = l * ex2_approx(m - base) + v.y * ex2_approx(v.x - base);
                m = mn;
            }
            float top = m;
#pragma unroll
            for (int off = 16; off; off >>= 1)
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float base = top == -INFINITY ? 0.f : top;
            l *= ex2_approx(m - base);
#pragma unroll
            for (int off = 16; off; off >>= 1)
                l += __shfl_xor_sync(0xffffffffu, l, off);
            if (lane == 0) {
                stat[2 * j] = base;
                stat[2 * j + 1] = 1.f / l;
            }
        }
        __syncthreads();
        const uint64_t first = l2_evict_first_policy();
        float *w = a.weights + (size_t)bg * a.slots;
        const float *x = a.scores + ((size_t)b * a.Hq + (size_t)g * a.G) * a.score_stride;
        const int end = (int)min((long long)L, (long long)(chunk + 1) * kJoinTokens);
        for (int t0 = chunk * kJoinTokens + threadIdx.x; t0 < end; t0 += kJoinThreads * kJoinPer) {
            float old[kJoinPer], p[kJoinPer];
#pragma unroll
            for (int i = 0; i < kJoinPer; ++i) {
                const int t = t0 + i * kJoinThreads;
                old[i] = a.decay != 0.f && t < end ? w[t] : 0.f;
                p[i] = 0.f;
            }
#pragma unroll 2
            for (int j = 0; j < a.G; ++j) {
                const float m = stat[2 * j], il = stat[2 * j + 1];
                const float *xj = x + (size_t)j * a.score_stride;
                float y[kJoinPer];
#pragma unroll
                for (int i = 0; i < kJoinPer; ++i)
                    y[i] = t0 + i * kJoinThreads < end ? take_score(xj + t0 + i * kJoinThreads, first) : 0.f;
#pragma unroll
                for (int i = 0; i < kJoinPer; ++i)
                    p[i] = fmaf(ex2_approx(fmaf(y[i], a.c2, -m)), il, p[i]);
            }
#pragma unroll
            for (int i = 0; i < kJoinPer; ++i) {
                const int t = t0 + i * kJoinThreads;
                if (t < end)
                    w[t] = a.decay != 0.f ? fmaf(a.decay, old[i], p[i]) : p[i];
            }
        }
    }
}

// ------------------------------------------------------------------ launch

struct Layout {
    size_t plan, span_p, span_x, rec_p, rec_x, scores, total;
    int RP, RTP;
};

static size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

template <typename T>
static Layout layout(int B, int Hq, int Hkv, int dd, int w, int maxp, bool scored)
{
    constexpr int kR = unit_rows<T>();
    Layout y;
    const int G = Hq / Hkv;
    y.RP = G < kR ? G : kR;
    y.RTP = (G + kR - 1) / kR;
    const size_t units = (size_t)B * Hkv * y.RTP + kMaxCtas;
    const size_t rows_p = (size_t)(kWarps / row_warps<T>(y.RP)) * y.RP;
    // a group of n rows has ceil(n / R) tiles, and there are at most B / 2 groups of two or more
    const size_t units_x = (size_t)Hkv * ((size_t)B * G / kR + B / 2 + 1) + kMaxCtas;
    const size_t slots = ((size_t)maxp * kPage + w + 3) / 4 * 4;
    y.plan = 0;
    y.span_p = y.plan + up256((size_t)B * sizeof(PlanSeq));
    y.span_x = y.span_p + up256(units * sizeof(int2));
    y.rec_p = y.span_x + up256(units_x * sizeof(int2));
    y.rec_x = y.rec_p + up256(units * rows_p * (4 + kHeadDim + dd) * sizeof(float));
    y.scores = y.rec_x + (scored ? 0 : up256(units_x * kR * (4 + dd) * sizeof(float)));
    y.total = y.scores + (scored ? up256((size_t)B * Hq * slots * sizeof(float)) : 0);
    return y;
}

template <typename T, int DD, bool SCORED, bool SMALL, bool FINE>
static cudaError_t launch_t(const SegmentArgs &s, void *workspace, cudaStream_t st)
{
    const Layout y = layout<T>(s.B, s.Hq, s.Hkv, DD, s.w, s.maxp, SCORED);
    char *ws = static_cast<char *>(workspace);
    Args a;
    a.q = s.q;
    a.out = s.out;
    a.block_table = s.block_table;
    a.seq_lens = s.seq_lens;
    a.group = s.group;
    a.prefix_pages = s.prefix_pages;
    a.status = s.status;
    a.Uk = s.Uk;
    a.Uv = s.Uv;
    a.plan = reinterpret_cast<PlanSeq *>(ws + y.plan);
    a.span_p = reinterpret_cast<int2 *>(ws + y.span_p);
    a.span_x = reinterpret_cast<int2 *>(ws + y.span_x);
    a.rec_p = reinterpret_cast<float *>(ws + y.rec_p);
    a.rec_x = reinterpret_cast<float *>(ws + y.rec_x);
    a.scores = SCORED ? reinterpret_cast<float *>(ws + y.scores) : nullptr;
    a.weights = s.weights;
    a.slots = (long long)s.maxp * kPage + s.w;
    a.score_stride = (a.slots + 3) / 4 * 4;
    a.B = s.B;
    a.Hq = s.Hq;
    a.Hkv = s.Hkv;
    a.G = s.Hq / s.Hkv;
    a.w = s.w;
    a.maxp = s.maxp;
    a.num_pages = s.num_pages;
    a.ngroups = s.n_groups;
    a.RP = y.RP;
    a.RTP = y.RTP;
    a.c2 = s.c2;
    a.decay = s.decay;
    constexpr int PL = kPage * DD * (int)sizeof(T) / 128;
    const unsigned long long ring_lines = (unsigned long long)s.B * s.Hkv * s.w * kHeadDim * sizeof(T) / 128;
    const unsigned long long pool_lines = (unsigned long long)(s.num_pages > 0 ? s.num_pages : 1) * s.Hkv * PL;
    const int box = PL < kLines ? PL : kLines;
    // 128-byte lines whatever the type: 64 two-byte elements each
    CUtensorMap wk, wv, pk{}, pv{};
    if (!make_tma_2d_bf16(&wk, s.win_k, ring_lines, 64, kLines) || !make_tma_2d_bf16(&wv, s.win_v, ring_lines, 64, kLines))
        return cudaErrorInvalidValue;
    if (s.maxp > 0 && (!make_tma_2d_bf16(&pk, s.pool_kd, pool_lines, 64, box) ||
                       !make_tma_2d_bf16(&pv, s.pool_vd, pool_lines, 64, box)))
        return cudaErrorInvalidValue;
    auto kern = segments_kernel<T, DD, SCORED, SMALL, FINE>;
    // CTAs per SM by registers (once per device); by shared memory below
    static PerDeviceOnce once;
    int fit = 0, sms = 0, dev = 0;
    cudaError_t e = per_device_once(
        once,
        [&](int d) {
            cudaError_t e2 = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                  (int)segments_smem<T>(DAR_DECODE_MAX_BATCH, DAR_DECODE_MAX_BATCH));
            if (e2 == cudaSuccess)
                e2 = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&once.value[d], kern, kThreads, 0);
            return e2;
        },
        &fit);
    if (e == cudaSuccess)
        e = cudaGetDevice(&dev);
    if (e == cudaSuccess)
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess)
        return e;
    const size_t smem = segments_smem<T>(s.B, s.n_groups);
    const int per_sm = min(min(max(fit, 1), 3), max(1, (int)(kSmemPerSm / (smem + 1024))));
    const int grid = min(per_sm * sms, kMaxCtas);
    kern<<<grid, kThreads, smem, st>>>(wk, wv, pk, pv, a);
    e = cudaGetLastError();
    if (e != cudaSuccess)
        return e;
    cudaLaunchAttribute pdl[1];
    pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    pdl[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cfg.attrs = pdl;
    cfg.numAttrs = 1;
    const int chunks = SCORED ? (int)((a.slots + kJoinTokens - 1) / kJoinTokens) : 0, rows = s.B * s.Hq;
    cfg.gridDim = dim3((unsigned)(rows + s.B * s.Hkv * chunks));
    cfg.dynamicSmemBytes = SCORED ? a.G * 2 * sizeof(float) : 0;
    // Few rows may have a partial result of every CTA's four warps each, and many rows few, of which two warps
    // are soon done.  Calls with 4 / 16 warps, us: one row over 32768 tokens 21 / 13, 128 shared rows 14.3 / 11.8,
    // 512 shared rows 12.6 / 19.7; with 4 / 2: 2048 shared rows 36.2 / 34.1.  Scored blocks also update weights:
    // 96 rows 14.9 / 16.6, and 2 warps are no faster.
    const int warps = rows < (SCORED ? 64 : 192) ? 16 : rows < 1024 || SCORED ? 4 : 2;
    cfg.blockDim = dim3(warps * 32);
    if (warps == 16)
        return cudaLaunchKernelEx(&cfg, join_kernel<T, DD, SCORED, 16>, a, chunks);
    if (warps == 4)
        return cudaLaunchKernelEx(&cfg, join_kernel<T, DD, SCORED, 4>, a, chunks);
    return cudaLaunchKernelEx(&cfg, join_kernel<T, DD, SCORED, SCORED ? 4 : 2>, a, chunks);
}

template <typename T, int DD, bool SCORED>
static cudaError_t launch_rows(const SegmentArgs &s, void *ws, cudaStream_t st)
{
    constexpr bool kMma = sizeof(T) == 2;
    const int G = s.Hq / s.Hkv;
    if constexpr (kMma && !SCORED && DD == 16) {  // dar_attn_decode takes an odd number of heads one by one
        if (G % 2)
            return G <= 8 ? launch_t<T, DD, SCORED, true, true>(s, ws, st)
                          : launch_t<T, DD, SCORED, false, true>(s, ws, st);
    }
    constexpr bool kFine = kMma && (SCORED || DD == 8);
    return kMma && G <= 8 ? launch_t<T, DD, SCORED, kMma, kFine>(s, ws, st)
                          : launch_t<T, DD, SCORED, false, kFine>(s, ws, st);
}

template <typename T, bool SCORED>
static cudaError_t launch_dd(int dd, const SegmentArgs &s, void *ws, cudaStream_t st)
{
    switch (dd) {
    case 8: return launch_rows<T, 8, SCORED>(s, ws, st);
    case 16: return launch_rows<T, 16, SCORED>(s, ws, st);
    case 32: return launch_rows<T, 32, SCORED>(s, ws, st);
    case 64: return launch_rows<T, 64, SCORED>(s, ws, st);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace seg

size_t segments_workspace_bytes(dar_dtype dt, int B, int Hq, int Hkv, int dd, int w, int maxp, bool scored)
{
    return dt == DAR_F32 ? seg::layout<float>(B, Hq, Hkv, dd, w, maxp, scored).total
                         : seg::layout<bf16>(B, Hq, Hkv, dd, w, maxp, scored).total;
}

// Blocks of the joining kernel: one per output row and, scored, one per kJoinTokens tokens of a (sequence, KV head).
double segments_join_blocks(int B, int Hq, int Hkv, int w, int maxp, bool scored)
{
    const long long chunks = scored ? ((long long)maxp * kPage + w + seg::kJoinTokens - 1) / seg::kJoinTokens : 0;
    return (double)B * Hq + (double)B * Hkv * chunks;
}

// Upper bound of the line's length: every sequence at capacity, as private units and once more as
// prefix units.
double segments_line_bound(dar_dtype dt, int B, int Hq, int Hkv, int dd, int w, int maxp)
{
    const int es = dt == DAR_F32 ? 4 : 2, G = Hq / Hkv;
    const double stages = (double)w * kHeadDim * es / seg::kHalf + (double)maxp * kPage * dd * es / seg::kHalf + 2;
    const int R = dt == DAR_F32 ? seg::unit_rows<float>() : seg::unit_rows<bf16>();
    return (double)B * Hkv * ((G + R - 1) / R) * (stages * (seg::kCostPrivate + seg::kCostMax) + 2 * seg::kCostUnit);
}

cudaError_t launch_segments(dar_dtype dt, int dd, const SegmentArgs &s, void *workspace, cudaStream_t st)
{
    if (s.B == 0)
        return cudaSuccess;
    if (s.weights)
        return dt == DAR_F32 ? seg::launch_dd<float, true>(dd, s, workspace, st)
                             : seg::launch_dd<bf16, true>(dd, s, workspace, st);
    return dt == DAR_F32 ? seg::launch_dd<float, false>(dd, s, workspace, st)
                         : seg::launch_dd<bf16, false>(dd, s, workspace, st);
}

}  // namespace dar
