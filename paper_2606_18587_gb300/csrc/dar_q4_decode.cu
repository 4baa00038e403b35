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
constexpr int kWarps = 8;        // of a CTA
constexpr int kMaxShares = 1920; // the workspace holds partial results of this many warps
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
                read_pair<GS, false>(page + i * F::kBlock, 2 * lane, x0, x1);
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
                read_pair<GS, true>(page + i * F::kBlock, 2 * lane, x0, x1);
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

template <typename T, int DD>
__global__ void __launch_bounds__(kWarps * 32) attend_kernel(Args a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const Tables t = tables_at(reinterpret_cast<int *>(smem + kWarps * sizeof(LaneSmem)), a.c.B);
    grid_dep_launch();
    build_tables<DD>(a, t);
    attend_lanes<T, DD>(a, t, reinterpret_cast<LaneSmem *>(smem)[threadIdx.x >> 5]);
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
    auto kern = attend_kernel<T, DD>;
    static PerDeviceOnce once;
    int sms = 0;
    cudaError_t e = per_device_once(
        once,
        [&](int d) {
            const cudaError_t e2 = cudaDeviceGetAttribute(&once.value[d], cudaDevAttrMultiProcessorCount, d);
            return e2 != cudaSuccess ? e2
                                     : cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                            (int)(kWarps * sizeof(LaneSmem) + (2 * DAR_DECODE_MAX_BATCH + 1) * 4));
        },
        &sms);
    if (e != cudaSuccess)
        return e;
    const int grid = std::min(sms, kMaxShares / kWarps);
    a.shares = grid * kWarps;
    kern<<<grid, kWarps * 32, kWarps * sizeof(LaneSmem) + (2 * (size_t)c.B + 1) * 4, s>>>(a);
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
