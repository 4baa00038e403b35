// dar_evict.cu -- eviction from the mixed-dimension cache by accumulated attention
// weight.  A sequence with n = L - w > keep distant tokens gives up n - keep of them,
// per KV head: the first `protect` tokens stay, and of the others the keep - protect
// with the largest weights (of equal ones the lower positions; NaN ranks lowest).
//
// Attention does not depend on the order of distant tokens (positions are encoded
// before the cache, and every distant token is farther than the window), so what stays
// is not packed in order: tokens that stay at positions >= keep move, in ascending
// order, into the positions < keep that evicted tokens leave.  Sources and
// destinations are disjoint, so the moves run in any order and in place, and no other
// row is read or written: at most min(keep, n - keep) rows of each head instead of keep.
//
// One cluster of C thread blocks per (sequence, KV head) selects and moves; C grows as
// there are fewer of them.  The blocks share the candidates in C consecutive slices, a block's warps its
// slice in consecutive parts:
//   1. the smallest weight that stays: a radix selection on an ordered key, 11 + 11 + 10
//      bits, from the cluster's histograms (each block's in its own shared memory, read
//      by all); then two bits for every key, larger than that weight and equal to it,
//      and each warp's counts of holes, movers and equal keys in its part;
//   2. with the counts of the parts before, each warp knows which of its equal keys stay and
//      where its lists begin, and lists the positions of its holes and movers in order;
//   3. hole i is filled from mover i, by all threads of the cluster; rows pass through
//      shared memory by asynchronous copies, which hold no registers while they are in flight.
// A second cluster per head turns the ring meanwhile: it holds position p in slot p mod w,
// and positions drop by e = n - keep, so by e mod w slots.  Through shared memory where the
// cluster's holds it, else in place by the reflections s -> -s and s -> -s - e (mod w),
// whose swaps are disjoint, one after the other.
// A second kernel sets the lengths, which the clusters of other heads read before.
// Bound: HBM for the rows that move and the weights, read once from there and then from
// L2; short calls, which a cluster of one block takes, by the selection's chain of scans and
// barriers.
#include <cooperative_groups.h>

#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_sm100.cuh"

namespace dar {
namespace evict {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;  // the largest portable cluster

struct Work {
    // [B * Hkv][maxp * 32] each: there are as many holes as movers, at most half the distant tokens
    int32_t *holes, *movers;
    uint4 *bits;        // [B * Hkv][maxp + 5 * kMaxCluster]: for slices whose bits shared memory does not hold
    float *window;      // [B * Hkv][w] the window's weights on their way down
    int32_t *new_lens;  // [B], -1: unchanged
};

// Order of weights as unsigned numbers: larger weight, larger key; NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);  // -0 + 0 = +0
    return x == x ? u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u) : 0u;
}

constexpr int kBins = 2048;
constexpr int kCoarse = 64;    // sums of 32 bins each, read first
constexpr int kBitRuns = 256;  // runs of 128 candidates whose bits fit there: slices of 32768
constexpr int kAhead = 4;      // 16-byte loads of a thread in flight
constexpr int kStage = 8;      // 16-byte pieces of rows of a thread in flight

// Counts of a part of the candidates: keys equal to the smallest that stays below and from the budget's
// position on, and the others' holes and movers.
struct __align__(16) Counts {
    int eq_lo, eq_hi, hole, mover;
};

// The candidates of a slice in runs of 128, the first one shorter so that the others are aligned: candidate
// origin + 128 c + 4 lane + v is bit `lane` of word v of run c, in `up` (it stays) and `eq` (equal to the
// smallest that stays).
struct Select {
    int hist[2][kBins], coarse[2][kCoarse];
    uint4 bits[2 * kBitRuns];
};
union Shared {
    Select s;
    uint4 stage[kStage * kThreads];
};

// Calls f(c, valid, x) for the runs c0 .. c1 - 1 in order, whole warps: candidates origin + 128 c + 4 lane + v,
// bit v of valid for those in [i0, i1).
template <typename F>
__device__ __forceinline__ void runs_each(const float *cand, int origin, int i0, int i1, int c0, int c1, F f)
{
    const int lane = threadIdx.x & 31;
    auto ragged = [&](int c) {
        const int i = origin + 128 * c + 4 * lane;
        float y[4];
        unsigned valid = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const bool in = i + v >= i0 && i + v < i1;
            y[v] = in ? cand[i + v] : 0.f;
            valid |= in ? 1u << v : 0u;
        }
        f(c, valid, y);
    };
    int c = c0;
    if (c < c1 && origin + 128 * c < i0)
        ragged(c++);
    for (; c + kAhead <= c1 && origin + 128 * (c + kAhead) <= i1; c += kAhead) {
        float4 x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            x[u] = *reinterpret_cast<const float4 *>(cand + origin + 128 * (c + u) + 4 * lane);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const float y[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
            f(c + u, 15u, y);
        }
    }
    for (; c < c1; ++c)
        ragged(c);
}

// The lanes' bits v of `nibble` as the words of a run, stored by one lane.
__device__ __forceinline__ void put_run(uint4 *to, unsigned nibble)
{
    uint4 w;
    w.x = __ballot_sync(0xffffffffu, nibble & 1u);
    w.y = __ballot_sync(0xffffffffu, nibble & 2u);
    w.z = __ballot_sync(0xffffffffu, nibble & 4u);
    w.w = __ballot_sync(0xffffffffu, nibble & 8u);
    if ((threadIdx.x & 31) == 0)
        *to = w;
}
__device__ __forceinline__ unsigned nibble_of(const uint4 &w, int lane)
{
    return (w.x >> lane & 1u) | (w.y >> lane & 1u) << 1 | (w.z >> lane & 1u) << 2 | (w.w >> lane & 1u) << 3;
}
// Of a lane's four candidates from i on, those in [lo, hi).
__device__ __forceinline__ unsigned nibble_in(int i, int lo, int hi)
{
    const int a = lo - i, b = hi - i;
    const unsigned from = a <= 0 ? 15u : a >= 4 ? 0u : 15u << a & 15u, to = b >= 4 ? 15u : b <= 0 ? 0u : (1u << b) - 1u;
    return from & to;
}

// The bits set in the nibbles of the lanes before this one, and *all = in those of all lanes.
__device__ __forceinline__ int rank4(unsigned nibble, int &all)
{
    const unsigned c = __popc(nibble), below = (1u << (threadIdx.x & 31)) - 1u;
    const unsigned b0 = __ballot_sync(0xffffffffu, c & 1u), b1 = __ballot_sync(0xffffffffu, c & 2u),
                   b2 = __ballot_sync(0xffffffffu, c & 4u);
    all = __popc(b0) + 2 * __popc(b1) + 4 * __popc(b2);
    return __popc(b0 & below) + 2 * __popc(b1 & below) + 4 * __popc(b2 & below);
}

// A cluster of one block needs no cluster barrier.
__device__ __forceinline__ void sync_cluster(cg::cluster_group &cl, int C)
{
    if (C > 1)
        cl.sync();
    else
        __syncthreads();
}

// Slot s of head id's rings goes to slot s - turn (mod w).
__device__ __forceinline__ void turn_ring(const EvictArgs &a, uint4 *stage, cg::cluster_group &cl, int id, int turn)
{
    if (turn == 0)
        return;
    const int C = (int)cl.num_blocks(), r = (int)cl.block_rank(), rp = a.ring_bytes / 16;
    uint4 *k = static_cast<uint4 *>(a.win_k) + (size_t)id * a.w * rp, *v = static_cast<uint4 *>(a.win_v) + (size_t)id * a.w * rp;
    const int share = (a.w + C - 1) / C, s0 = min(a.w, r * share), s1 = min(a.w, s0 + share);
    if ((long long)share * 2 * rp <= kStage * kThreads) {
        const int pieces = (s1 - s0) * rp;
        for (int x = threadIdx.x; x < pieces; x += kThreads) {
            sm100::cp_async16(sm100::smem_u32(&stage[x]), k + (size_t)s0 * rp + x);
            sm100::cp_async16(sm100::smem_u32(&stage[pieces + x]), v + (size_t)s0 * rp + x);
        }
        sm100::cp_async_wait_all();
        sync_cluster(cl, C);  // every slot is read
        for (int x = threadIdx.x; x < pieces; x += kThreads) {
            const int s = s0 + x / rp, to = s >= turn ? s - turn : s - turn + a.w;
            k[(size_t)to * rp + x % rp] = stage[x];
            v[(size_t)to * rp + x % rp] = stage[pieces + x];
        }
        return;
    }
    const int all = r * kThreads + threadIdx.x, step = C * kThreads;
    auto reflect = [&](int c) {  // swaps slot s with (c - s) mod w, 0 <= c < w
        for (long long x = all; x < (long long)a.w * rp; x += step) {
            const int s = (int)(x / rp), j = (int)(x % rp), o = c - s + (c < s ? a.w : 0);
            if (s >= o)
                continue;
            const size_t ps = (size_t)s * rp + j, po = (size_t)o * rp + j;
            const uint4 ks = k[ps], ko = k[po], vs = v[ps], vo = v[po];
            k[ps] = ko;
            k[po] = ks;
            v[ps] = vo;
            v[po] = vs;
        }
    };
    reflect(0);
    sync_cluster(cl, C);
    reflect(a.w - turn);
}

__global__ void __launch_bounds__(kThreads, 5) evict_kernel(EvictArgs a, Work wk)
{
    __shared__ __align__(16) Shared sh;
    __shared__ int pick[3];           // digit, how many keys lie above it, how many have it
    __shared__ Counts parts[kWarps];  // of the warps' parts
    __shared__ Counts mine;           // of the block's slice
    cg::cluster_group cl = cg::this_cluster();
    const int C = (int)cl.num_blocks(), r = (int)cl.block_rank();
    const int heads = a.B * a.Hkv, which = blockIdx.x / C;
    const bool turns = which >= heads;  // this cluster turns a ring
    const int id = turns ? which - heads : which, b = id / a.Hkv, g = id % a.Hkv;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    // ---- what this sequence has to do; every block of it decides the same
    const int L = a.seq_lens[b], keep = a.keep[b], first = a.protect ? a.protect[b] : 0;
    const long long slots = (long long)a.maxp * kPage + a.w;
    int err = DAR_OK;
    if (L < 0 || (long long)L > slots)
        err = DAR_ERR_CAPACITY;
    else if (keep < 0 || first < 0 || first > keep)
        err = DAR_ERR_INVALID_ARG;
    const int n = L > a.w ? L - a.w : 0;
    const bool go = err == DAR_OK && n > keep;
    const int32_t *table = a.block_table + (size_t)b * a.maxp;
    if (go) {
        int bad = 0;
        for (int p = first / kPage + tid; p < (n + kPage - 1) / kPage; p += kThreads) {
            const int v = __ldg(table + p);
            bad |= v < 0 || v >= a.num_pages;
        }
        if (__syncthreads_or(bad))
            err = DAR_ERR_CAPACITY;
    }
    if (g == 0 && r == 0 && tid == 0 && !turns) {
        if (err != DAR_OK)
            report(a.status, err);
        wk.new_lens[b] = go && err == DAR_OK ? keep + a.w : -1;
    }
    if (!go || err != DAR_OK)
        return;

    if (turns) {
        turn_ring(a, sh.stage, cl, id, (n - keep) % a.w);
        return;
    }
    float *w = a.weights + (size_t)id * slots;
    const int m = n - first, need = keep - first;
    const int sl = (m + C - 1) / C, i0 = min(m, r * sl), i1 = min(m, i0 + sl);
    const float *cand = w + first;
    const int edge = need;  // candidates from here on lie at positions >= keep
    // runs of 128 and each warp's part of them
    const int origin = i0 - (int)((reinterpret_cast<uintptr_t>(cand + i0) & 15u) >> 2);
    const int runs = i1 > i0 ? (i1 - origin + 127) / 128 : 0, per = (runs + kWarps - 1) / kWarps;
    const int c0 = min(runs, warp * per), c1 = min(runs, c0 + per);
    // up and eq: a slice has m / C + 3 candidates at most, so a block's share of the workspace holds them
    const int most = (m + C - 1) / C / 128 + 2;
    uint4 *up_runs = runs <= kBitRuns ? sh.s.bits
                                      : wk.bits + (size_t)id * (a.maxp + 5 * kMaxCluster) + (size_t)r * 2 * most;
    uint4 *eq_runs = up_runs + (runs <= kBitRuns ? kBitRuns : most);

    // ---- 1. the smallest key that stays, and how many of its equals do
    uint32_t prefix = 0xffffffffu;  // above every key: nothing stays
    int left = need;                // the key sought is the left-th largest of those that match prefix
    if (need > 0) {
        prefix = 0;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            int *h = sh.s.hist[pass & 1], *co = sh.s.coarse[pass & 1];
            for (int i = tid; i < kBins / 4; i += kThreads)
                reinterpret_cast<int4 *>(h)[i] = make_int4(0, 0, 0, 0);
            __syncthreads();
            const uint32_t above = pass == 0 ? 0u : ~0u << (pass == 1 ? 21 : 10);  // digits known already
            const uint32_t bins = pass == 2 ? 1023u : 2047u;
            runs_each(cand, origin, i0, i1, c0, c1, [&](int, unsigned valid, const float (&x)[4]) {
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const uint32_t key = key_of(x[v]);
                    if ((valid >> v & 1u) && ((key ^ prefix) & above) == 0)
                        atomicAdd(&h[key >> shift & bins], 1);
                }
            });
            __syncthreads();
            for (int c = warp; c < kCoarse; c += kWarps) {
                const int v = __reduce_add_sync(0xffffffffu, h[c * 32 + lane]);
                if (lane == 0)
                    co[c] = v;
            }
            sync_cluster(cl, C);
            if (warp == 0) {
                // lane 0 has the largest digits: first two sums of 32 bins per lane, then the bins of one
                auto descend = [&](const int *hist, int base, int n, int &above, int &count) {  // n: 1 or 2 per lane
                    int own[2] = {0, 0};
#pragma unroll
                    for (int q = 0; q < kMaxCluster; ++q)
                        if (q < C) {
                            const int *p = cl.map_shared_rank(hist, q) + base;
                            own[0] += p[n * (31 - lane) + n - 1];
                            if (n == 2)
                                own[1] += p[2 * (31 - lane)];
                        }
                    int upto = own[0] + own[1];
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int y = __shfl_up_sync(0xffffffffu, upto, o);
                        if (lane >= o)
                            upto += y;
                    }
                    // the first lane whose sums reach the key sought
                    const unsigned m = __ballot_sync(0xffffffffu, above + upto >= left);
                    const int src = __ffs(m) - 1;
                    const int before = above + upto - own[0] - own[1];
                    const bool second = n == 2 && before + own[0] < left;
                    const int digit = n * (31 - lane) + (n == 2 && !second ? 1 : 0);
                    above = __shfl_sync(0xffffffffu, before + (second ? own[0] : 0), src);
                    count = __shfl_sync(0xffffffffu, second ? own[1] : own[0], src);
                    return __shfl_sync(0xffffffffu, digit, src);
                };
                int above = 0, count;
                const int c = descend(co, 0, 2, above, count);
                const int d = 32 * c + descend(h, 32 * c, 1, above, count);
                if (lane == 0) {
                    pick[0] = d;
                    pick[1] = above;
                    pick[2] = count;
                }
            }
            __syncthreads();
            prefix |= (uint32_t)pick[0] << shift;
            left -= pick[1];
            if (left == pick[2]) {  // all of them stay (most often the only one): what lies above the key below them
                --prefix;           // (not 0: fewer stay than there are, so smaller keys exist)
                left = 0;
                break;
            }
        }
        Counts k{0, 0, 0, 0};  // of this warp's part
        runs_each(cand, origin, i0, i1, c0, c1, [&](int c, unsigned valid, const float (&x)[4]) {
            unsigned same = 0, up = 0;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const uint32_t key = key_of(x[v]);
                up |= key > prefix ? 1u << v : 0u;
                same |= key == prefix ? 1u << v : 0u;
            }
            up &= valid;
            same &= valid;
            put_run(up_runs + c, up);
            put_run(eq_runs + c, same);
            const int over = origin + 128 * c + 4 * lane - edge;
            const unsigned hi = over >= 0 ? 15u : over <= -4 ? 0u : 15u << -over;
            k.eq_lo += __popc(same & ~hi);
            k.eq_hi += __popc(same & hi);
            k.hole += __popc(valid & ~hi & ~(up | same));
            k.mover += __popc(up & hi);
        });
        k.eq_lo = __reduce_add_sync(0xffffffffu, k.eq_lo);
        k.eq_hi = __reduce_add_sync(0xffffffffu, k.eq_hi);
        k.hole = __reduce_add_sync(0xffffffffu, k.hole);
        k.mover = __reduce_add_sync(0xffffffffu, k.mover);
        if (lane == 0)
            parts[warp] = k;
    } else if (lane == 0) {  // nothing stays, so nothing moves
        parts[warp] = Counts{0, 0, 0, 0};
    }
    __syncthreads();
    if (tid == 0) {
        Counts s{0, 0, 0, 0};
        for (int i = 0; i < kWarps; ++i) {
            s.eq_lo += parts[i].eq_lo;
            s.eq_hi += parts[i].eq_hi;
            s.hole += parts[i].hole;
            s.mover += parts[i].mover;
        }
        mine = s;
    }
    sync_cluster(cl, C);

    // ---- 2. holes and movers of this slice, in order.  Equal keys are in the order of their positions, so
    // of the first `left` that stay those below the budget's position come first.
    int32_t *holes = wk.holes + (size_t)id * a.maxp * (kPage / 2), *movers = wk.movers + (size_t)id * a.maxp * (kPage / 2);
    int pairs = 0;
    if (need > 0) {
        // holes and movers of a part with eq equal keys before it
        auto split = [&](const Counts &c, int eq, int &hole, int &mover) {
            const int stay = min(max(left - eq, 0), c.eq_lo + c.eq_hi), lo = min(stay, c.eq_lo);
            hole = c.hole + c.eq_lo - lo;
            mover = c.mover + stay - lo;
        };
        int eq = 0, nh = 0, nm = 0, tm = 0, te = 0;
        Counts of[kMaxCluster];
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q)
            of[q] = q < C ? *cl.map_shared_rank(&mine, q) : Counts{0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q) {  // the slices before
            int x, y;
            split(of[q], te, x, y);
            if (q < r)
                eq = te + of[q].eq_lo + of[q].eq_hi, nh = pairs + x, nm = tm + y;
            te += of[q].eq_lo + of[q].eq_hi;
            pairs += x;
            tm += y;
        }
        for (int i = 0; i < warp; ++i) {  // the parts before
            int x, y;
            const Counts c = parts[i];
            split(c, eq, x, y);
            nh += x;
            nm += y;
            eq += c.eq_lo + c.eq_hi;
        }
        uint4 next_up = {}, next_eq = {};
        if (c0 < c1)
            next_up = up_runs[c0], next_eq = eq_runs[c0];
        for (int c = c0; c < c1; ++c) {
            // lane order and then order within a lane is the order of positions
            const int i = origin + 128 * c + 4 * lane;
            unsigned up = nibble_of(next_up, lane);
            const unsigned same = nibble_of(next_eq, lane);
            if (c + 1 < c1)
                next_up = up_runs[c + 1], next_eq = eq_runs[c + 1];
            int all;
            if (__any_sync(0xffffffffu, same != 0)) {
                int before = eq + rank4(same, all);
                eq += all;
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (same >> v & 1u)
                        up |= before++ < left ? 1u << v : 0u;
            }
            auto list = [&](unsigned some, int32_t *to, int &at) {
                if (!__any_sync(0xffffffffu, some != 0))
                    return;
                int x = at + rank4(some, all);
                at += all;
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (some >> v & 1u)
                        to[x++] = first + i + v;
            };
            list(nibble_in(i, i0, min(edge, i1)) & ~up, holes, nh);
            list(nibble_in(i, edge, i1) & up, movers, nm);
        }
    }
    sync_cluster(cl, C);

    // ---- 3. hole i is filled from mover i
    // a thread's pieces of rows are all the same one of the 2 * gk 16-byte pieces of a vector's keys and
    // values (a power of two that divides the number of threads)
    const int gk = a.row_bytes / 16, lg = __ffs(gk);
    const int all = r * kThreads + tid, step = C * kThreads, j = all & (2 * gk - 1);
    uint4 *pool = static_cast<uint4 *>(j < gk ? a.pool_kd : a.pool_vd) + (size_t)g * kPage * gk + (j & (gk - 1));
    auto piece = [&](int pos) {
        return pool + ((size_t)__ldg(table + pos / kPage) * a.Hkv * kPage + pos % kPage) * gk;
    };
    for (int x0 = all >> lg; x0 < pairs; x0 += kStage * (step >> lg)) {
        int to[kStage], at[kStage];
        float wv[kStage];
#pragma unroll
        for (int u = 0; u < kStage; ++u) {
            const int x = x0 + u * (step >> lg);
            to[u] = x < pairs ? holes[x] : -1;
            at[u] = x < pairs ? movers[x] : -1;
        }
#pragma unroll
        for (int u = 0; u < kStage; ++u)
            if (at[u] >= 0)
                sm100::cp_async16(sm100::smem_u32(&sh.stage[u * kThreads + tid]), piece(at[u]));
        if (j == 0) {
#pragma unroll
            for (int u = 0; u < kStage; ++u)
                wv[u] = at[u] >= 0 ? w[at[u]] : 0.f;
#pragma unroll
            for (int u = 0; u < kStage; ++u)
                if (to[u] >= 0)
                    w[to[u]] = wv[u];
        }
        sm100::cp_async_wait_all();
#pragma unroll
        for (int u = 0; u < kStage; ++u)
            if (to[u] >= 0)
                *piece(to[u]) = sh.stage[u * kThreads + tid];
    }
    // the window's weights come down to the new end
    float *win = wk.window + (size_t)id * a.w;
    for (int i = all; i < a.w; i += step)
        win[i] = w[n + i];
    sync_cluster(cl, C);
    for (int i = all; i < a.w; i += step)
        w[keep + i] = win[i];
    for (int i = keep + a.w + all; i < L; i += step)
        w[i] = 0.f;
}

__global__ void evict_lens_kernel(int32_t *seq_lens, const int32_t *new_lens, int B)
{
    sm100::grid_dep_wait();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B && new_lens[b] >= 0)
        seq_lens[b] = new_lens[b];
}

struct Layout {
    size_t lists, list, bits, window, lens, total;  // list: bytes of one of the two
};
static size_t up256(size_t x) { return (x + 255) & ~size_t(255); }
static Layout layout(int B, int Hkv, int w, int maxp)
{
    const size_t heads = (size_t)B * Hkv;
    Layout y;
    y.list = up256(heads * maxp * (kPage / 2) * sizeof(int32_t));
    y.lists = 0;
    y.bits = 2 * y.list;
    y.window = y.bits + up256(heads * (maxp + 5 * kMaxCluster) * sizeof(uint4));
    y.lens = y.window + up256(heads * w * sizeof(float));
    y.total = y.lens + up256((size_t)B * sizeof(int32_t));
    return y;
}

}  // namespace evict

size_t evict_workspace_bytes(int B, int Hkv, int w, int maxp) { return evict::layout(B, Hkv, w, maxp).total; }

cudaError_t launch_evict(const EvictArgs &a, void *workspace, cudaStream_t st)
{
    if (a.B == 0)
        return cudaSuccess;
    const evict::Layout y = evict::layout(a.B, a.Hkv, a.w, a.maxp);
    char *ws = static_cast<char *>(workspace);
    evict::Work wk;
    wk.holes = reinterpret_cast<int32_t *>(ws + y.lists);
    wk.movers = reinterpret_cast<int32_t *>(ws + y.lists + y.list);
    wk.bits = reinterpret_cast<uint4 *>(ws + y.bits);
    wk.window = reinterpret_cast<float *>(ws + y.window);
    wk.new_lens = reinterpret_cast<int32_t *>(ws + y.lens);
    const int heads = a.B * a.Hkv;
    // Blocks per head: enough of them to fill the GPU, each with a slice worth the cluster's barriers, by capacity (the
    // lengths are on the device).  us a call that keeps half (w 128, rows of 32 bytes) with 1 / 2 / 4 / 8 blocks:
    //   heads  tokens                                 heads  tokens
    //       8    1024    9.5 / 13.0 / 13.4 / 14.5        96    8192   26.8 / 26.2 / 24.0 / 34.1
    //       8    4096   16.6 / 16.8 / 15.0 / 14.6       152    8192   29.1 / 30.0 / 30.5 / 44.2
    //       8    8192   23.6 / 21.6 / 18.3 / 15.5       152   32768    113 /   93 /   90 /   98
    //       8   32768   82.0 / 53.4 / 37.3 / 29.5       304   32768    160 /  152 /  160 /  180
    //      64    2048   13.5 / 15.2 / 16.5 / 18.5       512    2048   22.4 / 34.0 / 52.0 / 99.7
    //      64    8192   26.0 / 24.0 / 22.2 / 21.8       512    8192   69.2 / 80.1 / 94.7 /  133
    // The rule is within 1.5 us or 1 % of the best of the four, but for 2048 tokens, where one block is 1 to 4 us faster
    // than two, and 4096 tokens of 152 and 304 heads, 6.5 and 3.3 us.
    int C = evict::kMaxCluster;
    while (C > 1 && (heads * C > 4 * kSms || a.maxp * kPage < 1024 * C))
        C /= 2;
    cudaLaunchAttribute at[1];
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(2 * heads * C);  // the second half turns the rings
    cfg.blockDim = dim3(evict::kThreads);
    cudaError_t e = cudaLaunchKernelEx(&cfg, evict::evict_kernel, a, wk);
    if (e != cudaSuccess)
        return e;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((a.B + 255) / 256);
    cfg.blockDim = dim3(256);
    return cudaLaunchKernelEx(&cfg, evict::evict_lens_kernel, a.seq_lens, (const int32_t *)wk.new_lens, a.B);
}

}  // namespace dar
