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
// The ring holds position p in slot p mod w; positions drop by e = n - keep, so it turns
// by e mod w slots: the reflections s -> -s and s -> -s - e (mod w), whose swaps are
// disjoint, one after the other.
//
// One cluster of C thread blocks per (sequence, KV head); C grows as there are fewer of
// them.  The blocks share the candidates in C consecutive slices:
//   1. the smallest weight that stays: a radix selection, 8 bits of the ordered key a
//      pass, from the cluster's histogram (each block's in its own shared memory, read
//      by all);
//   2. each block lists the holes and the movers of its slice in order, which needs the
//      number of equal weights in the slices before;
//   3. hole i is filled from mover i, by all threads of the cluster.
// A second kernel sets the lengths, which the clusters of other heads read before.
// Bound: HBM for the rows that move and the weights, read once from there and then from
// L2; short calls by the cluster's barriers.
#include <cooperative_groups.h>

#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_sm100.cuh"

namespace dar {
namespace evict {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;  // the largest portable cluster

struct Work {
    int32_t *holes, *movers;  // [B * Hkv][maxp * 64]
    float *window;            // [B * Hkv][w] the window's weights on their way down
    int32_t *new_lens;        // [B], -1: unchanged
};

// Order of weights as unsigned numbers: larger weight, larger key; NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x)
        return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);  // -0 + 0 = +0
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Exclusive rank of `flag` among the block's threads and the number of flags; `part` holds kWarps ints.
__device__ __forceinline__ int block_rank(bool flag, int *part, int &count)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned m = __ballot_sync(0xffffffffu, flag);
    __syncthreads();  // the values of the call before are read
    if (lane == 0)
        part[warp] = __popc(m);
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        const int v = part[i];
        before += i < warp ? v : 0;
        all += v;
    }
    count = all;
    return before + __popc(m & ((1u << lane) - 1u));
}

__global__ void __launch_bounds__(kThreads) evict_kernel(EvictArgs a, Work wk)
{
    __shared__ int hist[2][256];
    __shared__ int sum[256];
    __shared__ int pick[2];      // digit, and how many keys lie above it
    __shared__ int counts[2];    // holes and movers of this block's slice
    __shared__ int part[kWarps];
    cg::cluster_group cl = cg::this_cluster();
    const int C = (int)cl.num_blocks(), r = (int)cl.block_rank();
    const int id = blockIdx.x / C, b = id / a.Hkv, g = id % a.Hkv;
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
    if (g == 0 && r == 0 && tid == 0) {
        if (err != DAR_OK)
            report(a.status, err);
        wk.new_lens[b] = go && err == DAR_OK ? keep + a.w : -1;
    }
    if (!go || err != DAR_OK)
        return;

    float *w = a.weights + (size_t)id * slots;
    const int m = n - first, need = keep - first, e = n - keep;
    const int sl = (m + C - 1) / C, i0 = min(m, r * sl), i1 = min(m, i0 + sl);
    const float *cand = w + first;

    // ---- 1. the smallest key that stays, and how many of its equals do
    uint32_t prefix = 0, mask = 0;
    int left = need;  // the key sought is the left-th largest of those that match prefix
    if (need > 0) {
        for (int pass = 0; pass < 4; ++pass) {
            const int shift = 24 - 8 * pass;
            int *h = hist[pass & 1];
            for (int i = tid; i < 256; i += kThreads)
                h[i] = 0;
            __syncthreads();
            for (int i = i0 + tid; i < i1; i += kThreads) {
                const uint32_t k = key_of(cand[i]);
                if (((k ^ prefix) & mask) == 0)
                    atomicAdd(&h[(k >> shift) & 255u], 1);
            }
            cl.sync();
            if (tid < 256) {
                int s = 0;
                for (int q = 0; q < C; ++q)
                    s += cl.map_shared_rank(h, q)[tid];
                sum[tid] = s;
            }
            __syncthreads();
            if (warp == 0) {  // lane 0 holds the eight largest digits
                int own = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    own += sum[255 - (8 * lane + j)];
                int upto = own;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o)
                        upto += y;
                }
                int above = upto - own;
                if (above < left && left <= upto) {
                    int j = 0;
                    while (above + sum[255 - (8 * lane + j)] < left) {
                        above += sum[255 - (8 * lane + j)];
                        ++j;
                    }
                    pick[0] = 255 - (8 * lane + j);
                    pick[1] = above;
                }
            }
            __syncthreads();
            prefix |= (uint32_t)pick[0] << shift;
            mask |= 255u << shift;
            left -= pick[1];
        }
    }
    // equal keys in the slices before: the last pass's histograms count exactly these
    int eq = 0;
    if (need > 0)
        for (int q = 0; q < r; ++q)
            eq += cl.map_shared_rank(hist[1], q)[prefix & 255u];

    // ---- 2. holes and movers of this slice, in order
    int32_t *holes = wk.holes + (size_t)id * a.maxp * kPage + i0, *movers = wk.movers + (size_t)id * a.maxp * kPage + i0;
    int nh = 0, nm = 0;
    for (int c0 = i0; c0 < i1; c0 += kThreads) {
        const int i = c0 + tid, pos = first + i;
        const bool in = i < i1;
        const uint32_t k = in ? key_of(cand[i]) : 0u;
        const bool same = in && need > 0 && k == prefix;
        int cnt;
        const int er = eq + block_rank(same, part, cnt);
        eq += cnt;
        const bool stays = in && need > 0 && (k > prefix || (same && er < left));
        const bool hole = in && !stays && pos < keep, mover = stays && pos >= keep;
        const int hr = nh + block_rank(hole, part, cnt);
        nh += cnt;
        const int mr = nm + block_rank(mover, part, cnt);
        nm += cnt;
        if (hole)
            holes[hr] = pos;
        if (mover)
            movers[mr] = pos;
    }
    if (tid == 0) {
        counts[0] = nh;
        counts[1] = nm;
    }
    cl.sync();

    // ---- 3. hole i is filled from mover i
    int hb[kMaxCluster + 1], mb[kMaxCluster + 1];
    hb[0] = mb[0] = 0;
    for (int q = 0; q < C; ++q) {
        const int *p = cl.map_shared_rank(counts, q);
        hb[q + 1] = hb[q] + p[0];
        mb[q + 1] = mb[q] + p[1];
    }
    const int pairs = hb[C];
    const int32_t *hl = wk.holes + (size_t)id * a.maxp * kPage, *ml = wk.movers + (size_t)id * a.maxp * kPage;
    const int gk = a.row_bytes / 16;  // 16-byte pieces of a vector
    const int all = r * kThreads + tid, step = C * kThreads;
    for (long long x = all; x < (long long)pairs * 2 * gk; x += step) {
        const int i = (int)(x / (2 * gk)), j = (int)(x % (2 * gk));
        int qh = 0, qm = 0;
        for (int q = 1; q < C; ++q) {
            qh += i >= hb[q];
            qm += i >= mb[q];
        }
        const int to = hl[qh * sl + i - hb[qh]], at = ml[qm * sl + i - mb[qm]];
        const int pt = __ldg(table + to / kPage), pa = __ldg(table + at / kPage);
        uint4 *pool = static_cast<uint4 *>(j < gk ? a.pool_kd : a.pool_vd);
        const int jj = j < gk ? j : j - gk;
        const size_t dst = (((size_t)pt * a.Hkv + g) * kPage + to % kPage) * gk + jj;
        const size_t src = (((size_t)pa * a.Hkv + g) * kPage + at % kPage) * gk + jj;
        pool[dst] = pool[src];
        if (j == 0)
            w[to] = w[at];
    }
    // the window's weights leave for their new place, and the ring's first reflection
    float *win = wk.window + (size_t)id * a.w;
    for (int i = all; i < a.w; i += step)
        win[i] = w[n + i];
    const int turn = e % a.w, rp = a.ring_bytes / 16;
    uint4 *rings[2] = {static_cast<uint4 *>(a.win_k) + (size_t)id * a.w * rp,
                       static_cast<uint4 *>(a.win_v) + (size_t)id * a.w * rp};
    auto reflect = [&](int c) {  // swaps slot s with (c - s) mod w, 0 <= c < w
        for (long long x = all; x < (long long)a.w * 2 * rp; x += step) {
            const int s = (int)(x / (2 * rp)), j = (int)(x % (2 * rp));
            const int o = c - s + (c < s ? a.w : 0);
            if (s >= o)
                continue;
            uint4 *ring = rings[j >= rp];
            const int jj = j >= rp ? j - rp : j;
            const uint4 u = ring[(size_t)s * rp + jj], v = ring[(size_t)o * rp + jj];
            ring[(size_t)s * rp + jj] = v;
            ring[(size_t)o * rp + jj] = u;
        }
    };
    if (turn)
        reflect(0);
    cl.sync();
    for (int i = all; i < a.w; i += step)
        w[keep + i] = win[i];
    for (int i = keep + a.w + all; i < L; i += step)
        w[i] = 0.f;
    if (turn)
        reflect(a.w - turn);
}

__global__ void evict_lens_kernel(int32_t *seq_lens, const int32_t *new_lens, int B)
{
    sm100::grid_dep_wait();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B && new_lens[b] >= 0)
        seq_lens[b] = new_lens[b];
}

struct Layout {
    size_t holes, movers, window, lens, total;
};
static size_t up256(size_t x) { return (x + 255) & ~size_t(255); }
static Layout layout(int B, int Hkv, int w, int maxp)
{
    const size_t heads = (size_t)B * Hkv;
    Layout y;
    y.holes = 0;
    y.movers = up256(heads * maxp * kPage * sizeof(int32_t));
    y.window = 2 * y.movers;
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
    wk.holes = reinterpret_cast<int32_t *>(ws + y.holes);
    wk.movers = reinterpret_cast<int32_t *>(ws + y.movers);
    wk.window = reinterpret_cast<float *>(ws + y.window);
    wk.new_lens = reinterpret_cast<int32_t *>(ws + y.lens);
    const int heads = a.B * a.Hkv;
    int C = evict::kMaxCluster;
    while (C > 1 && heads * C > 4 * kSms)
        C /= 2;
    cudaLaunchAttribute at[1];
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(heads * C);
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
