// dar_q4_cache.cu -- writing the 4-bit pages of a cache (dar_q4.cuh) and reading
// them back: the append of new tokens, and conversion of pages to and from the
// storage type.
#include <algorithm>
#include <type_traits>

#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_project.cuh"
#include "dar_q4.cuh"
#include "dar_q4_append.cuh"
#include "dar_sm100.cuh"

namespace dar {
namespace q4 {

// ------------------------------------------------------------------ append
//
// As append_bulk_kernel (dar_append.cu): a CTA takes the new tokens j of one
// (sequence, KV head, keys or values) that push positions m = L + j - w out of the
// window, projects these (the same fp32 chains, rounded to T), and puts the tokens
// that stay into the ring slots that they leave.  Its tile starts at a position that
// is a multiple of a page, so that tokens that share words of a page have the same CTA; a
// warp then quantises and writes a page's group.
template <typename T, int DD, int RPT, int NR>
__global__ void __launch_bounds__(NR *slices<DD>()) append_kernel(AppendArgs a, int tiles)
{
    constexpr int R = RPT * NR, NT = NR * slices<DD>();
    constexpr int CW = cols_per_thread<DD>();
    constexpr int E = Granule<T>::kElems;
    constexpr int CPR = kHeadDim / E;
    using F = Fmt<DD>;
    __shared__ __align__(16) unsigned char rows[R * kHeadDim * sizeof(T)];
    __shared__ __align__(16) float Ws[kHeadDim * DD];
    const int tid = threadIdx.x, kv = blockIdx.y;
    const int bg = blockIdx.x / tiles;
    const int b = bg / a.Hkv, g = bg % a.Hkv;
    const int n = a.n, w = a.w;
    const int L = a.seq_lens[b], nb = a.n_per_seq ? a.n_per_seq[b] : n;
    if (append_error(L, nb, a) != DAR_OK)
        return;
    const int off = ((L - w) % kPage + kPage) % kPage;  // new token 0 pushes out a position this far into its page
    const int j0 = (int)(blockIdx.x % tiles) * R - off;
    if (j0 >= nb)
        return;
    const T *xnew = static_cast<const T *>(kv ? a.v_new : a.k_new) + (size_t)bg * n * kHeadDim;
    T *ring = static_cast<T *>(kv ? a.win_v : a.win_k) + (size_t)bg * w * kHeadDim;
    const int m0 = L + j0 - w;                     // a multiple of a page
    const int ra = max(max(0, -j0), -m0), nr = min(R, nb - j0);  // rows [ra, nr) leave the window
    if (ra < nr) {
        const uint32_t rows_s = sm100::smem_u32(rows);
        for (int i = tid; i < nr * CPR; i += NT) {
            const int r = i / CPR, c = i % CPR, m = m0 + r;
            if (r >= ra) {
                const T *src = m < L ? ring + (size_t)(m % w) * kHeadDim : xnew + (size_t)(m - L) * kHeadDim;
                sm100::cp_async16(rows_s + (r * CPR + (c ^ (r & 7))) * 16, src + c * E);
            }
        }
        const float *W = (kv ? a.Dv : a.Dk) + (size_t)g * kHeadDim * DD;
        for (int i = tid; i < kHeadDim * DD / 4; i += NT)
            reinterpret_cast<float4 *>(Ws)[i] = __ldg(reinterpret_cast<const float4 *>(W) + i);
        const int r0 = tid % NR, c0 = slices<DD>() > 1 ? tid / NR * CW : 0;  // this thread's rows r0 + k * NR and columns
        sm100::cp_async_wait_all();
        __syncthreads();  // every ring row this CTA reads is in shared memory
        float acc[RPT][CW];
        project_rows<T, DD, CW, RPT>(rows, Ws + c0, r0, NR, acc);  // (rows outside [ra, nr): of stale bytes, not used)
        __syncthreads();
        // the vectors, rounded to T, over the rows they come from
        T *vec = reinterpret_cast<T *>(rows);
#pragma unroll
        for (int k = 0; k < RPT; ++k)
            store_row<T, CW>(vec + (size_t)(r0 + k * NR) * DD + c0, acc[k]);
        __syncthreads();
        unsigned char *pool = static_cast<unsigned char *>(a.pool_kd);
        for (int i = tid / 32; i < R / kPage * F::kGroups; i += NT / 32) {
            const int p = i % (R / kPage), sb = i / (R / kPage), m = m0 + p * kPage;
            const int first = max(0, ra - p * kPage), end = min(kPage, nr - p * kPage);
            if (first >= end)
                continue;
            const int id = a.block_table[(size_t)b * a.maxp + m / kPage];
            if (id < 0 || id >= a.num_pages) {
                report(a.status, DAR_ERR_CAPACITY);
                continue;
            }
            unsigned char *block = pool + ((size_t)id * a.Hkv + g) * F::kBytes + sb * F::kBlock;
            const T *v = vec + (size_t)p * kPage * DD + sb * F::kGroup;
            if (kv)
                write_page<T, F::kGroup, true>(block, v, DD, first, end, tid & 31);
            else
                write_page<T, F::kGroup, false>(block, v, DD, first, end, tid & 31);
        }
    }
    // ring slots (L + j) % w, j < min(nb, w): the last new token of each
    const int jr = max(0, j0), slots = min(min(nb, w), j0 + R) - jr;
    for (int i = tid; i < slots * CPR; i += NT) {
        const int c = i % CPR, j = jr + i / CPR, last = j + (nb - 1 - j) / w * w;
        *reinterpret_cast<uint4 *>(ring + (size_t)((L + j) % w) * kHeadDim + c * E) =
            *reinterpret_cast<const uint4 *>(xnew + (size_t)last * kHeadDim + c * E);
    }
}

template <typename T, int DD>
__global__ void __launch_bounds__(kFewThreads) append_few_kernel(AppendArgs a)
{
    append_few<T, DD>(a);
}

template <typename T, int DD>
static cudaError_t append_few_launch(const AppendArgs &a, cudaStream_t s)
{
    static PerDeviceOnce once;  // opt-in to more than 48 KB of shared memory, once per device
    const cudaError_t e = per_device_once(once, [](int) {
        return cudaFuncSetAttribute(append_few_kernel<T, DD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    kFewStageBytes);
    });
    if (e != cudaSuccess)
        return e;
    append_few_kernel<T, DD><<<a.B, kFewThreads, few_smem<T>(a.Hkv), s>>>(a);
    return cudaGetLastError();
}

// Advances the lengths (and reports refused sequences) once every CTA of the append has read them.
__global__ void append_lens(AppendArgs a)
{
    sm100::grid_dep_wait();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= a.B)
        return;
    const int L = a.seq_lens[b], nb = a.n_per_seq ? a.n_per_seq[b] : a.n;
    const int e = append_error(L, nb, a);
    if (e != DAR_OK)
        report(a.status, e);
    else
        a.seq_lens[b] = L + nb;
}

template <typename T, int DD, int RPT, int NR>
static cudaError_t append_tiles(const AppendArgs &a, cudaStream_t s)
{
    const int tiles = (int)(((long long)a.n + kPage - 1 + RPT * NR - 1) / (RPT * NR));
    append_kernel<T, DD, RPT, NR><<<dim3((unsigned)(a.B * a.Hkv * tiles), 2), NR * slices<DD>(), 0, s>>>(a, tiles);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess)
        return e;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((a.B + 127) / 128);
    cfg.blockDim = dim3(128);
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, append_lens, a);
}

// ------------------------------------------------------------------ conversion
//
// A warp takes a page of a (sequence, KV head), or a group of its keys or values where the pages are few.
constexpr int kConvertWarps = 8;
constexpr long long kSplitPages = kSms * 32;  // pages by capacity: a warp each fills the chip

template <typename T, int DD, bool PACK>
__global__ void __launch_bounds__(kConvertWarps * 32) convert_kernel(Q4ConvertArgs a, int parts)
{
    using F = Fmt<DD>;
    constexpr int GS = F::kGroup;
    const int lane = threadIdx.x & 31, b = blockIdx.y;
    const long long item = (long long)blockIdx.x * kConvertWarps + (threadIdx.x >> 5);
    const int L = a.seq_lens[b], first = a.first ? a.first[b] : 0;
    const int most = min(a.maxp, a.maxp4);
    if (L < 0 || (long long)L - a.w > (long long)most * kPage || first < 0) {
        if (item == 0 && lane == 0)
            report(a.status, first < 0 ? DAR_ERR_INVALID_ARG : DAR_ERR_CAPACITY);
        return;
    }
    const int end = max(0, L - a.w), page0 = first / kPage;
    const int part = (int)(item % parts), g = (int)(item / parts % a.Hkv);
    const long long lp = page0 + item / parts / a.Hkv;
    if (first >= end || lp * kPage >= end)
        return;
    const int id = a.table[(size_t)b * a.maxp + lp], id4 = a.table4[(size_t)b * a.maxp4 + lp];
    if (id < 0 || id >= a.num_pages || id4 < 0 || id4 >= a.num_pages4) {
        if (lane == 0)
            report(a.status, DAR_ERR_CAPACITY);
        return;
    }
    unsigned char *page = static_cast<unsigned char *>(a.pool) + ((size_t)id4 * a.Hkv + g) * F::kBytes;
    const size_t row = ((size_t)id * a.Hkv + g) * kPage * DD;
    T *k = static_cast<T *>(a.pool_kd) + row, *v = static_cast<T *>(a.pool_vd) + row;
    const int from = (int)max(0ll, first - lp * kPage), to = (int)min((long long)kPage, end - lp * kPage);
    auto keys = [&](int i) {
        if constexpr (PACK)
            write_page<T, GS, false>(page + i * F::kBlock, k + i * GS, DD, from, to, lane);
        else
            read_page<T, GS, false>(page + i * F::kBlock, k + i * GS, DD, from, to, lane);
    };
    auto values = [&](int i) {
        if constexpr (PACK)
            write_page<T, GS, true>(page + i * F::kBlock, v + i * GS, DD, from, to, lane);
        else
            read_page<T, GS, true>(page + i * F::kBlock, v + i * GS, DD, from, to, lane);
    };
    if (parts == 1) {
        if (PACK && lane == 0) {  // (all contexts of the 1B shape: 5 % less)
            sm100::prefetch_l2(k, kPage * DD * sizeof(T));
            sm100::prefetch_l2(v, kPage * DD * sizeof(T));
        }
        // code that the instruction cache holds: of four groups together 610 us instead of 296 (pack of 64000 bf16 pages of
        // 64 entries), of two 126 and 136 (32 entries); fp32 1008 and 400
        constexpr int kTogether = sizeof(T) == 2 && F::kGroups <= 2 ? 2 : 1;
#pragma unroll kTogether
        for (int i = 0; i < F::kGroups; ++i) {
            keys(i);
            values(i);
        }
    } else if (part < F::kGroups) {
        keys(part);
    } else {
        values(part - F::kGroups);
    }
}

template <typename F>
static cudaError_t by_width(int dd, F &&f)
{
    switch (dd) {
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    case 32: return f(std::integral_constant<int, 32>());
    case 64: return f(std::integral_constant<int, 64>());
    default: return cudaErrorInvalidValue;
    }
}

constexpr long long kPairTiles = 4 * kSms;

template <typename T>
static cudaError_t append_t(int dd, const AppendArgs &a, cudaStream_t s)
{
    return by_width(dd, [&](auto width) {
        constexpr int DD = decltype(width)::value;
        if (append_is_few<T>(a, DD))
            return append_few_launch<T, DD>(a, s);
        // A tile is a page, a row to a thread; two rows for every read of W where that leaves work for all SMs: of 64
        // entries, whose tiles have four threads a row (bf16, 8 KV heads, 32 x 2048 tokens: 246 us, 316 with one; 1 x
        // 2048: 15.3 and 16.8), and from bf16 in tiles of two pages once these fill the chip a few times over (12 KV
        // heads, d_down 16, 32 x 2048: 111 and 128; 32 x 64, 768 tiles: 13.9 and 15.5; 4 x 512, 480 tiles: 13.5 and
        // 11.3).  fp32 rows are twice as long: 212 and 210 at 32 x 2048.  d_down 8: 62 and 63, but 14.7 and 13.1 at 4 x
        // 2048.  Not used: four rows a thread (64 entries in tiles of two pages 229 and 246 at 32 x 2048, 242 and 254 at 64 x
        // 1024, but 19.4 and 15.6 at 4 x 512; else 4 % less to twice as long), tiles of four pages (32 entries 133 and 142 at
        // 32 x 2048, but 22 and 17 at 32 x 64; 16 entries 2 % less there and 24 % more here; else longer).
        if constexpr (DD == 64) {
            return append_tiles<T, DD, 2, kPage / 2>(a, s);
        } else {
            if constexpr (DD >= 16 && sizeof(T) == 2) {
                const long long tiles = ((long long)a.n + kPage - 1 + 2 * kPage - 1) / (2 * kPage);
                if (tiles * a.B * a.Hkv * 2 >= kPairTiles)
                    return append_tiles<T, DD, 2, kPage>(a, s);
            }
            return append_tiles<T, DD, 1, kPage>(a, s);
        }
    });
}

template <typename T, bool PACK>
static cudaError_t convert_t(int dd, const Q4ConvertArgs &a, cudaStream_t s)
{
    return by_width(dd, [&](auto width) {
        // 72 pages of fp32 vectors of 32 entries: 22 us a page to a warp, 7 a group; all contexts of the 1B shape (133 thousand
        // pages, bf16): 158 and 192.  Pages are counted by capacity, since lengths and `first` are on the device: the last 128
        // tokens of 64 sequences of 8 heads take 3.2 us in a cache with room for no more, 8.5 with room for 3840 and 38 for
        // 32512, most of them of warps that find nothing to do.
        const long long pages = (long long)std::min(a.maxp, a.maxp4) * a.Hkv;
        const int parts = pages * a.B < kSplitPages ? 2 * Fmt<decltype(width)::value>::kGroups : 1;
        const long long items = pages * parts;
        const dim3 grid((unsigned)std::max(1ll, (items + kConvertWarps - 1) / kConvertWarps), (unsigned)a.B);
        convert_kernel<T, decltype(width)::value, PACK><<<grid, kConvertWarps * 32, 0, s>>>(a, parts);
        return cudaGetLastError();
    });
}

}  // namespace q4

size_t q4_page_bytes(int dd)
{
    return dd == 8 ? q4::Fmt<8>::kBytes : (size_t)(dd / 16) * q4::Fmt<16>::kBytes;
}

cudaError_t launch_append_q4(dar_dtype dt, int dd, const AppendArgs &a, cudaStream_t s)
{
    if (a.B == 0)
        return cudaSuccess;
    return dt == DAR_F32 ? q4::append_t<float>(dd, a, s) : q4::append_t<bf16>(dd, a, s);
}

cudaError_t launch_convert_q4(dar_dtype dt, int dd, bool pack, const Q4ConvertArgs &a, cudaStream_t s)
{
    if (a.B == 0)
        return cudaSuccess;
    if (pack)
        return dt == DAR_F32 ? q4::convert_t<float, true>(dd, a, s) : q4::convert_t<bf16, true>(dd, a, s);
    return dt == DAR_F32 ? q4::convert_t<float, false>(dd, a, s) : q4::convert_t<bf16, false>(dd, a, s);
}

}  // namespace dar
