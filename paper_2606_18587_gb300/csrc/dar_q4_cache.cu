// dar_q4_cache.cu -- writing the 4-bit pages of a cache (dar_q4.cuh) and reading
// them back: the append of new tokens, and conversion of pages to and from the
// storage type.
#include <algorithm>
#include <type_traits>

#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_project.cuh"
#include "dar_q4.cuh"
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

// Few tokens a sequence: one CTA per sequence, as cache_append_kernel (dar_append.cu), so that its length can be
// advanced at the end and a call is one launch.  A thread runs one chain (keys or values, KV head, entry) for the
// tokens that leave; the lanes that have a group quantise it together.
constexpr int kFewThreads = 512;
constexpr int kFewRows = 8;               // tokens of a round
constexpr int kFewStageBytes = 96 << 10;  // their rows of 64

template <typename T>
__host__ __device__ constexpr int few_rows(int Hkv)
{
    const int r = kFewStageBytes / (2 * Hkv * kHeadDim * (int)sizeof(T));
    return r > kFewRows ? kFewRows : r;
}

// Rows on their way into a block, an entry a thread: GS consecutive lanes have a group.  Words that several of the
// unit's rows share are written once.
template <int GS>
struct FewWords {
    uint32_t x0 = 0u, x1 = 0u, m0 = 0u, m1 = 0u;  // of the rows so far: words and masks (keys: of even and of odd rows)
    // Entry e of a row of a page, in this lane; all lanes.  last: the last row of its unit, or of all.
    __device__ __forceinline__ void add(float x, int e, bool values, int row, unsigned char *block, bool last)
    {
        uint32_t a = magnitude(x);
#pragma unroll
        for (int o = 1; o < GS; o <<= 1)
            a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
        const float s = group_scale(a);
        // where the entry is: keys, slot c + 2 (e / 2 mod 2) of half e mod 2; values, slot 2 c + (e / 2 mod 2) of half o
        const int o = row & 1, c = (row >> 1) & 1, i = (row >> 2) & 1, k = (e >> 1) & 1;
        const int slot = GS == 16 ? (values ? 2 * c + k : c + 2 * k) : 2 * i + c, half = values ? o : e & 1;
        uint32_t y = code_of(x, s) << slot_shift(slot, half);
        // the other entries of the word: keys, of four (two) consecutive ones; values, of e and e + 2
        uint32_t m = 15u << slot_shift(slot, half);
#pragma unroll
        for (int q = 1; q < 4; q <<= 1) {
            const uint32_t yo = __shfl_xor_sync(0xffffffffu, y, q), mo = __shfl_xor_sync(0xffffffffu, m, q);
            if (GS == 16 ? !values || q == 2 : !values && q == 1) {
                y |= yo;
                m |= mo;
            }
        }
        if (values || o == 0)
            x0 |= y, m0 |= m;
        else
            x1 |= y, m1 |= m;
        if (block && e == 0)
            reinterpret_cast<uint16_t *>(block + kPage * GS + (values ? 2 * kPage : 0))[scale_index(row)] =
                (uint16_t)(__float_as_uint(s) >> 16);
        if (!last)
            return;
        const int row0 = row & ~(GS == 16 ? 3 : 7);
        auto put = [&](int j, uint32_t x, uint32_t mask) {
            uint32_t *p = reinterpret_cast<uint32_t *>(
                block + (values ? kPage * GS / 2 + word_offset<GS, true>(row0, j) : word_offset<GS, false>(row0, j)));
            *p = (*p & ~mask) | x;
        };
        if (block) {
            if (values) {
                if (GS == 8)
                    put(e, x0, m0);
                else if ((e & 2) == 0)
                    put(2 * (e >> 2) + (e & 1), x0, m0);
            } else {  // words 4 o + u, u = e / 4 (e / 2): one lane writes the even rows', the next one the odd rows'
                const int u = GS == 16 ? e >> 2 : e >> 1, l = GS == 16 ? e & 3 : e & 1;
                if (l == 0 && m0)
                    put(u, x0, m0);
                else if (l == 1 && m1)
                    put(4 + u, x1, m1);
            }
        }
        x0 = x1 = m0 = m1 = 0u;
    }
};

template <typename T, int DD>
__device__ __forceinline__ void append_few(const AppendArgs &a)
{
    using F = Fmt<DD>;
    constexpr int E = Granule<T>::kElems, GPR = kHeadDim / E, GS = F::kGroup;
    extern __shared__ __align__(16) unsigned char few[];
    __shared__ int s_L, s_nb, s_ok;
    __shared__ int s_pid[kFewRows];  // page of each staged row (-1: invalid)
    const int b = blockIdx.x, tid = threadIdx.x, Hkv = a.Hkv, n = a.n, w = a.w;
    const int chains = 2 * Hkv * DD, R = few_rows<T>(Hkv);
    T *rows = reinterpret_cast<T *>(few);           // [R][kv][Hkv][64]
    const T *knew = static_cast<const T *>(a.k_new), *vnew = static_cast<const T *>(a.v_new);
    T *wk = static_cast<T *>(a.win_k), *wv = static_cast<T *>(a.win_v);
    unsigned char *pool = static_cast<unsigned char *>(a.pool_kd);
    if (tid == 0) {
        s_L = a.seq_lens[b];
        s_nb = a.n_per_seq ? a.n_per_seq[b] : n;
    }
    // what does not depend on the length: the first chain's column of W, and a granule of the last new rows
    float wc[kHeadDim];
    auto load_w = [&](int ch) {
        const int kv = ch / (Hkv * DD), g = (ch / DD) % Hkv, c = ch % DD;
        const float *W = (kv ? a.Dv : a.Dk) + (size_t)g * kHeadDim * DD + c;
#pragma unroll
        for (int t = 0; t < kHeadDim; ++t)
            wc[t] = __ldg(W + (size_t)t * DD);
    };
    if (tid < chains)
        load_w(tid);
    auto new_granule = [&](int i, int j0) {  // i over [row][kv][g][granule]
        const int q = i % GPR, rest = i / GPR, g = rest % Hkv, kv = (rest / Hkv) & 1, j = j0 + rest / (2 * Hkv);
        return (kv ? vnew : knew) + (((size_t)b * Hkv + g) * n + j) * kHeadDim + q * E;
    };
    const int pre_rows = min(n, w);
    uint4 pre = make_uint4(0u, 0u, 0u, 0u);
    if (tid < 2 * Hkv * pre_rows * GPR)
        pre = *reinterpret_cast<const uint4 *>(new_granule(tid, n - pre_rows));
    __syncthreads();
    if (tid == 0) {
        const int e = append_error(s_L, s_nb, a);
        if (e != DAR_OK)
            report(a.status, e);
        s_ok = e == DAR_OK;
    }
    __syncthreads();
    if (!s_ok || s_nb == 0)
        return;
    const int L = s_L, nb = s_nb, Lnew = L + nb;
    const int lo = max(0, L - w), hi = max(0, Lnew - w);  // positions that leave the window
    for (int m0 = lo; m0 < hi; m0 += R) {
        const int nr = min(R, hi - m0);
        for (int i = tid; i < nr * 2 * Hkv * GPR; i += kFewThreads) {
            const int q = i % GPR, rest = i / GPR, g = rest % Hkv, kv = (rest / Hkv) & 1, p = m0 + rest / (2 * Hkv);
            const T *src = p < L ? (kv ? wv : wk) + (((size_t)b * Hkv + g) * w + p % w) * kHeadDim
                                 : (kv ? vnew : knew) + (((size_t)b * Hkv + g) * n + (p - L)) * kHeadDim;
            reinterpret_cast<uint4 *>(rows)[i] = *reinterpret_cast<const uint4 *>(src + q * E);
        }
        if (tid < nr) {
            const int lp = (m0 + tid) / kPage, id = lp < a.maxp ? a.block_table[(size_t)b * a.maxp + lp] : -1;
            const bool valid = id >= 0 && id < a.num_pages;
            if (!valid)
                report(a.status, DAR_ERR_CAPACITY);
            s_pid[tid] = valid ? id : -1;
        }
        __syncthreads();
        for (int ch0 = 0; ch0 < chains; ch0 += kFewThreads) {  // (whole warps take part: chains is a multiple of 16)
            const int ch = ch0 + tid, kg = ch / DD, c = ch % DD;
            if (ch0 > 0 && ch < chains)
                load_w(ch);
            if (ch0 + (tid & ~31) >= chains)
                break;
            FewWords<GS> out;
            const bool mine = ch < chains;
            unsigned char *heads = pool + (size_t)(kg % Hkv) * F::kBytes + c / GS * F::kBlock;
            for (int r = 0; r < nr; ++r) {
                float acc = 0.0f;  // Eq. 1: one fp32 FMA chain over t = 0..63
                if (mine) {
                    const uint4 *x4 = reinterpret_cast<const uint4 *>(rows + ((size_t)r * 2 * Hkv + kg) * kHeadDim);
#pragma unroll
                    for (int q = 0; q < GPR; ++q) {
                        float xf[E];
                        unpack(x4[q], xf, T());
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            acc = __fmaf_rn(xf[e], wc[q * E + e], acc);
                    }
                }
                const int m = m0 + r, id = s_pid[r];
                out.add(to_f32(from_f32<T>(acc)), c % GS, kg >= Hkv, m % kPage,
                        mine && id >= 0 ? heads + (size_t)id * Hkv * F::kBytes : nullptr, r + 1 == nr || (m + 1) % F::kUnit == 0);
            }
        }
        if (chains > kFewThreads && m0 + R < hi && tid < chains)  // the first chains' columns again
            load_w(tid);
        __syncthreads();
    }
    // new tokens that stay in the window: every ring row above is read
    const int j0 = max(0, nb - w), granules = 2 * Hkv * (nb - j0) * GPR;
    for (int i = tid; i < granules; i += kFewThreads) {
        const int q = i % GPR, rest = i / GPR, g = rest % Hkv, kv = (rest / Hkv) & 1, j = j0 + rest / (2 * Hkv);
        const uint4 v = nb == n && i == tid ? pre : *reinterpret_cast<const uint4 *>(new_granule(i, j0));
        *reinterpret_cast<uint4 *>((kv ? wv : wk) + (((size_t)b * Hkv + g) * w + (L + j) % w) * kHeadDim + q * E) = v;
    }
    __syncthreads();
    if (tid == 0)
        a.seq_lens[b] = Lnew;
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
    append_few_kernel<T, DD><<<a.B, kFewThreads, (size_t)few_rows<T>(a.Hkv) * 2 * a.Hkv * kHeadDim * sizeof(T), s>>>(a);
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
// A warp takes a page of a (sequence, KV head), one group after the other.
constexpr int kConvertWarps = 8;

template <typename T, int DD, bool PACK>
__global__ void __launch_bounds__(kConvertWarps * 32) convert_kernel(Q4ConvertArgs a)
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
    const long long lp = page0 + item / a.Hkv;
    if (first >= end || lp * kPage >= end)
        return;
    const int g = (int)(item % a.Hkv);
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
#pragma unroll
    for (int sb = 0; sb < F::kGroups; ++sb) {
        unsigned char *block = page + sb * F::kBlock;
        if constexpr (PACK) {
            write_page<T, GS, false>(block, k + sb * GS, DD, from, to, lane);
            write_page<T, GS, true>(block, v + sb * GS, DD, from, to, lane);
        } else {
            read_page<T, GS, false>(block, k + sb * GS, DD, from, to, lane);
            read_page<T, GS, true>(block, v + sb * GS, DD, from, to, lane);
        }
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

constexpr long long kBigTiles = kSms * 6 * 2;

template <typename T>
static cudaError_t append_t(int dd, const AppendArgs &a, cudaStream_t s)
{
    return by_width(dd, [&](auto width) {
        constexpr int DD = decltype(width)::value;
        if (a.n <= kFewRows && few_rows<T>(a.Hkv) > 0)
            return append_few_launch<T, DD>(a, s);
        // Large tiles, whose threads have several rows for a read of W, once they fill the chip a few times over and are
        // not mostly empty (the rule of dar_append.cu, whose tiles these are).
        constexpr int R = rows_bulk<T>();
        const long long tiles = ((long long)a.n + kPage - 1 + R - 1) / R;
        if (tiles * a.B * a.Hkv * 2 >= kBigTiles && a.n >= 4 * R)
            return append_tiles<T, DD, rows_per_thread<DD>(), R / rows_per_thread<DD>()>(a, s);
        return append_tiles<T, DD, 1, kPage>(a, s);
    });
}

template <typename T, bool PACK>
static cudaError_t convert_t(int dd, const Q4ConvertArgs &a, cudaStream_t s)
{
    const long long items = (long long)std::min(a.maxp, a.maxp4) * a.Hkv;
    const dim3 grid((unsigned)std::max(1ll, (items + kConvertWarps - 1) / kConvertWarps), (unsigned)a.B);
    return by_width(dd, [&](auto width) {
        convert_kernel<T, decltype(width)::value, PACK><<<grid, kConvertWarps * 32, 0, s>>>(a);
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
