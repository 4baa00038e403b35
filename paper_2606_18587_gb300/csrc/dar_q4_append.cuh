// dar_q4_append.cuh -- the append of few tokens to a cache in 4 bits, as blocks of a kernel of its own or of the
// serving step's first kernel.
#pragma once

#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_project.cuh"
#include "dar_q4.cuh"

namespace dar {
namespace q4 {

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
template <typename T>
inline size_t few_smem(int Hkv)
{
    return (size_t)few_rows<T>(Hkv) * 2 * Hkv * kHeadDim * sizeof(T);
}
// Whether a call is one of this kernel's.  A sequence takes it some 4 us and 1 us for every token and round of chains, as
// many sequences as SMs no longer; the tiles of dar_q4_cache.cu take 6.4 us up to 8 tokens and more with every CTA.
// Here and there, d_down 16, us (B, Hkv, n): 1, 12, 1: 5.0 and 6.4; 1, 12, 4: 8.6 and 6.6; 32, 1, 4: 7.4 and 7.0; 32, 12, 8:
// 13.0 and 13.6; 32, 32, 4: 15.6 and 18.3; 32, 32, 8: 25 and 19; 128, 12, 8: 13.2 and 25.4; of 64 entries 32, 8, 4: 13.3 and
// 17.3; 32, 8, 8: 20.8 and 18.0.  (Of these the rule gives 32, 12, 8 to the tiles.)
template <typename T>
inline bool append_is_few(const AppendArgs &a, int dd)
{
    const long long chains = 2ll * a.Hkv * dd, rounds = (chains + kFewThreads - 1) / kFewThreads;
    return a.n <= kFewRows && few_rows<T>(a.Hkv) > 0 && a.n * rounds <= 2 + a.B * chains / (8 * kFewThreads);
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
            put_word(reinterpret_cast<uint32_t *>(block + (values ? kPage * GS / 2 + word_offset<GS, true>(row0, j)
                                                                  : word_offset<GS, false>(row0, j))), x, mask);
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

}  // namespace q4
}  // namespace dar
