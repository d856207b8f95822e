// gba_q4.hip -- products of a few rows with 4-bit weights, act(A.W + bias).
//
// W(k,j) = s(g,j) (q(k,j) - z(g,j)), g = k / group.  A code's four bits, put
// into the top of the fraction of the 16-bit float 16.0, are the float 16 + q
// with no conversion; so a group's sum is
//     sum_k a_k (q_k - z) = sum_k a_k (16 + q_k) - (16 + z) sum_k a_k
// and both sums are matrix instructions: the second one takes A times ones,
// or, where every z is 8, A times -24 into the same accumulator.  The products
// are exact and the sums fp32; the scale multiplies a group's fp32 sum.
//
// A workgroup owns 16 columns and 16 MT rows; its waves take the 128-deep
// chunks of K in turn (a chunk of a column block is 1 KB, contiguous: 16 bytes
// a lane, the lane's operands of four 32-deep matrix instructions) and add
// their sums through LDS in wave order.
#include "gba_decode.hpp"

namespace gba {
namespace {

struct Q4Args {
    const u4 *codes;
    const void *scales, *zeros, *A, *bias;
    void *C;
    int64_t lda, ldc;
    int M, N, K;
    int KB, GB;  // 128-deep chunks, groups
    int act;
};

constexpr int WAVES = 8;

template <class T>
__device__ __forceinline__ typename T::vec8 unpack(unsigned w)
{
    constexpr unsigned M = 0x000F000Fu << T::TOP;
    u4 r;
    r[0] = ((w << T::TOP) & M) | T::SIXTEEN;
    if constexpr (T::TOP >= 4) r[1] = ((w << (T::TOP - 4)) & M) | T::SIXTEEN;
    else r[1] = ((w >> (4 - T::TOP)) & M) | T::SIXTEEN;
    r[2] = ((w >> (8 - T::TOP)) & M) | T::SIXTEEN;
    r[3] = ((w >> (12 - T::TOP)) & M) | T::SIXTEEN;
    return __builtin_bit_cast(typename T::vec8, r);
}

template <class T>
__device__ __forceinline__ typename T::vec8 splat(float v)
{
    typename T::vec8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (typename T::elem)v;
    return r;
}

// Eight elements of a row from k on, zeros beyond K.
template <class T>
__device__ __forceinline__ typename T::vec8 load_row8(const typename T::elem *row, int k, int K)
{
    typedef typename T::vec8 unaligned __attribute__((aligned(2)));
    if (k + 8 <= K) return *reinterpret_cast<const unaligned *>(row + k);
    typename T::vec8 r = splat<T>(0.f);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (k + e < K) r[e] = row[k + e];
    return r;
}

// STEPS: 32-deep steps of a group
template <class T, int MT, int STEPS, bool ZEROS>
__global__ void __launch_bounds__(64 * WAVES) q4_kernel(Q4Args p)
{
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, kq = 8 * (lane >> 4);
    const int nb = blockIdx.x, row0 = blockIdx.y * (16 * MT);
    const u4 *codes = p.codes + (int64_t)nb * p.KB * 64 + lane;
    const elem *scales = static_cast<const elem *>(p.scales) + (int64_t)nb * p.GB * 16 + c;
    const elem *zeros = static_cast<const elem *>(p.zeros) + (int64_t)nb * p.GB * 16 + c;
    const elem *rows[MT];
    bool there[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int row = row0 + 16 * t + c;
        there[t] = row < p.M;
        rows[t] = static_cast<const elem *>(p.A) + (there[t] ? row : 0) * p.lda;
    }
    const vec8 fixed = splat<T>(ZEROS ? 1.f : -24.f), none = splat<T>(0.f);
    f4 acc[MT] = {};
    for (int kb = wave; kb < p.KB; kb += WAVES) {
        const u4 w = codes[(int64_t)kb * 64];
#pragma unroll
        for (int g = 0; g < 4 / STEPS; ++g) {
            int group = kb * (4 / STEPS) + g;
            if (group >= p.GB) group = p.GB - 1;  // beyond K: A's elements there are zeros
            const float scale = (float)scales[group * 16];
            f4 sum[MT] = {}, ones[MT] = {};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int j = g * STEPS + i;
                const vec8 b = unpack<T>(w[j]);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const vec8 a = there[t] ? load_row8<T>(rows[t], kb * 128 + 32 * j + kq, p.K) : none;
                    sum[t] = T::mfma(a, b, sum[t]);
                    if (ZEROS) ones[t] = T::mfma(a, fixed, ones[t]);
                    else sum[t] = T::mfma(a, fixed, sum[t]);
                }
            }
            const float shift = ZEROS ? 16.f + (float)zeros[group * 16] : 0.f;
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[t][e] += scale * (ZEROS ? sum[t][e] - shift * ones[t][e] : sum[t][e]);
        }
    }
    __shared__ f4 part[WAVES][MT][64];
#pragma unroll
    for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    for (int e = threadIdx.x; e < 256 * MT; e += 64 * WAVES) {
        const int row = row0 + e / 16, col = 16 * nb + e % 16;
        float x[1] = {0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x[0] += part[w][e / 256][(e / 64 % 4) * 16 + e % 16][e / 16 % 4];
        if (row < p.M && col < p.N) {
            if (p.bias != nullptr) x[0] += (float)static_cast<const elem *>(p.bias)[col];
            activate(p.act, x);
            static_cast<elem *>(p.C)[row * p.ldc + col] = (elem)x[0];
        }
    }
}

template <class T, int MT>
gba_status run_q4(const Q4Args &a, int group, hipStream_t s)
{
    const dim3 grid((unsigned)div_up(a.N, 16), (unsigned)div_up(a.M, 16 * MT)), block(64 * WAVES);
    const bool z = a.zeros != nullptr;
    if (group == 32) return z ? launch(q4_kernel<T, MT, 1, true>, grid, block, s, a) : launch(q4_kernel<T, MT, 1, false>, grid, block, s, a);
    if (group == 64) return z ? launch(q4_kernel<T, MT, 2, true>, grid, block, s, a) : launch(q4_kernel<T, MT, 2, false>, grid, block, s, a);
    return z ? launch(q4_kernel<T, MT, 4, true>, grid, block, s, a) : launch(q4_kernel<T, MT, 4, false>, grid, block, s, a);
}

template <class T>
gba_status run_q4(const Q4Args &a, int group, hipStream_t s)
{
    if (a.M <= 16) return run_q4<T, 1>(a, group, s);
    return a.M <= 32 ? run_q4<T, 2>(a, group, s) : run_q4<T, 4>(a, group, s);
}

// One thread a word.
__global__ void __launch_bounds__(256) q4_pack_kernel(int64_t words, int KB, int K, int N, const uint8_t *codes,
                                                      int64_t ld, uint32_t *packed)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= words) return;
    const int j = (int)(i & 3), l = (int)(i >> 2) & 63;
    const int64_t chunk = i >> 8;
    const int64_t col = chunk / KB * 16 + l % 16, k = chunk % KB * 128 + 32 * j + 8 * (l / 16);
    uint32_t w = 0;
    for (int e = 0; e < 8; ++e)
        if (k + e < K && col < N) w |= (uint32_t)(codes[(k + e) * ld + col] & 15) << (4 * (e / 2) + 16 * (e % 2));
    packed[i] = w;
}

}  // namespace
}  // namespace gba

using namespace gba;

extern "C" gba_status gba_q4_pack(int64_t K, int64_t N, const void *codes, int64_t ld, void *packed, gba_stream_t stream)
{
    if (K < 0 || N < 0 || ld < 0) return GBA_EINVAL;
    if (K > INT_MAX || N > INT_MAX) return GBA_EUNSUPPORTED;
    if (K == 0 || N == 0) return GBA_OK;
    if (codes == nullptr || packed == nullptr || ld < N) return GBA_EINVAL;
    const int64_t words = div_up(N, 16) * div_up(K, 128) * 256;
    if (!aligned_to(packed, 16) || div_up(words, 256) > INT_MAX / 256) return GBA_EUNSUPPORTED;
    return launch(q4_pack_kernel, dim3((unsigned)div_up(words, 256)), dim3(256), reinterpret_cast<hipStream_t>(stream), words,
                  (int)div_up(K, 128), (int)K, (int)N, static_cast<const uint8_t *>(codes), ld, static_cast<uint32_t *>(packed));
}

extern "C" gba_status gba_q4_linear(const gba_q4_weight *w, int64_t M, const void *A, int64_t lda, const void *bias,
                                    gba_act act, void *C, int64_t ldc, gba_stream_t stream)
{
    if (w == nullptr || !is_dtype(w->dtype) || !is_act(act)) return GBA_EINVAL;
    if (w->group != 32 && w->group != 64 && w->group != 128) return GBA_EINVAL;
    const int64_t K = w->K, N = w->N;
    if (M < 0 || N < 0 || K < 0 || lda < 0 || ldc < 0) return GBA_EINVAL;
    if (M > INT_MAX || N > INT_MAX || K > INT_MAX || M > 64 * (int64_t)65535) return GBA_EUNSUPPORTED;
    if (M == 0 || N == 0) return GBA_OK;
    if (C == nullptr || ldc < N) return GBA_EINVAL;
    if (K > 0 && (A == nullptr || lda < K || w->codes == nullptr || w->scales == nullptr)) return GBA_EINVAL;
    if (!aligned_to(w->codes, 16) || !aligned_to(w->scales, 2) || !aligned_to(w->zeros, 2) || !aligned_to(A, 2) ||
        !aligned_to(bias, 2) || !aligned_to(C, 2))
        return GBA_EUNSUPPORTED;
    // the launch runtime takes grids of less than 2^32 threads a dimension
    if (div_up(N, 16) > (int64_t)UINT_MAX / (64 * WAVES)) return GBA_EUNSUPPORTED;
    Q4Args a;
    a.codes = static_cast<const u4 *>(w->codes);
    a.scales = w->scales;
    a.zeros = w->zeros;
    a.A = A;
    a.bias = bias;
    a.C = C;
    a.lda = lda;
    a.ldc = ldc;
    a.M = (int)M;
    a.N = (int)N;
    a.K = (int)K;
    a.KB = (int)div_up(K, 128);
    a.GB = (int)div_up(K, w->group);
    a.act = act;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return w->dtype == GBA_F16 ? run_q4<F16>(a, w->group, s) : run_q4<BF16>(a, w->group, s);
}
