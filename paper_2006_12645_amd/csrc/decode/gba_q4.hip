// gba_q4.hip -- products of a few rows with 4-bit weights, act(A.W + bias).
//
// W(k,j) = s(g,j) (q(k,j) - z(g,j)), g = k / group.  A code's four bits, put
// into the top of the fraction of the 16-bit float 16.0, are the float 16 + q
// with no conversion; so a group's sum is
//     sum_k a_k (q_k - z) = sum_k a_k (16 + q_k) - (16 + z) sum_k a_k
// and both sums are matrix instructions, the second one of A and ones, for all
// columns of a wave at once.  The products are exact and the sums fp32; the
// scale multiplies a group's fp32 sum.  Where an element's sum is not finite,
// the first form is computed for it instead.
//
// The bound is reading W once.  A workgroup owns 16 NT columns and 16 MT rows;
// its waves take the 128-deep chunks of K in turn and never wait for each
// other before the end, where their sums are added through LDS in wave order.
// A chunk of a column block is 1 KB, contiguous: 16 bytes a lane, the lane's
// operands of four 32-deep matrix instructions.  A wave holds the codes,
// scales and rows of A of its next chunks in registers; A passes through the
// wave's own corner of LDS on its way to the matrix instructions' order, so
// that it is read in whole rows, of which the address unit takes four times
// as much a clock as of 16-byte pieces.
#include "gba_decode.hpp"
#include "gba_kernel.hpp"

namespace gba {
namespace {

struct Q4Args {
    const u4 *codes;
    const void *scales, *zeros, *A, *bias;
    void *C;
    int64_t lda, ldc;
    int M, N, K;
    int NB, KB, GB;  // 16-column blocks, 128-deep chunks, groups
    int act;
};

constexpr int WAVES = 8;

// The 16-bit floats 16 + q of eight codes.
template <class T>
__device__ __forceinline__ typename T::vec8 unpack(unsigned w)
{
    // in a vector register, or a mask and a constant are two instructions
    unsigned M = 0x000F000Fu << T::TOP;
    asm("" : "+v"(M));
    u4 r;
    r[0] = ((w << T::TOP) & M) | T::SIXTEEN;
    if constexpr (T::TOP >= 4) r[1] = ((w << (T::TOP - 4)) & M) | T::SIXTEEN;
    else r[1] = ((w >> (4 - T::TOP)) & M) | T::SIXTEEN;
    r[2] = ((w >> (8 - T::TOP)) & M) | T::SIXTEEN;
    r[3] = ((w >> (12 - T::TOP)) & M) | T::SIXTEEN;
    return __builtin_bit_cast(typename T::vec8, r);
}

// Eight elements of a row from k on, zeros beyond K.
template <class T>
__device__ __forceinline__ u4 load_row8(const typename T::elem *row, int k, int K)
{
    typedef u4 unaligned __attribute__((aligned(2)));
    if (k <= K - 8) return *reinterpret_cast<const unaligned *>(row + k);  // (k + 8 may be 2^31)
    typename T::vec8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = k + e < K ? row[k + e] : (typename T::elem)0.f;
    return __builtin_bit_cast(u4, r);
}

// sum_k a_k s (q_k - z) of one element, as it is written and in 64 bits.
template <class T>
__device__ __forceinline__ float q4_plainly(const Q4Args &p, int group, int row, int col)
{
    typedef typename T::elem elem;
    const int nb = col / 16, j = col % 16;
    const elem *a = static_cast<const elem *>(p.A) + row * p.lda;
    const uint32_t *codes = reinterpret_cast<const uint32_t *>(p.codes) + (int64_t)nb * p.KB * 256 + j * 4;
    const int64_t at = (int64_t)nb * p.GB * 16 + j;
    const elem *scales = static_cast<const elem *>(p.scales) + at, *zeros = static_cast<const elem *>(p.zeros) + at;
    double all = 0.;
    for (int g = 0; g < p.GB; ++g) {
        const double zero = p.zeros != nullptr ? (double)(float)zeros[(int64_t)g * 16] : 8.;
        double sum = 0.;
        for (int i = 0; i < group && g * group + i < p.K; i += 8) {
            const int k = g * group + i;
            const uint32_t w = codes[(int64_t)(k / 128) * 256 + k % 32 / 8 * 64 + k % 128 / 32];
            for (int e = 0; e < 8 && k + e < p.K; ++e) sum += (double)(float)a[k + e] * ((double)((w >> (4 * (e / 2) + 16 * (e % 2))) & 15) - zero);
        }
        all += (double)(float)scales[(int64_t)g * 16] * sum;
    }
    return (float)all;
}

// The waves' sums, added in wave order, bias, activation, and the one rounding.
// A sum that is not finite says little: infinity times 16 + q less infinity
// times 16 + z is NaN, and so is what the two sums of large inputs leave where
// each passes the largest float.  Such elements are computed again, plainly (one
// infinite input, 1 x 8192 x 32768: 0.65 ms).
template <class T, int MT, int NT, int W>
__device__ __forceinline__ void q4_store(const Q4Args &p, int group, const f4 (&acc)[MT][NT], char *smem, int row0, int nb0)
{
    typedef typename T::elem elem;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    f4 *part = reinterpret_cast<f4 *>(smem);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) part[((wave * MT + t) * NT + n) * 64 + lane] = acc[t][n];
    __syncthreads();
    const float *sums = reinterpret_cast<const float *>(smem);
    auto element = [&](int i, int &row, int &col) {
        const int t = i / (256 * NT), r = i / (16 * NT) % 16, n = i / 16 % NT, j = i % 16;
        row = row0 + 16 * t + r;
        col = 16 * (nb0 + n) + j;
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) x += sums[(((w * MT + t) * NT + n) * 64 + (r / 4) * 16 + j) * 4 + r % 4];
        return x;
    };
    auto finite = [](float x) { return (__builtin_bit_cast(unsigned, x) & 0x7F800000u) != 0x7F800000u; };
    auto store = [&](int row, int col, float sum) {
        float x[1] = {sum};
        if (p.bias != nullptr) x[0] += (float)static_cast<const elem *>(p.bias)[col];
        if (x[0] == x[0]) activate(p.act, x);  // (NaN stays NaN)
        static_cast<elem *>(p.C)[row * p.ldc + col] = (elem)x[0];
    };
    bool odd = false;
    int row, col;
    for (int i = threadIdx.x; i < 256 * MT * NT; i += 64 * W) {
        const float x = element(i, row, col);
        if (row >= p.M || col >= p.N) continue;
        odd |= !finite(x);
        store(row, col, x);
    }
    if (!odd) return;
#pragma unroll 1
    for (int i = threadIdx.x; i < 256 * MT * NT; i += 64 * W)
        if (!finite(element(i, row, col)) && row < p.M && col < p.N) store(row, col, q4_plainly<T>(p, group, row, col));
}

// Up to 16 rows.  STEPS: 32-deep steps of a group.  W: waves.  AHEAD: chunks
// that each holds in registers.  Bound by HBM for a large W: 1 x 8192 x 32768,
// 139 MB, 28.7 to 29.5 us (4.7 to 4.8 TB/s); 1 x 8192 x 8192, 35 MB, 9.3 us (3.7);
// 1 x 1024 x 1024 2.6 us, latency.
template <class T, int NT, int STEPS, bool ZEROS, int W, int AHEAD>
__global__ void __launch_bounds__(64 * W) q4_kernel(Q4Args p)
{
    constexpr int MT = 1;
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    constexpr int GROUPS = 4 / STEPS;              // of a chunk
    constexpr int ROWS = 16 * MT, LOADS = ROWS / 4;  // a load: four rows of 256 bytes
    constexpr int CORNER = ROWS * 256, PART = MT * NT * 1024;
    __shared__ __attribute__((aligned(16))) char smem[W * (CORNER > PART ? CORNER : PART)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int nb0 = blockIdx.x * NT, row0 = blockIdx.y * ROWS;
    char *corner = smem + wave * CORNER;

    // column blocks beyond the last one repeat it; they are not stored
    const u4 *codes[NT];
    const elem *scales[NT], *zeros[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int64_t nb = nb0 + n < p.NB ? nb0 + n : p.NB - 1;
        codes[n] = p.codes + nb * p.KB * 64 + lane;
        scales[n] = static_cast<const elem *>(p.scales) + nb * p.GB * 16 + c;
        zeros[n] = static_cast<const elem *>(p.zeros) + nb * p.GB * 16 + c;
    }
    const int rows = p.M - row0 < ROWS ? p.M - row0 : ROWS;
    const elem *A = static_cast<const elem *>(p.A) + row0 * p.lda;

    u4 code[AHEAD][NT], a[AHEAD][LOADS];
    elem scale[AHEAD][NT], zero[AHEAD][NT];  // of group lane / 16 of the chunk
    auto load = [&](int d, int kb) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            code[d][n] = codes[n][(int64_t)kb * 64];
            int group = kb * GROUPS + g % GROUPS;
            if (group >= p.GB) group = p.GB - 1;  // beyond K: A's elements there are zeros
            scale[d][n] = scales[n][group * 16];
            if (ZEROS) zero[d][n] = zeros[n][group * 16];
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (4 * i < rows) {
                const int row = 4 * i + g;
                a[d][i] = load_row8<T>(A + (row < rows ? row : rows - 1) * p.lda, kb * 128 + 8 * c, p.K);
            }
    };
    vec8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (elem)1.f;
    f4 acc[MT][NT] = {};
    auto use = [&](int d) {
        // row r's 16-byte piece j stands at j ^ (r % 16)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) *reinterpret_cast<u4 *>(corner + (4 * i + g) * 256 + 16 * (c ^ ((4 * i + g) & 15))) = a[d][i];
        lanes_meet();
#pragma unroll
        for (int s = 0; s < GROUPS; ++s) {
            f4 sum[MT][NT] = {}, all[MT] = {};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int j = s * STEPS + i;
                vec8 b[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) b[n] = unpack<T>(code[d][n][j]);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const vec8 x = *reinterpret_cast<const vec8 *>(corner + (16 * t + c) * 256 + 16 * ((4 * j + g) ^ c));
                    all[t] = T::mfma(x, ones, all[t]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) sum[t][n] = T::mfma(x, b[n], sum[t][n]);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float f = (float)scale[d][n], shift = ZEROS ? 16.f + (float)zero[d][n] : 24.f;
                if (GROUPS > 1) {
                    f = __shfl(f, 16 * s + c);
                    if (ZEROS) shift = __shfl(shift, 16 * s + c);
                }
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][n][e] += f * (sum[t][n][e] - shift * all[t][e]);
            }
        }
        lanes_meet();
    };

#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
        if (wave + W * d < p.KB) load(d, wave + W * d);
    for (int kb = wave; kb < p.KB; kb += W * AHEAD) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int at = kb + W * d;
            if (at < p.KB) use(d);
            if (at + W * AHEAD < p.KB) load(d, at + W * AHEAD);
        }
    }

    __syncthreads();
    q4_store<T, MT, NT, W>(p, 32 * STEPS, acc, smem, row0, nb0);
}

// 16 MT rows, MT 2 or 4, of which a wave could not hold the next chunks in
// registers.  DIRECT (16-byte aligned rows of A and K a multiple of 8): A goes
// straight to the wave's own part of LDS, AHEAD half chunks (16 MT rows of 64
// k) before it is used; rows beyond M and k beyond K are read past the end of
// a buffer, which gives zeros.  Else one half chunk ahead is in registers.
// The codes, scales and zeros of the next two chunks stay in registers.  Bound by
// instructions, about 430 a chunk and wave (48 of them matrix instructions), and
// by all of A going through each compute unit: 64 x 8192 x 8192, groups of 64 with
// zeros, 21.1 to 23.7 us (360 to 410 TFLOP/s, 1.7 to 1.9 TB/s).
template <int MT, int NT, bool DIRECT>
struct Q4Lds {
    static constexpr int AHEAD = MT == 4 || !DIRECT ? 1 : 3, SLOTS = DIRECT ? AHEAD + 1 : 1;
    static constexpr int HALF = 16 * MT * 128, COPIES = 2 * MT, WAVE = SLOTS * HALF, PART = MT * NT * 1024;
    static constexpr int SIZE = WAVES * (WAVE > PART ? WAVE : PART);
};

template <class T, int MT, int NT, int STEPS, bool ZEROS, bool DIRECT>
__global__ void __launch_bounds__(64 * WAVES) q4_rows_kernel(Q4Args p)
{
    typedef Q4Lds<MT, NT, DIRECT> L;
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    constexpr int GROUPS = 4 / STEPS, ROWS = 16 * MT;
    __shared__ __attribute__((aligned(16))) char smem[L::SIZE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int nb0 = blockIdx.x * NT, row0 = blockIdx.y * ROWS;
    char *mine = smem + wave * L::WAVE;
    const int count = p.KB > wave ? (p.KB - wave + WAVES - 1) / WAVES : 0;

    const u4 *codes[NT];
    const elem *scales[NT], *zeros[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int64_t nb = nb0 + n < p.NB ? nb0 + n : p.NB - 1;
        codes[n] = p.codes + nb * p.KB * 64 + lane;
        scales[n] = static_cast<const elem *>(p.scales) + nb * p.GB * 16 + c;
        zeros[n] = static_cast<const elem *>(p.zeros) + nb * p.GB * 16 + c;
    }
    u4 code[2][NT];
    elem scale[2][NT], zero[2][NT];  // of group lane / 16 of the chunk
    auto load = [&](int d, int i) {
        const int kb = wave + WAVES * i;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            code[d][n] = codes[n][(int64_t)kb * 64];
            int group = kb * GROUPS + g % GROUPS;
            if (group >= p.GB) group = p.GB - 1;
            scale[d][n] = scales[n][group * 16];
            if (ZEROS) zero[d][n] = zeros[n][group * 16];
        }
    };

    // row r's 16-byte piece j of a half chunk stands at j ^ (r % 8)
    const int piece = (lane & 7) ^ (lane >> 3);
    int off[DIRECT ? L::COPIES : 1];
    if constexpr (DIRECT) {
#pragma unroll
        for (int i = 0; i < L::COPIES; ++i) {
            const int row = 8 * i + (lane >> 3);
            off[i] = row0 + row < p.M ? (int)(row * p.lda * 2) + 16 * piece : OOB_OFFSET;
        }
    }
    const elem *A = static_cast<const elem *>(p.A) + row0 * p.lda;
    const int rows = p.M - row0 < ROWS ? p.M - row0 : ROWS;
    u4 next[DIRECT ? 1 : L::COPIES];
    // half chunk u; DIRECT: those past the wave's last one are of length 0, so
    // that the number of copies under way is always the same
    auto copy = [&](int u) {
        const unsigned k0 = (unsigned)(wave + WAVES * (u >> 1)) * 128 + 64 * (u & 1);  // past the last one it may pass 2^31
        const bool real = (u >> 1) < count;
        if constexpr (DIRECT) {
            const bool past = k0 + 8 * piece >= (unsigned)p.K;
            const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<elem *>(A + (real ? k0 : 0)), (short)0,
                                                                                real ? MAX_RECORDS : 0, RSRC_WORD3);
#pragma unroll
            for (int j = 0; j < L::COPIES; ++j)
                buffer_load16_lds(rs, mine + u % L::SLOTS * L::HALF + 1024 * j, past ? OOB_OFFSET : off[j], 0);
        } else if (real) {
#pragma unroll
            for (int j = 0; j < L::COPIES; ++j)
                if (8 * j < rows) {
                    const int row = 8 * j + (lane >> 3);
                    next[j] = load_row8<T>(A + (row < rows ? row : rows - 1) * p.lda, (int)k0 + 8 * piece, p.K);
                }
        }
    };

    vec8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (elem)1.f;
    f4 acc[MT][NT] = {};
    f4 sum[MT][NT], all[MT];
    auto use = [&](int d, int i) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int u = 2 * i + half;
            if constexpr (DIRECT) {
                wait_vm_lgkm0<63>();  // the slot's last fragments have been read
                copy(u + L::AHEAD);
                wait_vm_lgkm0<L::COPIES * L::AHEAD>();
            } else {
                lanes_meet();
#pragma unroll
                for (int j = 0; j < L::COPIES; ++j) *reinterpret_cast<u4 *>(mine + 1024 * j + 16 * lane) = next[j];
                copy(u + 1);
            }
            lanes_meet();
            const char *a = mine + u % L::SLOTS * L::HALF;
#pragma unroll
            for (int j = 2 * half; j < 2 * half + 2; ++j) {
                if (j % STEPS == 0) {
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        all[t] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int n = 0; n < NT; ++n) sum[t][n] = f4{0.f, 0.f, 0.f, 0.f};
                    }
                }
                vec8 b[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) b[n] = unpack<T>(code[d][n][j]);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const vec8 x = *reinterpret_cast<const vec8 *>(a + (16 * t + c) * 128 + 16 * ((4 * (j & 1) + g) ^ (c & 7)));
                    all[t] = T::mfma(x, ones, all[t]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) sum[t][n] = T::mfma(x, b[n], sum[t][n]);
                }
                if (j % STEPS == STEPS - 1) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float f = (float)scale[d][n], shift = ZEROS ? 16.f + (float)zero[d][n] : 24.f;
                        if (GROUPS > 1) {
                            f = __shfl(f, 16 * (j / STEPS) + c);
                            if (ZEROS) shift = __shfl(shift, 16 * (j / STEPS) + c);
                        }
#pragma unroll
                        for (int t = 0; t < MT; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[t][n][e] += f * (sum[t][n][e] - shift * all[t][e]);
                    }
                }
            }
        }
    };
    if (count > 0) {
        load(0, 0);
        if (count > 1) load(1, 1);
#pragma unroll
        for (int u = 0; u < L::AHEAD; ++u) copy(u);
    }
    for (int i = 0; i < count; i += 2) {
        use(0, i);
        if (i + 2 < count) load(0, i + 2);
        if (i + 1 < count) {
            use(1, i + 1);
            if (i + 3 < count) load(1, i + 3);
        }
    }
    wait_vm_lgkm0<0>();
    __syncthreads();
    q4_store<T, MT, NT, WAVES>(p, 32 * STEPS, acc, smem, row0, nb0);
}

template <class T, int MT, int NT, bool DIRECT>
gba_status run_rows(const Q4Args &a, int group, hipStream_t s)
{
    const dim3 grid((unsigned)div_up(a.NB, NT), (unsigned)div_up(a.M, 16 * MT)), block(64 * WAVES);
    const bool z = a.zeros != nullptr;
    // groups of 32 and two column blocks of 64 rows need more registers than
    // there are (64 x 8192 x 8192: 75 us against 41 on one)
    if constexpr (MT * NT < 8)
        if (group == 32)
            return z ? launch(q4_rows_kernel<T, MT, NT, 1, true, DIRECT>, grid, block, s, a) : launch(q4_rows_kernel<T, MT, NT, 1, false, DIRECT>, grid, block, s, a);
    if (group == 64)
        return z ? launch(q4_rows_kernel<T, MT, NT, 2, true, DIRECT>, grid, block, s, a) : launch(q4_rows_kernel<T, MT, NT, 2, false, DIRECT>, grid, block, s, a);
    return z ? launch(q4_rows_kernel<T, MT, NT, 4, true, DIRECT>, grid, block, s, a) : launch(q4_rows_kernel<T, MT, NT, 4, false, DIRECT>, grid, block, s, a);
}

template <class T, int NT, int W, int AHEAD>
gba_status run_few(const Q4Args &a, int group, hipStream_t s)
{
    const dim3 grid((unsigned)div_up(a.NB, NT)), block(64 * W);
    const bool z = a.zeros != nullptr;
    // groups of 32, two column blocks: more than the 128 registers of 16 waves
    if constexpr (NT != 2 || W != 16)
        if (group == 32) return z ? launch(q4_kernel<T, NT, 1, true, W, AHEAD>, grid, block, s, a) : launch(q4_kernel<T, NT, 1, false, W, AHEAD>, grid, block, s, a);
    if (group == 64) return z ? launch(q4_kernel<T, NT, 2, true, W, AHEAD>, grid, block, s, a) : launch(q4_kernel<T, NT, 2, false, W, AHEAD>, grid, block, s, a);
    return z ? launch(q4_kernel<T, NT, 4, true, W, AHEAD>, grid, block, s, a) : launch(q4_kernel<T, NT, 4, false, W, AHEAD>, grid, block, s, a);
}

// Which kernel: one 16-row block with its chunks in registers up to 16 rows,
// else blocks of 32 or 64 rows.  Column blocks of a workgroup: as many as
// leave 256 workgroups, since a workgroup reads all of its rows of A (1 x 8192 x
// 8192: 9.3 us with two, 12.0 with one; 1 x 4096 x 4096 4.5 with one, 5.3 with two;
// 64 x 8192 x 8192 22.0 with two, 30.5 with one; 32 x 4096 x 4096 7.4 with one, 8.4
// with two).
template <class T>
gba_status run_q4(const Q4Args &a, int group, hipStream_t s)
{
    if (a.M <= 16) {
        // One chunk ahead on four column blocks, two on fewer: more waves fit
        // with fewer registers (1 x 8192 x 32768: 28.5 us against 32.2 with
        // twice as many ahead).  16 waves with one ahead where each has a
        // chunk: 1 x 8192 x 8192 9.3 us against 10.5 with 8, 16 x 8192 x 1024
        // 6.9 against 8.2; half of them idle, 1024 x 32768 12.1 against 7.7.
        if (a.NB >= 1024) return run_few<T, 4, WAVES, 1>(a, group, s);
        if (a.KB >= 16 && a.NB < 512) return run_few<T, 1, 16, 1>(a, group, s);
        if (a.KB >= 16 && group != 32) return run_few<T, 2, 16, 1>(a, group, s);
        return a.NB >= 512 ? run_few<T, 2, WAVES, 2>(a, group, s) : run_few<T, 1, WAVES, 2>(a, group, s);
    }
    const bool direct = a.lda % 8 == 0 && a.K % 8 == 0 && a.lda < (1 << 23) && aligned_to(a.A, 16);
    if (!direct) return a.M <= 32 ? run_rows<T, 2, 1, false>(a, group, s) : run_rows<T, 4, 1, false>(a, group, s);
    if (a.NB >= 512 && (a.M <= 32 || group != 32)) return a.M <= 32 ? run_rows<T, 2, 2, true>(a, group, s) : run_rows<T, 4, 2, true>(a, group, s);
    return a.M <= 32 ? run_rows<T, 2, 1, true>(a, group, s) : run_rows<T, 4, 1, true>(a, group, s);
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
    if (div_up(N, 16) > (int64_t)UINT_MAX / 1024) return GBA_EUNSUPPORTED;
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
    a.NB = (int)div_up(N, 16);
    a.KB = (int)div_up(K, 128);
    a.GB = (int)div_up(K, w->group);
    a.act = act;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return w->dtype == GBA_F16 ? run_q4<F16>(a, w->group, s) : run_q4<BF16>(a, w->group, s);
}
