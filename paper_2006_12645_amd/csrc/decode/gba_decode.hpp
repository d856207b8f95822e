// gba_decode.hpp -- element types and host helpers shared by the kernels of
// a decoding step (4-bit weights, paged cache, tree attention).
#pragma once

#include <limits.h>
#include <stdint.h>

#include "gba.h"
#include "gba_common.hpp"

namespace gba {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

// fp16 and bf16: the matrix instruction, the bits of 16 + q for a code q (the
// code in the top bits of the fraction: no conversion is needed), and
// those of infinity and of the exponent's lowest bit, all twice.  SLACK, LIFT:
// how far, in powers of two, a softmax weight may pass that of the running
// maximum before the maximum moves, and what that one's weight is.
struct F16 {
    typedef _Float16 elem;
    typedef h8 vec8;
    static constexpr unsigned SIXTEEN = 0x4C004C00u;  // 16.0 twice
    static constexpr int TOP = 6;                     // lowest bit of the four fraction bits that hold a code
    static constexpr unsigned INFINITE = 0x7C007C00u, EXPONENT_ONE = 0x04000400u;
    static constexpr float SLACK = 4.f, LIFT = 11.f;
    static constexpr float LARGEST = 65504.f;
    static __device__ __forceinline__ f4 mfma(vec8 a, vec8 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};
struct BF16 {
    typedef __bf16 elem;
    typedef b8 vec8;
    static constexpr unsigned SIXTEEN = 0x41804180u;
    static constexpr int TOP = 3;
    static constexpr unsigned INFINITE = 0x7F807F80u, EXPONENT_ONE = 0x00800080u;
    static constexpr float SLACK = 8.f, LIFT = 0.f;
    static constexpr float LARGEST = 0x1.FEp127f;
    static __device__ __forceinline__ f4 mfma(vec8 a, vec8 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};

// First index i of [0, n] with before[i + 1] > v, for a rising array of n + 1
// (n where there is none): the owner of item v, before[] being where each
// owner's items begin.
template <class P>
__device__ __forceinline__ int owner_of(const P *before, int n, int64_t v)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (before[mid + 1] > v) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// What one lane of a wave has written to LDS, another one reads after this: a
// wave's accesses run in order, so only the compiler has to keep it.
__device__ __forceinline__ void lanes_meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

inline bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool is_dtype(int d) { return d == GBA_F16 || d == GBA_BF16; }
inline bool is_act(int a) { return a >= GBA_ACT_NONE && a <= GBA_ACT_TANH; }
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Launch, and the library's status for it.
template <class F, class... A>
gba_status launch(F kernel, dim3 grid, dim3 block, hipStream_t s, const A &...args)
{
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, grid, block, 0, s, args...);
    return hipGetLastError() == hipSuccess ? GBA_OK : GBA_EHIP;
}

}  // namespace gba
