// gba_q4_cache.hip -- new keys and values into the paged cache in 4 bits, and
// back out of it.
//
// A thread takes eight elements of a row, one word of codes: 16 bytes in and 4
// out, or the reverse; the threads of a group (4, 8 or 16) have its ends from
// lane exchanges.  Bound by HBM for prompts, by the launch for single tokens.
#include "gba_q4_cache.hpp"

namespace gba {
namespace {

struct Q4StoreArgs {
    const uint16_t *src[2];  // load: dst
    int64_t src_token[2], src_head[2];
    void *codes[2], *scales[2];
    const int32_t *slots;
    int64_t words;           // of all tokens
    int heads, dim, block_size, group_words;  // words of a group
    int64_t capacity;
};

// Where word w of thread i is: a token's head, its row in the cache (or -1).
struct Place {
    int64_t token, row;
    int head, word;
};

template <int WORDS>
__device__ __forceinline__ Place place_of(const Q4StoreArgs &p, int64_t i)
{
    Place at;
    const int64_t t = i / (p.heads * WORDS);
    const int in_token = (int)(i - t * (p.heads * WORDS));
    at.token = t;
    at.head = in_token / WORDS;
    at.word = in_token % WORDS;
    const int slot = p.slots[t];
    at.row = -1;
    if (slot >= 0 && slot < p.capacity) {
        const int block = slot / p.block_size;
        at.row = ((int64_t)block * p.heads + at.head) * p.block_size + (slot - block * p.block_size);
    }
    return at;
}

// The place of a key's word in its row: the words that a lane of a matrix
// instruction takes stand together.
template <int WORDS>
__device__ __forceinline__ int key_word(int w)
{
    return w % 4 * (WORDS / 4) + w / 4;
}

// WIDE: rows are read 16 bytes at a time.  Every group is stored from its own
// ends: scale = (high - low) / 15 and offset = low + 8 scale, each rounded to
// the cache's type; the codes are those nearest to the values, given these two.
// The steps are those of include/gba.h, in fp32, and nothing is contracted that
// would round differently: 0.5 high, 0.5 low and 8 scale are exact.
template <class T, int WORDS, bool WIDE>
__global__ void __launch_bounds__(256) q4_store_kernel(Q4StoreArgs p)
{
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    const int which = blockIdx.y;
    // (words is a multiple of a row's, so the threads of a group stay together)
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.words; i += (int64_t)gridDim.x * 256) {
        const Place at = place_of<WORDS>(p, i);
        const int d = 8 * at.word;
        const bool real = d < p.dim;
        float x[8];
        const uint16_t *src = p.src[which] + at.token * p.src_token[which] + at.head * p.src_head[which] + d;
        vec8 v = {};
        if (real && at.row >= 0) {
            if constexpr (WIDE) {
                v = *reinterpret_cast<const vec8 *>(src);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __builtin_bit_cast(elem, src[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
        float high = real ? x[0] : -INFINITY, low = real ? x[0] : INFINITY;
#pragma unroll
        for (int e = 1; e < 8; ++e) {
            high = real ? __builtin_elementwise_maximum(high, x[e]) : high;  // (NaN if either is)
            low = real ? __builtin_elementwise_minimum(low, x[e]) : low;
        }
#pragma unroll
        for (int s = 1; s < WORDS; s *= 2)
            if (s < p.group_words) {
                high = __builtin_elementwise_maximum(high, __shfl_xor(high, s));
                low = __builtin_elementwise_minimum(low, __shfl_xor(low, s));
            }
        const bool finite = high - high == 0.f && low - low == 0.f;
        float scale = finite ? (float)(elem)((0.5f * high - 0.5f * low) * (2.f / 15.f)) : 0.f;
        if (scale < SMALLEST_SCALE) scale = 0.f;
        const float offset = finite ? (float)(elem)(low + 8.f * scale) : high < low ? 0.f : NAN;  // (padding: no value)
        const float inverse = scale > 0.f ? 1.f / scale : 0.f;
        unsigned word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float steps = (x[e] - offset) * inverse;
            const float code = real && scale > 0.f ? __builtin_rintf(steps) + 8.f : 8.f;
            word |= (unsigned)__builtin_fminf(__builtin_fmaxf(code, 0.f), 15.f) << (4 * e);
        }
        if (at.row < 0) continue;
        unsigned *codes = static_cast<unsigned *>(p.codes[which]) + at.row * WORDS;
        codes[which == 0 ? key_word<WORDS>(at.word) : at.word] = word;
        if (at.word % p.group_words == 0) {
            typedef elem pair_t __attribute__((ext_vector_type(2)));
            pair_t pair = {(elem)scale, (elem)offset};
            static_cast<pair_t *>(p.scales[which])[at.row * (WORDS / p.group_words) + at.word / p.group_words] = pair;
        }
    }
}

template <class T, int WORDS, bool WIDE>
__global__ void __launch_bounds__(256) q4_load_kernel(Q4StoreArgs p)
{
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    typedef elem pair_t __attribute__((ext_vector_type(2)));
    const int which = blockIdx.y;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.words; i += (int64_t)gridDim.x * 256) {
        const Place at = place_of<WORDS>(p, i);
        if (8 * at.word >= p.dim) continue;
        vec8 v = {};
        if (at.row >= 0) {
            const unsigned word = static_cast<const unsigned *>(p.codes[which])[at.row * WORDS + (which == 0 ? key_word<WORDS>(at.word) : at.word)];
            const pair_t pair = static_cast<const pair_t *>(p.scales[which])[at.row * (WORDS / p.group_words) + at.word / p.group_words];
            const float scale = (float)pair[0], offset = (float)pair[1], nan = 0.f * scale + 0.f * offset;  // (0 of finite ones)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __builtin_fmaf(scale, (float)(int)((word >> (4 * e)) & 15) - 8.f, offset);
                v[e] = (elem)(__builtin_elementwise_minimum(__builtin_elementwise_maximum(x, -T::LARGEST), T::LARGEST) + nan);
            }
        }
        uint16_t *dst = const_cast<uint16_t *>(p.src[which]) + at.token * p.src_token[which] + at.head * p.src_head[which] + 8 * at.word;
        if constexpr (WIDE) {
            *reinterpret_cast<vec8 *>(dst) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const elem one = v[e];
                dst[e] = __builtin_bit_cast(uint16_t, one);
            }
        }
    }
}

template <class T, int WORDS, bool WIDE>
gba_status run_rows(const Q4StoreArgs &a, bool load, hipStream_t s)
{
    const int64_t groups = div_up(a.words, 256);
    const dim3 grid((unsigned)(groups < 16384 ? groups : 16384), 2), block(256);
    return load ? launch(q4_load_kernel<T, WORDS, WIDE>, grid, block, s, a) : launch(q4_store_kernel<T, WORDS, WIDE>, grid, block, s, a);
}

template <class T, bool WIDE>
gba_status run_rows(const Q4StoreArgs &a, bool load, int words, hipStream_t s)
{
    return words == 8 ? run_rows<T, 8, WIDE>(a, load, s) : words == 16 ? run_rows<T, 16, WIDE>(a, load, s) : run_rows<T, 32, WIDE>(a, load, s);
}

gba_status rows(const gba_q4_cache *c, int64_t tokens, const int32_t *slots, const void *k, int64_t k_token, int64_t k_head, const void *v,
                int64_t v_token, int64_t v_head, bool load, gba_stream_t stream)
{
    if (c == nullptr || tokens < 0) return GBA_EINVAL;
    const gba_status st = validate_q4_cache(*c);
    if (st != GBA_OK) return st;
    if (tokens > INT_MAX) return GBA_EUNSUPPORTED;
    if (tokens == 0 || c->heads == 0 || c->dim == 0 || (c->num_blocks == 0 && !load)) return GBA_OK;
    if (k == nullptr || v == nullptr || slots == nullptr) return GBA_EINVAL;
    if (!aligned_to(k, 2) || !aligned_to(v, 2) || !aligned_to(slots, 4)) return GBA_EUNSUPPORTED;
    Q4StoreArgs a;
    const void *src[2] = {k, v};
    const int64_t strides[2][2] = {{k_token, k_head}, {v_token, v_head}};
    bool wide = true;
    for (int i = 0; i < 2; ++i) {
        a.src[i] = static_cast<const uint16_t *>(src[i]);
        a.src_token[i] = strides[i][0];
        a.src_head[i] = strides[i][1];
        wide = wide && aligned_to(src[i], 16) && (tokens == 1 || strides[i][0] % 8 == 0) && (c->heads == 1 || strides[i][1] % 8 == 0);
    }
    const int words = q4_width(c->dim) / 8;
    a.codes[0] = c->k_codes;
    a.codes[1] = c->v_codes;
    a.scales[0] = c->k_scales;
    a.scales[1] = c->v_scales;
    a.slots = slots;
    a.words = tokens * c->heads * words;
    a.heads = (int)c->heads;
    a.dim = (int)c->dim;
    a.block_size = (int)c->block_size;
    a.group_words = c->group / 8 < words ? c->group / 8 : words;
    a.capacity = c->num_blocks * c->block_size;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (c->dtype == GBA_F16) return wide ? run_rows<F16, true>(a, load, words, s) : run_rows<F16, false>(a, load, words, s);
    return wide ? run_rows<BF16, true>(a, load, words, s) : run_rows<BF16, false>(a, load, words, s);
}

}  // namespace
}  // namespace gba

using namespace gba;

extern "C" gba_status gba_q4_cache_store(const gba_q4_cache *cache, int64_t tokens, const void *k, int64_t k_token, int64_t k_head,
                                         const void *v, int64_t v_token, int64_t v_head, const int32_t *slots, gba_stream_t stream)
{
    return rows(cache, tokens, slots, k, k_token, k_head, v, v_token, v_head, false, stream);
}

extern "C" gba_status gba_q4_cache_load(const gba_q4_cache *cache, int64_t tokens, const int32_t *slots, void *k, int64_t k_token,
                                        int64_t k_head, void *v, int64_t v_token, int64_t v_head, gba_stream_t stream)
{
    return rows(cache, tokens, slots, k, k_token, k_head, v, v_token, v_head, true, stream);
}
