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
    int tokens, heads, dim, block_size, group_words;  // words of a group
    int token_words, block_tokens;                    // words of a token; tokens of a workgroup
    unsigned token_factor;                            // 2^32 / token_words, rounded up
    int64_t capacity;
};

// Words of a thread, whose reads are under way together: two where there are
// many (16384 tokens of 8 heads of 128 in groups of 32: 24.5 us stored and 20.6
// read back; 28 and 24 with one, 26.1 and 20.8 with four), one where each thread
// is one more to share the latency (8 tokens: 3.2 and 3.0 us).
constexpr int64_t MANY_WORDS = 1 << 18;

// A word of a token: which one, of which head.
struct Place {
    int token, head, word;
    bool real;
};

// Word u of this thread: a workgroup has block_tokens whole tokens, or with
// longer ones a part of one.
template <int WORDS, int AT_ONCE>
__device__ __forceinline__ Place place_of(const Q4StoreArgs &p, int u)
{
    Place at;
    const unsigned i = threadIdx.x + 256 * u;
    const unsigned t = p.block_tokens > 1 ? __umulhi(i, p.token_factor) : 0;  // (exact: i is below 2^10)
    const unsigned in_token = i - t * p.token_words + blockIdx.z * (256 * AT_ONCE);
    at.token = (int)(blockIdx.x * p.block_tokens + t);
    at.head = (int)(in_token / WORDS);
    at.word = (int)(in_token % WORDS);
    at.real = t < (unsigned)p.block_tokens && in_token < (unsigned)p.token_words && at.token < p.tokens;
    return at;
}

// The row of a head's token in the cache, or -1.
__device__ __forceinline__ int64_t row_of(const Q4StoreArgs &p, const Place &at)
{
    const int slot = at.real ? p.slots[at.token] : -1;
    if (slot < 0 || slot >= p.capacity) return -1;
    const int block = slot / p.block_size;
    return ((int64_t)block * p.heads + at.head) * p.block_size + (slot - block * p.block_size);
}

// The higher and the lower of two lanes' ends (NaN if either is).
template <int CTRL>
__device__ __forceinline__ void ends(float &high, float &low)
{
    const int h = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, high), CTRL, 0xF, 0xF, false);
    const int l = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, low), CTRL, 0xF, 0xF, false);
    high = __builtin_elementwise_maximum(high, __builtin_bit_cast(float, h));
    low = __builtin_elementwise_minimum(low, __builtin_bit_cast(float, l));
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
// would round differently: 0.5 high and 0.5 low are exact.
template <class T, int WORDS, bool WIDE, int AT_ONCE>
__global__ void __launch_bounds__(256) q4_store_kernel(Q4StoreArgs p)
{
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    const int which = blockIdx.y;
    Place at[AT_ONCE];
    vec8 v[AT_ONCE];
    int64_t row[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        at[u] = place_of<WORDS, AT_ONCE>(p, u);
        const int d = 8 * at[u].word;
        v[u] = vec8{};
        if (!at[u].real || d >= p.dim) continue;
        const uint16_t *src = p.src[which] + at[u].token * p.src_token[which] + at[u].head * p.src_head[which] + d;
        if constexpr (WIDE) {
            v[u] = *reinterpret_cast<const vec8 *>(src);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = __builtin_bit_cast(elem, src[e]);
        }
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) row[u] = row_of(p, at[u]);
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        const int word_of_row = at[u].word;
        const bool real = 8 * word_of_row < p.dim;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[u][e];
        float high = x[0], low = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) {
            high = __builtin_elementwise_maximum(high, x[e]);  // (NaN if either is)
            low = __builtin_elementwise_minimum(low, x[e]);
        }
        if (!real) {
            high = -INFINITY;
            low = INFINITY;
        }
        // (a workgroup begins with a whole row, so the threads of a group stay
        // together: its quad, then the other quad of eight, then the other eight)
        ends<0xB1>(high, low);
        ends<0x4E>(high, low);
        if (p.group_words > 4) ends<0x141>(high, low);
        if (p.group_words > 8) ends<0x140>(high, low);
        const bool finite = high - high == 0.f && low - low == 0.f;
        float scale = finite ? (float)(elem)((0.5f * high - 0.5f * low) * (2.f / 15.f)) : 0.f;
        if (scale < SMALLEST_SCALE) scale = 0.f;
        const float offset = finite ? (float)(elem)q4_offset(low, scale) : high < low ? 0.f : NAN;  // (padding: no value)
        const float inverse = scale > 0.f ? 1.f / scale : 0.f;
        // 1.5 2^23 + 8 + steps, rounded to a whole number by that sum, has the code
        // in its low bits; what else these numbers hold adds up to a constant.
        unsigned word = 0, constant = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float steps = __builtin_amdgcn_fmed3f((x[e] - offset) * inverse, -8.f, 7.f);
            word += __builtin_bit_cast(unsigned, steps + 12582920.f) << (4 * e);
            constant += 0x4B400000u << (4 * e);
        }
        word = real && scale > 0.f ? word - constant : 0x88888888u;
        if (row[u] < 0) continue;
        static_cast<unsigned *>(p.codes[which])[row[u] * WORDS + (which == 0 ? key_word<WORDS>(word_of_row) : word_of_row)] = word;
        if (word_of_row % p.group_words == 0) {
            typedef elem pair_t __attribute__((ext_vector_type(2)));
            static_cast<pair_t *>(p.scales[which])[row[u] * (WORDS / p.group_words) + word_of_row / p.group_words] = pair_t{(elem)scale, (elem)offset};
        }
    }
}

template <class T, int WORDS, bool WIDE, int AT_ONCE>
__global__ void __launch_bounds__(256) q4_load_kernel(Q4StoreArgs p)
{
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    typedef elem pair_t __attribute__((ext_vector_type(2)));
    const int which = blockIdx.y;
    Place at[AT_ONCE];
    int64_t row[AT_ONCE];
    unsigned word[AT_ONCE];
    pair_t pair[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        at[u] = place_of<WORDS, AT_ONCE>(p, u);
        row[u] = row_of(p, at[u]);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        word[u] = 0;
        pair[u] = pair_t{};
        if (row[u] < 0) continue;
        word[u] = static_cast<const unsigned *>(p.codes[which])[row[u] * WORDS + (which == 0 ? key_word<WORDS>(at[u].word) : at[u].word)];
        pair[u] = static_cast<const pair_t *>(p.scales[which])[row[u] * (WORDS / p.group_words) + at[u].word / p.group_words];
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        if (!at[u].real || 8 * at[u].word >= p.dim) continue;
        vec8 v = {};
        const float scale = (float)pair[u][0], offset = (float)pair[u][1], nan = 0.f * scale + 0.f * offset;  // (0 of finite ones)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = __builtin_fmaf(scale, (float)(int)((word[u] >> (4 * e)) & 15) - 8.f, offset);
            v[e] = (elem)(__builtin_elementwise_minimum(__builtin_elementwise_maximum(x, -T::LARGEST), T::LARGEST) + nan);
        }
        uint16_t *dst = const_cast<uint16_t *>(p.src[which]) + at[u].token * p.src_token[which] + at[u].head * p.src_head[which] + 8 * at[u].word;
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

template <class T, int WORDS, bool WIDE, int AT_ONCE>
gba_status run_rows(Q4StoreArgs a, bool load, hipStream_t s)
{
    a.block_tokens = a.token_words < 256 * AT_ONCE ? 256 * AT_ONCE / a.token_words : 1;
    const int64_t groups = div_up(a.tokens, a.block_tokens);
    if (groups > (int64_t)UINT_MAX / 256) return GBA_EUNSUPPORTED;
    const dim3 grid((unsigned)groups, 2, (unsigned)div_up(a.token_words, 256 * AT_ONCE)), block(256);
    return load ? launch(q4_load_kernel<T, WORDS, WIDE, AT_ONCE>, grid, block, s, a) : launch(q4_store_kernel<T, WORDS, WIDE, AT_ONCE>, grid, block, s, a);
}

template <class T, int WORDS, bool WIDE>
gba_status run_rows(const Q4StoreArgs &a, bool load, hipStream_t s)
{
    return (int64_t)a.tokens * a.token_words >= MANY_WORDS ? run_rows<T, WORDS, WIDE, 2>(a, load, s) : run_rows<T, WORDS, WIDE, 1>(a, load, s);
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
    a.tokens = (int)tokens;
    a.token_words = (int)(c->heads * words);
    a.token_factor = (unsigned)(((uint64_t)1 << 32) / a.token_words + 1);
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
