// gba_tree_attention.hip -- attention of each request's new tokens over a
// paged cache.
//
// One wave a token and query head: 64 keys at a time, a lane each, with the
// running maximum and sum of a softmax; then a lane for every 64th element of
// the output.
#include "gba_decode.hpp"

namespace gba {
namespace {

struct AttentionArgs {
    const void *q, *k, *v;
    void *out;
    const int32_t *table, *lens, *offsets;
    const uint64_t *mask;
    int64_t k_block, k_token, k_head, v_block, v_token, v_head, q_token, q_head, out_token, out_head;
    int requests, width, tokens, max_new, q_heads, share, num_blocks, block_size, dim;
    float scale;
};

template <class T>
__global__ void __launch_bounds__(64) attention_simple(AttentionArgs p)
{
    typedef typename T::elem elem;
    __shared__ float query[256], weight[64];
    __shared__ int64_t value_at[64];
    const int lane = threadIdx.x, t = blockIdx.x, head = blockIdx.y, key_head = head / p.share;
    const int r = owner_of(p.offsets, p.requests, t);
    if (r >= p.requests || t < p.offsets[r]) return;
    const int first = p.offsets[r], T_new = min(p.offsets[r + 1], p.tokens) - first;
    if (T_new > p.max_new) return;
    const int64_t kept = max(p.lens[r], 0), end = min(kept + T_new, (int64_t)p.width * p.block_size);
    const uint64_t mask = p.mask == nullptr ? 0 : p.mask[t];
    const elem *q = static_cast<const elem *>(p.q) + t * p.q_token + head * p.q_head;
    for (int d = lane; d < p.dim; d += 64) query[d] = (float)q[d];
    __syncthreads();
    float top = -INFINITY, total = 0.f, o[4] = {};
    for (int64_t base = 0; base < end; base += 64) {
        const int64_t pos = base + lane, draft = pos - kept;
        bool sees = pos < end && (draft < 0 || (p.mask == nullptr ? draft <= t - first : draft < 64 && ((mask >> draft) & 1)));
        int block = -1;
        if (sees) {
            block = p.table[(int64_t)r * p.width + pos / p.block_size];
            sees = block >= 0 && block < p.num_blocks;
        }
        float s = -INFINITY;
        if (sees) {
            const int64_t token = pos % p.block_size;
            const elem *k = static_cast<const elem *>(p.k) + block * p.k_block + token * p.k_token + key_head * p.k_head;
            s = 0.f;
            for (int d = 0; d < p.dim; ++d) s += query[d] * (float)k[d];
            s *= p.scale;
            value_at[lane] = block * p.v_block + token * p.v_token + key_head * p.v_head;
        }
        float m = s;
        for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
        m = fmaxf(m, top);
        if (m == -INFINITY) continue;
        const float keep = top == -INFINITY ? 0.f : __expf(top - m);
        const float w = sees ? (float)(elem)__expf(s - m) : 0.f;
        weight[lane] = sees ? w : -1.f;
        float sum = w;
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        total = total * keep + sum;
        top = m;
        __syncthreads();
        for (int i = 0; i < 4; ++i) o[i] *= keep;
        for (int j = 0; j < 64; ++j) {
            if (weight[j] < 0.f) continue;
            const elem *v = static_cast<const elem *>(p.v) + value_at[j];
            for (int i = 0; i < 4; ++i)
                if (lane + 64 * i < p.dim) o[i] += weight[j] * (float)v[lane + 64 * i];
        }
        __syncthreads();
    }
    elem *out = static_cast<elem *>(p.out) + t * p.out_token + head * p.out_head;
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < p.dim) out[lane + 64 * i] = (elem)(total > 0.f ? o[i] / total : 0.f);
}

gba_status validate(const gba_attention &d)
{
    const gba_paged_cache &c = d.cache;
    if (!is_dtype(c.dtype)) return GBA_EINVAL;
    if (c.num_blocks < 0 || c.block_size < 1 || c.heads < 0 || c.dim < 0 || d.requests < 0 || d.width < 0 || d.tokens < 0 ||
        d.max_new < 0 || d.q_heads < 0)
        return GBA_EINVAL;
    if (d.workspace != nullptr && !aligned_to(d.workspace, 256)) return GBA_EINVAL;
    if (d.requests > GBA_MAX_REQUESTS || d.width > INT_MAX || d.tokens > INT_MAX || c.num_blocks > INT_MAX ||
        c.block_size > INT_MAX || d.q_heads > 65535 || c.heads > 65535 || c.num_blocks * c.block_size > INT_MAX ||
        d.requests * d.width > INT_MAX || d.width * c.block_size > INT_MAX)
        return GBA_EUNSUPPORTED;
    if (d.mask != nullptr && d.max_new > 64) return GBA_EUNSUPPORTED;
    if (d.tokens == 0 || d.requests == 0 || d.q_heads == 0 || d.max_new == 0 || c.dim == 0) return GBA_OK;
    if (c.heads == 0 || d.q_heads % c.heads != 0) return GBA_EINVAL;
    if (c.dim % 8 != 0 || c.dim > 256) return GBA_EUNSUPPORTED;
    if (d.q == nullptr || d.out == nullptr || d.lens == nullptr || d.offsets == nullptr) return GBA_EINVAL;
    if (d.width > 0 && d.table == nullptr) return GBA_EINVAL;
    if (c.num_blocks > 0 && (c.k == nullptr || c.v == nullptr)) return GBA_EINVAL;
    const int64_t eights[] = {c.k_block, c.k_token, c.k_head, c.v_block, c.v_token, c.v_head, d.q_token, d.q_head};
    for (int64_t s : eights)
        if (s % 8 != 0) return GBA_EUNSUPPORTED;
    if (d.out_token % 4 != 0 || d.out_head % 4 != 0) return GBA_EUNSUPPORTED;
    if (!aligned_to(d.q, 16) || !aligned_to(d.out, 16) || !aligned_to(c.k, 16) || !aligned_to(c.v, 16) ||
        !aligned_to(d.table, 4) || !aligned_to(d.lens, 4) || !aligned_to(d.offsets, 4) || !aligned_to(d.mask, 8))
        return GBA_EUNSUPPORTED;
    return GBA_OK;
}

}  // namespace
}  // namespace gba

using namespace gba;

extern "C" gba_status gba_tree_attention_workspace_size(const gba_attention *desc, size_t *bytes)
{
    if (desc == nullptr || bytes == nullptr) return GBA_EINVAL;
    *bytes = 0;
    return validate(*desc);
}

extern "C" gba_status gba_tree_attention(const gba_attention *desc, gba_stream_t stream)
{
    if (desc == nullptr) return GBA_EINVAL;
    const gba_attention &d = *desc;
    const gba_paged_cache &c = d.cache;
    const gba_status st = validate(d);
    if (st != GBA_OK || d.tokens == 0 || d.requests == 0 || d.q_heads == 0 || d.max_new == 0 || c.dim == 0) return st;
    AttentionArgs a;
    a.q = d.q;
    a.k = c.k;
    a.v = c.v;
    a.out = d.out;
    a.table = d.table;
    a.lens = d.lens;
    a.offsets = d.offsets;
    a.mask = d.mask;
    a.k_block = c.k_block;
    a.k_token = c.k_token;
    a.k_head = c.k_head;
    a.v_block = c.v_block;
    a.v_token = c.v_token;
    a.v_head = c.v_head;
    a.q_token = d.q_token;
    a.q_head = d.q_head;
    a.out_token = d.out_token;
    a.out_head = d.out_head;
    a.requests = (int)d.requests;
    a.width = (int)d.width;
    a.tokens = (int)d.tokens;
    a.max_new = (int)d.max_new;
    a.q_heads = (int)d.q_heads;
    a.share = (int)(d.q_heads / c.heads);
    a.num_blocks = (int)c.num_blocks;
    a.block_size = (int)c.block_size;
    a.dim = (int)c.dim;
    a.scale = d.scale;
    const dim3 grid((unsigned)d.tokens, (unsigned)d.q_heads), block(64);
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return c.dtype == GBA_F16 ? launch(attention_simple<F16>, grid, block, s, a) : launch(attention_simple<BF16>, grid, block, s, a);
}
