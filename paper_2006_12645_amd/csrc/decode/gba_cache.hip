// gba_cache.hip -- new keys and values into the paged cache, by slot.
//
// A copy: every new row is read once and written once.  A thread moves 16
// bytes (one element where a stride or an address does not allow it);
// consecutive threads move consecutive pieces of a token's row.  Bound by HBM:
// 16384 tokens of 8 heads of 128, 134 MB, in 27.1 us (5.0 TB/s; a plain copy
// reaches 4.8 here); by the launch below some hundred tokens (8 tokens 2.8 us).
#include "gba_decode.hpp"

namespace gba {
namespace {

struct StoreArgs {
    const uint16_t *src[2];
    uint16_t *dst[2];
    int64_t src_token[2], src_head[2], dst_block[2], dst_token[2], dst_head[2];
    const int32_t *slots;
    int64_t pieces;       // of all tokens
    int per_row, per_head;  // pieces of a token's row, of a head
    int block_size;
    int64_t capacity;     // slots of the cache
};

template <class V>
__global__ void __launch_bounds__(256) store_kernel(StoreArgs p)
{
    constexpr int E = sizeof(V) / 2;
    const int which = blockIdx.y;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / p.per_row;
        const int piece = (int)(i - t * p.per_row), head = piece / p.per_head, d = (piece - head * p.per_head) * E;
        const int slot = p.slots[t];
        if (slot < 0 || slot >= p.capacity) continue;
        const int block = slot / p.block_size, token = slot - block * p.block_size;
        const uint16_t *src = p.src[which] + t * p.src_token[which] + head * p.src_head[which] + d;
        uint16_t *dst = p.dst[which] + block * p.dst_block[which] + token * p.dst_token[which] + head * p.dst_head[which] + d;
        *reinterpret_cast<V *>(dst) = *reinterpret_cast<const V *>(src);
    }
}

}  // namespace
}  // namespace gba

using namespace gba;

extern "C" gba_status gba_cache_store(const gba_paged_cache *c, int64_t tokens, const void *k, int64_t k_token, int64_t k_head,
                                      const void *v, int64_t v_token, int64_t v_head, const int32_t *slots,
                                      gba_stream_t stream)
{
    if (c == nullptr || !is_dtype(c->dtype)) return GBA_EINVAL;
    if (c->num_blocks < 0 || c->block_size < 1 || c->heads < 0 || c->dim < 0 || tokens < 0) return GBA_EINVAL;
    if (tokens > INT_MAX || c->num_blocks > INT_MAX || c->block_size > INT_MAX || c->heads > INT_MAX || c->dim > INT_MAX ||
        c->num_blocks * c->block_size > INT_MAX || c->heads * c->dim > INT_MAX)
        return GBA_EUNSUPPORTED;
    if (tokens == 0 || c->num_blocks == 0 || c->heads == 0 || c->dim == 0) return GBA_OK;
    if (k == nullptr || v == nullptr || slots == nullptr || c->k == nullptr || c->v == nullptr) return GBA_EINVAL;
    if (!aligned_to(k, 2) || !aligned_to(v, 2) || !aligned_to(c->k, 2) || !aligned_to(c->v, 2) || !aligned_to(slots, 4))
        return GBA_EUNSUPPORTED;
    StoreArgs a;
    const void *src[2] = {k, v};
    void *dst[2] = {c->k, c->v};
    const int64_t strides[2][5] = {{k_token, k_head, c->k_block, c->k_token, c->k_head},
                                   {v_token, v_head, c->v_block, c->v_token, c->v_head}};
    bool wide = c->dim % 8 == 0;
    for (int i = 0; i < 2; ++i) {
        a.src[i] = static_cast<const uint16_t *>(src[i]);
        a.dst[i] = static_cast<uint16_t *>(dst[i]);
        a.src_token[i] = strides[i][0];
        a.src_head[i] = strides[i][1];
        a.dst_block[i] = strides[i][2];
        a.dst_token[i] = strides[i][3];
        a.dst_head[i] = strides[i][4];
        wide = wide && aligned_to(src[i], 16) && aligned_to(dst[i], 16);
        for (int64_t s : strides[i]) wide = wide && s % 8 == 0;
    }
    const int e = wide ? 8 : 1;
    a.slots = slots;
    a.per_head = (int)(c->dim / e);
    a.per_row = (int)(c->heads * c->dim / e);
    a.pieces = tokens * a.per_row;
    a.block_size = (int)c->block_size;
    a.capacity = c->num_blocks * c->block_size;
    const int64_t groups = div_up(a.pieces, 256);
    const dim3 grid((unsigned)(groups < 16384 ? groups : 16384), 2), block(256);
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return wide ? launch(store_kernel<u4>, grid, block, s, a) : launch(store_kernel<uint16_t>, grid, block, s, a);
}
