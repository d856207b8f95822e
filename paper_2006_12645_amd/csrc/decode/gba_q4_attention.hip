// gba_q4_attention.hip -- attention over the paged cache in 4 bits: checks, the
// choice of a kernel and its launch.
#include "gba_q4_kernel.hpp"

namespace gba {
namespace {

// No request has more new tokens than there are rows.
int64_t most_new(const gba_q4_attention &d) { return min_of(d.max_new, d.tokens); }

bool nothing_to_do(const gba_q4_attention &d)
{
    return d.tokens == 0 || d.requests == 0 || d.q_heads == 0 || d.max_new == 0 || d.cache.dim == 0;
}

gba_status validate(const gba_q4_attention &d)
{
    const gba_q4_cache &c = d.cache;
    if (d.requests < 0 || d.width < 0 || d.tokens < 0 || d.max_new < 0 || d.q_heads < 0 || d.window < 0 || d.sinks < 0) return GBA_EINVAL;
    if (d.workspace != nullptr && !aligned_to(d.workspace, 256)) return GBA_EINVAL;
    if ((__builtin_bit_cast(uint32_t, d.scale * LOG2_E) & 0x7F800000u) == 0x7F800000u) return GBA_EINVAL;  // infinite or NaN
    const gba_status st = validate_q4_cache(c);
    if (st != GBA_OK) return st;
    if (d.requests > GBA_MAX_REQUESTS || d.width > INT_MAX || d.tokens > INT_MAX || d.q_heads > 65535 || d.requests * d.width > INT_MAX ||
        d.width * c.block_size > INT_MAX)
        return GBA_EUNSUPPORTED;
    if (d.mask != nullptr && d.max_new > 64) return GBA_EUNSUPPORTED;
    if (nothing_to_do(d)) return GBA_OK;
    if (c.heads == 0 || d.q_heads % c.heads != 0) return GBA_EINVAL;
    if (most_new(d) * (d.q_heads / c.heads) > INT_MAX - 255) return GBA_EUNSUPPORTED;  // rows of a request and head, in tiles of 16
    if (d.q == nullptr || d.out == nullptr || d.lens == nullptr || d.offsets == nullptr) return GBA_EINVAL;
    if (d.width > 0 && d.table == nullptr) return GBA_EINVAL;
    // (a stride of a dimension of one element is not used)
    const struct { int64_t extent, stride; int of; } strides[] = {
        {d.tokens, d.q_token, 8}, {d.q_heads, d.q_head, 8}, {d.tokens, d.out_token, 4}, {d.q_heads, d.out_head, 4}};
    for (const auto &s : strides)
        if (s.extent > 1 && s.stride % s.of != 0) return GBA_EUNSUPPORTED;
    if (!aligned_to(d.q, 16) || !aligned_to(d.out, 16) || !aligned_to(d.table, 4) || !aligned_to(d.lens, 4) || !aligned_to(d.offsets, 4) ||
        !aligned_to(d.mask, 8))
        return GBA_EUNSUPPORTED;
    return GBA_OK;
}

// What a workgroup does beside its keys, as keys: a window of 128 requests and 4
// heads (4236 keys, 512 pairs) is one run, 43 us; as three, 47.
constexpr int64_t FIXED_KEYS = 512;

// Workgroups that are counted as running at once when windows are cut: one a
// compute unit.  All kernels but those of dim 256 have room for two or more, so
// from 129 to 256 pairs of request and head this leaves half of it empty: 16
// requests of 8 heads in a window of 4096 are two runs each, 24 us, and 24 requests
// one, 36.5.
constexpr int64_t WINDOW_ROOM = 256;

struct Shape {
    int dp, groups, row_tiles, target, slots, length, each;
    size_t bytes;  // of the workspace: counters, then the sums
};

// Runs to aim at.  A compute unit has room for two workgroups or more, and each
// request and head adds half a run on average, its last one: few requests, all
// runs at once (four of up to 131071 keys, 32 pairs of request and head: 103 us
// with 512, 129 with 768, where some wait for others); more of them, two rounds,
// to even out (64 of up to 8192, 512 pairs: 38 us with 256, 34 with 512, 31 with
// 768).
int64_t runs_to_aim_at(int64_t pairs) { return pairs <= 128 ? 512 : pairs < 1024 ? 768 : 2048; }

Shape shape_of(const gba_q4_attention &d)
{
    const gba_q4_cache &c = d.cache;
    Shape s;
    s.dp = q4_width(c.dim);
    s.groups = s.dp > c.group ? s.dp / c.group : 1;
    const int64_t rows = most_new(d) * (d.q_heads / c.heads);
    s.row_tiles = (int)div_up(rows, Q4_ROWS);
    s.target = 0;
    s.slots = (int)d.requests;
    s.length = s.each = 0;
    s.bytes = 0;
    int64_t most_keys = d.width * c.block_size;  // of a request
    const int64_t bounded = min_of(d.window, INT_MAX) + min_of(d.sinks, INT_MAX);
    if (d.window != 0) most_keys = min_of(most_keys, bounded + most_new(d) + 2 * Q4_KEYS);  // (sinks and window in whole tiles)
    // Tiles of rows that fill the chip, or have few keys, are left whole, with the keys that their own rows see.
    const int64_t tokens = div_up(Q4_ROWS * c.heads, d.q_heads);
    const bool alone = s.row_tiles > 1 && (d.requests * c.heads * s.row_tiles >= 512 || (d.window != 0 && bounded + tokens <= 1024));
    if (d.requests > SPLIT_REQUESTS || most_keys <= SHORTEST || alone) return s;
    const int64_t tiles = c.heads * (int64_t)s.row_tiles, pairs = d.requests * tiles;
    int64_t slots = 0;
    const int64_t sums = Q4_ROWS * (c.dim + 2) * (int64_t)sizeof(float);
    if (d.window != 0) {
        const int64_t length = run_of_window(pairs, sums, most_keys, WINDOW_ROOM, FIXED_KEYS, Q4_KEYS * Q4_WAVES);
        const int64_t each = div_up(most_keys, length);
        if (each == 1) return s;
        s.length = (int)length;
        s.each = (int)each;
        slots = d.requests * each;
    } else {
        slots = d.requests + div_up(runs_to_aim_at(pairs), tiles);
        if (slots * tiles > (int64_t)COUNTERS) return s;  // (more than fill the chip as they are)
    }
    s.target = (int)div_up(runs_to_aim_at(pairs), tiles);
    s.slots = (int)slots;
    s.bytes = COUNTER_BYTES + (size_t)(slots * tiles * sums);
    return s;
}

template <class T, int DP, int G>
gba_status run_attention(const Q4Args &a, hipStream_t s)
{
    const int64_t groups = div_up((int64_t)a.slots * a.heads, 8) * 8 * a.row_tiles;
    if (groups > (int64_t)UINT_MAX / (64 * Q4_WAVES)) return GBA_EUNSUPPORTED;
    return launch(q4_attention_kernel<T, DP, G>, dim3((unsigned)groups), dim3(64 * Q4_WAVES), s, a);
}

template <class T>
gba_status run_attention(const Q4Args &a, const Shape &sh, hipStream_t s)
{
    switch (sh.dp + sh.groups) {
    case 64 + 1: return run_attention<T, 64, 1>(a, s);
    case 64 + 2: return run_attention<T, 64, 2>(a, s);
    case 128 + 1: return run_attention<T, 128, 1>(a, s);
    case 128 + 2: return run_attention<T, 128, 2>(a, s);
    case 128 + 4: return run_attention<T, 128, 4>(a, s);
    case 256 + 2: return run_attention<T, 256, 2>(a, s);
    case 256 + 4: return run_attention<T, 256, 4>(a, s);
    default: return run_attention<T, 256, 8>(a, s);
    }
}

}  // namespace
}  // namespace gba

using namespace gba;

extern "C" gba_status gba_q4_attend_workspace_size(const gba_q4_attention *desc, size_t *bytes)
{
    if (desc == nullptr || bytes == nullptr) return GBA_EINVAL;
    const gba_status st = validate(*desc);
    if (st == GBA_OK) *bytes = nothing_to_do(*desc) ? 0 : shape_of(*desc).bytes;
    return st;
}

extern "C" gba_status gba_q4_attend(const gba_q4_attention *desc, gba_stream_t stream)
{
    if (desc == nullptr) return GBA_EINVAL;
    const gba_q4_attention &d = *desc;
    const gba_q4_cache &c = d.cache;
    const gba_status st = validate(d);
    if (st != GBA_OK || nothing_to_do(d)) return st;
    Shape sh = shape_of(d);
    if (sh.target != 0 && (d.workspace == nullptr || d.workspace_bytes < sh.bytes)) {
        sh.target = 0;
        sh.slots = (int)d.requests;
    }
    Q4Args a = {};
    a.q = d.q;
    a.k = c.k_codes;
    a.v = c.v_codes;
    a.k_scales = c.k_scales;
    a.v_scales = c.v_scales;
    a.out = d.out;
    a.table = d.table;
    a.lens = d.lens;
    a.offsets = d.offsets;
    a.mask = d.mask;
    a.q_token = d.q_token;
    a.q_head = d.q_head;
    a.out_token = d.out_token;
    a.out_head = d.out_head;
    a.requests = (int)d.requests;
    a.width = c.num_blocks > 0 ? (int)d.width : 0;  // an empty cache: no keys
    a.tokens = (int)d.tokens;
    a.max_new = (int)most_new(d);
    a.q_heads = (int)d.q_heads;
    a.heads = (int)c.heads;
    a.share = (int)(d.q_heads / c.heads);
    a.num_blocks = (int)c.num_blocks;
    a.block_size = (int)c.block_size;
    a.dim = (int)c.dim;
    const float scale2 = d.scale * LOG2_E;
    a.sign = scale2 > 0.f ? 1.f : scale2 < 0.f ? -1.f : 0.f;
    a.scale2 = scale2 > 0.f ? scale2 : scale2 < 0.f ? -scale2 : 1.f;
    if (c.dtype == GBA_BF16) {  // what keys were divided by, or with a scale that has no room for it the queries
        if (a.scale2 < 0x1p119f) a.scale2 *= 1.f / KEYS_DOWN<BF16>;
        else a.sign *= 1.f / KEYS_DOWN<BF16>;
    }
    a.window = d.window != 0 ? d.window : INT64_MAX;
    a.sinks = d.window != 0 ? (int)min_of(d.sinks, INT_MAX) : 0;
    a.row_tiles = sh.row_tiles;
    a.slots = sh.slots;
    a.target = sh.target;
    a.length = sh.length;
    a.each = sh.each;
    if (sh.target != 0) {
        a.arrived = static_cast<int32_t *>(d.workspace);
        a.part = reinterpret_cast<float *>(static_cast<char *>(d.workspace) + COUNTER_BYTES);
    }
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return c.dtype == GBA_F16 ? run_attention<F16>(a, sh, s) : run_attention<BF16>(a, sh, s);
}
