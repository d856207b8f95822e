// gba_q4_kernel.hpp -- attention over the paged cache in 4 bits.
//
// A value is scale (code - 8) + offset, with a scale and an offset for a group
// of dim.  Codes become 16-bit floats 16 + code by a shift, a mask and an or, and
// nothing else of a value is rounded: with x the query and X its sum over a group
//     k.x = sum over groups of scale sum (16 + code) x + (offset - 24 scale) X
//     sum p v = sum (p scale) (16 + code) - 24 sum p scale + sum p offset
// the first sum of each is a matrix instruction's, the rest fp32.  Weights
// p scale enter it in bf16, which has the range that scales need, and for fp16
// results as two numbers, the second one what the first's rounding left.
//
// Tiles of 64 keys.  Key 16 g + 4 h + e of a tile is row 4 g + e of the h-th
// 16-key product, so that lane group g has the scores of keys 16 g .. 16 g + 15:
// those of one nibble-transposing LDS read, of which lane c gets element c of 16
// rows.  Their scales and offsets are in the lanes of the same row, a key each,
// and reach the others as row broadcasts.  K goes from the cache to registers as
// the products take it, V through a wave's own part of LDS.
#pragma once

#include <type_traits>

#include "gba_attention.hpp"
#include "gba_q4_cache.hpp"

namespace gba {
namespace {

constexpr int Q4_KEYS = 64;   // of a tile
constexpr int Q4_WAVES = 4;   // take the tiles of a run in turn
constexpr int Q4_ROWS = 16;   // of a workgroup

struct Q4Args : AttentionArgs {  // k, v: the codes
    const void *k_scales, *v_scales;
};

// Eight codes as 16 + code, in the order 0 4 1 5 2 6 3 7.  The two constants are
// in a vector and a scalar register, or the and and the or are not one
// instruction.
template <class T>
struct Unpack {
    unsigned mask = 0x000F000Fu << T::TOP, sixteen = T::SIXTEEN;

    __device__ __forceinline__ Unpack() { asm("" : "+v"(mask), "+s"(sixteen)); }
    __device__ __forceinline__ u4 operator()(unsigned x) const
    {
        u4 v;
        v[0] = ((x << T::TOP) & mask) | sixteen;
        v[1] = ((T::TOP >= 4 ? x << (T::TOP >= 4 ? T::TOP - 4 : 0) : x >> (T::TOP < 4 ? 4 - T::TOP : 0)) & mask) | sixteen;
        v[2] = ((x >> (8 - T::TOP)) & mask) | sixteen;
        v[3] = ((x >> (12 - T::TOP)) & mask) | sixteen;
        return v;
    }
};

typedef float f2 __attribute__((ext_vector_type(2)));

// Two bf16 numbers in a word, the first one in its low half.
__device__ __forceinline__ unsigned two_bf16(f2 x)
{
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector(x, b2));
}

// What lane J of the 16 lanes of a row holds.
template <int J>
__device__ __forceinline__ float from_lane(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x150 + J, 0xF, 0xF, true));
}

__device__ __forceinline__ int64_t shuffled(int64_t v, int lane)
{
    const unsigned lo = __shfl((unsigned)v, lane), hi = __shfl((unsigned)(v >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t from_lane_uniform(int64_t v, int lane)
{
    const unsigned lo = __builtin_amdgcn_readlane((unsigned)v, lane), hi = __builtin_amdgcn_readlane((unsigned)(v >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// From this on a scale or an offset is a large one, if there are such numbers.
// Below it no sum overflows: of less than 2^31 keys, weights of up to 2^8 and
// numbers of up to 31 scales, or of an offset, it is below 2^(31 + 8 + 5 + 80).  A row
// that sees a large one has weights that are 2^LOWER smaller, its sum of weights
// among them, and so room for any value of the type; scales times weights then lose
// bits below 2^-78, more than 150 powers of two below that value.
template <class T>
constexpr float LARGE = std::is_same_v<T, BF16> ? 0x1p80f : INFINITY;
constexpr float LOWER = 48.f;

// Keys are taken 2^-8 times in bf16, where 24 scales, and scores of (16 + code)
// scales, may have no place in fp32 otherwise; scores are multiplied by 2^8 again
// with the scale of the softmax.  Exact: what that leaves of the smallest
// numbers fp32 holds as they are.
template <class T>
constexpr float KEYS_DOWN = std::is_same_v<T, BF16> ? 0x1p-8f : 1.f;

// The query of a row that has an element of 2^65 or more is taken 2^-16 times in
// bf16, where a sum of (16 + code) of them may have no place in fp32 otherwise.
// (Not with a scale of the softmax that has no room for it: scores of such queries
// have none either.)
constexpr float QUERY_DOWN = 0x1p-16f, NO_ROOM = 0x1p100f;

// A value of the even rows of 16 lanes in both rows of their pair, and that of
// the odd ones; the same of the wave's halves.
struct Two {
    unsigned even, odd;
};
__device__ __forceinline__ Two rows_of_pairs(unsigned x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return {r[0], r[1]};
}
__device__ __forceinline__ Two halves(unsigned x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return {r[0], r[1]};
}
__device__ __forceinline__ float as_float(unsigned x) { return __builtin_bit_cast(float, x); }
__device__ __forceinline__ unsigned as_bits(float x) { return __builtin_bit_cast(unsigned, x); }

// The sum over the four lanes c, c + 16, ...
__device__ __forceinline__ float across_sum(float x)
{
    const Two t = rows_of_pairs(as_bits(x));
    x = as_float(t.even) + as_float(t.odd);
    const Two u = halves(as_bits(x));
    return as_float(u.even) + as_float(u.odd);
}

// What is computed from these comes after what is written before: left to
// itself the compiler makes every broadcast of a tile first, and runs out of
// registers.
__device__ __forceinline__ void in_order(float &a, float &b) { asm volatile("" : "+v"(a), "+v"(b)); }
__device__ __forceinline__ void in_order(f4 &a) { asm volatile("" : "+v"(a)); }

template <int N, class F>
__device__ __forceinline__ void each(F f)
{
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// Where there are a few times as many workgroups as the chip holds, and requests
// may have many keys, those of long requests go first, so that no long one is left
// for the end: 16 trees of 64 tokens over 500 to 4096 keys, 2048 workgroups, 103 us
// as they come and 83, of 36 tokens over 100 to 8000 keys 96 and 65; over 4000 keys
// each 179 and 181; 64 trees of 64 over 100 to 4000 keys, 8192 workgroups, 271 and 285.
// Below, the look at all lengths costs more: trees of 64 over 500 to 4096 keys, 768
// workgroups 44 and 47, 1024 of them 75 and 66; 16 trees over up to 512 keys 37.1 and
// 38.5, up to 1024 51.5 and 48.7, up to 2048 78 and 72.
constexpr int64_t Q4_SORTED_FROM = 1024, Q4_SORTED_TO = 4096, Q4_SORTED_KEYS = 2048;

// The x-th longest of up to 64 requests, in steps of 64 keys; of equal ones, the
// first first.
__device__ __forceinline__ int nth_longest(const Q4Args &p, int x, int lane)
{
    const int key = lane < p.requests ? (max(p.lens[lane], 0) & ~63) | (63 - lane) : -1;
    int before = 0;
#pragma unroll 1
    for (int r = 0; r < p.requests; r += 16)
#pragma unroll
        for (int i = 0; i < 16; ++i) before += __builtin_amdgcn_readlane(key, r + i) > key;
    return __builtin_ctzll(__ballot(lane < p.requests && before == x));
}

// DP: dim, padded.  G: groups of dim.  A workgroup has 16 rows of a request and
// key head, and its waves the tiles of a run in turn.
//
// Bound by HBM where tiles are many and groups few: four requests of 60000 to
// 131071 keys, 8 key heads of 128 in groups of 128, 506 MB, in 102 to 105 us (4.9
// TB/s).  Else by vector instructions, about 740 a tile of dim 128 in two groups,
// of which 224 unpack codes: 64 requests of up to 8192 keys, 79 MB, 32 us; 16 trees
// of 64 tokens, four heads a key head, 83 us.  Two blocks of 16 rows a wave would
// share what is unpacked, but leave one wave a SIMD: 124 us, where these took 103
// with requests as they come.  With rows and keys exchanged in the first product a
// lane has one key, and scales need no broadcasts, but weights go through LDS to the
// second: 33 us and, of 128 windows of 4096 keys for 16 rows, 51 in place of 43.
template <class T, int DP, int G>
__global__ void __launch_bounds__(64 * Q4_WAVES, DP <= 128 ? 2 : 1) q4_attention_kernel(Q4Args p)
{
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    typedef elem pair_t __attribute__((ext_vector_type(2)));
    constexpr int STEPS = DP / 32, BLOCKS = DP / 16, ROWS = Q4_ROWS, ROW = DP / 2, TILE = Q4_KEYS * ROW, LOADS = TILE / 1024;
    constexpr int SUMS = ROWS * 4 * DP;  // bytes of LDS of a wave: first a tile of V, then the sums of its rows
    static_assert(TILE <= SUMS, "a tile of V is no larger than the sums");
    // Weights as two bf16 numbers in fp16; one in bf16, whose results are rounded as
    // it is (38.5 us with two in place of 36 for 64 requests of up to 8192 keys).
    constexpr int TERMS = std::is_same_v<T, F16> ? 2 : 1;
    __shared__ __attribute__((aligned(128))) char smem[Q4_WAVES * SUMS];
    __shared__ float tops[Q4_WAVES][ROWS], sums[Q4_WAVES][ROWS];

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    // The row tiles of one run and head have ids 8 apart: the same XCD's L2.
    const int xcd = blockIdx.x & 7, rest = blockIdx.x >> 3;
    const int row_tile = rest % p.row_tiles, item = rest / p.row_tiles * 8 + xcd;
    const int head = item % p.heads;
    int x = item / p.heads;
    if (x >= p.slots) return;
    const int64_t workgroups = (int64_t)p.slots * p.heads * p.row_tiles;
    if (p.target == 0 && p.requests <= 64 && workgroups >= Q4_SORTED_FROM && workgroups <= Q4_SORTED_TO &&
        min((int64_t)p.width * p.block_size, p.window) >= Q4_SORTED_KEYS)
        x = nth_longest(p, x, lane);
    const int row0 = row_tile * ROWS;
    const Run run = run_of<true, Q4_KEYS, true>(p, x, lane, Q4_KEYS * Q4_WAVES, row0, ROWS);
    if (run.r < 0) return;
    const Request rq = run.q;
    const int rows = rq.fresh * p.share;
    if (row0 >= rows) return;

    // ---- tiles: 16 keys are in one block.  A lane looks up a quarter of one of
    // the next 16 tiles: the row of its first key in the cache (row 0 where there
    // is none: codes are finite whatever they are) and how many keys exist.
    char *mine = smem + wave * SUMS;
    const int tiles = (int)(((unsigned)(run.to - run.from) + Q4_KEYS - 1) / Q4_KEYS);
    const int count = tiles > wave ? (tiles - wave + Q4_WAVES - 1) / Q4_WAVES : 0;
    const int32_t *entries = p.table + (int64_t)run.r * p.width;
    auto key0 = [&](int n) -> unsigned { return (unsigned)run.from + Q4_KEYS * (unsigned)(wave + Q4_WAVES * n); };
    int64_t first_row = 0;
    unsigned keys = 0;
    int looked_up = 0;
    auto look_up = [&](int n) {
        const unsigned pos = key0(n + lane / 4) + 16 * (lane & 3);
        first_row = 0;
        keys = 0;
        if (pos < (unsigned)run.to) {
            const unsigned at = position_of<true>(rq, pos);
            const int page = (int)(at / (unsigned)p.block_size), within = (int)at - page * p.block_size, b = entries[page];
            if (b >= 0 && b < p.num_blocks) {
                first_row = ((int64_t)b * p.heads + head) * p.block_size + within;
                keys = min((unsigned)run.to - pos, 16u);
            }
        }
        looked_up = n;
    };
    typedef unsigned words_t __attribute__((ext_vector_type(STEPS < 4 ? STEPS : 4)));
    constexpr int PIECES = STEPS <= 4 ? 1 : STEPS / 4;
    words_t k_next[4][PIECES];
    u4 v_next[LOADS];
    pair_t ks_next[G], vs_next[G];
    unsigned there_next = 0;  // of keys 16 g .. 16 g + 15, those that exist
    const char *k_codes = static_cast<const char *>(p.k), *v_codes = static_cast<const char *>(p.v);
    auto fetch_k = [&](int n) {
        const char *k = k_codes + shuffled(first_row, 4 * (n - looked_up) + (c >> 2)) * ROW + (c & 3) * ROW + g * (ROW / 4);
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) k_next[h][i] = *reinterpret_cast<const words_t *>(k + 4 * h * ROW + 16 * i);
    };
    // V, and the scales and offsets of both.
    auto fetch = [&](int n) {
        if (n - looked_up == 16) look_up(n);
        const int at = 4 * (n - looked_up);
        const int64_t pairs = (shuffled(first_row, at + g) + c) * G;
        there_next = (1u << __shfl(keys, at + g)) - 1;
        typedef elem pairs_t __attribute__((ext_vector_type(2 * G)));
        const pairs_t ks = *reinterpret_cast<const pairs_t *>(static_cast<const pair_t *>(p.k_scales) + pairs);
        const pairs_t vs = *reinterpret_cast<const pairs_t *>(static_cast<const pair_t *>(p.v_scales) + pairs);
#pragma unroll
        for (int i = 0; i < G; ++i) {
            ks_next[i] = pair_t{ks[2 * i], ks[2 * i + 1]};
            vs_next[i] = pair_t{vs[2 * i], vs[2 * i + 1]};
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {  // 1 KB each: 2048 / DP sixteens of keys
            if constexpr (DP == 64) {
                const int64_t row = shuffled(first_row, at + 2 * i + (lane >> 5));
                v_next[i] = *reinterpret_cast<const u4 *>(v_codes + row * ROW + 16 * (lane & 31));
            } else {
                const int64_t row = from_lane_uniform(first_row, at + i * 128 / DP);
                v_next[i] = *reinterpret_cast<const u4 *>(v_codes + row * ROW + 1024 * (i % (DP / 128)) + 16 * lane);
            }
        }
    };
    if (count > 0) {
        look_up(0);
        fetch(0);
        fetch_k(0);
    }

    // ---- this wave's rows, row c: the second operand, dim 32 s + 8 g on in the
    // order of Unpack
    vec8 query[STEPS];
    float X[G];
    const int my_row = row0 + c;
    const bool real = my_row < rows;
    const int index = real ? my_row / p.share : 0, token = rq.first + index;  // its token among the new ones, among all
    const elem *q = static_cast<const elem *>(p.q) + token * p.q_token + (head * p.share + (real ? my_row % p.share : 0)) * p.q_head;
    float scale2 = p.scale2;
    unsigned large = 0;  // at the top of an element's exponent: two ones, which it has from 2^65 on
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int d = 32 * s + 8 * g;
        u4 y = {};
        if (real && d < p.dim) y = *reinterpret_cast<const u4 *>(q + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) large |= y[e] & (y[e] << 1);
        const vec8 values = __builtin_bit_cast(vec8, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) query[s][2 * (e % 4) + e / 4] = p.sign != 1.f ? (elem)((float)values[e] * p.sign) : values[e];
    }
    if constexpr (std::is_same_v<T, BF16>) {
        uint64_t row = __ballot((large & 0x40004000u) != 0 && p.scale2 < NO_ROOM);
        if (row != 0) {
            row |= row >> 32;
            row |= row >> 16;
            if (row >> c & 1) {
                scale2 *= 1.f / QUERY_DOWN;
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) query[s][e] = (elem)((float)query[s][e] * QUERY_DOWN);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < G; ++j) {
        f4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = j * (STEPS / G); s < (j + 1) * (STEPS / G); ++s) sum = T::mfma(vec8{1, 1, 1, 1, 1, 1, 1, 1}, query[s], sum);
        X[j] = sum[0] + (sum[0] - sum[0]);  // (NaN where the query is not finite)
    }
    const bool masked = p.mask != nullptr;
    uint64_t sees = masked ? p.mask[token] : 0;  // bits of the new tokens that the row sees
    if (masked && rq.fresh < 64) sees &= ((uint64_t)1 << rq.fresh) - 1;
    const int begin = begin_of(p, rq.kept, masked ? __popcll(sees) : index + 1);
    if (masked) sees = bounded_mask(p, rq.kept, sees);
    const Edges edges = edges_of(p, rq, row0 / p.share, (int)(min((int64_t)row0 + ROWS, (int64_t)rows) - 1) / p.share);

    f4 out[BLOCKS] = {}, scales[G] = {};  // sums of weights times scales times 16 + code, and of weights times scales
    // of the keys of this lane group: sums of weights and of weights times offsets
    float total = 0.f, offsets[G], top = -INFINITY, limit = -INFINITY, base2 = 0.f;
    unsigned lower = 0;  // bits of the rows that have seen a large value
#pragma unroll
    for (int j = 0; j < G; ++j) offsets[j] = 0.f;
    u4 ones_bits = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    asm("" : "+v"(ones_bits));  // four registers of them, or they are made anew each time
    const BF16::vec8 ones = __builtin_bit_cast(BF16::vec8, ones_bits);

    // 16-byte chunk of a row of V in LDS: chunk ^ swap, over the banks
    constexpr int CHUNKS = DP / 32;
    auto swap_of = [](int row) { return DP == 64 ? (row >> 2) & 1 : DP == 128 ? (row >> 1) & 3 : row & 7; };
    typedef int i2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) i2 lds_i2;
    const Unpack<T> unpack_k;
    const Unpack<BF16> unpack_v;
    // row 16 g + c of V in LDS: the blocks of dim are at this, but for the bits of their chunk
    const unsigned v_row = (unsigned)(uintptr_t)(lds_void *)mine + lane * ROW + 16 * swap_of(lane);

    for (int n = 0; n < count; ++n) {
        float ksc[G], kof[G], vsc[G], vof[G];  // scales and offsets of key `lane`; of K, offset - 24 scale
        float largest = 0.f;  // of V's (NaN if one is)
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const bool used = j * (DP / G) < p.dim;  // (what stands past dim is not)
            ksc[j] = used ? (float)ks_next[j][0] * KEYS_DOWN<T> : 0.f;
            const float of = used ? (float)ks_next[j][1] * KEYS_DOWN<T> : 0.f;
            kof[j] = __builtin_fmaf(-24.f, ksc[j], of);
            ksc[j] += 0.f * ksc[j] + 0.f * of;  // (NaN where one is not finite: a score of -infinity would be no key)
            vsc[j] = used ? (float)vs_next[j][0] : 0.f;
            vof[j] = used ? (float)vs_next[j][1] : 0.f;
            largest = larger(larger(largest, __builtin_fabsf(vsc[j])), __builtin_fabsf(vof[j]));
        }
        const unsigned there = there_next;
        lanes_meet();  // the last tile's V has been read
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int chunk = 64 * i + lane, row = chunk / CHUNKS;
            *reinterpret_cast<u4 *>(mine + row * ROW + 16 * ((chunk % CHUNKS) ^ swap_of(row))) = v_next[i];
        }
        if (n + 1 < count) fetch(n + 1);
        lanes_meet();

        // ---- scores: keys 16 g + 4 h + e, row c
        f4 score[4];
        each<4>([&](auto half) {
            constexpr int H = decltype(half)::value;
#pragma unroll
            for (int j = 0; j < G; ++j) in_order(ksc[j], kof[j]);
            f4 part[G];
#pragma unroll
            for (int j = 0; j < G; ++j) part[j] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const vec8 a = __builtin_bit_cast(vec8, unpack_k(k_next[H][s / 4][s % 4]));
                part[s / (STEPS / G)] = T::mfma(a, query[s], part[s / (STEPS / G)]);
            }
            each<4>([&](auto element) {
                constexpr int E = decltype(element)::value;
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    const float sc = from_lane<4 * H + E>(ksc[j]), of = from_lane<4 * H + E>(kof[j]);
                    const float scaled = j == 0 ? sc * part[j][E] : __builtin_fmaf(sc, part[j][E], score[H][E]);
                    score[H][E] = __builtin_fmaf(of, X[j], scaled);
                }
            });
            in_order(score[H]);
        });
        if (n + 1 < count) fetch_k(n + 1);
        // ---- which keys the row sees
        const int first = (int)position_of<true>(rq, key0(n));
        const bool edge = __ballot(there != 0xFFFFu) != 0 || first > edges.sure - Q4_KEYS ||
                          (first < edges.latest && (unsigned)first + (Q4_KEYS - 1) >= (unsigned)p.sinks);
        unsigned seen = 0xFFFFu;
        if (edge) {
            const int mine_first = first + 16 * g;
            seen = there & seen_of(masked, sees, index, mine_first - rq.kept) &
                   (bits_from(begin - mine_first) | ~bits_from(p.sinks - mine_first) | (masked ? bits_from(rq.kept - mine_first) : 0u));
#pragma unroll
            for (int e = 0; e < 16; ++e) {  // (as bits: a score that is left out may be NaN)
                const float is = score[e / 4][e % 4];
                const unsigned bits = (seen >> e) & 1 ? __builtin_bit_cast(unsigned, is) : 0xFF800000u;
                score[e / 4][e % 4] = __builtin_bit_cast(float, bits);
            }
        }
        // What a value stands for whose scale or offset is not finite is NaN, and
        // 0 times it has to be 0 where it is not seen: it is taken out, and the
        // offsets of the rows that see it are NaN.
        bool lowered = false;
        const uint64_t large_keys = __ballot(!(largest < LARGE<T>));
        if (large_keys != 0) {
#pragma unroll
            for (int j = 0; j < G; ++j) {
                const bool is = 0.f * vsc[j] + 0.f * vof[j] != 0.f;
                const unsigned which = (unsigned)(__ballot(is) >> (16 * g)) & 0xFFFFu;
                if (is) vsc[j] = vof[j] = 0.f;
                if (which & seen) offsets[j] = NAN;
            }
            if constexpr (LARGE<T> < INFINITY) {
                uint64_t row = __ballot(((unsigned)(large_keys >> (16 * g)) & seen) != 0);  // (seen: 16 bits)
                row |= row >> 32;
                row |= row >> 16;
                const unsigned now = (unsigned)row & 0xFFFFu;
                lowered = (now & ~lower) != 0;
                lower |= now;
            }
        }
        // ---- softmax: the maximum moves when a score passes it by 2^8
        float most = score[0][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) most = larger(most, score[e / 4][e % 4]);
        most *= scale2;
        if (__ballot(most > limit) != 0 || lowered) {
            const float now = larger(across_max(most), top);
            const float next = now == -INFINITY ? 0.f : LARGE<T> < INFINITY && (lower >> c & 1) ? now + LOWER : now;
            const float keep = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(base2 - next);
            top = now;
            limit = now + 8.f;
            base2 = next;
            total *= keep;
#pragma unroll
            for (int j = 0; j < G; ++j) {
                scales[j] *= keep;
                offsets[j] *= keep;
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) out[b] *= keep;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            score[e / 4][e % 4] = __builtin_amdgcn_exp2f(__builtin_fmaf(score[e / 4][e % 4], scale2, -base2));
            total += score[e / 4][e % 4];
        }
        // ---- weights of each group and its blocks of dim
        each<G>([&](auto group) {
            constexpr int J = decltype(group)::value;
            in_order(vsc[J], vof[J]);
            u4 weight[TERMS][2];
            each<8>([&](auto pair) {  // keys 8 half + e and 8 half + 4 + e, next to each other as Unpack has them
                constexpr int HALF = decltype(pair)::value / 4, E = decltype(pair)::value % 4;
                const float sc0 = from_lane<8 * HALF + E>(vsc[J]), of0 = from_lane<8 * HALF + E>(vof[J]);
                const float sc1 = from_lane<8 * HALF + 4 + E>(vsc[J]), of1 = from_lane<8 * HALF + 4 + E>(vof[J]);
                const float p0 = score[2 * HALF][E], p1 = score[2 * HALF + 1][E];
                const f2 w = {p0 * sc0, p1 * sc1};
                const unsigned high = two_bf16(w);
                offsets[J] = __builtin_fmaf(p1, of1, __builtin_fmaf(p0, of0, offsets[J]));
                weight[0][HALF][E] = high;
                if constexpr (TERMS == 2)
                    weight[1][HALF][E] = two_bf16(f2{w[0] - __builtin_bit_cast(float, high << 16), w[1] - __builtin_bit_cast(float, high & 0xFFFF0000u)});
            });
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
#pragma unroll
                for (int half = 0; half < 2; ++half) scales[J] = BF16::mfma(ones, __builtin_bit_cast(BF16::vec8, weight[t][half]), scales[J]);
#pragma unroll
            for (int b = J * (BLOCKS / G); b < (J + 1) * (BLOCKS / G); ++b) {
                const i2 words = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i2 *)(uintptr_t)(v_row ^ (16 * (b >> 1) + 8 * (b & 1))));
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const BF16::vec8 v = __builtin_bit_cast(BF16::vec8, unpack_v((unsigned)words[half]));
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) out[b] = BF16::mfma(v, __builtin_bit_cast(BF16::vec8, weight[t][half]), out[b]);
                }
            }
        });
    }

    // ---- this wave's sums, joined with the others' through LDS: row c, chunks of
    // four of dim, chunk j of a row at j ^ c
    lanes_meet();
    total = across_sum(total);
    if (g == 0) {
        tops[wave][c] = top == -INFINITY ? top : base2;  // (what the sums are relative to)
        sums[wave][c] = total;
    }
#pragma unroll
    for (int j = 0; j < G; ++j) {
        const float rest_of = across_sum(offsets[j]) - 24.f * scales[j][0];
#pragma unroll
        for (int b = j * (BLOCKS / G); b < (j + 1) * (BLOCKS / G); ++b)
            *reinterpret_cast<f4 *>(mine + c * (4 * DP) + 16 * ((4 * b + g) ^ c)) = out[b] + rest_of;
    }
    __syncthreads();
    const bool whole_request = run.n == 1;
    typedef elem four_t __attribute__((ext_vector_type(4)));
    float *part = whole_request ? nullptr : p.part + (((int64_t)x * p.heads + head) * p.row_tiles + row_tile) * ROWS * (int64_t)(p.dim + 2);
    constexpr int FOURS = DP / 4;
    for (int j = threadIdx.x; j < ROWS * FOURS; j += 64 * Q4_WAVES) {
        const int row = j / FOURS, four = j % FOURS, d = 4 * four;
        if (row0 + row >= rows || d >= p.dim) continue;
        float m = tops[0][row];
#pragma unroll
        for (int w = 1; w < Q4_WAVES; ++w) m = larger(m, tops[w][row]);
        f4 o = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < Q4_WAVES; ++w) {
            const float share = tops[w][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(tops[w][row] - m);
            l += share * sums[w][row];
            o += share * *reinterpret_cast<const f4 *>(smem + w * SUMS + row * (4 * DP) + 16 * (four ^ (row & 15)));
        }
        if (whole_request) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            const int token = rq.first + (row0 + row) / p.share, h = head * p.share + (row0 + row) % p.share;
            four_t r4;
#pragma unroll
            for (int e = 0; e < 4; ++e) r4[e] = (elem)(o[e] * inv);
            *reinterpret_cast<four_t *>(static_cast<elem *>(p.out) + token * p.out_token + h * p.out_head + d) = r4;
        } else {
            to_other_xcds(part + row * p.dim + d, o);
            if (four == 0) {
                to_other_xcds(part + ROWS * p.dim + row, m);
                to_other_xcds(part + ROWS * (p.dim + 1) + row, l);
            }
        }
    }
    if (!whole_request) join_by_last<T, DP, ROWS, 64 * Q4_WAVES, true>(p, run, rq, head, row_tile, rows);
}

}  // namespace
}  // namespace gba
