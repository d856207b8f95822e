// gba_attention.hpp -- what the kernels of attention over a paged cache share:
// a request's keys, cut into runs of one length over all requests, and the
// joins of a request's runs in their order.
#pragma once

#include "gba_decode.hpp"
#include "gba_kernel.hpp"

namespace gba {
namespace {

struct AttentionArgs {
    const void *q, *k, *v;
    void *out;
    const int32_t *table, *lens, *offsets;
    const uint64_t *mask;
    int64_t k_block, k_token, k_head, v_block, v_token, v_head, q_token, q_head, out_token, out_head;
    int requests, width, tokens, max_new, q_heads, heads, share, num_blocks, block_size, dim;
    float scale2;      // |scale| * log2(e); its sign, or 0, goes to the queries
    float sign;
    int64_t window;    // (windows only) what a token sees of its text: the last ones
    int sinks;         // and the first
    int row_tiles;     // of a request and head
    int slots;         // runs of keys there is room for: at least as many as there are
    int target;        // runs to aim at (0: one for each request)
    int length, each;  // (windows only) if not 0: keys of a run, and how many of them are set aside for each request
    int32_t *arrived;    // [slots][heads][row_tiles], zeros: runs that have ended, at a request's first one; or null
    int32_t *first_run;  // [requests][2]: a request's first run and how many it has
    float *part;       // [slots][heads][row_tiles]: rows x dim sums, then as many maxima and sums of weights
};

constexpr int SHORTEST = 256;   // keys of a run, but a request's last

// A request's new tokens and keys, none for one with too many, or whose
// offsets fall or begin past the tokens.  With a window, keys are counted
// without the `gap` from position `split` on that none of the rows sees: key v
// is position v, or v + gap from split on.
struct Request {
    int first, fresh, kept, end;
    int split, gap;
};

template <bool WINDOW>
__device__ __forceinline__ unsigned position_of(const Request &q, unsigned key)
{
    return WINDOW && key >= (unsigned)q.split ? key + (unsigned)q.gap : key;
}

// Where the window begins of a token whose text is as long as `seen` positions
// after the cached ones make it.
__device__ __forceinline__ int begin_of(const AttentionArgs &p, int kept, int seen)
{
    const int64_t begin = (int64_t)kept + seen - p.window;
    return (int)(begin < 0 ? 0 : begin < INT_MAX ? begin : INT_MAX);
}

// Of new tokens `from` to `to`: every one sees the positions from `latest` on
// that are before `sure`.
struct Edges {
    int latest, sure;
};
__device__ __forceinline__ Edges edges_of(const AttentionArgs &p, const Request &q, int from, int to)
{
    if (p.mask != nullptr) return {begin_of(p, q.kept, q.fresh), q.kept};
    const int64_t past = (int64_t)q.kept + from + 1;
    return {begin_of(p, q.kept, to + 1), (int)(past < INT_MAX ? past : INT_MAX)};
}

// The keys of new tokens `from` to `to` of a request (of all of them with a
// mask: the shortest text is the cached one), sinks and window in whole tiles
// of TILE.
template <int TILE>
__device__ __forceinline__ void bound_keys(const AttentionArgs &p, int from, int to, Request &q)
{
    constexpr unsigned WHOLE = ~(unsigned)(TILE - 1);
    const int64_t past = (int64_t)q.kept + to + 1;
    if (p.mask == nullptr && past < q.end) q.end = (int)past;
    const int low = (int)((unsigned)min(begin_of(p, q.kept, p.mask == nullptr ? from + 1 : 0), q.end) & WHOLE);
    const unsigned sinks = ((unsigned)min(p.sinks, q.end) + (TILE - 1)) & WHOLE;
    q.split = (int)min(sinks, (unsigned)INT_MAX & WHOLE);
    q.gap = low > q.split ? low - q.split : 0;
    q.end -= q.gap;  // (low is not past it)
}

__device__ __forceinline__ Request request_of(const AttentionArgs &p, int r)
{
    Request q;
    q.first = p.offsets[r];
    const int end = min(p.offsets[r + 1], p.tokens);
    q.fresh = (int)((unsigned)end - (unsigned)q.first);
    if (q.first < 0 || end < q.first || q.fresh > p.max_new) q.fresh = 0;
    q.kept = max(p.lens[r], 0);
    q.end = (int)min((int64_t)q.kept + q.fresh, (int64_t)p.width * p.block_size);
    q.split = q.gap = 0;
    return q;
}

// Running sums over a wave, in the order of its lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int wave_sums(int x)
{
    x += moved<0x111, 0xF>(x);  // one lane up, within 16
    x += moved<0x112, 0xF>(x);
    x += moved<0x114, 0xF>(x);
    x += moved<0x118, 0xF>(x);
    x += moved<0x142, 0xA>(x);  // lanes 15 and 47 to the 16 after them
    x += moved<0x143, 0xC>(x);  // lane 31 to the 32 after it
    return x;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float x)
{
    return __builtin_bit_cast(float, moved<CTRL, ROWS>(__builtin_bit_cast(int, x)));
}
__device__ __forceinline__ float wave_total(float x)
{
    x += moved<0x111, 0xF>(x);
    x += moved<0x112, 0xF>(x);
    x += moved<0x114, 0xF>(x);
    x += moved<0x118, 0xF>(x);
    x += moved<0x142, 0xA>(x);
    x += moved<0x143, 0xC>(x);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Run number x: keys [from, to) of request r, one of the n runs that begin
// with number `first`; r = -1 where there is no such run.
struct Run {
    int r, n, first, from, to;
    Request q;
};

// Every run but a request's last is of one length, a multiple of `step`:
// the mean of all keys over p.target runs, so there are no more than
// p.target + p.requests; a mean next to 2^31 or above makes one run of each
// request.  The sum of the lengths is one in 24 bits; the
// factor covers its rounding.
//
// With a window, a run that is all of a request's is that of the row tile: its
// `rows` rows from row0 on alone say which keys it has.  Not BY_MEAN: runs, where
// there are any, are of p.length.
template <bool WINDOW, int TILE, bool BY_MEAN>
__device__ __forceinline__ Run run_of(const AttentionArgs &p, int x, int lane, int step, int row0, int rows)
{
    Run u;
    if (p.target == 0) {
        Request q = request_of(p, x);
        if constexpr (WINDOW) {
            const int last = (int)(min((int64_t)row0 + rows, (int64_t)q.fresh * p.share) - 1) / p.share;
            if (q.fresh > 0 && row0 < q.fresh * p.share) bound_keys<TILE>(p, row0 / p.share, last, q);
        }
        u.q = {uniform(q.first), uniform(q.fresh), uniform(q.kept), uniform(q.end), uniform(q.split), uniform(q.gap)};
        u.r = u.q.fresh > 0 ? x : -1;
        u.n = 1;
        u.first = x;
        u.from = 0;
        u.to = u.q.end;
        return u;
    }
    u.r = -1;
    if constexpr (WINDOW) {
        if (!BY_MEAN || p.length != 0) {
            const int r = x / p.each, i = x - r * p.each;
            Request q = request_of(p, r);
            if (q.fresh == 0) return u;
            bound_keys<TILE>(p, 0, q.fresh - 1, q);
            u.q = {uniform(q.first), uniform(q.fresh), uniform(q.kept), uniform(q.end), uniform(q.split), uniform(q.gap)};
            u.n = u.q.end > p.length ? (u.q.end - 1) / p.length + 1 : 1;
            if (i >= u.n) return u;
            u.r = r;
            u.first = x - i;
            u.from = i * p.length;
            u.to = u.q.end - u.from > p.length ? u.from + p.length : u.q.end;
            return u;
        }
    }
    if constexpr (BY_MEAN) {
        float keys = 0.f;
        Request q = {0, 0, 0, 0, 0, 0};
        auto look = [&](int r) {
            q = request_of(p, r);
            if constexpr (WINDOW) bound_keys<TILE>(p, 0, q.fresh - 1, q);
        };
        for (int r = lane; r < p.requests; r += 64) {
            look(r);
            if (q.fresh > 0) keys += (float)q.end;
        }
        const float mean = wave_total(keys) / (float)p.target * 1.00001f;
        int length = mean < (float)(INT_MAX / step * step - step) ? ((int)mean / step + 1) * step : INT_MAX;
        if (length < SHORTEST) length = SHORTEST;
        length = uniform(length);
        int before = 0;
        for (int base = 0; base < p.requests; base += 64) {
            const int r = base + lane;
            if (p.requests > 64 && r < p.requests) look(r);
            int n = 0;
            if (r < p.requests && q.fresh > 0) n = q.end > length ? (q.end - 1) / length + 1 : 1;
            const int upto = wave_sums(n);
            const uint64_t past = __ballot(before + upto > x);
            if (past != 0) {
                const int l = __ffsll((unsigned long long)past) - 1;
                u.r = base + l;
                u.n = __builtin_amdgcn_readlane(n, l);
                u.first = before + __builtin_amdgcn_readlane(upto, l) - u.n;
                u.from = (x - u.first) * length;
                u.q = {__builtin_amdgcn_readlane(q.first, l), __builtin_amdgcn_readlane(q.fresh, l), __builtin_amdgcn_readlane(q.kept, l),
                       __builtin_amdgcn_readlane(q.end, l), WINDOW ? __builtin_amdgcn_readlane(q.split, l) : 0,
                       WINDOW ? __builtin_amdgcn_readlane(q.gap, l) : 0};
                u.to = u.q.end - u.from > length ? u.from + length : u.q.end;
                return u;
            }
            before += __builtin_amdgcn_readlane(upto, 63);
        }
    }
    return u;
}

// The larger one, NaN if either is: one instruction, where fmaxf takes
// two more to make its operands quiet.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The largest of the four lanes that hold one row.
__device__ __forceinline__ float across_max(float x)
{
    x = larger(x, __shfl_xor(x, 32));
    return larger(x, __shfl_xor(x, 16));
}

// Which of 32 keys from new token `first` on (below 0: from the cached ones)
// a row sees, if they exist: the bits of its mask, or with no mask those up to
// its own token; all cached ones.
__device__ __forceinline__ unsigned seen_of(bool masked, uint64_t mask, int index, int first)
{
    if (first <= -32) return 0xFFFFFFFFu;
    if (!masked) {
        const int n = index - first + 1;
        return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1;
    }
    if (first < 0) return (unsigned)(mask << -first) | ((1u << -first) - 1);
    return first < 64 ? (unsigned)(mask >> first) : 0u;
}

// Two 16-bit floats: 0x8000 for each that is infinite or NaN (the exponent's top
// carries into the sign's place).
template <class T>
__device__ __forceinline__ unsigned not_finite(unsigned w)
{
    return ((w & T::INFINITE) + T::EXPONENT_ONE) & 0x80008000u;
}

// Bits of 32 positions: those from number n on (below 0: all of them).
__device__ __forceinline__ unsigned bits_from(int n) { return n <= 0 ? 0xFFFFFFFFu : n >= 32 ? 0u : 0xFFFFFFFFu << n; }

// The new tokens in a mask that are among the last `window` places of a text of
// `kept` cached tokens and these, or among its first `sinks`.
__device__ __forceinline__ uint64_t bounded_mask(const AttentionArgs &p, int kept, uint64_t mask)
{
    const int64_t firsts = (int64_t)p.sinks - kept;
    uint64_t out = mask;
    for (int i = 0, drop = p.window < 64 ? __popcll(mask) - (int)p.window : 0; i < drop; ++i) {
        const uint64_t lowest = mask & (0 - mask);
        mask ^= lowest;
        if (i >= firsts) out ^= lowest;
    }
    return out;
}

// Stores that write through to where every XCD sees them, and loads from there:
// a workgroup that has written its sums so need not write back its XCD's L2
// before another one reads them, which costs more than the sums.
__device__ __forceinline__ void to_other_xcds(float *to, float x) { __hip_atomic_store(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void to_other_xcds(float *to, f4 x)
{
    typedef uint64_t l2 __attribute__((ext_vector_type(2)));
    const l2 v = __builtin_bit_cast(l2, x);
    __hip_atomic_store(reinterpret_cast<uint64_t *>(to), v[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(reinterpret_cast<uint64_t *>(to) + 1, v[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <bool OTHERS>
__device__ __forceinline__ float load_one(const float *at)
{
    return OTHERS ? __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : *at;
}
template <bool OTHERS>
__device__ __forceinline__ f4 load_four(const float *at)
{
    if constexpr (!OTHERS) {
        return *reinterpret_cast<const f4 *>(at);
    } else {
        typedef uint64_t l2 __attribute__((ext_vector_type(2)));
        const uint64_t *p = reinterpret_cast<const uint64_t *>(at);
        return __builtin_bit_cast(f4, l2{__hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                                         __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)});
    }
}

// Until this wave's stores have arrived: those before this in the source, which the
// compiler moves past no assembly that may touch memory.
__device__ __forceinline__ void stores_arrive() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Four elements of a row of `n` runs, added in their order.  A run's maximum is
// -infinity where the row sees none of its keys, and where all of its scores
// are NaN: its sums, zeros or NaN, are added all the same.
template <class T, bool OTHERS>
__device__ __forceinline__ void join_runs(const float *sum_at, const float *top_at, const float *l_at, int64_t stride, int n, typename T::elem *to)
{
    typedef typename T::elem elem;
    typedef elem four_t __attribute__((ext_vector_type(4)));
    float m = -INFINITY, l = 0.f;
    f4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; i += 4) {
        f4 v[4];
        float t[4], w[4], next = m;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bool real = i + u < n;
            const int64_t at = (real ? i + u : i) * stride;
            const f4 sums = load_four<OTHERS>(sum_at + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = real ? sums[e] : 0.f;
            const float its_top = load_one<OTHERS>(top_at + at), its_l = load_one<OTHERS>(l_at + at);
            t[u] = real ? its_top : -INFINITY;
            w[u] = real ? its_l : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) next = larger(next, t[u]);
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next);
        l *= keep;
        o *= keep;
        m = next;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float share = t[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(t[u] - next);
            l += share * w[u];
            o += share * v[u];
        }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    four_t r4;
#pragma unroll
    for (int e = 0; e < 4; ++e) r4[e] = (elem)(o[e] * inv);
    *reinterpret_cast<four_t *>(to) = r4;
}

// A workgroup whose sums of one run, ROWS rows of `row_tile`, are written: the
// one that is the request's last joins them all.  Every wave's stores are done at
// the barrier.
//
// Not WRITTEN_THROUGH: one thread's release makes them visible to other XCDs
// before it counts the run, and who counts the last one acquires those of all
// others.
//
// WRITTEN_THROUGH, with to_other_xcds: the language orders nothing here, since the
// count is relaxed: a release would write back the XCD's L2.  What is relied upon is
// this hardware's: a store that writes through has arrived where every XCD reads it
// when the wave's vmcnt no longer counts it, each wave waits for that before the
// barrier, and so before the count; loads of agent scope are not served from an L2
// that may be out of date.  To the compiler the assembly before the count and after
// it is an order of memory.
template <class T, int DP, int ROWS, int THREADS, bool WRITTEN_THROUGH>
__device__ __forceinline__ void join_by_last(const AttentionArgs &p, const Run &run, const Request &rq, int head, int row_tile, int rows)
{
    __shared__ int last;
    if constexpr (WRITTEN_THROUGH) stores_arrive();
    else wait_vm_lgkm0<0>();
    __syncthreads();
    const int64_t place = ((int64_t)run.first * p.heads + head) * p.row_tiles + row_tile;
    if (threadIdx.x == 0) {
        last = __hip_atomic_fetch_add(p.arrived + place, 1, WRITTEN_THROUGH ? __ATOMIC_RELAXED : __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == run.n - 1;
        if (last) __hip_atomic_store(p.arrived + place, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last) return;
    if constexpr (WRITTEN_THROUGH) asm volatile("" ::: "memory");
    else __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    const int64_t stride = (int64_t)p.heads * p.row_tiles * ROWS * (p.dim + 2);
    const float *first_part = p.part + place * ROWS * (int64_t)(p.dim + 2);
    constexpr int FOURS = DP / 4;
    const int row0 = row_tile * ROWS;
    for (int j = threadIdx.x; j < ROWS * FOURS; j += THREADS) {
        const int row = j / FOURS, d = 4 * (j % FOURS);
        if (row0 + row >= rows || d >= p.dim) continue;
        const float *top_at = first_part + ROWS * p.dim + row;
        const int token = rq.first + (row0 + row) / p.share, h = head * p.share + (row0 + row) % p.share;
        join_runs<T, WRITTEN_THROUGH>(first_part + row * p.dim + d, top_at, top_at + ROWS, stride, run.n,
                                      static_cast<typename T::elem *>(p.out) + token * p.out_token + h * p.out_head + d);
    }
}

// A token's request and its runs: false where there is nothing to join.
__device__ __forceinline__ bool runs_of(const AttentionArgs &p, int t, int lane, int &x0, int &n, Request &rq)
{
    int r = 0;  // the number of requests that end at or before t
    for (int base = 0; base < p.requests; base += 64)
        r += __popcll(__ballot(base + lane < p.requests && p.offsets[base + lane + 1] <= t));
    if (r >= p.requests) return false;
    x0 = p.first_run[2 * r];
    n = p.first_run[2 * r + 1];
    rq = request_of(p, r);
    // (where offsets fall, the one that is found may not be the token's)
    return rq.fresh != 0 && t >= rq.first && t - rq.first < rq.fresh && n > 1;
}

// The runs of a request, added in their order: many rows, each of few runs; a
// workgroup a token, a thread four elements of a row.  Bound by reading the
// sums, which other XCDs wrote: 32768 rows of 128, most of two or three runs, 8.8 us
// (11.8 with a wave a row).
template <class T>
__global__ void __launch_bounds__(512) join_rows_kernel(AttentionArgs p, int tile_rows)
{
    const int t = blockIdx.x;
    int x0, n;
    Request rq;
    if (!runs_of(p, t, threadIdx.x & 63, x0, n, rq)) return;
    const int64_t tile_size = (int64_t)tile_rows * (p.dim + 2), stride = tile_size * p.heads * p.row_tiles;
    const int fours = p.dim / 4;
    for (int j = threadIdx.x; j < p.q_heads * fours; j += 512) {
        const int head = j / fours, d = 4 * (j - head * fours), kv = head / p.share;
        const int row = (t - rq.first) * p.share + head - kv * p.share, tile = row / tile_rows, in_tile = row - tile * tile_rows;
        const float *part = p.part + (((int64_t)x0 * p.heads + kv) * p.row_tiles + tile) * tile_size, *top_at = part + tile_rows * p.dim + in_tile;
        join_runs<T, false>(part + in_tile * p.dim + d, top_at, top_at + tile_rows, stride, n,
                     static_cast<typename T::elem *>(p.out) + t * p.out_token + head * p.out_head + d);
    }
}

// The same for few rows of many runs: one wave a token and query
// head, lane l four elements of every (256 / DP)-th run: its share of the
// weight comes from the lane that holds that run's maximum and sum.  Bound by
// latency: 2048 rows of up to 9 runs 4.8 us.
template <class T, int DP>
__global__ void __launch_bounds__(256) join_kernel(AttentionArgs p, int tile_rows)
{
    typedef typename T::elem elem;
    constexpr int FOURS = DP / 4, AT_ONCE = 64 / FOURS;
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6);
    const int t = (int)(id / p.q_heads), head = (int)(id - (int64_t)t * p.q_heads);
    if (t >= p.tokens) return;
    int x0, n;
    Request rq;
    if (!runs_of(p, t, lane, x0, n, rq)) return;
    const int row = (t - rq.first) * p.share + head % p.share, tile = row / tile_rows, in_tile = row % tile_rows;
    const int64_t tile_size = (int64_t)tile_rows * (p.dim + 2), stride = tile_size * p.heads * p.row_tiles;
    const float *part = p.part + (((int64_t)x0 * p.heads + head / p.share) * p.row_tiles + tile) * tile_size;
    const float *tops = part + tile_rows * p.dim + in_tile, *sums = tops + tile_rows;
    const int d = 4 * (lane % FOURS), which = lane / FOURS;
    const float *mine = part + (int64_t)in_tile * p.dim + (d < p.dim ? d : 0);
    float m = -INFINITY, l = 0.f;
    f4 o = {0.f, 0.f, 0.f, 0.f};
    for (int base = 0; base < n; base += 64) {
        const int here = n - base < 64 ? n - base : 64;
        const float top = lane < here ? tops[(base + lane) * stride] : -INFINITY;
        const float sum = lane < here ? sums[(base + lane) * stride] : 0.f;
        float next = top;
        for (int s = 32; s; s >>= 1) next = larger(next, __shfl_xor(next, s));
        next = larger(next, m);
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next);
        const float share = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - next);
        m = next;
        l = l * keep + share * sum;
        o *= keep;
        for (int i = 0; i < here; i += 4 * AT_ONCE) {
            f4 v[4];
            float f[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int from = i + u * AT_ONCE + which;
                const bool real = from < here;
                f[u] = __shfl(share, from & 63);
                const f4 sums = *reinterpret_cast<const f4 *>(mine + (base + (real ? from : 0)) * stride);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[u][e] = real ? sums[e] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) o += f[u] * v[u];
        }
    }
    for (int s = 32; s; s >>= 1) l += __shfl_xor(l, s);
    for (int s = 32; s >= FOURS; s >>= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], s);
    if (which != 0 || d >= p.dim) return;
    typedef elem four_t __attribute__((ext_vector_type(4)));
    const float inv = l > 0.f ? 1.f / l : 0.f;
    four_t r4;
#pragma unroll
    for (int e = 0; e < 4; ++e) r4[e] = (elem)(o[e] * inv);
    *reinterpret_cast<four_t *>(static_cast<elem *>(p.out) + t * p.out_token + head * p.out_head + d) = r4;
}

constexpr float LOG2_E = 1.44269504088896340736f;

// A workgroup's release writes back its XCD's L2: that costs less than the
// second kernel while there are few runs of 16 rows (one request of 1000 keys:
// 9.5 us against 10.8, two: 9.8 and 10.9), and more from about a hundred on (8
// trees of 8, 128 of them: 17.0 us against 14.7; 64 requests of up to 8192: 94
// and 81).
constexpr int FEW_RUNS = 64;

// The workspace begins with the counters, zeros whatever calls used it before.
constexpr size_t COUNTERS = 65536, COUNTER_BYTES = COUNTERS * sizeof(int32_t);

constexpr int SPLIT_REQUESTS = 1024;           // above that each request is one run

inline int64_t min_of(int64_t a, int64_t b) { return a < b ? a : b; }

// Runs of windows have sums of no more than this: a workspace is kept, and where
// there are as many runs as that, they gain little (1020 requests of 131072 keys, 32
// heads of 256: 666 ms, 665 with 1 GB of sums).
constexpr int64_t MOST_SUMS = (int64_t)512 << 20;

// Length of the runs, a multiple of `step`, that windows of `keys` keys at most
// are cut into, for `pairs` of a request's rows and a head, each run with `sums`
// bytes, where `room` workgroups run at once: what takes the fewest rounds of
// them, each as long as a run and, for what a workgroup does beside its keys,
// `fixed` keys more.
inline int64_t run_of_window(int64_t pairs, int64_t sums, int64_t keys, int64_t room, int64_t fixed, int64_t step)
{
    const int64_t most = min_of(min_of(256, div_up(keys, SHORTEST)), min_of((int64_t)COUNTERS / pairs, MOST_SUMS / (pairs * sums)));
    int64_t best = div_up(keys, step) * step, least = INT64_MAX;
    for (int64_t n = 1; n <= most; ++n) {
        const int64_t length = div_up(div_up(keys, n), step) * step;
        const int64_t cost = div_up(pairs * div_up(keys, length), room) * (length + fixed);
        if (cost < least) {
            least = cost;
            best = length;
        }
    }
    return best;
}

// A thread for four elements from this many rows on (16 trees of 64, 32768 rows:
// 54.7 us in all, 56.4 with a wave a row), a wave a row below (one request of
// 32000 keys, 32 rows of 32 runs: 34.7 against 42.2; 2048 rows: 81.3 and 82.5).
constexpr int JOIN_ROWS = 4096;

// Joins the runs of every request, where the last workgroup has not.
template <class T, int DP>
gba_status launch_joins(const AttentionArgs &a, int tile_rows, hipStream_t s)
{
    if (a.tokens * (int64_t)a.q_heads >= JOIN_ROWS) return launch(join_rows_kernel<T>, dim3((unsigned)a.tokens), dim3(512), s, a, tile_rows);
    return launch(join_kernel<T, DP>, dim3((unsigned)div_up((int64_t)a.tokens * a.q_heads, 4)), dim3(256), s, a, tile_rows);
}

}  // namespace
}  // namespace gba
