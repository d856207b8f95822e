// gba_tree_attention.hip -- attention of each request's new tokens over a
// paged cache.
//
// The query rows of a request that share a key head (its new tokens times the
// query heads a key head) are taken 16 RT at a time.  With K a tile of 32
// keys and Q the rows, one matrix instruction per 32 of dim gives 16 keys by
// 16 rows of S = K Q^T, so that a lane holds the scores of one row; with the
// keys of the two 16-key halves in the order in which those registers hold
// them, exp(S - m) is the operand of O = V^T P as it stands, with no exchange
// between lanes.  V^T comes from transposing LDS reads.
//
// One pass: every row has a running maximum m and sum l.  m follows the scores
// only when one passes it by more than SLACK (in the base-2 exponent), so that
// the accumulators are seldom scaled.  Weights are 2^(score - m + LIFT), in 16
// bits for the matrix instruction.  In bf16 (slack 8, lift 0) their relative
// rounding is the same at any size.  In fp16 they have to stay below 2^16 and
// lose bits below 2^-14: a slack of 4 and a lift of 11 use that range up, so
// that the keys after a dominant one keep 11 bits down to 2^-25 of its weight
// and none vanishes above 2^-36 (a slack of 8 and a lift of 7: 16 trees of 64
// 52 us, not 53, but 4 bits fewer; 1 and 14: 57.5).  l is one more matrix
// instruction, of ones and the rounded weights, and has the same factor 2^LIFT.
//
// Few rows read a whole cache: the bound is HBM.  A wave copies its tiles
// straight into its own part of LDS, two tiles ahead, and waits for nothing but
// its own copies; the waves of a workgroup take the tiles of a run of keys in
// turn and meet once, at its end.  Runs are cut to one length for all
// requests, from the sum of their lengths, which every wave reads for itself.
// The runs of one request are joined in their order, by a second kernel, or,
// where there are few of them, by the workgroup that ends last.
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
    int row_tiles;     // of a request and head
    int slots;         // runs of keys there is room for: at least as many as there are
    int target;        // runs to aim at (0: one for each request)
    int32_t *arrived;    // [slots][heads][row_tiles], zeros: runs that have ended, at a request's first one; or null
    int32_t *first_run;  // [requests][2]: a request's first run and how many it has
    float *part;       // [slots][heads][row_tiles]: rows x dim sums, then as many maxima and sums of weights
};

constexpr int KEYS = 32;        // of a tile
constexpr int SHORTEST = 256;   // keys of a run, but a request's last

// A request's new tokens and keys, none for one with too many, or whose
// offsets fall or begin past the tokens.
struct Request {
    int first, fresh, kept, end;
};

__device__ __forceinline__ Request request_of(const AttentionArgs &p, int r)
{
    Request q;
    q.first = p.offsets[r];
    const int end = min(p.offsets[r + 1], p.tokens);
    q.fresh = (int)((unsigned)end - (unsigned)q.first);
    if (q.first < 0 || end < q.first || q.fresh > p.max_new) q.fresh = 0;
    q.kept = max(p.lens[r], 0);
    q.end = (int)min((int64_t)q.kept + q.fresh, (int64_t)p.width * p.block_size);
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
__device__ __forceinline__ Run run_of(const AttentionArgs &p, int x, int lane, int step)
{
    Run u;
    if (p.target == 0) {
        const Request q = request_of(p, x);
        u.q = {uniform(q.first), uniform(q.fresh), uniform(q.kept), uniform(q.end)};
        u.r = u.q.fresh > 0 ? x : -1;
        u.n = 1;
        u.first = x;
        u.from = 0;
        u.to = u.q.end;
        return u;
    }
    float keys = 0.f;
    Request q = {0, 0, 0, 0};
    for (int r = lane; r < p.requests; r += 64) {
        q = request_of(p, r);
        if (q.fresh > 0) keys += (float)q.end;
    }
    const float mean = wave_total(keys) / (float)p.target * 1.00001f;
    int length = mean < (float)(INT_MAX / step * step - step) ? ((int)mean / step + 1) * step : INT_MAX;
    if (length < SHORTEST) length = SHORTEST;
    length = uniform(length);
    u.r = -1;
    int before = 0;
    for (int base = 0; base < p.requests; base += 64) {
        const int r = base + lane;
        if (p.requests > 64 && r < p.requests) q = request_of(p, r);
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
                   __builtin_amdgcn_readlane(q.end, l)};
            u.to = u.q.end - u.from > length ? u.from + length : u.q.end;
            return u;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return u;
}

// Chunk permutations of a tile's rows in LDS: 16-byte chunk c of key r stands
// at c ^ swap(r).  K is read 16 keys at one chunk, V eight keys at a pair of
// chunks a half wave: all banks each time.
template <int DP>
__device__ __forceinline__ int swap_k(int key)
{
    return DP == 64 ? (key >> 1) & 7 : key & 15;
}
template <int DP>
__device__ __forceinline__ int swap_v(int key)
{
    return DP == 64 ? ((key >> 1) & 3) << 1 : (key & 7) << 1;
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

// Reads of 16 bytes, OFF bytes past each address, in one block of assembly that
// waits for them: before a load from LDS of its own the compiler waits for
// every copy to LDS that is under way, the next tile's too.
template <int O0, int O1, int O2, int O3>
__device__ __forceinline__ void read_four(unsigned a0, unsigned a1, unsigned a2, unsigned a3, u4 (&v)[4])
{
    asm volatile(
        "ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%9\n\t"
        "ds_read_b128 %2, %6 offset:%10\n\tds_read_b128 %3, %7 offset:%11\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
        : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(O0), "n"(O1), "n"(O2), "n"(O3));
}

// Four blocks of 16 of dim, transposed: keys 4 j .. 4 j + 3 of the lane's group
// OFF bytes past each address, and those FURTHER bytes on.
template <int OFF, int FURTHER>
__device__ __forceinline__ void read_transposed(const unsigned *at, u4 (&v)[4])
{
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    u2 r[8];
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
        "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
        "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
        "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(OFF), "n"(OFF + FURTHER));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = u4{r[2 * i][0], r[2 * i][1], r[2 * i + 1][0], r[2 * i + 1][1]};
}

// Two 16-bit floats: 0x8000 for each that is infinite or NaN (the exponent's top
// carries into the sign's place).
template <class T>
__device__ __forceinline__ unsigned not_finite(unsigned w)
{
    return ((w & T::INFINITE) + T::EXPONENT_ONE) & 0x80008000u;
}

template <int N>
struct Const {
    static constexpr int value = N;
};

// A workgroup's waves: RG of them take 16 RT rows each of the same keys, and
// KG such groups the tiles of a run in turn.  A group keeps two stages of SUB
// tiles in LDS; its waves meet once a stage.
template <int DP, int RG>
struct Shared {
    static constexpr int KG = RG == 8 ? 1 : RG == 4 || DP == 256 ? 2 : 4, WAVES = RG * KG;
    static constexpr int SUB = RG == 8 ? 4 : RG == 4 ? 2 : 1;
    static constexpr int CPR = DP / 8;                   // 16-byte chunks of a row
    static constexpr int KPI = 64 / CPR;                 // keys that one 64-lane copy covers
    static constexpr int COPIES = KEYS / KPI;            // of a tile of K or V
    static constexpr int ROW = 2 * DP, TILE = KEYS * ROW, PAIR = 2 * TILE, GROUP = 2 * SUB * PAIR;
};

// The join of several key groups needs 16 RT rows of fp32 for each wave.
template <int DP, int RT, int RG>
constexpr int lds_bytes()
{
    typedef Shared<DP, RG> S;
    return S::KG == 1 || S::KG * S::GROUP > S::WAVES * 16 * RT * 4 * DP ? S::KG * S::GROUP : S::WAVES * 16 * RT * 4 * DP;
}
template <int DP, int RG>
constexpr int threads_of()
{
    return 64 * Shared<DP, RG>::WAVES;
}

// Four elements of a row of `n` runs, added in their order.  A run's maximum is
// -infinity where the row sees none of its keys, and where all of its scores
// are NaN: its sums, zeros or NaN, are added all the same.
template <class T>
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
            const f4 sums = *reinterpret_cast<const f4 *>(sum_at + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = real ? sums[e] : 0.f;
            t[u] = real ? top_at[at] : -INFINITY;
            w[u] = real ? l_at[at] : 0.f;
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

// DP: dim, padded.  RT: blocks of 16 rows of a wave.  WHOLE: 16 consecutive
// keys, from a multiple of 16 on, are in one block, and go straight to LDS;
// else (RG 1 only) they pass through registers, which hold the next tile.
//
// RG 1 is bound by HBM: 64 requests of 16 to 8192 keys, 8 key heads of 128, 349
// MB: 76 us (4.6 TB/s); two of 100000 to 131071, 16 of 64, 976 MB: 200 us
// (4.9 TB/s); one of 1000 keys, bound by the latency of lengths, table, tiles and
// join: 9.0 us.  RG 8 by a tile's instructions and LDS waits, about 2500 clocks
// of which 1088 are matrix instructions: 16 trees of 64 tokens over 500 to 4096
// keys, 8 key heads of 128 with four query heads each, 45 us (390 TFLOP/s).
template <class T, int DP, int RT, int RG, bool WHOLE>
__global__ void __launch_bounds__((threads_of<DP, RG>()), (RG == 1 ? 1 : 2)) attention_kernel(AttentionArgs p)
{
    typedef Shared<DP, RG> S;
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    static_assert(WHOLE || RG == 1, "waves share only what goes straight to LDS");
    constexpr int WAVES = S::WAVES, KG = S::KG, SUB = S::SUB, SLOTS = WHOLE ? 2 * SUB : 1;
    constexpr int CPR = S::CPR, KPI = S::KPI, COPIES = S::COPIES, ROW = S::ROW, TILE = S::TILE;
    constexpr int STEPS = DP / 32, BLOCKS = DP / 16, ROWS = 16 * RT * RG;
    __shared__ __attribute__((aligned(16))) char smem[lds_bytes<DP, RT, RG>()];
    __shared__ float tops[WAVES][16 * RT], sums[WAVES][16 * RT];
    __shared__ int odd_from[RG > 1 ? KG : WAVES];  // first key of the first tile whose V has been cleaned

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), rg = wave % RG, kg = wave / RG;
    const int c = lane & 15, g = lane >> 4;
    // The row tiles of one run and head have ids 8 apart: the same XCD's L2.
    const int xcd = blockIdx.x & 7, rest = blockIdx.x >> 3;
    const int row_tile = rest % p.row_tiles, item = rest / p.row_tiles * 8 + xcd;
    const int head = item % p.heads, x = item / p.heads;
    if (x >= p.slots) return;
    const Run run = run_of(p, x, lane, KEYS * KG);
    if (run.r < 0) return;
    const Request rq = run.q;
    const int rows = rq.fresh * p.share, row0 = row_tile * ROWS;
    if (p.target != 0 && p.arrived == nullptr && run.first == x && head == 0 && row_tile == 0 && threadIdx.x == 0) {
        p.first_run[2 * run.r] = x;
        p.first_run[2 * run.r + 1] = run.n;
    }
    if (row0 >= rows) return;

    // ---- copies of a tile: 1 KB each, lane l the chunk at byte 16 l
    char *mine = smem + kg * S::GROUP;
    const int tiles = (int)(((unsigned)(run.to - run.from) + KEYS - 1) / KEYS);
    const int count = tiles > kg ? (tiles - kg + KG - 1) / KG : 0;  // of this group
    const int rounds = (tiles + KG * SUB - 1) / (KG * SUB);           // stages of every group, where waves meet
    const int32_t *entries = p.table + (int64_t)run.r * p.width;
    // (unsigned: tiles past the run's end are looked up too, and a run may end just below 2^31)
    auto key0 = [&](int n) -> unsigned { return (unsigned)run.from + KEYS * (unsigned)(kg + KG * n); };
    const int in_copy = lane / CPR, place = lane % CPR;
    constexpr int PER_HALF = COPIES / 2;
    const char *k_head = reinterpret_cast<const char *>(static_cast<const elem *>(p.k) + head * p.k_head);
    const char *v_head = reinterpret_cast<const char *>(static_cast<const elem *>(p.v) + head * p.v_head);
    // Byte offset of this lane's chunk of copy i of a half, or beyond the
    // buffer; of K or of V.
    auto chunk_of = [&](int i, bool v) {
        const int key = KPI * i + in_copy, chunk = place ^ (v ? swap_v<DP>(key) : swap_k<DP>(key));
        return 8 * chunk < p.dim ? (int)(key * (v ? p.v_token : p.k_token) * 2) + 16 * chunk : OOB_OFFSET;
    };
    // A tile's copies: those of K, then of V.  With waves that share tiles, half
    // of them copy K and half V, MINE each: from copy MINE * (rg % (RG / 2)) on.
    constexpr int MINE = 2 * COPIES / RG;
    const bool copies_v = RG > 1 && rg >= RG / 2;
    const int first_copy = RG > 1 ? MINE * (rg % (RG / 2 > 0 ? RG / 2 : 1)) : 0;
    int k_off[WHOLE ? PER_HALF : 1], v_off[WHOLE && RG == 1 ? PER_HALF : 1];  // RG > 1: k_off is of what it copies
    if constexpr (WHOLE) {
#pragma unroll
        for (int i = 0; i < PER_HALF; ++i) {
            if (RG == 1) {
                k_off[i] = chunk_of(i, false);
                v_off[i] = chunk_of(i, true);
            } else {
                k_off[i] = chunk_of((first_copy + i) % PER_HALF, copies_v);
            }
        }
    }
    // WHOLE: a lane for each half of the next 32 tiles: where its first key is,
    // the length of a buffer that ends with its last one (there are zeros
    // beyond), and bits of the keys that exist: those up to the run's end, if
    // their block does.  Else: the block and token of key lane % 32 of the next
    // tile, and its registers.
    int64_t k_from = 0, v_from = 0;
    int k_bytes = 0, v_bytes = 0, entries_from = 0;
    unsigned bits = 0;
    int entry = -1, within = 0;
    u4 k_next[WHOLE ? 1 : COPIES], v_next[WHOLE ? 1 : COPIES];
    auto look_up = [&](int n) {
        const unsigned pos = WHOLE ? key0(n + lane / 2) + 16 * (lane & 1) : key0(n) + (lane & 31);
        entry = -1;
        if (pos < (unsigned)run.to) {
            const int page = (int)(pos / (unsigned)p.block_size);
            within = (int)pos - page * p.block_size;
            const int b = entries[page];
            entry = b >= 0 && b < p.num_blocks ? b : -1;
        }
        if constexpr (WHOLE) {
            const int left = run.to - (int)pos, keys = entry < 0 ? 0 : left < 16 ? left : 16;
            bits = (1u << keys) - 1;
            k_from = keys ? 2 * (entry * p.k_block + within * p.k_token) : 0;
            v_from = keys ? 2 * (entry * p.v_block + within * p.v_token) : 0;
            k_bytes = keys ? (int)((keys - 1) * p.k_token + p.dim) * 2 : 0;
            v_bytes = keys ? (int)((keys - 1) * p.v_token + p.dim) * 2 : 0;
            entries_from = n;
        }
    };
    auto buffer_of = [&](const char *head_of, int64_t from, int bytes, int at, bool real) {
        const unsigned lo = __builtin_amdgcn_readlane((unsigned)from, at), hi = __builtin_amdgcn_readlane((unsigned)(from >> 32), at);
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(head_of + (int64_t)((uint64_t)hi << 32 | lo)), (short)0,
                                                 real ? __builtin_amdgcn_readlane(bytes, at) : 0, RSRC_WORD3);
    };
    // Copies K (part 0) or V (part 1) of tile n, or with waves that share tiles
    // the wave's share of both.  None are left out past the last tile, so that
    // the number under way is always the same.
    auto copy = [&](int n, int part) {
        char *k_lds = mine + n % SLOTS * S::PAIR, *v_lds = k_lds + TILE;
        const int at = 2 * (n - entries_from);
        const bool real = n < count;
        if constexpr (RG == 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const __amdgpu_buffer_rsrc_t rs = part ? buffer_of(v_head, v_from, v_bytes, at + h, real) : buffer_of(k_head, k_from, k_bytes, at + h, real);
#pragma unroll
                for (int i = 0; i < PER_HALF; ++i)
                    buffer_load16_lds(rs, (part ? v_lds : k_lds) + 1024 * (PER_HALF * h + i), part ? v_off[i] : k_off[i], 0);
            }
        } else {
            char *to = (copies_v ? v_lds : k_lds) + 1024 * first_copy;
            const char *head_of = copies_v ? v_head : k_head;
            const int64_t from = copies_v ? v_from : k_from;
            const int bytes = copies_v ? v_bytes : k_bytes;
            constexpr int HALVES = MINE > PER_HALF ? 2 : 1, EACH = MINE / HALVES;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const __amdgpu_buffer_rsrc_t rs = buffer_of(head_of, from, bytes, at + h + first_copy / PER_HALF, real);
#pragma unroll
                for (int i = 0; i < EACH; ++i) buffer_load16_lds(rs, to + 1024 * (EACH * h + i), k_off[i], 0);
            }
        }
    };
    // Which keys of tile n exist (WHOLE).
    auto keys_of = [&](int n) -> unsigned {
        const int at = 2 * (n - entries_from);
        return n < count ? __builtin_amdgcn_readlane(bits, at) | __builtin_amdgcn_readlane(bits, at + 1) << 16 : 0u;
    };
    // Else: tile n's keys and values into registers, and which of them exist.
    auto fetch = [&](int n) -> unsigned {
        const unsigned there = (unsigned)__ballot(entry >= 0);
        const int block = entry, token = within;
        if (n + 1 < count) look_up(n + 1);
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int key = KPI * i + in_copy, kc = place ^ swap_k<DP>(key), vc = place ^ swap_v<DP>(key);
            const int64_t b = __shfl(block, key), t = __shfl(token, key);
            const u4 none = {0, 0, 0, 0};
            k_next[i] = v_next[i] = none;
            if (b >= 0 && 8 * kc < p.dim) k_next[i] = *reinterpret_cast<const u4 *>(k_head + 2 * (b * p.k_block + t * p.k_token) + 16 * kc);
            if (b >= 0 && 8 * vc < p.dim) v_next[i] = *reinterpret_cast<const u4 *>(v_head + 2 * (b * p.v_block + t * p.v_token) + 16 * vc);
        }
        return there;
    };
    if (rounds > 0) look_up(0);
    if (lane == 0 && (RG == 1 || rg == 0)) odd_from[RG > 1 ? kg : wave] = INT_MAX;  // (before the first meeting)

    // ---- this wave's rows: as the second operand, row c of each block; dim
    // 32 s + 8 g on
    vec8 query[RT][STEPS];
    uint64_t sees[RT];  // bits of the new tokens that the row sees
    int index[RT];      // its token among the new ones
    const int wave_row0 = row0 + rg * 16 * RT;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int row = wave_row0 + 16 * i + c;
        const bool real = row < rows;
        index[i] = real ? row / p.share : 0;
        const int token = rq.first + index[i];
        const elem *q = static_cast<const elem *>(p.q) + token * p.q_token + (head * p.share + (real ? row % p.share : 0)) * p.q_head;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int d = 32 * s + 8 * g;
            const u4 none = {0, 0, 0, 0};
            query[i][s] = real && d < p.dim ? *reinterpret_cast<const vec8 *>(q + d) : __builtin_bit_cast(vec8, none);
            if (p.sign != 1.f)
#pragma unroll
                for (int e = 0; e < 8; ++e) query[i][s][e] = (elem)((float)query[i][s][e] * p.sign);
        }
        sees[i] = p.mask != nullptr ? p.mask[token] : 0;
    }
    const bool masked = p.mask != nullptr;

    f4 out[RT][BLOCKS] = {}, weights[RT] = {};
    // running maximum; what a score may be before it moves; what is subtracted
    // (0 while there is no maximum)
    float top[RT], limit[RT], base2[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        top[i] = limit[i] = -INFINITY;
        base2[i] = 0.f;
    }

    // ---- LDS addresses of the fragments
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_void *)mine;
    unsigned k_at[STEPS], v_at[BLOCKS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) k_at[s] = lds0 + c * ROW + 16 * ((4 * s + g) ^ swap_k<DP>(c));
    const int v_key = 4 * g + (c >> 2), v_swap = 16 * swap_v<DP>(v_key);
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) v_at[b] = lds0 + TILE + v_key * ROW + 16 * ((c & 3) >> 1) + 8 * (c & 1) + ((32 * b) ^ v_swap);
    u4 ones_bits = __builtin_bit_cast(u4, vec8{(elem)1.f, (elem)1.f, (elem)1.f, (elem)1.f, (elem)1.f, (elem)1.f, (elem)1.f, (elem)1.f});
    asm("" : "+v"(ones_bits));  // four registers of them, or they are made anew each time
    const vec8 ones = __builtin_bit_cast(vec8, ones_bits);

    f4 score[RT][2];
    vec8 weight[RT];
    // Scores of the tile OFF bytes past the addresses plus `slot`: keys 16 h +
    // 4 g + e, row c of each block.
    auto multiply_k = [&](auto off, unsigned slot) {
        constexpr int OFF = decltype(off)::value;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < RT; ++i) score[i][h] = f4{0.f, 0.f, 0.f, 0.f};
        auto four = [&](auto first) {
            constexpr int Q = decltype(first)::value, HALF = 16 * ROW;
            constexpr int S0 = Q % STEPS, S1 = (Q + 1) % STEPS, S2 = (Q + 2) % STEPS, S3 = (Q + 3) % STEPS;
            u4 k[4];
            read_four<OFF + Q / STEPS * HALF, OFF + (Q + 1) / STEPS * HALF, OFF + (Q + 2) / STEPS * HALF, OFF + (Q + 3) / STEPS * HALF>(
                k_at[S0] + slot, k_at[S1] + slot, k_at[S2] + slot, k_at[S3] + slot, k);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < RT; ++i)
                    score[i][(Q + e) / STEPS] = T::mfma(__builtin_bit_cast(vec8, k[e]), query[i][(Q + e) % STEPS], score[i][(Q + e) / STEPS]);
        };
        four(Const<0>{});
        if constexpr (2 * STEPS > 4) four(Const<4>{});
        if constexpr (2 * STEPS > 8) {
            four(Const<8>{});
            four(Const<12>{});
        }
    };
    // The weights of tile n, of which the keys in `there` exist; whether a row
    // does not see one of those.
    auto soften = [&](int n, unsigned there) -> bool {
        bool unseen = false;
        const int first_draft = (int)key0(n) - rq.kept;  // of the new tokens, or below 0
        if (there != 0xFFFFFFFFu || first_draft + KEYS > 0) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const unsigned all = there & seen_of(masked, sees[i], index[i], first_draft), seen = all >> (4 * g);
                unseen |= all != there;
#pragma unroll
                for (int e = 0; e < 8; ++e) {  // (as bits: a score that is left out may be NaN)
                    const float is = score[i][e >> 2][e & 3];
                    const unsigned bits = (seen >> (16 * (e >> 2) + (e & 3))) & 1 ? __builtin_bit_cast(unsigned, is) : 0xFF800000u;
                    score[i][e >> 2][e & 3] = __builtin_bit_cast(float, bits);
                }
            }
        }
        float most[RT];
        bool past = false;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            most[i] = score[i][0][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) most[i] = larger(most[i], score[i][e >> 2][e & 3]);
            most[i] *= p.scale2;
            past |= most[i] > limit[i];
        }
        if (__ballot(past)) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const float now = larger(across_max(most[i]), top[i]);
                const float next = now == -INFINITY ? 0.f : now - T::LIFT;
                const float keep = top[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(base2[i] - next);
                top[i] = now;
                limit[i] = now + T::SLACK;
                base2[i] = next;
                weights[i] *= keep;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) out[i][b] *= keep;
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                weight[i][e] = (elem)__builtin_amdgcn_exp2f(__builtin_fmaf(score[i][e >> 2][e & 3], p.scale2, -base2[i]));
            weights[i] = T::mfma(ones, weight[i], weights[i]);
        }
        return __ballot(unseen) != 0;
    };
    auto multiply_v = [&](auto off, unsigned slot) {
#pragma unroll
        for (int b = 0; b < BLOCKS; b += 4) {
            u4 v[4];
            const unsigned at[4] = {v_at[b] + slot, v_at[b + 1] + slot, v_at[b + 2] + slot, v_at[b + 3] + slot};
            read_transposed<decltype(off)::value, 16 * ROW>(at, v);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < RT; ++i) out[i][b + j] = T::mfma(__builtin_bit_cast(vec8, v[j]), weight[i], out[i][b + j]);
        }
    };
    // Where a row does not see a key that is there, 0 times what V holds has to
    // be 0, whatever that is: what is not finite is taken out of such a tile in
    // LDS, and added at the end to the rows that see it.  The `copies` of
    // tiles from n on from number `first` on.  Waves that share tiles share this, in
    // every stage with new tokens.
    auto clean = [&](int n, unsigned slot, int first, int copies) {
        for (int i = first; i < first + copies; ++i) {
            u4 *v = reinterpret_cast<u4 *>(mine + slot + i / COPIES * S::PAIR + TILE + 1024 * (i % COPIES) + 16 * lane);
            u4 x = *v;
            unsigned odd = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned bits = not_finite<T>(x[e]);
                odd |= bits;
                x[e] &= ~((bits << 1) - (bits >> 15));
            }
            if (odd != 0) {
                *v = x;
                atomicMin(&odd_from[RG > 1 ? kg : wave], (int)key0(n + i / COPIES));
            }
        }
        lanes_meet();
    };

    if constexpr (WHOLE && RG == 1) {
        // K and V are two tiles ahead each: K's slot is free as soon as the
        // scores are there, V's when the tile is done.
        wait_vm_lgkm0<0>();  // the rows and blocks: from here on only copies are under way
        unsigned now = 0, next = 0;
        if (count > 0) {
            now = keys_of(0);
            next = keys_of(1);
            copy(0, 0);
            copy(0, 1);
            copy(1, 0);
            copy(1, 1);
        }
        for (int n = 0; n < count; ++n) {
            const unsigned slot = (n & 1) * S::PAIR;
            wait_vm_lgkm0<3 * COPIES>();
            lanes_meet();
            multiply_k(Const<0>{}, slot);
            if (n + 2 - entries_from == 32) look_up(n + 2);
            const unsigned after = keys_of(n + 2);
            copy(n + 2, 0);
            const bool unseen = soften(n, now);
            wait_vm_lgkm0<3 * COPIES>();
            lanes_meet();
            if (unseen) clean(n, slot, 0, COPIES);
            multiply_v(Const<0>{}, slot);
            copy(n + 2, 1);
            now = next;
            next = after;
        }
    } else if constexpr (WHOLE) {
        wait_vm_lgkm0<0>();
        unsigned ahead[SUB];
        auto stage = [&](int first) {
            if (first - entries_from == 32) look_up(first);
#pragma unroll
            for (int j = 0; j < SUB; ++j) {
                ahead[j] = keys_of(first + j);
                copy(first + j, 0);
            }
        };
        if (rounds > 0) stage(0);
        for (int round = 0; round < rounds; ++round) {
            unsigned now[SUB];
#pragma unroll
            for (int j = 0; j < SUB; ++j) now[j] = ahead[j];
            wait_vm_lgkm0<0>();
            __builtin_amdgcn_s_barrier();  // every wave's share is there, and the other stage has been read
            const unsigned slot = (round & 1) * (SUB * S::PAIR);
            if (run.from + (int64_t)(KEYS * KG * SUB) * (round + 1) > rq.kept) {
                clean(round * SUB, slot, SUB * COPIES / RG * rg, SUB * COPIES / RG);
                wait_vm_lgkm0<0>();
                __builtin_amdgcn_s_barrier();
            }
            stage((round + 1) * SUB);
            lanes_meet();
            auto tile = [&](auto j) {
                constexpr int J = decltype(j)::value;
                if (now[J] != 0) {
                    multiply_k(Const<J * S::PAIR>{}, slot);
                    soften(round * SUB + J, now[J]);
                    multiply_v(Const<J * S::PAIR>{}, slot);
                }
            };
            tile(Const<0>{});
            if constexpr (SUB > 1) tile(Const<1>{});
            if constexpr (SUB > 2) {
                tile(Const<2>{});
                tile(Const<3>{});
            }
        }
    } else {
        unsigned next = count > 0 ? fetch(0) : 0;
        for (int n = 0; n < count; ++n) {
            const unsigned now = next;
            lanes_meet();  // the last tile's fragments have been read
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                *reinterpret_cast<u4 *>(mine + 1024 * i + 16 * lane) = k_next[i];
                *reinterpret_cast<u4 *>(mine + TILE + 1024 * i + 16 * lane) = v_next[i];
            }
            if (n + 1 < count) next = fetch(n + 1);
            lanes_meet();
            multiply_k(Const<0>{}, 0);
            const bool unseen = soften(n, now);
            if (unseen) clean(n, 0, 0, COPIES);
            multiply_v(Const<0>{}, 0);
        }
    }

    wait_vm_lgkm0<0>();
    if (RG > 1) __syncthreads();  // no copies are under way, and the tiles have been read

    // What has been taken out of V from key `from` on, for elements d .. d + 3
    // of a row.
    auto odd_at = [&](int from, int row, int d) {
        f4 o = {0.f, 0.f, 0.f, 0.f};
        const int own = row / p.share;
        const uint64_t bits = masked ? p.mask[rq.first + own] : 0;
        for (int pos = from; pos < run.to; ++pos) {
            const int page = pos / p.block_size, block = entries[page], draft = pos - rq.kept;
            if (block < 0 || block >= p.num_blocks || (draft >= 0 && !(masked ? draft < 64 && (bits >> draft & 1) : draft <= own))) continue;
            const uint16_t *v = reinterpret_cast<const uint16_t *>(v_head) + block * p.v_block + (pos - page * p.block_size) * p.v_token + d;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (not_finite<T>(v[e]) != 0) o[e] += (float)__builtin_bit_cast(elem, v[e]);
        }
        return o;
    };

    const bool whole_request = run.n == 1;
    typedef elem four_t __attribute__((ext_vector_type(4)));
    float *part = whole_request ? nullptr : p.part + (((int64_t)x * p.heads + head) * p.row_tiles + row_tile) * ROWS * (int64_t)(p.dim + 2);
    if constexpr (KG == 1) {  // one key group: the sums are these
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int row = wave_row0 + 16 * i + c;
            if (row >= rows) continue;
            const float l = weights[i][0], inv = l > 0.f ? 1.f / l : 0.f;
            elem *to = static_cast<elem *>(p.out) + (int64_t)(rq.first + index[i]) * p.out_token +
                       (int64_t)(head * p.share + row - index[i] * p.share) * p.out_head + 4 * g;
            float *to_part = part + (row - row0) * p.dim + 4 * g;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                if (16 * b + 4 * g >= p.dim) continue;
                if (whole_request) {
                    four_t r4;
#pragma unroll
                    for (int e = 0; e < 4; ++e) r4[e] = (elem)(out[i][b][e] * inv);
                    *reinterpret_cast<four_t *>(to + 16 * b) = r4;
                } else {
                    *reinterpret_cast<f4 *>(to_part + 16 * b) = out[i][b];
                }
            }
            if (!whole_request && g == 0) {
                part[ROWS * p.dim + row - row0] = top[i];
                part[ROWS * (p.dim + 1) + row - row0] = l;
            }
        }
        const int odd = uniform(odd_from[0]);
        if (odd == INT_MAX) return;
        for (int row = wave_row0 + c; row < rows && row < wave_row0 + 16 * RT; row += 16)
            for (int d = 4 * g; d < p.dim; d += 16) {
                const f4 more = odd_at(odd, row, d);
                elem *to = static_cast<elem *>(p.out) + (int64_t)(rq.first + row / p.share) * p.out_token + (int64_t)(head * p.share + row % p.share) * p.out_head + d;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (whole_request) to[e] = (elem)((float)to[e] + more[e]);
                    else part[(row - row0) * p.dim + d + e] += more[e];
                }
            }
        return;
    }

    // ---- the key groups' sums, joined through LDS: row c, chunks of four of
    // dim, chunk j of a row at j ^ c
    lanes_meet();
    char *sums_of_wave = smem + wave * (16 * RT * 4 * DP);
    if (RG == 1) sums_of_wave = mine;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        if (g == 0) {
            tops[wave][16 * i + c] = top[i];
            sums[wave][16 * i + c] = weights[i][0];
        }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
            *reinterpret_cast<f4 *>(sums_of_wave + (16 * i + c) * (4 * DP) + 16 * ((4 * b + g) ^ c)) = out[i][b];
    }
    __syncthreads();
    int odd = INT_MAX;
#pragma unroll
    for (int w = 0; w < (RG > 1 ? KG : WAVES); ++w) odd = min(odd, odd_from[w]);
    odd = uniform(odd);
    constexpr int FOURS = DP / 4;
    for (int j = threadIdx.x; j < ROWS * FOURS; j += 64 * WAVES) {
        const int row = j / FOURS, four = j % FOURS, d = 4 * four, w0 = row / (16 * RT), r = row % (16 * RT);
        if (row0 + row >= rows || d >= p.dim) continue;
        float m = tops[w0][r];
#pragma unroll
        for (int w = 1; w < KG; ++w) m = larger(m, tops[w0 + w * RG][r]);
        f4 o = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < KG; ++w) {
            const int from = w0 + w * RG;
            const float share = tops[from][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(tops[from][r] - m);
            l += share * sums[from][r];
            o += share * *reinterpret_cast<const f4 *>(smem + (RG == 1 ? from * S::GROUP : from * (16 * RT * 4 * DP)) + r * (4 * DP) + 16 * (four ^ (r & 15)));
        }
        if (odd != INT_MAX) o += odd_at(odd, row0 + row, d);
        if (whole_request) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            const int token = rq.first + (row0 + row) / p.share, h = head * p.share + (row0 + row) % p.share;
            four_t r4;
#pragma unroll
            for (int e = 0; e < 4; ++e) r4[e] = (elem)(o[e] * inv);
            *reinterpret_cast<four_t *>(static_cast<elem *>(p.out) + token * p.out_token + h * p.out_head + d) = r4;
        } else {
            *reinterpret_cast<f4 *>(part + row * p.dim + d) = o;
            if (four == 0) {
                part[ROWS * p.dim + row] = m;
                part[ROWS * (p.dim + 1) + row] = l;
            }
        }
    }
    if constexpr (RG <= 2) {
        if (whole_request || p.arrived == nullptr) return;
        // Every wave's stores are done at the barrier; one thread's release
        // makes them visible to other XCDs before it counts the run, and who
        // counts the last one acquires those of all others.
        __shared__ int last;
        wait_vm_lgkm0<0>();
        __syncthreads();
        const int64_t place = ((int64_t)run.first * p.heads + head) * p.row_tiles + row_tile;
        if (threadIdx.x == 0) {
            last = __hip_atomic_fetch_add(p.arrived + place, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == run.n - 1;
            if (last) __hip_atomic_store(p.arrived + place, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        const int64_t stride = (int64_t)p.heads * p.row_tiles * ROWS * (p.dim + 2);
        const float *first_part = p.part + place * ROWS * (int64_t)(p.dim + 2);
        for (int j = threadIdx.x; j < ROWS * FOURS; j += 64 * WAVES) {
            const int row = j / FOURS, d = 4 * (j % FOURS);
            if (row0 + row >= rows || d >= p.dim) continue;
            const float *top_at = first_part + ROWS * p.dim + row;
            const int token = rq.first + (row0 + row) / p.share, h = head * p.share + (row0 + row) % p.share;
            join_runs<T>(first_part + row * p.dim + d, top_at, top_at + ROWS, stride, run.n,
                         static_cast<elem *>(p.out) + token * p.out_token + h * p.out_head + d);
        }
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
        join_runs<T>(part + in_tile * p.dim + d, top_at, top_at + tile_rows, stride, n,
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

// No request has more new tokens than there are rows.
int64_t most_new(const gba_attention &d) { return d.max_new < d.tokens ? d.max_new : d.tokens; }

gba_status validate(const gba_attention &d)
{
    const gba_paged_cache &c = d.cache;
    if (!is_dtype(c.dtype)) return GBA_EINVAL;
    if (c.num_blocks < 0 || c.block_size < 1 || c.heads < 0 || c.dim < 0 || d.requests < 0 || d.width < 0 || d.tokens < 0 ||
        d.max_new < 0 || d.q_heads < 0)
        return GBA_EINVAL;
    if (d.workspace != nullptr && !aligned_to(d.workspace, 256)) return GBA_EINVAL;
    if ((__builtin_bit_cast(uint32_t, d.scale * LOG2_E) & 0x7F800000u) == 0x7F800000u) return GBA_EINVAL;  // infinite or NaN
    if (d.requests > GBA_MAX_REQUESTS || d.width > INT_MAX || d.tokens > INT_MAX || c.num_blocks > INT_MAX ||
        c.block_size > INT_MAX || d.q_heads > 65535 || c.heads > 65535 || c.num_blocks * c.block_size > INT_MAX ||
        d.requests * d.width > INT_MAX || d.width * c.block_size > INT_MAX)
        return GBA_EUNSUPPORTED;
    if (d.mask != nullptr && d.max_new > 64) return GBA_EUNSUPPORTED;
    if (d.tokens == 0 || d.requests == 0 || d.q_heads == 0 || d.max_new == 0 || c.dim == 0) return GBA_OK;
    if (c.heads == 0 || d.q_heads % c.heads != 0) return GBA_EINVAL;
    if (c.dim % 8 != 0 || c.dim > 256) return GBA_EUNSUPPORTED;
    if (most_new(d) * (d.q_heads / c.heads) > INT_MAX - 255) return GBA_EUNSUPPORTED;  // rows of a request and head, in tiles of up to 256
    if (d.q == nullptr || d.out == nullptr || d.lens == nullptr || d.offsets == nullptr) return GBA_EINVAL;
    if (d.width > 0 && d.table == nullptr) return GBA_EINVAL;
    if (c.num_blocks > 0 && (c.k == nullptr || c.v == nullptr)) return GBA_EINVAL;
    // (a stride of a dimension of one element is not used)
    const struct { int64_t extent, stride; int of; } strides[] = {
        {c.num_blocks, c.k_block, 8}, {c.block_size, c.k_token, 8}, {c.heads, c.k_head, 8}, {c.num_blocks, c.v_block, 8}, {c.block_size, c.v_token, 8},
        {c.heads, c.v_head, 8}, {d.tokens, d.q_token, 8}, {d.q_heads, d.q_head, 8}, {d.tokens, d.out_token, 4}, {d.q_heads, d.out_head, 4}};
    for (const auto &s : strides)
        if (s.extent > 1 && s.stride % s.of != 0) return GBA_EUNSUPPORTED;
    if (!aligned_to(d.q, 16) || !aligned_to(d.out, 16) || !aligned_to(c.k, 16) || !aligned_to(c.v, 16) ||
        !aligned_to(d.table, 4) || !aligned_to(d.lens, 4) || !aligned_to(d.offsets, 4) || !aligned_to(d.mask, 8))
        return GBA_EUNSUPPORTED;
    return GBA_OK;
}

// How a call runs: the kernel, tiles of rows, runs of keys and their room.
struct Shape {
    bool whole;
    int dp, rt, rg, row_tiles, target, slots;
    bool counts;           // runs are joined by the workgroup that ends last
    size_t header, bytes;  // of the workspace: what stands before the sums, all
};

// A workgroup's release writes back its XCD's L2: that costs less than the
// second kernel while there are few runs of 16 rows (one request of 1000 keys:
// 9.5 us against 10.8, two: 9.8 and 10.9), and more from about a hundred on (8
// trees of 8, 128 of them: 17.0 us against 14.7; 64 requests of up to 8192: 94
// and 81).
constexpr int FEW_RUNS = 64;

// The workspace begins with the counters, zeros whatever calls used it before.
constexpr size_t COUNTERS = 65536, COUNTER_BYTES = COUNTERS * sizeof(int32_t);

// Runs to aim at.  A compute unit has room for one workgroup (two of dim 64),
// and each request and head adds half a run on average, its last one.  Few
// requests: one run a compute unit (one of 32000 keys: 34 us, 52 with four).
// Many of different lengths: more and shorter ones, to even out (64 of up to
// 8192: 92 us with 256, 82 with 512, 87 with 1024; 128 of up to 4000: 139, 128,
// 123).  Tiles of more than 64 rows are bound by their products, not by HBM,
// and a run costs them more: all of them at once (16 trees of 64: 55 us with
// 192, 65 with 224, 80 with 512).
int64_t runs_to_aim_at(const gba_attention &d, int rg, int row_tiles)
{
    const int64_t pairs = d.requests * d.cache.heads * row_tiles;
    if (rg > 2) return pairs < 256 ? 256 - pairs / 2 : 128;
    return pairs <= 128 ? 256 : pairs < 1024 ? 512 : 1024;
}

constexpr int SPLIT_REQUESTS = 1024;           // above that each request is one run

Shape shape_of(const gba_attention &d)
{
    const gba_paged_cache &c = d.cache;
    Shape s;
    // 16 keys in one block, and their offsets in a buffer of 32 bits
    s.whole = c.block_size % 16 == 0 && c.k_token >= 0 && c.v_token >= 0 && c.k_token < (1 << 25) && c.v_token < (1 << 25);
    s.dp = c.dim <= 64 ? 64 : c.dim <= 128 ? 128 : 256;
    const int64_t rows = most_new(d) * (d.q_heads / c.heads);
    // 16 or 32 rows a wave (26 rows over 131k keys: 206 us, 368 as two tiles of
    // 16); more rows on more waves that share the tiles (64 rows, 32 requests of
    // up to 4096 keys, on 2 waves: 80 us, 117 on 8; 256 rows, 16 requests, on 8:
    // 56 us, 71 as two tiles on 4)
    s.rt = rows <= 16 || (s.dp == 256 && !s.whole) ? 1 : 2;
    s.rg = rows <= 32 || s.dp == 256 || !s.whole ? 1 : rows <= 64 ? 2 : rows <= 128 ? 4 : 8;
    s.row_tiles = (int)div_up(rows, 16 * s.rt * s.rg);
    s.target = 0;
    s.slots = (int)d.requests;
    s.counts = false;
    s.header = s.bytes = 0;
    if (d.requests <= SPLIT_REQUESTS && d.width * c.block_size > SHORTEST) {
        s.target = (int)div_up(runs_to_aim_at(d, s.rg, s.row_tiles), c.heads * (int64_t)s.row_tiles);
        s.slots = (int)d.requests + s.target;
        s.counts = s.rg <= 2 && s.rt * s.rg * d.requests * c.heads * s.row_tiles * div_up(d.width * c.block_size, SHORTEST) <= FEW_RUNS &&
                   (size_t)s.slots * c.heads * s.row_tiles <= COUNTERS;
        s.header = COUNTER_BYTES + (size_t)div_up(d.requests * 8, 256) * 256;
        s.bytes = s.header + (size_t)s.slots * c.heads * s.row_tiles * (16 * s.rt * s.rg) * (c.dim + 2) * sizeof(float);
    }
    return s;
}

// A thread for four elements from this many rows on (16 trees of 64, 32768 rows:
// 54.7 us in all, 56.4 with a wave a row), a wave a row below (one request of
// 32000 keys, 32 rows of 32 runs: 34.7 against 42.2; 2048 rows: 81.3 and 82.5).
constexpr int JOIN_ROWS = 4096;

template <class T, int DP, int RT, int RG, bool WHOLE>
gba_status run_attention(const AttentionArgs &a, hipStream_t s)
{
    const int64_t groups = div_up((int64_t)a.slots * a.heads, 8) * 8 * a.row_tiles;
    constexpr int threads = threads_of<DP, RG>();
    const bool joins = a.target != 0 && a.arrived == nullptr, joins_rows = joins && a.tokens * (int64_t)a.q_heads >= JOIN_ROWS;
    if (groups > (int64_t)UINT_MAX / threads || (joins_rows && a.tokens > UINT_MAX / 512)) return GBA_EUNSUPPORTED;
    const gba_status st = launch(attention_kernel<T, DP, RT, RG, WHOLE>, dim3((unsigned)groups), dim3(threads), s, a);
    if (st != GBA_OK || !joins) return st;
    if (joins_rows) return launch(join_rows_kernel<T>, dim3((unsigned)a.tokens), dim3(512), s, a, 16 * RT * RG);
    return launch(join_kernel<T, DP>, dim3((unsigned)div_up((int64_t)a.tokens * a.q_heads, 4)), dim3(256), s, a, 16 * RT * RG);
}

template <class T, int DP>
gba_status run_attention(const AttentionArgs &a, const Shape &sh, hipStream_t s)
{
    if constexpr (DP == 256) {
        if (!sh.whole) return run_attention<T, 256, 1, 1, false>(a, s);
        return sh.rt == 1 ? run_attention<T, 256, 1, 1, true>(a, s) : run_attention<T, 256, 2, 1, true>(a, s);
    } else {
        if (!sh.whole) return sh.rt == 1 ? run_attention<T, DP, 1, 1, false>(a, s) : run_attention<T, DP, 2, 1, false>(a, s);
        if (sh.rt == 1) return run_attention<T, DP, 1, 1, true>(a, s);
        switch (sh.rg) {
        case 1: return run_attention<T, DP, 2, 1, true>(a, s);
        case 2: return run_attention<T, DP, 2, 2, true>(a, s);
        case 4: return run_attention<T, DP, 2, 4, true>(a, s);
        default: return run_attention<T, DP, 2, 8, true>(a, s);
        }
    }
}

template <class T>
gba_status run_attention(const AttentionArgs &a, const Shape &sh, hipStream_t s)
{
    if (sh.dp == 64) return run_attention<T, 64>(a, sh, s);
    return sh.dp == 128 ? run_attention<T, 128>(a, sh, s) : run_attention<T, 256>(a, sh, s);
}

bool nothing_to_do(const gba_attention &d)
{
    return d.tokens == 0 || d.requests == 0 || d.q_heads == 0 || d.max_new == 0 || d.cache.dim == 0;
}

}  // namespace
}  // namespace gba

using namespace gba;

extern "C" gba_status gba_tree_attention_workspace_size(const gba_attention *desc, size_t *bytes)
{
    if (desc == nullptr || bytes == nullptr) return GBA_EINVAL;
    const gba_status st = validate(*desc);
    if (st == GBA_OK) *bytes = nothing_to_do(*desc) ? 0 : shape_of(*desc).bytes;
    return st;
}

extern "C" gba_status gba_tree_attention(const gba_attention *desc, gba_stream_t stream)
{
    if (desc == nullptr) return GBA_EINVAL;
    const gba_attention &d = *desc;
    const gba_paged_cache &c = d.cache;
    const gba_status st = validate(d);
    if (st != GBA_OK || nothing_to_do(d)) return st;
    Shape sh = shape_of(d);
    if (sh.target != 0 && (d.workspace == nullptr || d.workspace_bytes < sh.bytes)) {
        sh.target = 0;
        sh.slots = (int)d.requests;
        sh.counts = false;
    }
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
    a.row_tiles = sh.row_tiles;
    a.slots = sh.slots;
    a.target = sh.target;
    a.arrived = sh.counts ? static_cast<int32_t *>(d.workspace) : nullptr;
    a.first_run = sh.target != 0 ? reinterpret_cast<int32_t *>(static_cast<char *>(d.workspace) + COUNTER_BYTES) : nullptr;
    a.part = sh.target != 0 ? reinterpret_cast<float *>(static_cast<char *>(d.workspace) + sh.header) : nullptr;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return c.dtype == GBA_F16 ? run_attention<F16>(a, sh, s) : run_attention<BF16>(a, sh, s);
}
