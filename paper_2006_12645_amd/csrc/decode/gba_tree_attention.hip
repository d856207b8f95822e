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
// only when one passes it by more than 2^8 (in the base-2 exponent), so that
// the accumulators are seldom scaled; weights then stay below 2^8, and their
// relative rounding is the same at any size.  l is one more matrix
// instruction, of ones and the rounded weights.
//
// Few rows read a whole cache: the bound is HBM.  A wave copies its tiles
// straight into its own part of LDS, one tile ahead, and waits for nothing but
// its own copies; the waves of a workgroup take the tiles of a run of keys in
// turn and meet once, at its end.  Runs are cut to one length for all
// requests, from the sum of their lengths, which every wave reads for itself;
// the runs of one request are joined by a second kernel.
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
    float scale2;      // scale * log2(e)
    int row_tiles;     // of a request and head
    int slots;         // runs of keys there is room for: at least as many as there are
    int target;        // runs to aim at (0: one for each request)
    int32_t *first_run;  // [requests][2]: a request's first run and how many it has
    float *part;       // [slots][heads][row_tiles]: rows x dim sums, then as many maxima and sums of weights
};

constexpr int KEYS = 32;        // of a tile
constexpr int SHORTEST = 256;   // keys of a run, but a request's last
constexpr float SLACK = 8.f;

// A request's new tokens and keys, none for one with too many.
struct Request {
    int first, fresh, kept, end;
};

__device__ __forceinline__ Request request_of(const AttentionArgs &p, int r)
{
    Request q;
    q.first = p.offsets[r];
    q.fresh = min(p.offsets[r + 1], p.tokens) - q.first;
    if (q.first < 0 || q.fresh < 0 || q.fresh > p.max_new) q.fresh = 0;
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
};

// Every run but a request's last is of one length, a multiple of `step`:
// the mean of all keys over p.target runs, so there are no more than
// p.target + p.requests.  The sum of the lengths is one in 24 bits; the
// factor covers its rounding.
__device__ __forceinline__ Run run_of(const AttentionArgs &p, int x, int lane, int step)
{
    Run u;
    if (p.target == 0) {
        const Request q = request_of(p, x);
        u.r = uniform(q.fresh) > 0 ? x : -1;
        u.n = 1;
        u.first = x;
        u.from = 0;
        u.to = uniform(q.end);
        return u;
    }
    float keys = 0.f;
    Request q = {0, 0, 0, 0};
    for (int r = lane; r < p.requests; r += 64) {
        q = request_of(p, r);
        if (q.fresh > 0) keys += (float)q.end;
    }
    const float mean = wave_total(keys) / (float)p.target * 1.00001f;
    const int most = INT_MAX / step * step;
    int length = mean < (float)(most - step) ? ((int)mean / step + 1) * step : most;
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
            const int end = __builtin_amdgcn_readlane(q.end, l);
            u.to = end - u.from > length ? u.from + length : end;
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

// The largest of the four lanes that hold one row.
__device__ __forceinline__ float across_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 32));
    return fmaxf(x, __shfl_xor(x, 16));
}

// A workgroup's waves: RG of them take 16 RT rows each of the same keys, and
// KG such groups the tiles of a run in turn.  One group keeps STAGES tiles in
// LDS.
template <int DP, int RG>
struct Shared {
    static constexpr int KG = RG == 8 ? 1 : RG == 4 || DP == 256 ? 2 : 4, WAVES = RG * KG;
    static constexpr int STAGES = RG == 8 ? 4 : RG == 4 ? 3 : 2;
    static constexpr int CPR = DP / 8;                   // 16-byte chunks of a row
    static constexpr int KPI = 64 / CPR;                 // keys that one 64-lane copy covers
    static constexpr int COPIES = KEYS / KPI;            // of a tile of K or V
    static constexpr int ROW = 2 * DP, TILE = KEYS * ROW, STAGE = 2 * TILE, GROUP = STAGES * STAGE;
};

// The join of the key groups needs 16 RT rows of fp32 for each wave.
template <int DP, int RT, int RG>
constexpr int lds_bytes()
{
    typedef Shared<DP, RG> S;
    return S::KG * S::GROUP > S::WAVES * 16 * RT * 4 * DP ? S::KG * S::GROUP : S::WAVES * 16 * RT * 4 * DP;
}
template <int DP, int RG>
constexpr int threads_of()
{
    return 64 * Shared<DP, RG>::WAVES;
}

// DP: dim, padded.  RT: blocks of 16 rows of a wave.  WHOLE: 16 consecutive
// keys, from a multiple of 16 on, are in one block, and go straight to LDS;
// else (RG 1 only) they pass through registers, which hold the next tile.
template <class T, int DP, int RT, int RG, bool WHOLE>
__global__ void __launch_bounds__((threads_of<DP, RG>()), (RG == 1 ? 1 : 2)) attention_kernel(AttentionArgs p)
{
    typedef Shared<DP, RG> S;
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    static_assert(WHOLE || RG == 1, "waves share only what goes straight to LDS");
    constexpr int WAVES = S::WAVES, KG = S::KG, STAGES = WHOLE ? S::STAGES : 1;
    constexpr int CPR = S::CPR, KPI = S::KPI, COPIES = S::COPIES, ROW = S::ROW, TILE = S::TILE;
    constexpr int STEPS = DP / 32, BLOCKS = DP / 16, ROWS = 16 * RT * RG;
    __shared__ __attribute__((aligned(16))) char smem[lds_bytes<DP, RT, RG>()];
    __shared__ float tops[WAVES][16 * RT], sums[WAVES][16 * RT];

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), rg = wave % RG, kg = wave / RG;
    const int c = lane & 15, g = lane >> 4;
    // The row tiles of one run and head have ids 8 apart: the same XCD's L2.
    const int xcd = blockIdx.x & 7, rest = blockIdx.x >> 3;
    const int row_tile = rest % p.row_tiles, item = rest / p.row_tiles * 8 + xcd;
    const int head = item % p.heads, x = item / p.heads;
    if (x >= p.slots) return;
    const Run run = run_of(p, x, lane, KEYS * KG);
    if (run.r < 0) return;
    Request rq = request_of(p, run.r);
    rq.first = uniform(rq.first);
    rq.fresh = uniform(rq.fresh);
    rq.kept = uniform(rq.kept);
    const int rows = rq.fresh * p.share, row0 = row_tile * ROWS;
    if (p.target != 0 && run.first == x && head == 0 && row_tile == 0 && threadIdx.x == 0) {
        p.first_run[2 * run.r] = x;
        p.first_run[2 * run.r + 1] = run.n;
    }
    if (row0 >= rows) return;

    // ---- copies of a tile: 1 KB each, lane l the chunk at byte 16 l
    char *mine = smem + kg * S::GROUP;
    const int tiles = (run.to - run.from + KEYS - 1) / KEYS;
    const int count = tiles > kg ? (tiles - kg + KG - 1) / KG : 0;  // of this group
    const int rounds = RG == 1 ? count : (tiles + KG - 1) / KG;     // of every group, where waves wait for each other
    const int32_t *entries = p.table + (int64_t)run.r * p.width;
    auto key0 = [&](int n) { return run.from + KEYS * (kg + KG * n); };
    const int in_copy = lane / CPR, place = lane % CPR;
    constexpr int PER_HALF = COPIES / 2;
    const char *k_head = reinterpret_cast<const char *>(static_cast<const elem *>(p.k) + head * p.k_head);
    const char *v_head = reinterpret_cast<const char *>(static_cast<const elem *>(p.v) + head * p.v_head);
    int k_off[WHOLE ? PER_HALF : 1], v_off[WHOLE ? PER_HALF : 1];
    if constexpr (WHOLE) {
#pragma unroll
        for (int i = 0; i < PER_HALF; ++i) {
            const int key = KPI * i + in_copy, kc = place ^ swap_k<DP>(key), vc = place ^ swap_v<DP>(key);
            k_off[i] = 8 * kc < p.dim ? (int)(key * p.k_token * 2) + 16 * kc : OOB_OFFSET;
            v_off[i] = 8 * vc < p.dim ? (int)(key * p.v_token * 2) + 16 * vc : OOB_OFFSET;
        }
    }
    // WHOLE: the blocks of the next 32 tiles' halves, a lane each.  Else: the
    // block and token of key lane % 32 of the next tile, and its registers.
    int entry = -1, within = 0, entries_from = 0;
    u4 k_next[WHOLE ? 1 : COPIES], v_next[WHOLE ? 1 : COPIES];
    auto look_up = [&](int n) {
        const int pos = WHOLE ? key0(n + lane / 2) + 16 * (lane & 1) : key0(n) + (lane & 31);
        entry = -1;
        if (pos < run.to) {
            const int page = pos / p.block_size;
            within = pos - page * p.block_size;
            const int b = entries[page];
            entry = b >= 0 && b < p.num_blocks ? b : -1;
        }
        entries_from = n;
    };
    // How many keys of a half of tile n exist (WHOLE): those up to the run's
    // end, if its block does.
    auto keys_of = [&](int n, int h) {
        const int b = __builtin_amdgcn_readlane(entry, 2 * (n - entries_from) + h), left = run.to - (key0(n) + 16 * h);
        return b < 0 || left < 0 ? 0 : left < 16 ? left : 16;
    };
    // Copies tile n, and says which of its keys exist.  A share of a group's
    // copies for each of its waves; none are left out past the last tile, so
    // that the number under way is always the same.
    constexpr int MY_COPIES = 2 * COPIES / RG;
    auto copy = [&](int n) -> unsigned {
        if constexpr (WHOLE) {
            unsigned there = 0;
            char *k_lds = mine + n % STAGES * S::STAGE, *v_lds = k_lds + TILE;
            if (n - entries_from == 32) look_up(n);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = 2 * (n - entries_from) + h, keys = n < count ? keys_of(n, h) : 0;
                there |= ((1u << keys) - 1) << (16 * h);
                const int b = keys ? __builtin_amdgcn_readlane(entry, at) : 0, t = keys ? __builtin_amdgcn_readlane(within, at) : 0;
                // beyond the last key the buffer has ended: zeros
                const __amdgpu_buffer_rsrc_t kr =
                    __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(k_head + 2 * (b * p.k_block + t * p.k_token)), (short)0,
                                                      keys ? (int)((keys - 1) * p.k_token + p.dim) * 2 : 0, RSRC_WORD3);
                const __amdgpu_buffer_rsrc_t vr =
                    __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(v_head + 2 * (b * p.v_block + t * p.v_token)), (short)0,
                                                      keys ? (int)((keys - 1) * p.v_token + p.dim) * 2 : 0, RSRC_WORD3);
#pragma unroll
                for (int i = 0; i < PER_HALF; ++i) {
                    const int j = PER_HALF * h + i;
                    if (RG == 1 || (2 * j) % RG == rg) buffer_load16_lds(kr, k_lds + 1024 * j, k_off[i], 0);
                    if (RG == 1 || (2 * j + 1) % RG == rg) buffer_load16_lds(vr, v_lds + 1024 * j, v_off[i], 0);
                }
            }
            return there;
        } else {
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
        }
    };
    if (rounds > 0) look_up(0);

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
        }
        sees[i] = p.mask != nullptr ? p.mask[token] : 0;
    }
    const bool masked = p.mask != nullptr;

    f4 out[RT][BLOCKS] = {}, weights[RT] = {};
    float top[RT], base2[RT];  // running maximum; what is subtracted (0 while there is none)
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        top[i] = -INFINITY;
        base2[i] = 0.f;
    }

    // ---- LDS addresses of the fragments
    int k_at[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) k_at[s] = c * ROW + 16 * ((4 * s + g) ^ swap_k<DP>(c));
    const int v_key = 4 * g + (c >> 2), v_swap = 16 * swap_v<DP>(v_key);
    const int v_at = v_key * ROW + 16 * ((c & 3) >> 1) + 8 * (c & 1);
    vec8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (elem)1.f;

    unsigned ahead[WHOLE ? STAGES - 1 : 1];  // which keys of the tiles under way exist
    if constexpr (WHOLE) {
        wait_vm_lgkm0<0>();  // the rows and blocks: from here on only copies are under way
        if (rounds > 0) {
#pragma unroll
            for (int n = 0; n < STAGES - 1; ++n) ahead[n] = copy(n);
        }
    } else if (rounds > 0) {
        ahead[0] = copy(0);
    }
    for (int n = 0; n < rounds; ++n) {
        const char *k_lds = mine + n % STAGES * S::STAGE, *v_lds = k_lds + TILE;
        const unsigned there = ahead[0];
#pragma unroll
        for (int i = 0; i + 2 < STAGES; ++i) ahead[i] = ahead[i + 1];
        if constexpr (WHOLE && RG == 1) {
            wait_vm_lgkm0<63>();  // the slot's last fragments have been read
            ahead[STAGES - 2] = copy(n + STAGES - 1);
            wait_vm_lgkm0<(STAGES - 1) * MY_COPIES>();
        } else if constexpr (WHOLE) {
            wait_vm_lgkm0<(STAGES - 2) * MY_COPIES>();
            __builtin_amdgcn_s_barrier();  // every wave's share is there, and the last slot has been read
            ahead[STAGES - 2] = copy(n + STAGES - 1);
        } else {
            lanes_meet();  // the last tile's fragments have been read
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                *reinterpret_cast<u4 *>(mine + 1024 * i + 16 * lane) = k_next[i];
                *reinterpret_cast<u4 *>(mine + TILE + 1024 * i + 16 * lane) = v_next[i];
            }
            if (n + 1 < count) ahead[0] = copy(n + 1);
        }
        lanes_meet();
        if (there == 0) continue;

        // scores: keys 16 h + 4 g + e of the tile, row c of each block
        f4 score[RT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < RT; ++i) score[i][h] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const vec8 k = *reinterpret_cast<const vec8 *>(k_lds + 16 * h * ROW + k_at[s]);
#pragma unroll
                for (int i = 0; i < RT; ++i) score[i][h] = T::mfma(k, query[i][s], score[i][h]);
            }
        }
        const int first_draft = key0(n) - rq.kept;  // of the new tokens, or below 0
        const bool all = there == 0xFFFFFFFFu && first_draft + KEYS <= 0;
        vec8 weight[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = score[i][e >> 2][e & 3] * p.scale2;
            if (!all) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int key = 16 * (e >> 2) + 4 * g + (e & 3), draft = first_draft + key;
                    const bool in_tree = masked ? (draft < 64) & (int)((sees[i] >> (draft & 63)) & 1) : draft <= index[i];
                    const bool seen = ((there >> key) & 1) & ((draft < 0) | in_tree);
                    t[e] = seen ? t[e] : -INFINITY;
                }
            }
            float most = t[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) most = fmaxf(most, t[e]);
            if (__ballot(most > top[i] + SLACK)) {
                const float now = fmaxf(across_max(most), top[i]);
                const float next = now == -INFINITY ? 0.f : now;
                const float keep = top[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(base2[i] - next);
                top[i] = now;
                base2[i] = next;
                weights[i] *= keep;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) out[i][b] *= keep;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) weight[i][e] = (elem)__builtin_amdgcn_exp2f(t[e] - base2[i]);
            weights[i] = T::mfma(ones, weight[i], weights[i]);
        }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const char *at = v_lds + v_at + ((32 * b) ^ v_swap);
            const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)at);
            const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(at + 16 * ROW));
            const vec8 v = __builtin_bit_cast(vec8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int i = 0; i < RT; ++i) out[i][b] = T::mfma(v, weight[i], out[i][b]);
        }
    }

    // ---- the key groups' sums, joined through LDS: row c, chunks of four of
    // dim, chunk j of a row at j ^ c
    wait_vm_lgkm0<0>();
    if (RG > 1) __syncthreads();  // the tiles have been read
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
    const bool whole_request = run.n == 1;
    float *part = whole_request ? nullptr : p.part + (((int64_t)x * p.heads + head) * p.row_tiles + row_tile) * ROWS * (int64_t)(p.dim + 2);
    constexpr int FOURS = DP / 4;
    for (int j = threadIdx.x; j < ROWS * FOURS; j += 64 * WAVES) {
        const int row = j / FOURS, four = j % FOURS, d = 4 * four, w0 = row / (16 * RT), r = row % (16 * RT);
        if (row0 + row >= rows || d >= p.dim) continue;
        float m = tops[w0][r];
#pragma unroll
        for (int w = 1; w < KG; ++w) m = fmaxf(m, tops[w0 + w * RG][r]);
        f4 o = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < KG; ++w) {
            const int from = w0 + w * RG;
            const float share = tops[from][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(tops[from][r] - m);
            l += share * sums[from][r];
            o += share * *reinterpret_cast<const f4 *>(smem + (RG == 1 ? from * S::GROUP : from * (16 * RT * 4 * DP)) + r * (4 * DP) + 16 * (four ^ (r & 15)));
        }
        if (whole_request) {
            typedef elem four_t __attribute__((ext_vector_type(4)));
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
}

// The runs of a request, added in their order; one wave a token and query
// head, lane l four elements of every (256 / DP)-th run: its share of the
// weight comes from the lane that holds that run's maximum and sum.
template <class T, int DP>
__global__ void __launch_bounds__(256) join_kernel(AttentionArgs p, int tile_rows)
{
    typedef typename T::elem elem;
    constexpr int FOURS = DP / 4, AT_ONCE = 64 / FOURS;
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6);
    const int t = (int)(id / p.q_heads), head = (int)(id - (int64_t)t * p.q_heads);
    if (t >= p.tokens) return;
    int r = 0;  // the number of requests that end at or before t
    for (int base = 0; base < p.requests; base += 64)
        r += __popcll(__ballot(base + lane < p.requests && p.offsets[base + lane + 1] <= t));
    if (r >= p.requests) return;
    const int x0 = p.first_run[2 * r], n = p.first_run[2 * r + 1];
    const Request rq = request_of(p, r);
    if (rq.fresh == 0 || t < rq.first || n <= 1) return;
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
        for (int s = 32; s; s >>= 1) next = fmaxf(next, __shfl_xor(next, s));
        next = fmaxf(next, m);
        if (next == -INFINITY) continue;
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
                const float w = __shfl(share, from & 63);
                f[u] = from < here ? w : 0.f;
                v[u] = *reinterpret_cast<const f4 *>(mine + (base + (from < here ? from : 0)) * stride);
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

// How a call runs: the kernel, tiles of rows, runs of keys and their room.
struct Shape {
    bool whole;
    int dp, rt, rg, row_tiles, target, slots;
    size_t header, bytes;  // of the workspace
};

constexpr int RUNS = 1024, RUNS_SHARED = 512;  // workgroups to aim at
constexpr int SPLIT_REQUESTS = 1024;           // above that each request is one run

Shape shape_of(const gba_attention &d)
{
    const gba_paged_cache &c = d.cache;
    Shape s;
    // 16 keys in one block, and their offsets in a buffer of 32 bits
    s.whole = c.block_size % 16 == 0 && c.k_token >= 0 && c.v_token >= 0 && c.k_token < (1 << 25) && c.v_token < (1 << 25);
    s.dp = c.dim <= 64 ? 64 : c.dim <= 128 ? 128 : 256;
    const int64_t rows = d.max_new * (d.q_heads / c.heads);
    // 16 or 32 rows a wave; more rows on more waves that share the tiles
    s.rt = rows <= 16 || (s.dp == 256 && !s.whole) ? 1 : 2;
    s.rg = rows <= 32 || s.dp == 256 || !s.whole ? 1 : rows <= 64 ? 2 : rows <= 128 ? 4 : 8;
    s.row_tiles = (int)div_up(rows, 16 * s.rt * s.rg);
    s.target = 0;
    s.slots = (int)d.requests;
    s.header = s.bytes = 0;
    if (d.requests <= SPLIT_REQUESTS && d.width * c.block_size > SHORTEST) {
        s.target = (int)div_up(s.rg > 2 ? RUNS_SHARED : RUNS, c.heads * (int64_t)s.row_tiles);
        s.slots = (int)d.requests + s.target;
        s.header = (size_t)div_up(d.requests * 8, 256) * 256;
        s.bytes = s.header + (size_t)s.slots * c.heads * s.row_tiles * (16 * s.rt * s.rg) * (c.dim + 2) * sizeof(float);
    }
    return s;
}

template <class T, int DP, int RT, int RG, bool WHOLE>
gba_status run_attention(const AttentionArgs &a, hipStream_t s)
{
    const int64_t groups = div_up((int64_t)a.slots * a.heads, 8) * 8 * a.row_tiles;
    constexpr int threads = threads_of<DP, RG>();
    if (groups > (int64_t)UINT_MAX / threads || div_up((int64_t)a.tokens * a.q_heads, 4) > (int64_t)UINT_MAX / 256) return GBA_EUNSUPPORTED;
    const gba_status st = launch(attention_kernel<T, DP, RT, RG, WHOLE>, dim3((unsigned)groups), dim3(threads), s, a);
    if (st != GBA_OK || a.target == 0) return st;
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
    a.max_new = (int)d.max_new;
    a.q_heads = (int)d.q_heads;
    a.heads = (int)c.heads;
    a.share = (int)(d.q_heads / c.heads);
    a.num_blocks = (int)c.num_blocks;
    a.block_size = (int)c.block_size;
    a.dim = (int)c.dim;
    a.scale2 = d.scale * 1.44269504088896340736f;
    a.row_tiles = sh.row_tiles;
    a.slots = sh.slots;
    a.target = sh.target;
    a.first_run = static_cast<int32_t *>(d.workspace);
    a.part = sh.target != 0 ? reinterpret_cast<float *>(static_cast<char *>(d.workspace) + sh.header) : nullptr;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return c.dtype == GBA_F16 ? run_attention<F16>(a, sh, s) : run_attention<BF16>(a, sh, s);
}
