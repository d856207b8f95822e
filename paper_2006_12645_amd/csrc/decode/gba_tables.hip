// gba_tables.hip -- block tables and slot maps of a step, from the requests'
// lengths, on the GPU.
//
// Three running sums over the requests say everything: of the blocks given
// back, of the blocks wanted and of the new tokens.  They give each request its
// places on the stack of free blocks, so that all requests move their blocks
// at once, one wave each, and what happens does not depend on the order of the
// threads.  The stack is pushed before it is popped: two kernels, of which each
// workgroup of the first one takes the running sums for itself (they are a few
// kilobytes) and pushes for its 16 requests; the second one pops, clears what
// was given back, and writes what belongs to each token, whose new block it
// reads from the stack itself.  Between them nothing that either one reads is
// written.  A small step is one workgroup that does both.
//
// Bound by launches and by the latency of four dependent reads, not by bytes: 4
// requests 4.0 us; 256 trees of 64 tokens 6.3 and 3.9 us for the two kernels.
#include "gba_decode.hpp"

namespace gba {
namespace {

constexpr int TABLE_THREADS = 1024, TABLE_WAVES = TABLE_THREADS / 64;
constexpr int PER_THREAD = GBA_MAX_REQUESTS / TABLE_THREADS;
// What one workgroup does alone: its waves take the requests in turn.  16 trees
// of 64 tokens 6.4 us, 6.8 with two kernels; 64 trees of 16 11.0 and 7.7; 64
// single tokens 7.9 and 7.3, where the host's second launch is 3.4.
constexpr int SMALL_REQUESTS = 64, SMALL_TREES = 32, SMALL_TOKENS = 1024;

// What the second kernel knows of a request: blocks needed and held, the
// running sum of the blocks wanted before it, and its status; of the step,
// in the place after the last request's: blocks on the stack after the pushes,
// blocks handed out, tokens.
typedef int Plan __attribute__((ext_vector_type(4)));

struct TableArgs {
    int32_t *table, *held, *free_blocks, *free_count;
    const int32_t *lens, *count, *parents;
    int32_t *offsets, *slots, *positions, *status;
    uint64_t *mask;
    Plan *plan;
    int requests, width, num_blocks, block_size, tokens;
};

struct Pair {
    int a, b;
};

template <int CTRL, int ROWS>
__device__ __forceinline__ void add_moved(Pair &x)
{
    x.a += __builtin_amdgcn_update_dpp(0, x.a, CTRL, ROWS, 0xF, false);
    x.b += __builtin_amdgcn_update_dpp(0, x.b, CTRL, ROWS, 0xF, false);
}

// Exclusive running sums over the workgroup's threads; totals for every thread.
__device__ __forceinline__ Pair block_scan(Pair v, Pair *scratch, Pair &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    Pair x = v;
    add_moved<0x111, 0xF>(x);  // one lane up, within 16
    add_moved<0x112, 0xF>(x);
    add_moved<0x114, 0xF>(x);
    add_moved<0x118, 0xF>(x);
    add_moved<0x142, 0xA>(x);  // lanes 15 and 47 to the 16 after them
    add_moved<0x143, 0xC>(x);  // lane 31 to the 32 after it
    if (lane == 63) scratch[wave] = x;
    __syncthreads();
    Pair before = {x.a - v.a, x.b - v.b};
    total = {0, 0};
    for (int w = 0; w < waves; ++w) {
        const Pair y = scratch[w];
        before.a += w < wave ? y.a : 0;
        before.b += w < wave ? y.b : 0;
        total.a += y.a;
        total.b += y.b;
    }
    return before;
}

// The step's plan.  The whole workgroup takes part; it writes what it finds of
// requests [base, base + count): into `plan` (and what the step as a whole is
// into plan[count]), `to`, the place on the stack of the first block that each
// gives back, offsets and status.
__device__ __forceinline__ void make_plan(const TableArgs &p, int base, int count, Plan *plan, int64_t *to)
{
    __shared__ Pair scratch[2][TABLE_WAVES];
    __shared__ int handed_out;
    const int R = p.requests, W = p.width;
    // few requests: one a thread, so that their loads are all under way at once
    const int each = R > (int)blockDim.x ? PER_THREAD : 1, first = threadIdx.x * each;
    int fc = *p.free_count;
    fc = fc < 0 ? 0 : fc > p.num_blocks ? p.num_blocks : fc;
    if (threadIdx.x == 0) handed_out = 0;

    int state[PER_THREAD], need[PER_THREAD], held[PER_THREAD], fresh[PER_THREAD];
    Pair sum = {0, 0}, all;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        const int r = first + i;
        const bool real = i < each && r < R;
        const int n = real ? p.count[r] : 0, kept = real ? p.lens[r] : 0, h = real ? p.held[r] : 0;
        fresh[i] = n > 0 ? n : 0;
        const uint32_t end = (uint32_t)(kept > 0 ? kept : 0) + (uint32_t)fresh[i];
        const uint32_t want = end > 0 ? (end - 1) / (uint32_t)p.block_size + 1 : 0;
        state[i] = want > (uint32_t)W ? 2 : 0;
        need[i] = want > (uint32_t)W ? W : (int)want;
        held[i] = h < 0 ? 0 : h > W ? W : h;
        // tokens in two halves, whose sums fit 32 bits
        sum.a += fresh[i] >> 16;
        sum.b += fresh[i] & 0xFFFF;
    }
    const Pair start = block_scan(sum, scratch[0], all);
    int64_t at = ((int64_t)start.a << 16) + start.b;
    const int64_t total = ((int64_t)all.a << 16) + all.b;
    const int tokens = (int)(total < p.tokens ? total : p.tokens);
    // blocks given back and blocks wanted: each sum is at most requests * width
    sum = {0, 0};
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        const int r = first + i;
        const bool real = i < each && r < R;
        if (real && r >= base && r < base + count) p.offsets[r] = (int32_t)(at < p.tokens ? at : p.tokens);
        at += fresh[i];
        if (state[i] == 0 && (at > p.tokens || (p.parents != nullptr && fresh[i] > 64))) state[i] = 3;
        if (real && need[i] < held[i]) sum.a += held[i] - need[i];
        else if (real && state[i] == 0) sum.b += need[i] - held[i];
    }
    Pair before = block_scan(sum, scratch[1], all);
    const int64_t avail = (int64_t)fc + all.a;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        const int r = first + i;
        if (i >= each || r >= R) break;
        const int back = held[i] > need[i] ? held[i] - need[i] : 0, want = back == 0 && state[i] == 0 ? need[i] - held[i] : 0;
        if (want > 0 && before.b + (int64_t)want > avail) state[i] = 1;
        else if (want > 0) atomicMax(&handed_out, before.b + want);
        if (r >= base && r < base + count) {
            plan[r - base] = Plan{need[i], held[i], before.b, state[i]};
            to[r - base] = (int64_t)fc + before.a;
            p.status[r] = state[i];
        }
        before.a += back;
        before.b += want;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        // more on the stack than it has places: blocks that no request held
        plan[count] = Plan{avail < INT_MAX ? (int)avail : INT_MAX, handed_out, tokens, 0};
        if (base + count >= R) p.offsets[R] = tokens;
    }
    __syncthreads();
}

// One wave: the blocks that request r gives back, onto the stack.
__device__ __forceinline__ void push(const TableArgs &p, int r, const Plan &q, int64_t to, int lane)
{
    const int32_t *from = p.table + (int64_t)r * p.width + q[0];
    for (int i = lane; i < q[1] - q[0]; i += 64)
        if (to + i < p.num_blocks) p.free_blocks[to + i] = from[i];
}

// Entry `column` of a request's row after the step.
__device__ __forceinline__ int entry_of(const TableArgs &p, int r, const Plan &q, int avail, int column)
{
    if (column < q[1]) return p.table[(int64_t)r * p.width + column];
    const int from = avail - 1 - (q[2] + column - q[1]);
    return from >= 0 && from < p.num_blocks ? p.free_blocks[from] : -1;
}

// One wave: request r's row and holdings.
__device__ __forceinline__ void pop(const TableArgs &p, int r, const Plan &q, int avail, int lane)
{
    int32_t *row = p.table + (int64_t)r * p.width;
    const int end = q[3] == 0 && q[0] > q[1] ? q[0] : q[1];
    for (int i = q[1] + lane; i < end; i += 64) row[i] = entry_of(p, r, q, avail, i);
    for (int i = q[0] + lane; i < q[1]; i += 64) row[i] = -1;
    if (lane == 0) p.held[r] = q[0] < q[1] ? q[0] : end;
}

__device__ __forceinline__ void write_token(const TableArgs &p, int t, int slot, int64_t position)
{
    if (p.slots != nullptr) p.slots[t] = slot;
    if (p.positions != nullptr) p.positions[t] = (int32_t)position;
}

__device__ __forceinline__ int slot_of(const TableArgs &p, int r, const Plan &q, int avail, int64_t pos)
{
    if (q[3] != 0) return -1;
    const int column = (int)((uint32_t)pos / (uint32_t)p.block_size), entry = entry_of(p, r, q, avail, column);
    return entry < 0 ? -1 : (int)((int64_t)entry * p.block_size + (pos - (int64_t)column * p.block_size));
}

// One wave: the tokens of request r, a tree, one a lane.  A token's mask is its
// own bit and those of its ancestors, found by doubling: six rounds in which
// every token takes the mask of the token it points to and then points to where
// that one points.  T may be less than the request asks for: a tree of more than
// 64 has status 2 or 3.
__device__ __forceinline__ void tree(const TableArgs &p, int r, const Plan &q, int avail, int first, int T, int lane)
{
    if (q[3] >= 2 && p.count[r] > 64) {
        for (int i = lane; i < T; i += 64) {
            write_token(p, first + i, -1, -1);
            p.mask[first + i] = 0;
        }
        return;
    }
    const int n = p.lens[r], parent = lane < T ? p.parents[first + lane] : -1;
    const int64_t kept = n > 0 ? n : 0;
    const int slot = lane < T ? slot_of(p, r, q, avail, kept + lane) : -1;
    int up = parent >= 0 && parent < lane ? parent : lane;
    uint64_t mask = 1ull << lane;
    for (int i = 0; i < 6; ++i) {
        mask |= __shfl(mask, up);
        up = __shfl(up, up);
    }
    if (lane < T) {
        write_token(p, first + lane, slot, kept + __popcll(mask) - 1);
        p.mask[first + lane] = mask;
    }
}

// Entries past the last request's tokens.
__device__ __forceinline__ void pad(const TableArgs &p, int64_t t, int64_t step)
{
    for (; t < p.tokens; t += step) {
        write_token(p, (int)t, -1, -1);
        if (p.parents != nullptr) p.mask[t] = 0;
    }
}

__global__ void __launch_bounds__(TABLE_THREADS) small_kernel(TableArgs p)
{
    __shared__ Plan plan[SMALL_REQUESTS + 1];
    __shared__ int64_t to[SMALL_REQUESTS];
    __shared__ int begin[SMALL_REQUESTS + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    make_plan(p, 0, p.requests, plan, to);
    const int avail = plan[p.requests][0], tokens = plan[p.requests][2];
    if ((int)threadIdx.x <= p.requests) begin[threadIdx.x] = p.offsets[threadIdx.x];
    for (int r = wave; r < p.requests; r += waves) push(p, r, plan[r], to[r], lane);
    __syncthreads();
    // nothing that a token reads is written here: what its request keeps, and
    // the stack
    if (p.parents != nullptr) {
        for (int r = wave; r < p.requests; r += waves) tree(p, r, plan[r], avail, begin[r], begin[r + 1] - begin[r], lane);
    } else {
        for (int t = threadIdx.x; t < tokens; t += blockDim.x) {
            const int r = owner_of(begin, p.requests, t), n = p.lens[r];
            const int64_t pos = (int64_t)(n > 0 ? n : 0) + (t - begin[r]);
            write_token(p, t, slot_of(p, r, plan[r], avail, pos), pos);
        }
    }
    for (int r = wave; r < p.requests; r += waves) pop(p, r, plan[r], avail, lane);
    pad(p, tokens + threadIdx.x, blockDim.x);
    if (threadIdx.x == 0) *p.free_count = avail - plan[p.requests][1];
}

// A request a wave.
__global__ void __launch_bounds__(TABLE_THREADS) push_kernel(TableArgs p)
{
    __shared__ Plan plan[TABLE_WAVES + 1];
    __shared__ int64_t to[TABLE_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, base = blockIdx.x * waves;
    const int count = p.requests - base < waves ? p.requests - base : waves;
    make_plan(p, base, count, plan, to);
    if (wave < count) {
        push(p, base + wave, plan[wave], to[wave], lane);
        if (lane == 0) p.plan[base + wave] = plan[wave];
    }
    if (base + count >= p.requests && threadIdx.x == 0) p.plan[p.requests] = plan[count];
}

// The first workgroups: four requests each.  The others, for chains: 256
// tokens each.
__global__ void __launch_bounds__(256) pop_kernel(TableArgs p, int request_groups)
{
    __shared__ int begin[GBA_MAX_REQUESTS + 1];
    const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    const Plan step = p.plan[p.requests];
    if ((int)blockIdx.x < request_groups) {
        if (r < p.requests) {
            const Plan q = p.plan[r];
            if (p.parents != nullptr) tree(p, r, q, step[0], p.offsets[r], p.offsets[r + 1] - p.offsets[r], lane);
            pop(p, r, q, step[0], lane);
        }
        pad(p, step[2] + (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)request_groups * 256);
        if (blockIdx.x == 0 && threadIdx.x == 0) *p.free_count = step[0] - step[1];
        return;
    }
    const int64_t t = (int64_t)((int)blockIdx.x - request_groups) * 256 + threadIdx.x;
    for (int i = threadIdx.x; i <= p.requests; i += 256) begin[i] = p.offsets[i];
    __syncthreads();
    if (t >= step[2]) return;
    const int of = owner_of(begin, p.requests, t), n = p.lens[of];
    const int64_t pos = (int64_t)(n > 0 ? n : 0) + (t - begin[of]);
    write_token(p, (int)t, slot_of(p, of, p.plan[of], step[0], pos), pos);
}

}  // namespace
}  // namespace gba

using namespace gba;

extern "C" gba_status gba_tables_step(const gba_block_tables *b, const int32_t *lens, const int32_t *count,
                                      const int32_t *parents, int64_t tokens, int32_t *offsets, int32_t *slots,
                                      int32_t *positions, int32_t *status, uint64_t *mask, gba_stream_t stream)
{
    if (b == nullptr || b->requests < 0 || b->width < 0 || b->num_blocks < 0 || b->block_size < 1 || tokens < 0)
        return GBA_EINVAL;
    if (b->requests > GBA_MAX_REQUESTS || b->width > INT_MAX || b->num_blocks > INT_MAX || b->block_size > INT_MAX ||
        tokens > INT_MAX || b->requests * b->width > INT_MAX || b->num_blocks * b->block_size > INT_MAX)
        return GBA_EUNSUPPORTED;
    if (parents != nullptr && mask == nullptr) return GBA_EINVAL;
    if (b->requests == 0) return GBA_OK;
    if ((b->width > 0 && b->table == nullptr) || b->held == nullptr || (b->num_blocks > 0 && b->free_blocks == nullptr) ||
        b->free_count == nullptr || b->scratch == nullptr || lens == nullptr || count == nullptr || offsets == nullptr || status == nullptr)
        return GBA_EINVAL;
    const void *ints[] = {b->table, b->held, b->free_blocks, b->free_count, lens, count, parents, offsets, slots, positions, status};
    for (const void *x : ints)
        if (!aligned_to(x, 4)) return GBA_EUNSUPPORTED;
    if (!aligned_to(mask, 8) || !aligned_to(b->scratch, 16)) return GBA_EUNSUPPORTED;
    TableArgs a;
    a.table = b->table;
    a.held = b->held;
    a.free_blocks = b->free_blocks;
    a.free_count = b->free_count;
    a.lens = lens;
    a.count = count;
    a.parents = parents;
    a.offsets = offsets;
    a.slots = slots;
    a.positions = positions;
    a.status = status;
    a.mask = mask;
    a.plan = reinterpret_cast<Plan *>(b->scratch);
    a.requests = (int)b->requests;
    a.width = (int)b->width;
    a.num_blocks = (int)b->num_blocks;
    a.block_size = (int)b->block_size;
    a.tokens = (int)tokens;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (b->requests <= (parents != nullptr ? SMALL_TREES : SMALL_REQUESTS) && tokens <= SMALL_TOKENS)
        return launch(small_kernel, dim3(1), dim3(b->requests <= 4 && tokens <= 256 ? 256 : TABLE_THREADS), s, a);
    const int threads = b->requests <= 256 ? 256 : TABLE_THREADS;
    const gba_status st = launch(push_kernel, dim3((unsigned)div_up(b->requests, threads / 64)), dim3(threads), s, a);
    if (st != GBA_OK) return st;
    const int groups = (int)div_up(b->requests, 4);
    return launch(pop_kernel, dim3((unsigned)(groups + (parents != nullptr ? 0 : div_up(tokens, 256)))), dim3(256), s, a, groups);
}
