// gba_tables.hip -- block tables and slot maps of a step, from the requests'
// lengths, on the GPU.
//
// Three running sums over the requests say everything: of the blocks given
// back, of the blocks wanted and of the new tokens.  Block i given back and
// block j handed out then find their request by a search in those sums, so
// all of them move in parallel, and what happens does not depend on the order
// of the threads.  The first kernel is one workgroup (the stack is pushed
// before it is popped); the second one writes what belongs to each token.
#include "gba_decode.hpp"

namespace gba {
namespace {

constexpr int TABLE_THREADS = 1024;
constexpr int PER_THREAD = GBA_MAX_REQUESTS / TABLE_THREADS;

struct TableArgs {
    int32_t *table, *held, *free_blocks, *free_count;
    const int32_t *lens, *count, *parents;
    int32_t *offsets, *slots, *positions, *status;
    uint64_t *mask;
    int requests, width, num_blocks, block_size, tokens;
};

// Exclusive running sum over the workgroup's threads; total for every thread.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *scratch, int64_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = v;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) scratch[wave] = x;
    __syncthreads();
    int64_t before = 0;
    total = 0;
    for (int w = 0; w < TABLE_THREADS / 64; ++w) {
        if (w < wave) before += scratch[w];
        total += scratch[w];
    }
    return before + x - v;
}

__global__ void __launch_bounds__(TABLE_THREADS) tables_kernel(TableArgs p)
{
    __shared__ int32_t need_of[GBA_MAX_REQUESTS], held_of[GBA_MAX_REQUESTS];
    __shared__ int32_t back[GBA_MAX_REQUESTS + 1], want[GBA_MAX_REQUESTS + 1];  // running sums
    __shared__ int64_t scratch[TABLE_THREADS / 64];
    const int R = p.requests, W = p.width, first = threadIdx.x * PER_THREAD;
    int fc = *p.free_count;
    fc = fc < 0 ? 0 : fc > p.num_blocks ? p.num_blocks : fc;

    int state[PER_THREAD], wants[PER_THREAD], backs[PER_THREAD];
    int64_t fresh[PER_THREAD], sum_fresh = 0, total;
    for (int i = 0; i < PER_THREAD; ++i) {
        const int r = first + i;
        const int n = r < R ? p.count[r] : 0;
        fresh[i] = n > 0 ? n : 0;
        sum_fresh += fresh[i];
    }
    int64_t at = block_scan(sum_fresh, scratch, total);
    int64_t sum_back = 0, sum_want = 0;
    for (int i = 0; i < PER_THREAD; ++i) {
        const int r = first + i;
        state[i] = wants[i] = backs[i] = 0;
        if (r < R) {
            const int n = p.lens[r];
            const int64_t need = (((int64_t)(n > 0 ? n : 0) + fresh[i]) + p.block_size - 1) / p.block_size;
            int held = p.held[r];
            held = held < 0 ? 0 : held > W ? W : held;
            p.offsets[r] = (int32_t)(at < p.tokens ? at : p.tokens);
            at += fresh[i];
            if (need > W) state[i] = 2;
            else if (at > p.tokens || (p.parents != nullptr && fresh[i] > 64)) state[i] = 3;
            if (need < held) backs[i] = held - (int)need;
            else if (state[i] == 0) wants[i] = (int)need - held;
            need_of[r] = (int)(need < W ? need : W);
            held_of[r] = held;
        }
        sum_back += backs[i];
        sum_want += wants[i];
    }
    if (threadIdx.x == 0) p.offsets[R] = (int32_t)(total < p.tokens ? total : p.tokens);
    int64_t total_back, total_want;
    int64_t b = block_scan(sum_back, scratch, total_back), w = block_scan(sum_want, scratch, total_want);
    for (int i = 0; i < PER_THREAD; ++i) {
        back[first + i] = (int32_t)b;
        want[first + i] = (int32_t)w;
        b += backs[i];
        w += wants[i];
    }
    if (threadIdx.x == TABLE_THREADS - 1) {
        back[GBA_MAX_REQUESTS] = (int32_t)b;
        want[GBA_MAX_REQUESTS] = (int32_t)w;
    }
    __syncthreads();

    // blocks given back, onto the stack
    for (int64_t i = threadIdx.x; i < total_back; i += TABLE_THREADS) {
        const int r = owner_of(back, R, i);
        int32_t *entry = p.table + (int64_t)r * W + need_of[r] + (i - back[r]);
        if (fc + i < p.num_blocks) p.free_blocks[fc + i] = *entry;
        *entry = -1;
    }
    __syncthreads();

    // blocks handed out, from its top: to the requests whose running sum fits
    const int64_t avail = fc + total_back;
    const int first_short = owner_of(want, R, avail);  // the first one whose sum passes avail
    const int64_t given = want[first_short];
    for (int64_t i = threadIdx.x; i < given; i += TABLE_THREADS) {
        const int r = owner_of(want, R, i);
        const int64_t from = avail - 1 - i;
        p.table[(int64_t)r * W + held_of[r] + (i - want[r])] = from < p.num_blocks ? p.free_blocks[from] : -1;
    }
    for (int i = 0; i < PER_THREAD; ++i) {
        const int r = first + i;
        if (r >= R) break;
        if (wants[i] > 0 && r >= first_short) {
            state[i] = 1;
            wants[i] = 0;
        }
        p.held[r] = held_of[r] - backs[i] + wants[i];
        if (p.status != nullptr) p.status[r] = state[i];
    }
    if (threadIdx.x == 0) *p.free_count = (int32_t)(avail - given);
}

__device__ __forceinline__ int slot_of(const TableArgs &p, int r, int64_t pos)
{
    const int64_t column = pos / p.block_size;
    if (column >= p.width) return -1;
    // an entry is missing where the request got no blocks
    const int entry = column < p.held[r] ? p.table[(int64_t)r * p.width + column] : -1;
    return entry < 0 ? -1 : (int)((int64_t)entry * p.block_size + (pos - column * p.block_size));
}

// Chains: one thread a token.
__global__ void __launch_bounds__(256) chain_kernel(TableArgs p)
{
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= p.tokens) return;
    const int r = owner_of(p.offsets, p.requests, t);
    int64_t pos = -1;
    int slot = -1;
    if (r < p.requests) {
        const int n = p.lens[r];
        pos = (int64_t)(n > 0 ? n : 0) + (t - p.offsets[r]);
        if (p.status[r] == 0) slot = slot_of(p, r, pos);
    }
    if (p.slots != nullptr) p.slots[t] = slot;
    if (p.positions != nullptr) p.positions[t] = (int32_t)pos;
}

// Trees: one wave a request, one lane a token.  A token's mask is its own bit
// and those of its ancestors, found by doubling: six rounds in which every
// token takes the mask of the token it points to and then points to where
// that one points.
__global__ void __launch_bounds__(256) tree_kernel(TableArgs p)
{
    const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r < p.requests) {
        const int first = p.offsets[r], T = p.offsets[r + 1] - first;
        const int n = p.lens[r], status = p.status[r];
        if (T <= 64) {
            const int parent = lane < T ? p.parents[first + lane] : -1;
            int up = parent >= 0 && parent < lane ? parent : lane;
            uint64_t mask = 1ull << lane;
            for (int i = 0; i < 6; ++i) {
                mask |= __shfl(mask, up);
                up = __shfl(up, up);
            }
            if (lane < T) {
                const int64_t kept = n > 0 ? n : 0;
                if (p.slots != nullptr) p.slots[first + lane] = status == 0 ? slot_of(p, r, kept + lane) : -1;
                if (p.positions != nullptr) p.positions[first + lane] = (int32_t)(kept + __popcll(mask) - 1);
                p.mask[first + lane] = mask;
            }
        } else {
            for (int i = lane; i < T; i += 64) {
                if (p.slots != nullptr) p.slots[first + i] = -1;
                if (p.positions != nullptr) p.positions[first + i] = -1;
                p.mask[first + i] = 0;
            }
        }
    }
    for (int64_t t = p.offsets[p.requests] + (int64_t)blockIdx.x * 256 + threadIdx.x; t < p.tokens; t += (int64_t)gridDim.x * 256) {
        if (p.slots != nullptr) p.slots[t] = -1;
        if (p.positions != nullptr) p.positions[t] = -1;
        p.mask[t] = 0;
    }
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
        b->free_count == nullptr || lens == nullptr || count == nullptr || offsets == nullptr || status == nullptr)
        return GBA_EINVAL;
    const void *ints[] = {b->table, b->held, b->free_blocks, b->free_count, lens, count, parents, offsets, slots, positions, status};
    for (const void *x : ints)
        if (!aligned_to(x, 4)) return GBA_EUNSUPPORTED;
    if (!aligned_to(mask, 8)) return GBA_EUNSUPPORTED;
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
    a.requests = (int)b->requests;
    a.width = (int)b->width;
    a.num_blocks = (int)b->num_blocks;
    a.block_size = (int)b->block_size;
    a.tokens = (int)tokens;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const gba_status st = launch(tables_kernel, dim3(1), dim3(TABLE_THREADS), s, a);
    if (st != GBA_OK || tokens == 0) return st;
    if (parents != nullptr) return launch(tree_kernel, dim3((unsigned)div_up(b->requests, 4)), dim3(256), s, a);
    return launch(chain_kernel, dim3((unsigned)div_up(tokens, 256)), dim3(256), s, a);
}
