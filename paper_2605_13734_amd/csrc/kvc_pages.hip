// A step of the cache's sequences: their lengths, the starts, positions and slots of their new rows, and the pages that they take from the
// free ones or give back, from the tokens that they hold, keep and get.
//
// Everything is a few integers per sequence and a few words per page and row, so a call is bound by latency: one launch, in which every
// workgroup makes the running sums over all sequences for itself (in LDS) and then does its share of the rows and pages.  The
// numbers of the caller that change (held tokens, the free pages' count) are written by the workgroup that is done last, when no other
// reads them any more.
//
// Pages given back and pages taken meet in one list: the free stack and above it the given ones, the last given lowest.  The i-th page
// taken is the i-th from its top: given page i, and with no given ones left the stack's own downwards.  So a call either reads the
// stack or pushes onto it, and two calls that take and give back the same restore it.
#include "kvc_prompt_internal.h"
#include "../../include/kvc.h"

namespace kvc {

// The running sums stop here: more than any number of rows or pages that a call may have, so that a sum that has stopped fits none.
constexpr uint32_t kTop = 0x80000000u;

__device__ __forceinline__ uint32_t add_up(uint32_t a, uint32_t b)
{
    const uint32_t sum = __builtin_elementwise_add_sat(a, b);
    return sum < kTop ? sum : kTop;
}
// A sum as the largest word that callers have for it.
__device__ __forceinline__ int word_of(uint32_t sum) { return sum < kTop ? (int)sum : 0x7fffffff; }

template <int CONTROL, int ROWS = 0xf> __device__ __forceinline__ uint32_t from_lane(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, ROWS, 0xf, true);
}
// Sum of x over the workgroup's threads before this one; total: over all.
template <int THREADS> __device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t &total)
{
    uint32_t sum = x;                        // (lanes without a partner get zero)
    sum = add_up(sum, from_lane<0x111>(sum));          // 1, 2, 4, 8 lanes before in the row of 16
    sum = add_up(sum, from_lane<0x112>(sum));
    sum = add_up(sum, from_lane<0x114>(sum));
    sum = add_up(sum, from_lane<0x118>(sum));
    sum = add_up(sum, from_lane<0x142, 0xa>(sum));     // the last lane of the first and third row for the rows behind them
    sum = add_up(sum, from_lane<0x143, 0xc>(sum));     // that of the second for the third and fourth
    const uint32_t mine = from_lane<0x138>(sum);       // one lane before in the wave
    if constexpr (THREADS == 64) {
        total = (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
        return mine;
    } else {
        __shared__ uint32_t waves[THREADS / 64];
        __syncthreads();                     // (the words may still be read for another sum)
        if (lane_id() == 63) waves[wave_id()] = sum;
        __syncthreads();
        uint32_t before = 0;
        total = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w == wave_id()) before = total;
            total = add_up(total, waves[w]);
        }
        return add_up(before, mine);
    }
}

// The last place whose running sum is not above x (sums[0] = 0, x < sums[n]).
__device__ __forceinline__ int place_of(const uint32_t *sums, int n, uint32_t x)
{
    int low = 0, high = n;
    while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (sums[mid] <= x) low = mid;
        else high = mid;
    }
    return low;
}

struct Step {
    int held, kept, fresh;
    bool fits;                               // (but for the rows' room and the pages)
};
__device__ __forceinline__ Step step_of(const AdvanceArgs &a, int s)
{
    Step t;
    t.held = a.held[s];
    t.kept = a.kept ? a.kept[s] : t.held;
    t.fresh = a.fresh ? a.fresh[s] : 0;
    t.fits = t.kept >= 0 && t.kept <= t.held && t.held <= a.max_tokens && t.fresh >= 0 && t.fresh <= a.max_new &&
             (long long)t.kept + t.fresh <= a.max_tokens;
    return t;
}

// THREADS of a workgroup, which have EACH sequences at most.
template <int THREADS, int EACH> __global__ __launch_bounds__(THREADS) void advance_kernel(AdvanceArgs a)
{
    constexpr int kMost = THREADS * EACH;
    // per sequence: sums before it, tokens kept (-1: it is left out), pages held before
    __shared__ uint32_t start[kMost + 1], takes[kMost + 1], gives[kMost + 1];
    __shared__ int kept[kMost], held_pages[kMost];
    __shared__ uint32_t taken;
    __shared__ int last;
    const int tid = threadIdx.x, each = (a.n + THREADS - 1) / THREADS;
    const bool first = blockIdx.x == 0;
    int count = a.free_pages[0];
    count = count < 0 ? 0 : count > a.num_pages ? a.num_pages : count;
    auto pages = [&](int tokens) { return (int)(((long long)tokens + (1 << a.page_shift) - 1) >> a.page_shift); };

    Step mine[EACH];
    uint32_t sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int s = tid * each + i;
        mine[i] = Step{0, 0, 0, false};
        if (i < each && s < a.n) {
            mine[i] = step_of(a, s);
            sum = add_up(sum, (unsigned)mine[i].fresh <= (unsigned)a.max_new ? mine[i].fresh : 0);
        }
    }
    uint32_t total_rows, total_takes, total_gives;
    uint32_t row = sum_before<THREADS>(sum, total_rows);
    uint32_t take = 0, give = 0;
    if (tid == 0) taken = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int s = tid * each + i;
        if (i < each && s < a.n) {
            start[s] = row;
            if (first) a.new_start[s] = word_of(row);
            row = add_up(row, (unsigned)mine[i].fresh <= (unsigned)a.max_new ? mine[i].fresh : 0);
            mine[i].fits = mine[i].fits && (long long)row <= a.rows;
            if (mine[i].fits) {
                const int now = pages(mine[i].kept + mine[i].fresh), before = pages(mine[i].held);
                take = add_up(take, now > before ? now - before : 0);
                give = add_up(give, before > now ? before - now : 0);
            }
        }
    }
    uint32_t my_take = sum_before<THREADS>(take, total_takes), my_give = sum_before<THREADS>(give, total_gives);
    if (tid == 0) {
        start[a.n] = total_rows;
        takes[a.n] = total_takes;
        gives[a.n] = total_gives;
        if (first) a.new_start[a.n] = word_of(total_rows);
    }
    const uint32_t room = add_up((uint32_t)count, total_gives);
    int after[EACH];                         // tokens that are held afterwards
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int s = tid * each + i;
        if (i < each && s < a.n) {
            takes[s] = my_take;
            gives[s] = my_give;
            int report = KVC_DEV_BAD_ROW;
            bool done = mine[i].fits;
            const int before = pages(mine[i].held);
            if (done) {
                const int now = pages(mine[i].kept + mine[i].fresh);
                my_take = add_up(my_take, now > before ? now - before : 0);
                my_give = add_up(my_give, before > now ? before - now : 0);
                if (now > before) {
                    done = my_take <= room && my_take < kTop;
                    if (done) atomicMax(&taken, my_take);
                    else report = KVC_DEV_NO_PAGE;
                }
            }
            held_pages[s] = before;
            kept[s] = done ? mine[i].kept : -1;
            after[i] = done ? mine[i].kept + mine[i].fresh : mine[i].held;
            if (first) {
                a.tokens[s] = done ? after[i] : -1;
                if (!done) atomicOr(a.status + s, report);
            }
        }
    }
    __syncthreads();
    total_takes = taken;

    // page i of those taken (or, beyond them, of those given); who: the sequence that it is reported for
    auto page_taken = [&](uint32_t i, int who) {
        int page = -1;
        if (i < total_gives) {
            const int s = place_of(gives, a.n, i);
            // (the places behind the pages that it keeps)
            page = a.block_table[s * a.table_stride + held_pages[s] - (int)(gives[s + 1] - i)];
        } else if (i - total_gives < (uint32_t)count) page = a.free_pages[4 + count - 1 - (int)(i - total_gives)];
        if ((unsigned)page < (unsigned)a.num_pages) return page;
        atomicOr(a.status + who, KVC_DEV_BAD_BLOCK);
        return -1;
    };
    const long long at = (long long)blockIdx.x * THREADS + tid, stride = (long long)gridDim.x * THREADS;
    for (long long i = at; i < total_takes; i += stride) {
        const int s = place_of(takes, a.n, (uint32_t)i);
        a.block_table[s * a.table_stride + held_pages[s] + (i - takes[s])] = page_taken((uint32_t)i, s);
    }
    // what is left of the given ones (more than the pool has: the first are dropped)
    const long long dropped = (long long)count + total_gives - a.num_pages;
    for (long long i = (dropped > (long long)total_takes ? dropped : (long long)total_takes) + at; i < total_gives; i += stride)
        a.free_pages[4 + count + ((long long)total_gives - 1 - i)] = page_taken((uint32_t)i, place_of(gives, a.n, (uint32_t)i));
    if (a.positions || a.slots) {
        for (long long r = at; r < a.rows; r += stride) {
            int position = -1;
            long long slot = -1;
            if (r < total_rows) {
                const int s = place_of(start, a.n, (uint32_t)r), old = kept[s];
                if (old >= 0) {
                    position = old + (int)(r - start[s]);
                    if (a.slots) {
                        const int place = position >> a.page_shift, before = held_pages[s];
                        const int page = place < before ? a.block_table[s * a.table_stride + place] : page_taken(takes[s] + (place - before), s);
                        if ((unsigned)page < (unsigned)a.num_pages)
                            slot = ((long long)page << a.page_shift) + (position & ((1 << a.page_shift) - 1));
                        else atomicOr(a.status + s, KVC_DEV_BAD_BLOCK);
                    }
                }
            }
            if (a.positions) a.positions[r] = position;
            if (a.slots) a.slots[r] = slot;
        }
    }

    // the workgroup that is done last: all others have read what changes now (nothing that they have written is read here, so no fence
    // has to write back their L2s)
    if (gridDim.x > 1) {
        __syncthreads();
        if (tid == 0) last = atomicAdd(a.free_pages + 1, 1) == (int)gridDim.x - 1;
        __syncthreads();
        if (!last) return;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int s = tid * each + i;
        if (i < each && s < a.n) a.held[s] = after[i];
    }
    if (tid == 0) {
        const long long now = (long long)count + total_gives - total_takes;
        a.free_pages[0] = (int)(now < a.num_pages ? now : a.num_pages);
        if (gridDim.x > 1) a.free_pages[1] = 0;
    }
}

// Rows of positions and slots, or pages, that there may be, are divided among workgroups.  One wave alone makes the sums fastest: a step of 32
// sequences and back 6.6 us in a graph, 11.9 with 1024 threads.  One token each and back for 256 sequences 9.3 us, 1024 14.3, 1025 14.1, 2048 15.9,
// 4096 22.0.
template <int THREADS, int EACH> static void launch_threads(const AdvanceArgs &a, long long items, hipStream_t stream)
{
    const long long groups = (items + THREADS - 1) / THREADS;
    advance_kernel<THREADS, EACH><<<(int)(groups < 1 ? 1 : groups > 256 ? 256 : groups), THREADS, 0, stream>>>(a);
}
void launch_advance(const AdvanceArgs &a, hipStream_t stream)
{
    long long items = a.rows;
    if (!a.positions && !a.slots) {
        const long long rows = (long long)a.n * a.max_new;
        items = ((rows < a.rows ? rows : a.rows) >> a.page_shift) + a.n;
    }
    if (a.n <= 64 && items <= 64) launch_threads<64, 1>(a, items, stream);
    else if (a.n <= 1024) launch_threads<256, 4>(a, items, stream);
    else launch_threads<1024, KVC_MOST_ADVANCING / 1024>(a, items, stream);
}

}  // namespace kvc
