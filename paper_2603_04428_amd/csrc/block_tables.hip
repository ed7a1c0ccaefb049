// Block tables that live on the GPU: lengths of many rows changed at once, with the slots of the tokens that came in
// (q4kv_resize_tables), and rows that become copies of other rows (q4kv_beam_reorder).
//
// The state is a count per block: how many rows list it.  A block of count 0 is free; free blocks are handed out lowest id first,
// to rows in order, so that every result follows from the arguments alone (counts go up and down by atomics, whose order does not
// show).  The bookkeeping is a chain of prefix sums over at most 2,048 rows with a trip to memory between them: one workgroup,
// two rows a lane, sums in registers and LDS, no launch in between.  What it has to read beside the rows are the counts, in order until
// enough free ones are found.  Work of uneven size per row (blocks freed, blocks taken, tokens mapped) is laid out flat and the row
// of an item found by bisection in the prefix sums.
//
// Measured (kernel times): 40 rows a token longer 4.1 us, back 3.3; 500 rows of 15,500 blocks with 2,800 tokens mapped 8.1, back 4.7; 400
// prompts of 299,000 tokens admitted 6.2 and their map 4.4, released 5.5; rows of 4, 40 and 64 beams gathered 6.7, 8.2 and 8.2.  A wide call's
// time stamps (10,700 clocks) lie 600 to 2,100 clocks apart: no step of it is long, and none can begin before the one in front of it has ended.
// What is done where rows are refused or share their last blocks stands beside the straight path, not in a loop around it: in a loop
// the same calls took 0.2 us longer.
//
// A block in which a row ends and that others list too is copied by a kernel of its own (the pools of all layers; HBM-bound).
#include "q4_device.h"
#include "q4kv_internal.h"

namespace q4kv {
namespace {

constexpr int kRows = Q4KV_MAX_TABLE_ROWS;
constexpr int kWide = 1024, kNarrow = 256; // threads of a workgroup: kThreads of the functions below
constexpr int kPer = kRows / kWide;         // rows of a lane: consecutive ones
constexpr int kFree = 4096;            // free blocks kept in LDS; a call that takes more reads the counts twice
constexpr int kHash = 2 * kRows;       // places for the shared blocks that rows end in
constexpr int kRefs = 4;               // counts a lane reads at a time: 16 bytes, consecutive lanes consecutive ones

// Blocks to copy: counts[0] pairs; then sources, destinations, tokens.
struct Moves {
    int32_t *count, *src, *dst, *tokens;
};

struct TablesParams {
    int32_t *table, *len, *refs, *refused;
    int32_t agents, max_blocks, num_blocks;
    const int32_t *new_len; // resize
    const int32_t *parent;  // reorder
    int32_t max_tokens;
    int32_t *token_begin, *slot, *token_agent, *position;
    Moves moves;
    bool copies;  // shared blocks can be copied
    bool map_here; // the slot map is written by the same workgroup
};

struct Shared {
    int32_t before[kRows], after[kRows]; // lengths
    uint32_t items[kRows + 1];           // first item of a row: blocks freed, then blocks taken
    uint32_t tokens[kRows + 1];
    uint8_t copy[kRows];
    int32_t free[kFree];
    int32_t key[kHash], lowest[kHash], rows[kHash], left[kHash];
    uint32_t wave[10][kWide / kWave]; // what the waves tell each other, by the place that asks: one barrier each
    int32_t first_refused, moves, refused;
};
enum Place { kGone, kGoneSum, kWidest, kShared, kNeed, kMore, kBehind, kOver, kFound }; // kFound and the one behind it in turns

__device__ __forceinline__ int blocks_of(int tokens) { return (tokens >> 8) + ((tokens & 255) != 0); }
__device__ __forceinline__ uint32_t sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Counts of blocks.  A kernel of one workgroup has them to itself; where several share a table's columns they meet in memory.
template <bool ALONE>
__device__ __forceinline__ void count(int32_t *ref, int32_t by)
{
    (void)__hip_atomic_fetch_add(ref, by, __ATOMIC_RELAXED, ALONE ? __HIP_MEMORY_SCOPE_WORKGROUP : __HIP_MEMORY_SCOPE_AGENT);
}

// v and the sum of v over the lanes below, in steps of the data-parallel-primitive moves; sums that pass 32 bits stay at the top
__device__ __forceinline__ uint32_t wave_scan(uint32_t v)
{
#define Q4KV_SCAN_STEP(CTRL, ROWS) v = sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, (CTRL), (ROWS), 0xF, false))
    Q4KV_SCAN_STEP(0x111, 0xF); // row_shr 1, 2, 4, 8
    Q4KV_SCAN_STEP(0x112, 0xF);
    Q4KV_SCAN_STEP(0x114, 0xF);
    Q4KV_SCAN_STEP(0x118, 0xF);
    Q4KV_SCAN_STEP(0x142, 0xA); // row_bcast15 into rows 1 and 3
    Q4KV_SCAN_STEP(0x143, 0xC); // row_bcast31 into rows 2 and 3
#undef Q4KV_SCAN_STEP
    return v;
}

// Exclusive prefix sum of a number over the lanes of the workgroup out of its sum within the wave, and its total; behind a barrier
// between the waves' writing of s.wave[place] and here.
__device__ __forceinline__ void tell(Shared &s, int place, uint32_t v) { s.wave[place][threadIdx.x >> 6] = v; }
template <int kThreads>
__device__ __forceinline__ uint32_t told(const Shared &s, int place)
{
    const int lane = threadIdx.x & 63;
    return lane < kThreads / kWave ? s.wave[place][lane] : 0u;
}
template <int kThreads>
__device__ __forceinline__ uint32_t prefix(const Shared &s, int place, uint32_t inclusive, uint32_t &all)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t totals = wave_scan(told<kThreads>(s, place)); // the waves' totals in the lanes of every wave
    all = (uint32_t)__builtin_amdgcn_readlane((int)totals, kThreads / kWave - 1);
    const uint32_t below = wave ? (uint32_t)__builtin_amdgcn_readlane((int)totals, wave - 1) : 0u;
    return sat(below, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)inclusive, 0x138, 0xF, 0xF, false)); // wave_shr 1
}
template <int kThreads>
__device__ __forceinline__ uint32_t scan(Shared &s, int place, uint32_t v, uint32_t &all)
{
    const uint32_t inclusive = wave_scan(v);
    if ((threadIdx.x & 63) == 63) tell(s, place, inclusive);
    __syncthreads();
    return prefix<kThreads>(s, place, inclusive, all);
}
// Whether any lane of the workgroup says so.
template <int kThreads>
__device__ __forceinline__ bool any_of(Shared &s, int place, bool v)
{
    const bool here = __any(v);
    if ((threadIdx.x & 63) == 0) tell(s, place, here);
    __syncthreads();
    return __any(told<kThreads>(s, place) != 0);
}

// The row that item i belongs to: the last whose first item is not behind i.
__device__ __forceinline__ int row_of(const uint32_t *first, int rows, uint32_t i)
{
    int lo = 0, hi = rows;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

// What a lane reads of the counts: kRefs from `at` on, and bit i set where count i is 0.
struct Counts {
    int4 c;
};
__device__ __forceinline__ Counts counts_at(const TablesParams &p, int64_t at)
{
    Counts k;
    if (__builtin_expect(at + kRefs <= p.num_blocks, 1)) {
        k.c = *reinterpret_cast<const int4 *>(p.refs + at);
    } else {
        auto one = [&](int64_t i) { return i < p.num_blocks ? p.refs[i] : 1; }; // behind the last: taken
        k.c = make_int4(one(at), one(at + 1), one(at + 2), one(at + 3));
    }
    return k;
}
__device__ __forceinline__ uint32_t free_bits(const Counts &k)
{
    return (uint32_t)(k.c.x == 0) | (uint32_t)(k.c.y == 0) << 1 | (uint32_t)(k.c.z == 0) << 2 | (uint32_t)(k.c.w == 0) << 3;
}

// A free block becomes item i of the rows' items.
__device__ __forceinline__ void take_block(const TablesParams &p, Shared &s, uint32_t i, int32_t id)
{
    const int r = row_of(s.items, p.agents, i), at = min(s.before[r], s.after[r]);
    const int k = (int)(i - s.items[r]);
    int32_t *row = p.table + (int64_t)r * p.max_blocks;
    p.refs[id] = 1;
    if (s.copy[r] && k == 0) {
        const int32_t src = row[at >> 8];
        row[at >> 8] = id;
        const int m = atomicAdd(&s.moves, 1);
        p.moves.src[m] = src;
        p.moves.dst[m] = id;
        p.moves.tokens[m] = at & 255;
    } else {
        row[blocks_of(s.before[r]) + k - s.copy[r]] = id;
    }
}

// Lane's rows kPer t .. : lengths from `before` (blocks up to there are listed) to `after`; rows that get shorter have given their
// blocks back.  Finds the blocks that rows end in and share, takes free blocks, writes lengths and the map's bounds.
//
// Rows are served in order.  The first growing row that finds too few blocks or places in the map ends that for growing rows; what
// it and those behind it would have taken is there for the copies of rows that do not grow, as long as blocks last.  Of those
// a row that was cut, or that a reorder made, loses what it has of a block for which there is no copy, and any other stays in it.
// GROWS: of a resize; a reorder's rows have their lengths, before and after are the same.
template <int kThreads, bool GROWS>
__device__ __forceinline__ void settle(const TablesParams &p, Shared &s, const int (&before)[kPer], int (&after)[kPer], int refused)
{
    const int t = threadIdx.x;
    Counts counts = counts_at(p, (int64_t)t * kRefs); // on their way while rows are looked at
    bool shared[kPer], copy[kPer], keeps[kPer]; // keeps: grows, and is the row that goes on in a block of several
    int32_t last[kPer];
    int32_t listed[kPer];
    int place[kPer];
    bool any = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = kPer * t + i, at = min(before[i], after[i]);
        shared[i] = copy[i] = keeps[i] = false;
        last[i] = -1;
        place[i] = 0;
        if (r < p.agents && (at & 255) && (p.copies || after[i] < before[i])) {
            last[i] = p.table[(int64_t)r * p.max_blocks + (at >> 8)];
            if ((uint32_t)last[i] < (uint32_t)p.num_blocks) {
                listed[i] = p.refs[last[i]];
                shared[i] = listed[i] > 1;
            }
        }
        any |= shared[i];
    }
    if (t == 0) {
        s.moves = 0;
        s.refused = 0;
        s.first_refused = p.agents;
    }
    const bool sharing = any_of<kThreads>(s, kShared, any);
    if (__builtin_expect(sharing, 0)) {
        int places = 64; // twice as many as rows
        while (places < 2 * p.agents) places <<= 1;
        for (int i = t; i < places; i += kThreads) {
            s.key[i] = -1;
            s.lowest[i] = kRows;
            s.rows[i] = s.left[i] = 0;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!shared[i]) continue;
            int h = (int)(((uint32_t)last[i] * 2654435769u) >> 20) & (places - 1);
            while (true) { // at most as many keys as rows
                const int32_t was = atomicCAS(&s.key[h], -1, last[i]);
                if (was == -1 || was == last[i]) break;
                h = (h + 1) & (places - 1);
            }
            atomicMin(&s.lowest[h], kPer * t + i);
            atomicAdd(&s.rows[h], 1);
            place[i] = h;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!shared[i]) continue;
            copy[i] = !(s.lowest[place[i]] == kPer * t + i && s.rows[place[i]] == listed[i]);
            keeps[i] = !copy[i] && after[i] > before[i];
        }
    }
    uint32_t need[kPer], more[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (copy[i] && !p.copies) { // cut inside a shared block, and nothing to copy it with
            const int r = kPer * t + i;
            count<true>(&p.refs[last[i]], -1);
            p.table[(int64_t)r * p.max_blocks + (after[i] >> 8)] = -1;
            after[i] &= ~255;
            copy[i] = false;
            ++refused;
        }
        need[i] = (uint32_t)copy[i] + (uint32_t)max(0, blocks_of(after[i]) - blocks_of(before[i]));
        more[i] = p.max_tokens > 0 ? (uint32_t)max(0, after[i] - before[i]) : 0u;
    }
    uint32_t found = 0, all_need, all_more;
    uint32_t first_need[kPer], first_more[kPer];
    int64_t base = 0; // counts read up to here
    int turn = 0;
    // Sums of what rows need; free blocks, lowest first, as far as they are needed; the first growing row that cannot be served.
    auto serve = [&]() __attribute__((always_inline)) {
        const uint32_t in_need = wave_scan(sat(need[0], need[1])), in_more = wave_scan(sat(more[0], more[1]));
        if ((t & 63) == 63) {
            tell(s, kNeed, in_need);
            tell(s, kMore, in_more);
        }
        __syncthreads();
        first_need[0] = prefix<kThreads>(s, kNeed, in_need, all_need);
        first_more[0] = prefix<kThreads>(s, kMore, in_more, all_more);
        first_need[1] = sat(first_need[0], need[0]);
        first_more[1] = sat(first_more[0], more[0]);
        if (!(all_need | all_more)) return p.agents; // nobody wants anything
#pragma unroll 1
        for (; base < p.num_blocks && found < all_need; base += kThreads * kRefs) {
            const uint32_t bits = free_bits(counts);
            counts = counts_at(p, base + kThreads * kRefs + (int64_t)t * kRefs);
            uint32_t all;
            uint32_t rank = found + scan<kThreads>(s, kFound + turn, __popc(bits), all);
            turn ^= 1;
#pragma unroll 1
            for (uint32_t b = bits; b && rank < kFree; b &= b - 1, ++rank) s.free[rank] = (int32_t)(base + (int64_t)t * kRefs + __ffs(b) - 1);
            found += all;
        }
        if (!GROWS) return p.agents;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const bool fails = after[i] > before[i] && ((need[i] && sat(first_need[i], need[i]) > found) ||
                                                        (p.max_tokens > 0 && sat(first_more[i], more[i]) > (uint32_t)p.max_tokens));
            if (fails) atomicMin(&s.first_refused, kPer * t + i);
        }
        __syncthreads();
        return s.first_refused;
    };
    int stop = serve();
    const bool wanted = (all_need | all_more) != 0;
    uint32_t taken = min(all_need, found), mapped = all_more; // blocks and places that are given out
    if (GROWS && __builtin_expect(stop < p.agents || (sharing && wanted), 0)) {
#pragma unroll 1
        while (true) {
            // the items and tokens of the rows in front of the refused one, and behind them the copies of rows that do not grow
            uint32_t behind[kPer], all_behind;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = kPer * t + i;
                behind[i] = r > stop && after[i] <= before[i] ? need[i] : 0u;
                if (r == stop) {
                    s.items[p.agents] = min(first_need[i], found);
                    s.tokens[p.agents] = first_more[i];
                }
            }
            const uint32_t ex = scan<kThreads>(s, kBehind, behind[0] + behind[1], all_behind);
            if (stop < p.agents) {
                const uint32_t used = s.items[p.agents];
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (kPer * t + i >= stop) first_need[i] = used + ex + (i ? behind[0] : 0u);
                taken = min(used + all_behind, found);
                mapped = s.tokens[p.agents];
            }
            if (!sharing) break;
            // A row goes on in a block of several only if nobody stays there who has more tokens in it: else it gets a copy as well.
            bool over = false;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const bool served = after[i] > before[i] ? kPer * t + i < stop : first_need[i] < found;
                if (copy[i] && !served && after[i] >= before[i]) atomicMax(&s.left[place[i]], before[i] & 255);
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (!keeps[i] || kPer * t + i >= stop || s.left[place[i]] <= (before[i] & 255)) continue;
                keeps[i] = false;
                copy[i] = over = true;
                ++need[i];
            }
            if (!any_of<kThreads>(s, kOver, over)) break;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (shared[i]) s.left[place[i]] = 0;
            if (t == 0) s.first_refused = p.agents;
            stop = serve();
            taken = min(all_need, found);
            mapped = all_more;
        }
    }
    bool leaves[kPer] = {}; // the block it shared
    if (__builtin_expect(sharing, 0)) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!copy[i]) continue;
            const bool served = GROWS && after[i] > before[i] ? kPer * t + i < stop : first_need[i] < found;
            leaves[i] = served || !GROWS || after[i] < before[i];
            copy[i] = served;
            if (leaves[i] && !served) {
                p.table[(int64_t)(kPer * t + i) * p.max_blocks + (after[i] >> 8)] = -1;
                after[i] &= ~255;
                ++refused;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = kPer * t + i;
        if (r >= p.agents) continue;
        if (GROWS && r >= stop && after[i] > before[i]) { // stays as it was
            ++refused;
            after[i] = before[i];
        }
        p.len[r] = after[i];
        if (wanted) {
            s.before[r] = before[i];
            s.after[r] = after[i];
            s.items[r] = min(first_need[i], taken);
            s.tokens[r] = min(first_more[i], mapped);
            s.copy[r] = copy[i];
        }
    }
    if (refused) atomicAdd(&s.refused, refused);
    if (wanted) __syncthreads();
    uint32_t seen = 0;
    if (__builtin_expect(taken > kFree, 0)) {
        // more than LDS holds: those behind are taken while the counts are read once more (before any of them changes)
#pragma unroll 1
        for (int64_t base = 0; base < p.num_blocks && seen < taken; base += kThreads * kRefs) {
            const uint32_t bits = free_bits(counts_at(p, base + (int64_t)t * kRefs));
            uint32_t all;
            uint32_t rank = seen + scan<kThreads>(s, kFound + turn, __popc(bits), all);
            turn ^= 1;
#pragma unroll 1
            for (uint32_t b = bits; b && rank < taken; b &= b - 1, ++rank)
                if (rank >= kFree) take_block(p, s, rank, (int32_t)(base + (int64_t)t * kRefs + __ffs(b) - 1));
            seen += all;
        }
        __syncthreads();
    }
    for (uint32_t i = t; i < min(taken, (uint32_t)kFree); i += kThreads) take_block(p, s, i, s.free[i]);
    if (__builtin_expect(sharing, 0)) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (leaves[i]) count<true>(&p.refs[last[i]], -1); // behind the last look at the counts: such a block may be free from here on
    }
    if (p.max_tokens > 0) {
        for (int r = t; r < p.agents; r += kThreads) p.token_begin[r] = mapped ? (int32_t)s.tokens[r] : 0;
        if (t == 0) p.token_begin[p.agents] = (int32_t)mapped;
    }
    __syncthreads();
    if (t == 0) {
        if (p.refused) *p.refused = s.refused;
        if (p.copies) *p.moves.count = s.moves;
    }
    if (p.max_tokens > 0 && p.map_here) {
        for (int i = t; i < p.max_tokens; i += kThreads) {
            int32_t slot = -1, agent = -1, position = -1;
            if ((uint32_t)i < mapped) {
                agent = row_of(s.tokens, p.agents, i);
                position = s.before[agent] + (int)(i - s.tokens[agent]);
                const int32_t id = p.table[(int64_t)agent * p.max_blocks + (position >> 8)];
                if ((uint32_t)id < (uint32_t)p.num_blocks) slot = id * kBlockTokens + (position & 255);
            }
            p.slot[i] = slot;
            if (p.token_agent) p.token_agent[i] = agent;
            if (p.position) p.position[i] = position;
        }
    }
}

__device__ __forceinline__ int length_of(const TablesParams &p, int r)
{
    const int64_t most = min((int64_t)p.max_blocks * kBlockTokens, (int64_t)0x7fffffff);
    return (int)min((int64_t)max(p.len[r], 0), most);
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void resize_kernel(TablesParams p)
{
    __shared__ Shared s;
    const int t = threadIdx.x;
    int before[kPer], after[kPer], refused = 0;
    uint32_t gone[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = kPer * t + i;
        before[i] = after[i] = 0;
        if (r < p.agents) {
            before[i] = after[i] = length_of(p, r);
            const int32_t wanted = p.new_len[r];
            if (wanted > (int64_t)p.max_blocks * kBlockTokens) ++refused;
            else if (wanted >= 0) after[i] = wanted;
        }
        gone[i] = (uint32_t)max(0, blocks_of(before[i]) - blocks_of(after[i]));
    }
    if (any_of<kThreads>(s, kGone, (gone[0] | gone[1]) != 0)) {
        uint32_t all;
        const uint32_t ex = scan<kThreads>(s, kGoneSum, sat(gone[0], gone[1]), all);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = kPer * t + i;
            if (r >= p.agents) continue;
            s.items[r] = i == 0 ? ex : sat(ex, gone[0]);
            s.after[r] = after[i];
        }
        __syncthreads();
#pragma unroll 1
        for (uint32_t i = t; i < all; i += kThreads) {
            const int r = row_of(s.items, p.agents, i);
            int32_t *entry = p.table + (int64_t)r * p.max_blocks + blocks_of(s.after[r]) + (i - s.items[r]);
            const int32_t id = *entry;
            if ((uint32_t)id < (uint32_t)p.num_blocks) count<true>(&p.refs[id], -1);
            *entry = -1;
        }
        __syncthreads(); // the counts are read from here on
    }
    settle<kThreads, true>(p, s, before, after, refused);
}

// The map of a call with many tokens, behind resize_kernel.
__global__ __launch_bounds__(256) void slot_map_kernel(TablesParams p)
{
    __shared__ uint32_t s_first[kRows + 1];
    for (int r = threadIdx.x; r <= p.agents; r += 256) s_first[r] = (uint32_t)p.token_begin[r];
    __syncthreads();
    const uint32_t mapped = s_first[p.agents];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.max_tokens; i += (int64_t)gridDim.x * 256) {
        int32_t slot = -1, agent = -1, position = -1;
        if (i < mapped) {
            agent = row_of(s_first, p.agents, (uint32_t)i);
            position = p.len[agent] - (int32_t)(s_first[agent + 1] - (uint32_t)i);
            const int32_t id = p.table[(int64_t)agent * p.max_blocks + (position >> 8)];
            if ((uint32_t)id < (uint32_t)p.num_blocks) slot = id * kBlockTokens + (position & 255);
        }
        p.slot[i] = slot;
        if (p.token_agent) p.token_agent[i] = agent;
        if (p.position) p.position[i] = position;
    }
}

// Rows' entries of a slab of columns become those of their parents.  All of a slab's entries are read before the first is
// written, kHeld a lane; columns have nothing to do with each other, so that any number of workgroups shares the table.
constexpr int kHeld = 8;
template <int kThreads, bool ALONE, int HELD>
__device__ __forceinline__ void gather_slabs(const TablesParams &p, Shared &s, int first_slab, int slabs, int widest, int cols)
{
    const int t = threadIdx.x;
    const int r0 = t / cols, c0 = t - r0 * cols, r_step = kThreads / cols, c_step = kThreads - r_step * cols;
#pragma unroll 1
    for (int64_t slab = (int64_t)first_slab * cols; slab < widest; slab += (int64_t)slabs * cols) {
        int32_t was[HELD], is[HELD], row[HELD], col[HELD];
        int r = r0, c = c0;
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int64_t at = slab + c;
            was[k] = is[k] = row[k] = -1;
            col[k] = (int)at;
            if (r < p.agents && s.key[r] != r) {
                const int64_t from = s.key[r];
                row[k] = at < max(s.before[r], s.after[r]) ? r : -1;
                if (at < s.before[r]) was[k] = p.table[(int64_t)r * p.max_blocks + at];
                if (at < s.after[r]) is[k] = p.table[from * p.max_blocks + at];
            }
            r += r_step;
            c += c_step;
            if (c >= cols) {
                c -= cols;
                ++r;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (row[k] < 0 || (was[k] == is[k] && col[k] < s.before[row[k]])) continue; // equal: the prefix that rows share
            if ((uint32_t)was[k] < (uint32_t)p.num_blocks) count<ALONE>(&p.refs[was[k]], -1);
            if ((uint32_t)is[k] < (uint32_t)p.num_blocks) count<ALONE>(&p.refs[is[k]], 1);
            p.table[(int64_t)row[k] * p.max_blocks + col[k]] = is[k];
        }
    }
}

// Leaves the rows' new lengths in s.items.
template <int kThreads, bool ALONE>
__device__ __forceinline__ void gather_rows(const TablesParams &p, Shared &s, int first_slab, int slabs)
{
    const int t = threadIdx.x;
    int widest = 0; // no row lists more blocks, before or after
    for (int r = t; r < p.agents; r += kThreads) {
        const int32_t from = p.parent[r];
        const bool has = from >= 0 && from < p.agents;
        const int length = has ? length_of(p, from) : 0, before = blocks_of(length_of(p, r)), after = blocks_of(length);
        s.key[r] = has ? from : -1;
        s.before[r] = before;
        s.after[r] = after;
        s.items[r] = (uint32_t)length;
        widest = max(widest, max(before, after));
    }
    // (as binary32: at most 2^23 blocks)
    const float here = wave_max((float)widest);
    if ((t & 63) == 0) tell(s, kWidest, (uint32_t)here);
    __syncthreads();
    widest = (int)wave_max((float)told<kThreads>(s, kWidest));
    const int most = max(1, kThreads * kHeld / p.agents); // columns that fit: at least kHeld / kPer
    const int cols = ALONE ? min(most, max(widest, 1)) : most;
    if ((int64_t)p.agents * cols <= kThreads) gather_slabs<kThreads, ALONE, 1>(p, s, first_slab, slabs, widest, cols);
    else gather_slabs<kThreads, ALONE, kHeld>(p, s, first_slab, slabs, widest, cols);
}

__global__ __launch_bounds__(kWide) void gather_kernel(TablesParams p)
{
    __shared__ Shared s;
    gather_rows<kWide, false>(p, s, blockIdx.x, gridDim.x);
}

template <int kThreads, bool ALONE>
__global__ __launch_bounds__(kThreads) void reorder_kernel(TablesParams p)
{
    __shared__ Shared s;
    int before[kPer], after[kPer];
    if (ALONE) gather_rows<kThreads, true>(p, s, 0, 1);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = kPer * (int)threadIdx.x + i;
        int length = 0;
        if (ALONE) {
            if (r < p.agents) length = (int)s.items[r];
        } else {
            int32_t from = -1;
            if (r < p.agents) from = p.parent[r];
            if (from >= 0 && from < p.agents) length = length_of(p, from);
        }
        before[i] = after[i] = length;
    }
    __syncthreads(); // lengths are read before the first is written, and counts from here on
    settle<kThreads, false>(p, s, before, after, 0);
}

// The first tokens of blocks copied to other blocks, on every layer.  In every (layer, head) plane of a block the tokens of each of
// the six arrays are one run that begins on a multiple of 16 bytes.  A workgroup has a plane and takes pairs in turn, or, where
// there are fewer pairs than workgroups to a plane, a part of a pair; kCopyLoads 16-byte loads per lane of K's and as many of
// V's codes are in flight in front of the first store, and a wave takes one of the four arrays of parameters.
constexpr int kCopyThreads = 256, kCopyLoads = 4;
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));
struct TailParams {
    unsigned char *codes[2], *params[4];
    int32_t code_bytes[2], param_bytes[2]; // of a token in a plane; 0 where there is no V
    int32_t heads, num_blocks;
    Moves moves;
};

__global__ __launch_bounds__(kCopyThreads) void tail_copy_kernel(TailParams p)
{
    const int pairs = *p.moves.count, t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
    if (pairs == 0) return;
    const int layer = blockIdx.x / p.heads, head = blockIdx.x - layer * p.heads;
    const int workers = gridDim.y, parts = max(1, workers / pairs), part = blockIdx.y / pairs;
    if (part >= parts) return;
    const int step = pairs < workers ? pairs : workers;
    for (int pair = blockIdx.y % pairs; pair < pairs; pair += step) {
        const int tokens = p.moves.tokens[pair];
        const int64_t from = ((int64_t)layer * p.num_blocks + p.moves.src[pair]) * p.heads + head;
        const int64_t to = ((int64_t)layer * p.num_blocks + p.moves.dst[pair]) * p.heads + head;
        const u4_t *in[2];
        u4_t *out[2];
        int first[2], end[2]; // granules of 16 bytes
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int64_t plane = (int64_t)p.code_bytes[k] * kBlockTokens;
            const int granules = tokens * (p.code_bytes[k] / 16);
            in[k] = reinterpret_cast<const u4_t *>(p.codes[k] + from * plane);
            out[k] = reinterpret_cast<u4_t *>(p.codes[k] + to * plane);
            first[k] = (int)((int64_t)granules * part / parts);
            end[k] = (int)((int64_t)granules * (part + 1) / parts);
        }
        const int rounds = (max(end[0] - first[0], end[1] - first[1]) + kCopyThreads * kCopyLoads - 1) / (kCopyThreads * kCopyLoads);
        for (int r = 0; r < rounds; ++r) {
            u4_t data[2][kCopyLoads];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < kCopyLoads; ++j) {
                    const int i = first[k] + (r * kCopyLoads + j) * kCopyThreads + t;
                    if (i < end[k]) data[k][j] = in[k][i];
                }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < kCopyLoads; ++j) {
                    const int i = first[k] + (r * kCopyLoads + j) * kCopyThreads + t;
                    if (i < end[k]) out[k][i] = data[k][j];
                }
        }
        const int bytes = tokens * p.param_bytes[wave >> 1];
        if (part == 0 && bytes > 0) {
            const int64_t plane = (int64_t)p.param_bytes[wave >> 1] * kBlockTokens;
            const unsigned char *src = p.params[wave] + from * plane;
            unsigned char *dst = p.params[wave] + to * plane;
            for (int at = lane * 16; at + 16 <= bytes; at += kWave * 16)
                *reinterpret_cast<u4_t *>(dst + at) = *reinterpret_cast<const u4_t *>(src + at);
            const int rest = (bytes & ~15) + lane * 2; // what does not fill a granule, two bytes a lane: what is behind it stays
            if (rest < bytes) *reinterpret_cast<uint16_t *>(dst + rest) = *reinterpret_cast<const uint16_t *>(src + rest);
        }
    }
}

TablesParams params_of(const TablesArgs &a)
{
    TablesParams p = {};
    p.table = a.tables->block_table;
    p.len = a.tables->seq_len;
    p.refs = a.tables->refs;
    p.refused = a.tables->refused;
    p.agents = a.tables->num_agents;
    p.max_blocks = a.tables->max_blocks;
    p.num_blocks = p.agents > 0 ? a.tables->num_blocks : 0; // a table of no rows may come without counts: none is read
    p.copies = a.spec != nullptr;
    if (p.copies) {
        int32_t *w = static_cast<int32_t *>(a.workspace);
        p.moves = Moves{w, w + 64, w + 64 + p.agents, w + 64 + 2 * p.agents};
    }
    return p;
}

// Whether a workgroup of 256 does: its four waves have a SIMD each, the sixteen of a wide one share them, which shows where a call is
// a chain of instructions (resize, 40 rows a token longer: 4.2 us for 4.4, and back 3.2 for 3.8).  Many rows, counts to read or tokens
// to map want more lanes (500 rows, 2,800 tokens: 13.2 for 8.0), and so do more entries to gather than lanes (64 rows of 17 blocks:
// 10.6 for 8.2).
bool narrow(const TablesParams &p)
{
    return p.agents <= kPer * kNarrow && p.num_blocks <= 16 * kNarrow * kRefs && (!p.map_here || p.max_tokens <= 4 * kNarrow);
}

hipError_t launch_tail_copy(const TablesArgs &a, const Moves &moves, hipStream_t stream)
{
    TailParams p = {};
    for (int i = 0; i < (a.v ? 2 : 1); ++i) {
        const q4kv_pool &pool = i ? *a.v : *a.k;
        const int dim = i ? a.spec->v_dim : a.spec->k_dim;
        p.codes[i] = reinterpret_cast<unsigned char *>(pool.codes);
        p.params[2 * i] = reinterpret_cast<unsigned char *>(pool.scale);
        p.params[2 * i + 1] = reinterpret_cast<unsigned char *>(pool.bias);
        p.code_bytes[i] = dim / 2;
        p.param_bytes[i] = dim / kGroup * 2;
    }
    p.heads = a.spec->num_kv_heads;
    p.num_blocks = a.k->num_blocks;
    p.moves = moves;
    // the planes of all layers side by side, and workgroups to a plane so that eight or so stand on every compute unit
    const int64_t planes = (int64_t)a.spec->num_layers * p.heads, wanted = 8LL * a.compute_units / planes;
    const int most = a.tables->num_agents > 16 ? a.tables->num_agents : 16;
    const int workers = (int)(wanted < 1 ? 1 : wanted > most ? most : wanted);
    hipLaunchKernelGGL(tail_copy_kernel, dim3((unsigned)planes, (unsigned)workers), dim3(kCopyThreads), 0, stream, p);
    return hipGetLastError();
}

} // namespace

size_t tables_workspace_bytes(int num_agents) { return (size_t)(64 + 3 * (size_t)num_agents) * sizeof(int32_t); }

hipError_t launch_resize_tables(const TablesArgs &a, hipStream_t stream)
{
    TablesParams p = params_of(a);
    p.new_len = a.new_len;
    p.max_tokens = a.max_tokens;
    p.token_begin = a.token_begin;
    p.slot = a.slot;
    p.token_agent = a.token_agent;
    p.position = a.position;
    p.map_here = a.max_tokens <= 4 * kWide; // four rounds of the workgroup's lanes: less than another launch
    if (narrow(p)) hipLaunchKernelGGL(resize_kernel<kNarrow>, dim3(1), dim3(kNarrow), 0, stream, p);
    else hipLaunchKernelGGL(resize_kernel<kWide>, dim3(1), dim3(kWide), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.max_tokens > 0 && !p.map_here) {
        const int64_t blocks = ((int64_t)p.max_tokens + 255) / 256, cap = 8LL * a.compute_units;
        hipLaunchKernelGGL(slot_map_kernel, dim3((unsigned)(blocks < cap ? blocks : cap)), dim3(256), 0, stream, p);
        e = hipGetLastError();
    }
    if (e == hipSuccess && p.copies && p.agents > 0) e = launch_tail_copy(a, p.moves, stream);
    return e;
}

hipError_t launch_beam_reorder(const TablesArgs &a, hipStream_t stream)
{
    TablesParams p = params_of(a);
    p.parent = a.parent;
    const int64_t entries = (int64_t)p.agents * p.max_blocks;
    hipError_t e = hipSuccess;
    if (narrow(p) && entries <= kNarrow) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(reorder_kernel<kNarrow, true>), dim3(1), dim3(kNarrow), 0, stream, p);
    } else if (entries <= 4 * kWide * kHeld) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(reorder_kernel<kWide, true>), dim3(1), dim3(kWide), 0, stream, p);
    } else {
        const int cols = kWide * kHeld / p.agents;
        const int64_t slabs = ((int64_t)p.max_blocks + cols - 1) / cols, cap = 2LL * a.compute_units;
        hipLaunchKernelGGL(gather_kernel, dim3((unsigned)(slabs < cap ? slabs : cap)), dim3(kWide), 0, stream, p);
        e = hipGetLastError();
        if (e == hipSuccess) hipLaunchKernelGGL(HIP_KERNEL_NAME(reorder_kernel<kWide, false>), dim3(1), dim3(kWide), 0, stream, p);
    }
    if (e == hipSuccess) e = hipGetLastError();
    if (e == hipSuccess) e = launch_tail_copy(a, p.moves, stream);
    return e;
}

} // namespace q4kv
