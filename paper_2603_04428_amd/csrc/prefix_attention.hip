// Decode attention of agents that share a prefix (forked from one parent: their block-table rows begin with the same blocks):
//   out[l][a][h] = softmax(sm * q K_hat^T) V_hat   over all of the agent's tokens, as in decode_attention.hip,
// with the tokens that a group of agents shares read and unpacked once for up to 32 of its query rows on a KV head (48 with 64-wide heads).
//
// A group's first prefix_len tokens are one unit per (layer, KV head, row tile) of its (agents of the group) * n_rep query rows; what
// lies behind them is one unit per (layer, KV head, agent) with n_rep rows.  A row's softmax over the two parts (and over the ranges
// that several workers take of a unit) is joined from their un-normalised sums, maxima and denominators:
//   m = max m_i,  out = sum_i 2^(m_i - m) acc_i / sum_i 2^(m_i - m) l_i.
//
// One pass over each unit's cache, 64 tokens at a time, per wave (no synchronisation inside the tile loop):
//  * code words and parameters travel HBM -> LDS directly (global_load_lds, 16 bytes a lane) into a ring of tile buffers; the K
//    part of a buffer is asked for again as soon as the scores of its tile are taken, the rest when its values are summed.  The
//    block ids of the tiles to come are in a register that a branch may load again, and behind that branch the compiler waits for all
//    vector memory, the transfers among it: when a tile's K is asked for, everything asked for before has arrived, so that one tile,
//    not RING - 1/2, is on its way while one is worked on.  Rows lie swizzled in LDS: 16-byte chunk c of token t at chunk
//    c ^ f(t), which spreads both kinds of reads below over all banks; the transfer fetches permuted chunks of one row.
//  * scores, transposed: S^T[t][row] = sum_g s[t,g] (C_g Q_g^T)[t][row] + (b Qsum^T)[t][row]: two v_mfma_f32_16x16x32_f16 per 16
//    tokens, group and 16 rows, operand A a code word masked in place (nibbles are binary16 subnormals), the scale applied to
//    the binary32 results; the bias term is one 16x16x16 instruction over the groups, group sums of q split in two binary16
//    parts.
//  * output, transposed: O^T[e][row] = sum_t (c[t,e] - 8) (p[row,t] s[t,g(e)]) + sum_t (b + 8 s)[t,g(e)] p[row,t]: the transposing 4-bit LDS read
//    gives a lane 16 tokens of one element, masks unpack 8 of them into operand A; the lane that received S^T of (row, four
//    tokens of each 16) supplies their p s as operand B, in two binary16 terms, so probabilities never leave their registers.
// Unpacking (about 10 vector instructions per 64 codes of a lane) is shared by CT column tiles of 16 rows.
// What bounds it: below about 2,000 tiles the chain plan - ids - tiles - meeting - records (23 us for 10 agents x 8,192 tokens, 256-wide,
// one layer), above that the issue of instructions (60 % of a wave's time; matrix pipe 27 %) and the waits for the ring (26 %): 12 such
// layers 105 us, 301 MB of cache = 2.9 TB/s; 32 agents of four rows x 16,384, 128-wide, two layers 89 us.
#include <algorithm>

#include "q4_device.h"
#include "prefix_plan.h"
#include "q4kv_internal.h"

namespace q4kv {
namespace {

template <int V> struct Int { static constexpr int value = V; };

constexpr int kThreads = 256;
constexpr int kWaves = kPlanWaves;
static_assert(kWaves == kThreads / kWave, "the plan counts four waves a workgroup");
constexpr int kCols = 16;          // query rows of a column tile
constexpr int kMaxAgents = 512;    // agents of a call: their lengths and tile counts are kept in LDS
constexpr float kNegBig = -1.0e30f; // "minus infinity" that survives subtraction
constexpr float kLog2e = 1.4426950408889634f;
// Largest value scales (binary16 bits) with which probabilities may reach 2^15 and 2^7: their products stay below 65504.
constexpr uint32_t kHighScaleBits = 0x3F9A; // 1.9
constexpr uint32_t kMidScaleBits = 0x5BE0;  // 252

typedef __attribute__((address_space(3))) void *lds_ptr_t;
typedef int int2_t __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) int2_t *lds_int2_ptr;
typedef uint32_t uint2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) short4_t *lds_short4_ptr;
typedef const __attribute__((address_space(3))) uint2_t *lds_uint2_ptr;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct PrefixParams {
    const uint32_t *k_codes, *v_codes;
    const uint16_t *k_scale, *k_bias, *v_scale, *v_bias;
    const uint16_t *q;
    uint16_t *out;
    const int32_t *block_table, *seq_len, *group_begin, *prefix_len;
    int32_t *plan;
    float *part_acc, *part_ml;
    int num_agents, num_groups, max_blocks, num_blocks, kv_heads, q_heads, n_rep, layer_begin, layers, max_seq_len;
    int slots;    // records reserved per row: those of the prefix from the front, of the agent's own tokens from the back
    int row_tile; // rows of a prefix unit: 16 * CT
    float score_scale;
    float inv_n_rep;
};

// What the merge needs to know of the plan, written by workgroup 0: header, then per agent what is counted in front of its own
// part, that part's tiles, where it begins (the tiles of the prefix it shares), what is counted in front of its group's units,
// and the group's first agent.
constexpr int kHeader = 4; // [0] tiles per worker  [1] tiles counted for a (layer, KV head)  [2] for its prefix units  [3] Plan::round
__host__ __device__ constexpr int plan_ints(int agents) { return kHeader + 5 * agents; }

// ---------------------------------------------------------------------------------------------- the plan

// The tiles of a (layer, KV head): all prefix units (group by group, row tile by row tile), then the agents' own parts.  Every
// workgroup works it out for itself, in LDS.  A unit may count for more tiles than it has: see spread().
struct Plan {
    int own[kMaxAgents + 1];   // tiles that the agents in front of an agent count for
    int group[kMaxAgents + 1]; // tiles that the prefix units of the groups in front of a group count for
    int len[kMaxAgents];       // visible tokens of an agent
    int start[kMaxAgents];     // tile its own part begins with
    int begin[kMaxAgents + 1]; // first agent of a group
    int wave_sum[4][kWaves];
    int mark[kWaves][kWave]; // of up to 64 agents
    int per, round, solo; // tiles of a worker; a unit's tiles are counted as the next multiple of `round`; 1: waves are the workers
};

__device__ __forceinline__ int tiles_of(int tokens) { return (tokens + kWave - 1) / kWave; }

// inclusive sum over the lanes of a wave
__device__ __forceinline__ int wave_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false); // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false); // row_bcast15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false); // row_bcast31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_scan(v), kWave - 1); }

// inclusive maximum over the lanes of values that are not negative
__device__ __forceinline__ int wave_scan_max(int v)
{
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));
    return v;
}

// the last index of 0 .. count - 1 whose entry is at most x (entries do not fall; entry 0 is at most x), by all lanes of a wave
__device__ __forceinline__ int last_at_most(const int *pre, int count, int x)
{
    int found = 0;
    for (int i0 = 0; i0 < count; i0 += kWave) {
        const int i = i0 + (int)(threadIdx.x % kWave);
        const uint64_t below = __builtin_amdgcn_ballot_w64(i < count && pre[i < count ? i : 0] <= x);
        if (below == 0) break;
        found = i0 + 63 - __builtin_clzll(below);
    }
    return found;
}
// the same by one lane, each its own x
__device__ __forceinline__ int lane_last_at_most(const int *pre, int count, int x)
{
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (pre[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// What a lane reads for the plan of up to 64 agents: lane a of agent a, lane g of group g.
struct PlanInputs {
    int len, prefix, bound, last;
};
__device__ __forceinline__ PlanInputs plan_inputs(const PrefixParams &p, int lane)
{
    // lanes behind the last agent or group read that one again: a load behind a branch of its own would be waited for at its end
    PlanInputs in = {p.seq_len[min(lane, p.num_agents - 1)], 0, 0, 0};
    if (p.num_groups > 0) {
        const int g = min(lane, p.num_groups - 1);
        in.prefix = p.prefix_len[g];
        in.bound = p.group_begin[g];
        in.last = p.group_begin[p.num_groups];
    }
    return in;
}

// For up to 64 agents every wave makes the plan for itself, in its lanes (all write the same).
__device__ __forceinline__ void make_plan_few(const PrefixParams &p, const PlanInputs &in, int lane, int wave, Plan &pl)
{
    {
        const int A = p.num_agents, G = p.num_groups;
        const int n = lane < A ? min(max(in.len, 0), p.max_seq_len) : 0, prefix = in.prefix, last = in.last;
        const int bound = lane < G ? in.bound : 0;
        const int begin = wave_scan_max(min(max(bound, 0), A)); // bounds that fall are raised: groups never overlap
        const int end = max(__builtin_amdgcn_readlane(begin, kWave - 1), min(max(last, 0), A));
        int next = __shfl_down(begin, 1, kWave);
        if (lane >= G - 1) next = end;
        const int agents = lane < G ? next - begin : 0;
        const int shared = agents > 1 ? min(max(prefix, 0), p.max_seq_len) / kWave : 0; // a group of one shares nothing
        const int row_tiles = quotient(agents * p.n_rep + p.row_tile - 1, p.row_tile);
        // lane a: the group its agent is in, from the first agents of the groups that have any
        pl.mark[wave][lane] = 0;
        wave_lds_sync();
        if (agents > 0) pl.mark[wave][begin] = lane + 1;
        wave_lds_sync();
        const int mark = pl.mark[wave][lane];
        const uint64_t upto = __builtin_amdgcn_ballot_w64(mark > 0) & (~0ull >> (63 - lane));
        const int of = __shfl(mark, upto ? 63 - __builtin_clzll(upto) : lane, kWave); // group number + 1
        const int of_end = __shfl(next, of - 1 < 0 ? 0 : of - 1, kWave), of_shared = __shfl(shared, of - 1 < 0 ? 0 : of - 1, kWave);
        const int start = of > 0 && lane < of_end ? of_shared : 0;
        const int own = lane < A ? max(0, tiles_of(n) - start) : 0;
        const int units = p.layers * p.kv_heads; // (layer, KV head) pairs
        int per, round;
        const int busy = __builtin_popcountll(__builtin_amdgcn_ballot_w64(own > 0)) + wave_total(shared > 0 ? row_tiles : 0);
        const bool solo = spread(wave_total(own + row_tiles * shared) * units, busy * units, gridDim.x, per, round,
                                 [&](int r) { return (long long)wave_total(rounded_up(own, r) + row_tiles * rounded_up(shared, r)) * units; });
        const int group_counts = row_tiles * rounded_up(shared, round), own_counts = rounded_up(own, round);
        const int group_incl = wave_scan(group_counts), own_incl = wave_scan(own_counts);
        if (lane < A) {
            pl.len[lane] = n;
            pl.start[lane] = start;
            pl.own[lane] = own_incl - own_counts;
        }
        if (lane < G) {
            pl.begin[lane] = begin;
            pl.group[lane] = group_incl - group_counts;
        }
        if (lane == kWave - 1) {
            pl.own[A] = own_incl;
            pl.group[G] = group_incl;
            pl.begin[G] = end;
            pl.per = per;
            pl.round = round;
            pl.solo = solo ? 1 : 0;
        }
    }
    wave_lds_sync();
}

__device__ __forceinline__ void make_plan_many(const PrefixParams &p, Plan &pl)
{
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    constexpr int EACH = kMaxAgents / kThreads; // agents (and groups) of a thread
    const int A = p.num_agents, G = p.num_groups;
    int n[EACH], shared[EACH], first[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int a = tid * EACH + i;
        n[i] = a < A ? min(max(p.seq_len[a], 0), p.max_seq_len) : 0;
        shared[i] = a < G ? min(max(p.prefix_len[a], 0), p.max_seq_len) / kWave : 0;
        if (a < A) pl.len[a] = n[i];
        first[i] = a < G ? min(max(p.group_begin[a], 0), A) : 0;
    }
    // bounds that fall are raised to the ones in front of them: groups never overlap, whatever the caller wrote
    int top = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) first[i] = top = max(top, first[i]);
    const int raised = wave_scan_max(top);
    if (lane == kWave - 1) pl.wave_sum[0][wave] = raised;
    __syncthreads();
    top = __shfl_up(raised, 1, kWave);
    if (lane == 0) top = 0;
    for (int w = 0; w < wave; ++w) top = max(top, pl.wave_sum[0][w]);
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (tid * EACH + i < G) pl.begin[tid * EACH + i] = max(top, first[i]);
    if (tid == kThreads - 1) pl.begin[G] = G > 0 ? max(max(top, first[EACH - 1]), min(max(p.group_begin[G], 0), A)) : 0;
    __syncthreads();
    // a group of one agent shares nothing
    int row_tiles[EACH], own[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int g = tid * EACH + i;
        row_tiles[i] = 0;
        if (g < G) {
            const int agents = pl.begin[g + 1] - pl.begin[g];
            if (agents < 2) shared[i] = 0;
            row_tiles[i] = quotient(agents * p.n_rep + p.row_tile - 1, p.row_tile);
            pl.group[g] = shared[i]; // for the agents, until the sums are taken
        }
    }
    __syncthreads();
    int sum = 0, busy = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int a = tid * EACH + i;
        own[i] = 0;
        if (a < A) {
            int start = 0;
            if (G > 0 && a >= pl.begin[0]) {
                const int g = lane_last_at_most(pl.begin, G, a);
                if (a < pl.begin[g + 1]) start = pl.group[g];
            }
            pl.start[a] = start;
            own[i] = max(0, tiles_of(n[i]) - start);
        }
        sum += own[i] + row_tiles[i] * shared[i];
        busy += (own[i] > 0 ? 1 : 0) + (shared[i] > 0 ? row_tiles[i] : 0);
    }
    auto total = [&](int v, int slot) { // over the workgroup; every thread
        const int of_wave = wave_total(v);
        if (lane == 0) pl.wave_sum[slot][wave] = of_wave;
        __syncthreads();
        long long t = 0;
        for (int w = 0; w < kWaves; ++w) t += pl.wave_sum[slot][w];
        __syncthreads();
        return t;
    };
    const int units = p.layers * p.kv_heads;
    int per, round;
    const int units_busy = (int)total(busy, 1) * units;
    const bool solo = spread((int)total(sum, 1) * units, units_busy, gridDim.x, per, round, [&](int r) {
        int v = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) v += rounded_up(own[i], r) + row_tiles[i] * rounded_up(shared[i], r);
        return total(v, 1) * units;
    });
    int group_sum = 0, own_sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        own[i] = rounded_up(own[i], round);
        row_tiles[i] *= rounded_up(shared[i], round);
        group_sum += row_tiles[i];
        own_sum += own[i];
    }
    const int group_incl = wave_scan(group_sum), own_incl = wave_scan(own_sum);
    if (lane == kWave - 1) {
        pl.wave_sum[2][wave] = group_incl;
        pl.wave_sum[3][wave] = own_incl;
    }
    __syncthreads();
    int group_at = group_incl - group_sum, own_at = own_incl - own_sum;
    for (int w = 0; w < wave; ++w) {
        group_at += pl.wave_sum[2][w];
        own_at += pl.wave_sum[3][w];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int a = tid * EACH + i;
        if (a <= G) pl.group[a] = group_at;
        if (a <= A) pl.own[a] = own_at;
        group_at += row_tiles[i];
        own_at += own[i];
    }
    if (tid == kThreads - 1) { // counts of exactly kMaxAgents
        if (G == kMaxAgents) pl.group[G] = group_at;
        if (A == kMaxAgents) pl.own[A] = own_at;
        pl.per = per;
        pl.round = round;
        pl.solo = solo ? 1 : 0;
    }
    __syncthreads();
}

__device__ __forceinline__ void write_plan(const PrefixParams &p, const Plan &pl)
{
    const int A = p.num_agents, G = p.num_groups;
    if (threadIdx.x == 0) {
        p.plan[0] = pl.per;
        p.plan[1] = pl.group[G] + pl.own[A];
        p.plan[2] = pl.group[G];
        p.plan[3] = pl.round;
    }
    for (int a = threadIdx.x; a < A; a += kThreads) {
        const int g = G > 0 && a >= pl.begin[0] ? lane_last_at_most(pl.begin, G, a) : 0;
        p.plan[kHeader + a] = pl.own[a];
        p.plan[kHeader + A + a] = max(0, tiles_of(pl.len[a]) - pl.start[a]);
        p.plan[kHeader + 2 * A + a] = pl.start[a];
        p.plan[kHeader + 3 * A + a] = pl.group[g];
        p.plan[kHeader + 4 * A + a] = pl.begin[g];
    }
}

// ---------------------------------------------------------------------------------------------- tiles in LDS

__device__ __forceinline__ float half_of(uint32_t pair, int hi)
{
    return half_bits_to_float((uint16_t)(hi ? pair >> 16 : pair & 0xffffu));
}

// binary16 of p * s, rounded once, into the lower or the upper half of a register; s is the lower or the upper half of a word.
// Written out: the compiler converts s, multiplies and converts back.
template <bool UPPER>
__device__ __forceinline__ uint32_t product_lower(float p, uint32_t s)
{
    uint32_t d;
    if constexpr (UPPER) asm("v_fma_mixlo_f16 %0, %1, %2, 0 op_sel:[0,1,0] op_sel_hi:[0,1,0]" : "=v"(d) : "v"(p), "v"(s));
    else asm("v_fma_mixlo_f16 %0, %1, %2, 0 op_sel_hi:[0,1,0]" : "=v"(d) : "v"(p), "v"(s));
    return d;
}
template <bool UPPER>
__device__ __forceinline__ uint32_t product_upper(uint32_t d, float p, uint32_t s)
{
    if constexpr (UPPER) asm("v_fma_mixhi_f16 %0, %1, %2, 0 op_sel:[0,1,0] op_sel_hi:[0,1,0]" : "+v"(d) : "v"(p), "v"(s));
    else asm("v_fma_mixhi_f16 %0, %1, %2, 0 op_sel_hi:[0,1,0]" : "+v"(d) : "v"(p), "v"(s));
    return d;
}

// What the product's rounding left: p s less a half of hi, exact but where it is subnormal.
template <bool UPPER>
__device__ __forceinline__ uint32_t rest_lower(float p, uint32_t s, uint32_t hi)
{
    uint32_t d;
    if constexpr (UPPER) asm("v_fma_mixlo_f16 %0, %1, %2, -%3 op_sel:[0,1,0] op_sel_hi:[0,1,1]" : "=v"(d) : "v"(p), "v"(s), "v"(hi));
    else asm("v_fma_mixlo_f16 %0, %1, %2, -%3 op_sel_hi:[0,1,1]" : "=v"(d) : "v"(p), "v"(s), "v"(hi));
    return d;
}
template <bool UPPER>
__device__ __forceinline__ uint32_t rest_upper(uint32_t d, float p, uint32_t s, uint32_t hi)
{
    if constexpr (UPPER) asm("v_fma_mixhi_f16 %0, %1, %2, -%3 op_sel:[0,1,1] op_sel_hi:[0,1,1]" : "+v"(d) : "v"(p), "v"(s), "v"(hi));
    else asm("v_fma_mixhi_f16 %0, %1, %2, -%3 op_sel:[0,0,1] op_sel_hi:[0,1,1]" : "+v"(d) : "v"(p), "v"(s), "v"(hi));
    return d;
}

// What the binary16 pair hi leaves of p0 f | p1 f.
__device__ __forceinline__ uint32_t remainder_of(uint32_t hi, float p0, float p1, float f)
{
    uint32_t d;
    asm("v_fma_mixlo_f16 %0, %1, %3, -%4 op_sel_hi:[0,0,1]\n\tv_fma_mixhi_f16 %0, %2, %3, -%4 op_sel:[0,0,1] op_sel_hi:[0,0,1]"
        : "=&v"(d) : "v"(p0), "v"(p1), "s"(f), "v"(hi));
    return d;
}

// Code rows of one width in LDS: UNITS chunks of 16 bytes per row, chunk c of token t at place c ^ swizzle(t).  A row is 8, 16,
// 24 or 32 banks long: with the swizzle the 16 rows 16 j .. 16 j + 15 (a set of the scores) and the 16 rows 16 j + 4 q + r of one q
// (a slot of the values) each spread one chunk per row over all 64 banks, as far as rows of 64 elements allow.
template <int DIM>
struct Rows {
    static constexpr int BYTES = DIM / 2;          // of a row
    static constexpr int UNITS = DIM / 32;
    static constexpr int LOADS = kWave * BYTES / 1024; // 1 KiB transfers of a tile
    __device__ __forceinline__ static constexpr int swizzle(int t)
    {
        if constexpr (UNITS == 8) return ((t >> 1) & 7) ^ (2 * ((t >> 4) & 3));
        else if constexpr (UNITS == 4) return ((t >> 2) & 3) ^ ((t >> 4) & 3);
        else return ((t >> 3) ^ (t >> 4)) & 1;
    }
    // byte offset in the tile's rows that lane `lane` fetches in transfer i, less 1024 i
    __device__ __forceinline__ static uint32_t source(int i, int lane)
    {
        const int u = i * kWave + lane, t = u / UNITS, c = (u % UNITS) ^ swizzle(t);
        return (uint32_t)((t * UNITS + c - i * kWave) * 16);
    }
    // which of the first SOURCES transfers has the same offsets
    static constexpr int SOURCES = LOADS < 4 ? LOADS : UNITS == 6 ? 3 : 4;
    static constexpr int source_of(int i) { return UNITS == 6 ? i % 3 : i < 4 ? i : (i - 4) ^ 1; }
    // for the rows 16 j + col of set j: what the swizzle adds to that of j == 0 and group g, and the offset behind the exclusive or
    static constexpr int set_xor(int j, int g)
    {
        if constexpr (UNITS == 8) return 2 * (g ^ j);
        else if constexpr (UNITS == 4) return (2 * g) ^ j;
        else return j & 1;
    }
    static constexpr int group_offset(int g) { return UNITS == 6 ? 32 * g : 0; }
};

template <int DK, int DV>
struct Shape {
    static constexpr int GK = DK / kGroup, GV = DV / kGroup;
    static constexpr int K_BYTES = kWave * DK / 2, V_BYTES = kWave * DV / 2;
    static constexpr int PARAM_UNITS = 16 * (GK + GV);                      // chunks of K scale, K bias, V scale, V bias of a tile
    static constexpr int PARAM_LOADS = (PARAM_UNITS + kWave - 1) / kWave;
    static constexpr int P_BYTES = PARAM_LOADS * 1024;
    static constexpr int TILE_BYTES = K_BYTES + V_BYTES + P_BYTES;
    static constexpr int WAVES_PER_SIMD = 1;
    static constexpr int RING = DK == 256 ? 2 : DK == 192 ? 3 : 4;
    static constexpr int WAVE_BYTES = RING * TILE_BYTES;
    static constexpr int ROW_PITCH = DV + 4;                                // floats of a row of sums in LDS
    // offsets of the parameter arrays in a tile's parameters
    static constexpr int KS_AT = 0, KB_AT = 128 * GK, VS_AT = 256 * GK, VB_AT = 256 * GK + 128 * GV;
};

// up to four transfers of 1 KiB from consecutive KiB of global memory to consecutive KiB of LDS
template <int N>
__device__ __forceinline__ void transfer(uint32_t lds, const void *src, uint32_t o0, uint32_t o1, uint32_t o2, uint32_t o3)
{
    if constexpr (N == 1)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1" ::"s"(lds), "s"(src), "v"(o0) : "memory");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024" ::"s"(lds),
                     "s"(src), "v"(o0), "v"(o1)
                     : "memory");
    else if constexpr (N == 3)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                     "global_load_lds_dwordx4 %4, %1 offset:2048" ::"s"(lds),
                     "s"(src), "v"(o0), "v"(o1), "v"(o2)
                     : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                     "global_load_lds_dwordx4 %4, %1 offset:2048\n\tglobal_load_lds_dwordx4 %5, %1 offset:%6" ::"s"(lds),
                     "s"(src), "v"(o0), "v"(o1), "v"(o2), "v"(o3), "n"(3 * 1024)
                     : "memory");
}
// the code rows of a tile
template <int DIM>
__device__ __forceinline__ void transfer_rows(uint32_t lds, const unsigned char *src, const uint32_t (&from)[Rows<DIM>::SOURCES])
{
    typedef Rows<DIM> R;
#pragma unroll
    for (int i = 0; i < R::LOADS; i += 4) {
        const uint32_t o0 = from[R::source_of(i)], o1 = from[R::source_of(i + 1 < R::LOADS ? i + 1 : i)];
        const uint32_t o2 = from[R::source_of(i + 2 < R::LOADS ? i + 2 : i)], o3 = from[R::source_of(i + 3 < R::LOADS ? i + 3 : i)];
        if (R::LOADS - i >= 4) transfer<4>(lds + i * 1024, src + i * 1024, o0, o1, o2, o3);
        else if (R::LOADS - i == 3) transfer<3>(lds + i * 1024, src + i * 1024, o0, o1, o2, o3);
        else if (R::LOADS - i == 2) transfer<2>(lds + i * 1024, src + i * 1024, o0, o1, o2, o3);
        else transfer<1>(lds + i * 1024, src + i * 1024, o0, o1, o2, o3);
    }
}
// the same from an address per lane
__device__ __forceinline__ void transfer_from(uint32_t lds, uint64_t address)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(address) : "memory");
}

template <int N>
__device__ __forceinline__ void wait_for_all_but()
{
    static_assert(N <= 63, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// A unit, or the part of it that a worker takes.
struct Part {
    int li, kvh;       // layer in call, KV head
    int agent, agents; // the agents whose rows read it: first, number
    int row0, rows;    // rows of this unit: row0 .. row0 + rows - 1 of those agents' rows
    int tile, count;   // the part: first tile (of the agent's tokens), number of tiles
    int counted;       // what it counts for in the plan
    int slot;          // the part's record among the unit's
    int which;         // 0: prefix, 1: own tokens
    int whole_row;     // 1: there is nothing else to join, the rows' outputs are final
};

__device__ __forceinline__ Part locate(const PrefixParams &p, const Plan &pl, int x, int x1, int per, int round, int worker)
{
    Part u;
    const int group_tiles = uniform(pl.group[p.num_groups]), head_tiles = group_tiles + uniform(pl.own[p.num_agents]);
    const int lk = quotient(x, head_tiles);
    int r = x - lk * head_tiles, tiles;
    u.li = quotient(lk, p.kv_heads);
    u.kvh = lk - u.li * p.kv_heads;
    if (r < group_tiles) {
        const int g = last_at_most(pl.group, p.num_groups, r);
        u.agent = uniform(pl.begin[g]);
        u.agents = uniform(pl.begin[g + 1]) - u.agent;
        tiles = uniform(pl.start[u.agent]);
        r -= uniform(pl.group[g]);
        const int counted = rounded_up(tiles, round), rt = quotient(r, counted);
        r -= rt * counted;
        u.row0 = rt * p.row_tile;
        u.rows = min(p.row_tile, u.agents * p.n_rep - u.row0);
        u.tile = r;
        u.which = 0;
    } else {
        r -= group_tiles;
        u.agent = last_at_most(pl.own, p.num_agents, r);
        u.agents = 1;
        const int start = uniform(pl.start[u.agent]);
        tiles = max(0, tiles_of(uniform(pl.len[u.agent])) - start);
        r -= uniform(pl.own[u.agent]);
        u.row0 = 0;
        u.rows = p.n_rep;
        u.tile = r + start;
        u.which = 1;
    }
    const int unit0 = x - r, counted = rounded_up(tiles, round);
    u.counted = min(counted - r, x1 - x);
    u.count = min(tiles - r, x1 - x); // at least one: what a unit counts for beyond its tiles is less than a worker's range
    // a unit that begins in front of this worker's range may have begun several ranges before
    u.slot = r == 0 ? 0 : worker - quotient(unit0, per);
    u.whole_row = u.which == 1 && u.tile == r && u.slot == 0 && u.count == tiles;
    u.li = uniform(u.li); u.kvh = uniform(u.kvh); u.agent = uniform(u.agent); u.agents = uniform(u.agents);
    u.row0 = uniform(u.row0); u.rows = uniform(u.rows); u.tile = uniform(u.tile); u.count = uniform(u.count);
    u.counted = uniform(u.counted); u.slot = uniform(u.slot); u.whole_row = uniform(u.whole_row); u.which = uniform(u.which);
    return u;
}

// the place of row `row` of a part: (layer, agent, query head)
__device__ __forceinline__ int64_t row_index(const PrefixParams &p, const Part &u, int row, int &agent)
{
    const int idx = u.row0 + row, in_group = (int)(((float)idx + 0.5f) * p.inv_n_rep); // idx / n_rep: below 2^21 this is exact
    agent = u.agent + in_group;
    return ((int64_t)u.li * p.num_agents + agent) * p.q_heads + u.kvh * p.n_rep + (idx - in_group * p.n_rep);
}

// CT: column tiles of 16 rows of the prefix units.  BF: scale and bias are stored as bfloat16.
template <int DK, int DV, int CTP, bool BF>
__global__ __launch_bounds__(kThreads, (Shape<DK, DV>::WAVES_PER_SIMD)) void prefix_attention_kernel(const PrefixParams p)
{
    typedef Shape<DK, DV> S;
    constexpr int GK = S::GK, GV = S::GV;
    __shared__ __attribute__((aligned(1024))) unsigned char tiles_lds[kWaves * S::WAVE_BYTES];
    __shared__ Plan plan;
    __shared__ float ml_lds[kWaves][CTP * kCols][2];

    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
    PlanInputs plan_in;
    if (p.num_agents <= kWave) plan_in = plan_inputs(p, lane); // on their way while the lane's places are worked out

    unsigned char *const region = tiles_lds + wave * S::WAVE_BYTES;
    const uint32_t region_at = (uint32_t)(uintptr_t)(lds_ptr_t)region;
    const int col = lane % 16, qk = lane / 16;

    // what a lane fetches of a tile's rows and parameters
    uint32_t k_src[Rows<DK>::SOURCES], v_src[Rows<DV>::SOURCES];
#pragma unroll
    for (int i = 0; i < Rows<DK>::SOURCES; ++i) k_src[i] = Rows<DK>::source(i, lane);
#pragma unroll
    for (int i = 0; i < Rows<DV>::SOURCES; ++i) v_src[i] = Rows<DV>::source(i, lane);
    uint64_t param_src[S::PARAM_LOADS];
    bool param_of_v[S::PARAM_LOADS];
#pragma unroll
    for (int i = 0; i < S::PARAM_LOADS; ++i) {
        const int u = min(i * kWave + lane, S::PARAM_UNITS - 1); // (behind the last: that one again)
        const bool of_v = u >= 16 * GK;
        const int in_pool = of_v ? u - 16 * GK : u, units = 8 * (of_v ? GV : GK);
        const uint16_t *base = of_v ? (in_pool < units ? p.v_scale : p.v_bias) : (in_pool < units ? p.k_scale : p.k_bias);
        param_src[i] = (uint64_t)(uintptr_t)base + 16 * (in_pool < units ? in_pool : in_pool - units);
        param_of_v[i] = of_v;
    }
    // where it reads them: row `col` of set 0 for the scores, row 16 (col / 4) + 4 qk + col % 4 for the values
    const uint32_t k_at = region_at + col * Rows<DK>::BYTES + (((qk >> 1) ^ Rows<DK>::swizzle(col)) << 4) + (qk & 1) * 8;
    const int v_row = 16 * (col / 4) + 4 * qk + col % 4;
    const uint32_t v_at = region_at + S::K_BYTES + v_row * Rows<DV>::BYTES + (Rows<DV>::swizzle(v_row) << 4);

    if (p.num_agents <= kWave) make_plan_few(p, plan_in, lane, wave, plan);
    else make_plan_many(p, plan);
    const int per = uniform(plan.per), round = uniform(plan.round);
    const int total = uniform(plan.group[p.num_groups] + plan.own[p.num_agents]) * p.kv_heads * p.layers; // below 2^31: see spread()
    const bool solo = uniform(plan.solo) != 0;
    if (blockIdx.x == 0) write_plan(p, plan);
    const int worker = solo ? (int)blockIdx.x * kWaves + wave : (int)blockIdx.x;
    const long long begin = (long long)worker * per;
    if (begin >= total) return; // a whole workgroup, or a wave on its own
    const int x1 = (int)min((long long)total, begin + per);

    auto run_part = [&](auto column_tiles, const Part &u) __attribute__((always_inline)) {
        constexpr int CT = decltype(column_tiles)::value;
        constexpr bool kTight = CT * (GK + GV) >= 16; // registers for everything only if loads from LDS do not move far ahead
        const int step = solo ? 1 : kWaves;
        const int first = solo ? 0 : wave;                                       // tiles of the part that are this wave's:
        const int mine = u.count > first ? (u.count - first + step - 1) / step : 0; // first, first + step, ...
        const int64_t unit_row = ((int64_t)(p.layer_begin + u.li) * p.num_blocks * p.kv_heads + u.kvh) * kBlockTokens;
        const int32_t *const table = p.block_table + (int64_t)u.agent * p.max_blocks;
        // block ids of 64 blocks from table_base on, one per lane
        int table_base = (u.tile + first) / 4;
        auto fetch_table = [&]() { return table_base + lane < p.max_blocks ? table[table_base + lane] : -1; };
        int table_ids = -1;
        auto block_of = [&](int t) __attribute__((always_inline)) { // wave-uniform
            const int b = t / 4;
            if (__builtin_expect(b >= table_base + kWave, 0)) {
                table_base = b;
                table_ids = fetch_table();
            }
            return __builtin_amdgcn_readlane(table_ids, b - table_base);
        };
        uint32_t reachable_bufs = 0; // bit: the block id of the tile in that buffer is inside the pool
        auto row_of = [&](int t, int buf) __attribute__((always_inline)) {
            const int blk = block_of(t);
            const bool inside = blk >= 0 && blk < p.num_blocks;
            reachable_bufs = (reachable_bufs & ~(1u << buf)) | (inside ? 1u << buf : 0u);
            // the loads of a tile whose id is outside the pool go to block 0; all they bring is masked
            return unit_row + (int64_t)(inside ? blk : 0) * (p.kv_heads * kBlockTokens) + (t % 4) * kWave;
        };
        int64_t row = 0; // of the tile asked for last: first its K, later the rest
        auto issue_k = [&](int t, int buf) __attribute__((always_inline)) {
            row = row_of(t, buf);
            const unsigned char *src = reinterpret_cast<const unsigned char *>(p.k_codes) + row * Rows<DK>::BYTES;
            const uint32_t dst = region_at + buf * S::TILE_BYTES;
            transfer_rows<DK>(dst, src, k_src);
        };
        auto issue_rest = [&](int buf) __attribute__((always_inline)) { // parameters, then V
            const uint32_t dst = region_at + buf * S::TILE_BYTES + S::K_BYTES;
#pragma unroll
            for (int i = 0; i < S::PARAM_LOADS; ++i)
                transfer_from(dst + S::V_BYTES + i * 1024, param_src[i] + (uint64_t)row * (2 * GK != 2 * GV && param_of_v[i] ? 2 * GV : 2 * GK));
            const unsigned char *src = reinterpret_cast<const unsigned char *>(p.v_codes) + row * Rows<DV>::BYTES;
            transfer_rows<DV>(dst, src, v_src);
        };
        // Of the transfers behind what is waited for, `ahead` tiles' (the tiles behind the current one that have been asked for) may
        // still be on their way; loads complete in order.
        constexpr int K_LOADS = Rows<DK>::LOADS, V_LOADS = Rows<DV>::LOADS, ALL = K_LOADS + V_LOADS + S::PARAM_LOADS;
        auto wait_scores = [&](int ahead) __attribute__((always_inline)) { // K and parameters of the current tile
            if (S::RING >= 4 && ahead >= 3) wait_for_all_but<V_LOADS + 3 * ALL>();
            else if (S::RING >= 3 && ahead >= 2) wait_for_all_but<V_LOADS + 2 * ALL>();
            else if (ahead >= 1) wait_for_all_but<V_LOADS + ALL>();
            else wait_for_all_but<V_LOADS>();
        };
        auto wait_values = [&](int ahead) __attribute__((always_inline)) { // V of the current tile; K of RING tiles on may have been asked for
            if (S::RING >= 4 && ahead >= 4) wait_for_all_but<3 * ALL + K_LOADS>();
            else if (S::RING >= 4 && ahead >= 3) wait_for_all_but<3 * ALL>();
            else if (S::RING == 3 && ahead >= 3) wait_for_all_but<2 * ALL + K_LOADS>();
            else if (S::RING >= 3 && ahead >= 2) wait_for_all_but<2 * ALL>();
            else if (S::RING == 2 && ahead >= 2) wait_for_all_but<ALL + K_LOADS>();
            else if (ahead >= 1) wait_for_all_but<ALL>();
            else wait_for_all_but<0>();
        };

        // ---- loads complete in order: the block ids, the rows' queries, the tiles
        table_ids = fetch_table();
        __builtin_amdgcn_sched_barrier(0);
        uint4 raw[CT][GK][2];
        int n_row[CT], n_min = 0x7fffffff, n_max = 0;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            int agent;
            const int64_t row = row_index(p, u, min(16 * ct + col, u.rows - 1), agent);
            n_row[ct] = agent;
            const uint16_t *qrow = p.q + row * DK + 16 * qk;
#pragma unroll
            for (int g = 0; g < GK; ++g) {
                raw[ct][g][0] = *reinterpret_cast<const uint4 *>(qrow + g * kGroup);
                raw[ct][g][1] = *reinterpret_cast<const uint4 *>(qrow + g * kGroup + 8);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // all reads of the tile buffers are done
#pragma unroll 1
        for (int i = 0; i < S::RING; ++i)
            if (i < mine) {
                issue_k(u.tile + first + i * step, i);
                issue_rest(i);
            }

        // ---- the query operand: the element order of code_operand, odd elements / 16 because their codes arrive 16 times larger;
        // group sums of q
        half8_t qop[CT][GK][2];
        half4_t qsop[CT];
        float sum_unit[CT]; // of the bias term: 2^-24, the unit of the products, times 2^6 for a row whose sums are taken down by that
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            n_row[ct] = plan.len[n_row[ct]];
            n_min = min(n_min, n_row[ct]);
            n_max = max(n_max, n_row[ct]);
            float qs[GK];
#pragma unroll
            for (int g = 0; g < GK; ++g) {
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint4 w = raw[ct][g][r];
                    const half2_t ones = half2_t{(half_t)1.0f, (half_t)1.0f}, sixteenth = half2_t{(half_t)0.0625f, (half_t)0.0625f};
                    const half2_t e15 = bits_to_half2(__builtin_amdgcn_perm(w.z, w.x, 0x07060302u)) * sixteenth;
                    const half2_t e37 = bits_to_half2(__builtin_amdgcn_perm(w.w, w.y, 0x07060302u)) * sixteenth;
                    qop[ct][g][r] = words_to_half8(__builtin_amdgcn_perm(w.z, w.x, 0x05040100u), half2_to_bits(e15),
                                                   __builtin_amdgcn_perm(w.w, w.y, 0x05040100u), half2_to_bits(e37));
                    sum = __builtin_amdgcn_fdot2(bits_to_half2(w.x), ones, sum, false);
                    sum = __builtin_amdgcn_fdot2(bits_to_half2(w.y), ones, sum, false);
                    sum = __builtin_amdgcn_fdot2(bits_to_half2(w.z), ones, sum, false);
                    sum = __builtin_amdgcn_fdot2(bits_to_half2(w.w), ones, sum, false);
                }
                qs[g] = xor32_sum(xor16_sum(sum));
            }
            // 64 finite values may sum up to 64 times the largest binary16 number; rows that stay below half of it keep their sums
            float largest = 0.0f;
#pragma unroll
            for (int g = 0; g < GK; ++g) largest = fmaxf(largest, fabsf(qs[g]));
            const float shrink = largest > 32768.0f ? 0x1p-6f : 1.0f;
            sum_unit[ct] = largest > 32768.0f ? 0x1p-18f : 0x1p-24f;
            // contraction index of the bias term: with up to two groups high and low parts side by side in slot 0, else the
            // high parts in slot 0 and the low parts in slot 1
            half_t part[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int g = GK <= 2 ? e % GK : e;
                const float v = g < GK && (GK > 2 || e < 2 * GK) ? qs[g < GK ? g : 0] * shrink : 0.0f;
                const half_t hi = (half_t)v;
                const bool low = GK <= 2 ? e >= GK : qk == 1;
                const half_t value = low ? (half_t)(v - (float)hi) : hi;
                part[e] = qk < (GK <= 2 ? 1 : 2) ? value : (half_t)0.0f;
            }
            qsop[ct] = half4_t{part[0], part[1], part[2], part[3]};
        }
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1) {
            n_min = min(n_min, __shfl_xor(n_min, off, 16));
            n_max = max(n_max, __shfl_xor(n_max, off, 16));
        }
        n_min = uniform(n_min);
        n_max = uniform(n_max);
        float4_t acc[CT][4 * GV], pbacc[CT];
        float m_run[CT], l_run[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
            for (int c = 0; c < 4 * GV; ++c) acc[ct][c] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
            pbacc[ct] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
            m_run[ct] = kNegBig;
            l_run[ct] = 0.0f;
        }

        // The query operand of two column tiles of wide heads lives in accumulator registers, which matrix instructions read directly.
        if constexpr (CT * GK >= 6) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int g = 0; g < GK; ++g) asm volatile("" : "+a"(qop[ct][g][0]), "+a"(qop[ct][g][1]));
        }

        int buf = 0;
        for (int i = 0; i < mine; ++i) {
            const int t = u.tile + first + i * step, t0 = t * kWave;
            const int ahead = min(mine - 1 - i, S::RING - 1);
            const uint32_t base = (uint32_t)buf * S::TILE_BYTES;
            const unsigned char *const params = region + base + S::K_BYTES + S::V_BYTES;
            wait_scores(ahead);
            const bool reachable = (reachable_bufs >> buf & 1u) != 0;
            const bool edge = !(reachable && t0 + kWave <= n_min);
            uint32_t s_top = 0;
            {
                // token `lane`'s parameters: converted from bfloat16, zero for tokens that no row sees (their slots may hold
                // anything, and no NaN or infinity may reach a matrix operand)
                const bool seen = reachable && t0 + lane < n_max;
                auto row_of_params = [&](int at, int groups) __attribute__((always_inline)) {
                    return reinterpret_cast<uint16_t *>(const_cast<unsigned char *>(params) + at) + lane * groups;
                };
                auto redo = [&](uint16_t *w, int groups) __attribute__((always_inline)) {
                    for (int g = 0; g < groups; ++g) {
                        const uint16_t v = BF ? float_to_half_bits(bf16_bits_to_float(w[g])) : w[g];
                        w[g] = seen ? v : (uint16_t)0;
                    }
                };
                if (BF || __builtin_expect(edge, 0)) {
                    redo(row_of_params(S::KS_AT, GK), GK);
                    redo(row_of_params(S::KB_AT, GK), GK);
                    redo(row_of_params(S::VS_AT, GV), GV);
                    redo(row_of_params(S::VB_AT, GV), GV);
                }
                const uint16_t *vs = row_of_params(S::VS_AT, GV);
#pragma unroll
                for (int g = 0; g < GV; ++g) s_top = max(s_top, (uint32_t)vs[g]);
                wave_lds_sync();
            }
            const bool mid = __builtin_amdgcn_ballot_w64(s_top > kHighScaleBits) != 0ull;
            const bool wide = mid && __builtin_amdgcn_ballot_w64(s_top > kMidScaleBits) != 0ull;

            // ---- scores: z[ct][j][r] is token 16 j + 4 qk + r, row 16 ct + col, in units of 2^-24 / score_scale
            float z[CT][4][4];
            const float4_t zero = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
            const uint32_t ka = k_at + base;
            auto read_keys = [&](int j, int g) __attribute__((always_inline)) {
                return *(lds_uint2_ptr)(uintptr_t)((ka ^ (uint32_t)(Rows<DK>::set_xor(j, g) << 4)) + (uint32_t)(16 * j * Rows<DK>::BYTES + Rows<DK>::group_offset(g)));
            };
            uint2_t keys[2][GK];
#pragma unroll
            for (int g = 0; g < GK; ++g) keys[0][g] = read_keys(0, g);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t b[2], s[2 * GK]; // bias row of token 16 j + col; scales of tokens 16 j + 4 qk .. + 3
                const unsigned char *brow = params + S::KB_AT + (16 * j + col) * (2 * GK), *srow = params + S::KS_AT + (16 * j + 4 * qk) * (2 * GK);
                if constexpr (GK == 4) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(brow);
                    b[0] = w.x;
                    b[1] = w.y;
                } else if constexpr (GK == 3) {
                    const uint16_t *w = reinterpret_cast<const uint16_t *>(brow);
                    b[0] = (uint32_t)w[0] | (uint32_t)w[1] << 16;
                    b[1] = w[2];
                } else if constexpr (GK == 2) {
                    b[0] = b[1] = *reinterpret_cast<const uint32_t *>(brow);
                } else {
                    const uint32_t w = *reinterpret_cast<const uint16_t *>(brow);
                    b[0] = w | w << 16;
                    b[1] = 0;
                }
                __builtin_memcpy(s, __builtin_assume_aligned(srow, GK % 2 == 0 ? 16 : 8), 8 * GK);
                const half4_t bop = __builtin_bit_cast(half4_t, make_uint2(b[0], b[1]));
                float4_t sum[CT];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    sum[ct] = __builtin_amdgcn_mfma_f32_16x16x16f16(bop, qsop[ct], zero, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[ct][r] *= sum_unit[ct];
                }
#pragma unroll
                for (int g = 0; g < GK; ++g) {
                    const uint2_t w = keys[j % 2][g];
                    if (j < 3) keys[(j + 1) % 2][g] = read_keys(j + 1, g); // ahead of their use
                    const half8_t a0 = code_operand(w.x), a1 = code_operand(w.y);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        float4_t d = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, qop[ct][g][0], zero, 0, 0, 0);
                        d = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, qop[ct][g][1], d, 0, 0, 0);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int at = r * GK + g;
                            sum[ct][r] = fmaf(half_of(s[at / 2], at & 1), d[r], sum[ct][r]);
                        }
                    }
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[ct][j][r] = sum[ct][r];
                if (kTight) __builtin_amdgcn_sched_barrier(0);
            }
            // wide tiles' scores are final here: or the scaling sinks behind the branches below, and all products wait for it in registers
            // (12 layers of 20 rows, 256-wide, 99.1 -> 93.3 us; 128-wide heads, which have room for that, are faster without: 82.4 for 84.6)
            if constexpr (kTight) {
#pragma unroll
                for (int k = 0; k < 16 * CT; ++k) asm volatile("" : "+v"(z[k / 16][k / 4 % 4][k % 4]));
            }
            // K of this buffer has been read: the next tile for it
            const bool more = i + S::RING < mine;
            if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                issue_k(t + S::RING * step, buf);
            }

            // ---- online softmax.  m_run is the reference the exponentials are taken against: it moves only when a tile's maximum
            // exceeds it by more than `above_by` (in log2 units), and then to `lift` below that maximum.  p as well as p s stay
            // inside binary16 (65504) then: p <= 2^15 with scales up to 1.9, 2^7 with scales up to 252, 2^2.5 with larger ones
            // (no binary16 row has one above 8734); and what is far below a row's maximum keeps its bits: tokens of which there are many
            // may weigh as much together as the few at the top.  The codes of the odd rows r arrive 16 times larger in operand A
            // (code_operand): z of an odd r becomes p / 16.
            const float above_by = wide ? 2.5f : mid ? 7.0f : 15.0f, lift = wide ? 0.0f : mid ? 4.0f : 12.0f;
            float zs = p.score_scale * kCodeScaleA;
            if (__builtin_expect(!(p.score_scale > 0.0f), 0)) { // the maximum may not be taken before the scale is applied
                asm volatile("");
#pragma unroll
                for (int k = 0; k < 16 * CT; ++k) z[k / 16][k / 4 % 4][k % 4] *= zs;
                zs = 1.0f;
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if (__builtin_expect(edge, 0)) {
                    asm volatile("");
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (!(reachable && t0 + 16 * j + 4 * qk + r < n_row[ct])) z[ct][j][r] = -INFINITY;
                }
                float mt = -INFINITY;
#pragma unroll
                for (int k = 0; k < 16; ++k) mt = fmaxf(mt, z[ct][k / 4][k % 4]);
                mt = xor32_max(xor16_max(mt)) * zs;
                asm("" : "+v"(mt)); // rounded here, and not once more with each of the differences below
                const bool above = mt - m_run[ct] > above_by;
                float m_new = above ? mt - lift : m_run[ct], factor = zs, taken = m_new;
                // The maximum is rounded once more than the exponents, by up to 2^-7 for scores of 2^18.  Beyond, where that would let
                // weights out of binary16 (from 2^22 on) or vanish, all scores of the tile are rounded like it.
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(fabsf(mt) > 0x1p18f) != 0ull, 0)) {
                    asm volatile("");
                    if (above && fabsf(mt) > 0x1p22f) m_new = mt; // `lift` may be less than a step there
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float score = z[ct][k / 4][k % 4] * zs;
                        asm("" : "+v"(score)); // a rounding of its own
                        z[ct][k / 4][k % 4] = score - m_new;
                    }
                    factor = 1.0f;
                    taken = 0.0f;
                }
                const float minus_even = -taken, minus_odd = -(taken + 4.0f);
                float even_sum = 0.0f, odd_sum = 0.0f;
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float pr = __builtin_amdgcn_exp2f(fmaf(z[ct][k / 4][k % 4], factor, (k & 1) ? minus_odd : minus_even));
                    z[ct][k / 4][k % 4] = pr;
                    if (k & 1) odd_sum += pr; else even_sum += pr;
                }
                if (i > 0 && __builtin_amdgcn_ballot_w64(above) != 0ull) {
                    const float alpha = __builtin_amdgcn_exp2f(m_run[ct] - m_new);
                    l_run[ct] *= alpha;
                    pbacc[ct] *= alpha;
#pragma unroll
                    for (int c = 0; c < 4 * GV; ++c) acc[ct][c] *= alpha;
                }
                l_run[ct] += fmaf(16.0f, odd_sum, even_sum);
                m_run[ct] = m_new;
            }

            // ---- values: V_hat = (c - 8) s + 8 s + b.  p s goes in as two binary16 terms, what the first one's rounding left being the
            // second, so that 2^-22 of it is lost, relative to |c - 8| s, the distance from the middle of the value's group: sum (c - 8) ps =
            // sum c ps - 8 sum ps with the ps that were rounded, two more instructions per group and half.  One term alone would be 2^-12
            // off, 2.6e-4 instead of 2.2e-4 of an output's size with the output's own rounding of 2.1e-4, and 82 us for 90 on two layers of
            // 128 rows behind 16,384 tokens, 94 for 105 on twelve of 20, 256-wide, 26 for 28 on one.  The middles may be any size, and cancel: sums of p b
            // and p s take p in two binary16 terms.  All these sums share an accumulator, whose rows 4 k + g are group g's: k = 0 takes
            // sum 8 ps, 2 sum p b and 3 sum p s.
            // Matrix instructions cut off what lies too far below the exponent of their largest summand, and a subnormal operand
            // counts with the exponent of the smallest normal number: sum c ps falls short by 2^-19 of itself, about, while outputs
            // over many tokens are only some hundredths of it.  So the eight is a code as well, cut off alike (8,192 tokens, 256-wide
            // heads, p s in one term: the error of the outputs goes from 3.0e-4 to 2.7e-4 of their size).
            // scales of tokens 16 j + 4 qk + r, four tokens a read; of 256-wide heads two groups at a time, in front of their products
            // (sixteen registers fewer: the sums need not be moved out of the way, 108.0 -> 103.8 us for 12 layers of 20 rows)
            constexpr bool kPairs = GV == 4;
            uint32_t s4[4][2 * GV];
            auto read_pair = [&](int g) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s4[j][(r * GV + g) / 2] = *reinterpret_cast<const uint32_t *>(params + S::VS_AT + (16 * j + 4 * qk + r) * (2 * GV) + 2 * g);
            };
            if (kPairs) read_pair(0);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!kPairs) __builtin_memcpy(s4[j], __builtin_assume_aligned(params + S::VS_AT + (16 * j + 4 * qk) * (2 * GV), 8), 8 * GV);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // operand A: row `col` is group col % 4, its elements zero (rows 0 to 7), b (to 11) or s of the tokens 4 qk + r of sets
                // 2 h and 2 h + 1, side by side for each r
                uint32_t word[4];
                if constexpr (GV == 4) {
                    // the transposing read gives lane `col` group col % 4 of four tokens, from the lanes col / 4, col / 4 + 4, .. of its 16:
                    // those point at the tokens
                    const int tok = 16 * (2 * h + ((col >> 2) & 1)) + 4 * qk + (col >> 3);
                    const uint32_t at = region_at + base + S::K_BYTES + S::V_BYTES + tok * 8 + (col % 4 == 3 ? S::VS_AT : S::VB_AT);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(uintptr_t)(at + 16 * k)));
                        word[2 * k] = w.x;
                        word[2 * k + 1] = w.y;
                    }
                } else {
                    uint32_t m[2][2 * GV];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        __builtin_memcpy(m[k], __builtin_assume_aligned(params + (col < 12 ? S::VB_AT : S::VS_AT) + (16 * (2 * h + k) + 4 * qk) * (2 * GV), 8), 8 * GV);
                    // which half of a token's word: the group's (rows behind the last group repeat it and are not used)
                    const uint32_t pick = GV == 2 && (col & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        word[r] = GV == 2 ? __builtin_amdgcn_perm(m[1][r], m[0][r], pick)
                                          : __builtin_amdgcn_perm(m[1][r / 2], m[0][r / 2], (r & 1) ? 0x07060302u : 0x05040100u);
                }
                const uint32_t used = col >= 8 ? 0xFFFFFFFFu : 0u;
                const half8_t bop = words_to_half8(word[0] & used, word[1] & used, word[2] & used, word[3] & used);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    uint32_t hi[4], lo[4]; // p of the same tokens
                    const half2_t sixteen = half2_t{(half_t)16.0f, (half_t)16.0f};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float p0 = z[ct][2 * h][r], p1 = z[ct][2 * h + 1][r];
                        half2_t v = half2_t{(half_t)p0, (half_t)p1};
                        if (r & 1) v *= sixteen;
                        hi[r] = half2_to_bits(v);
                        lo[r] = remainder_of(hi[r], p0, p1, (r & 1) ? 16.0f : 1.0f);
                    }
                    asm("s_nop 1" : "+v"(lo[0]), "+v"(lo[1]), "+v"(lo[2]), "+v"(lo[3])); // as below
                    pbacc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bop, words_to_half8(hi[0], hi[1], hi[2], hi[3]), pbacc[ct], 0, 0, 0);
                    pbacc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bop, words_to_half8(lo[0], lo[1], lo[2], lo[3]), pbacc[ct], 0, 0, 0);
                }
            }
            wait_values(min(mine - 1 - i, S::RING));
            const uint32_t va = v_at + base;
            auto read_codes = [&](int c) __attribute__((always_inline)) {
                return __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_int2_ptr)(uintptr_t)((va ^ (uint32_t)((c >> 1) << 4)) + (c & 1) * 8));
            };
            int2_t words[2] = {read_codes(0), read_codes(1)}; // read two ahead of their use: left to itself, the compiler waits for each
#pragma unroll
            for (int g = 0; g < GV; ++g) {
                if (kTight) __builtin_amdgcn_sched_barrier(0);
                half8_t ps[CT][2], rest[CT][2]; // p s in two binary16 terms
                const uint32_t eight = col == g ? 0x00080008u : 0u, sixteen_times = col == g ? 0x00800080u : 0u;
                const half8_t eights = words_to_half8(eight, sixteen_times, eight, sixteen_times);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t a[4], b[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int at = r * GV + g;
                            const uint32_t w0 = s4[2 * h][at / 2], w1 = s4[2 * h + 1][at / 2];
                            const float p0 = z[ct][2 * h][r], p1 = z[ct][2 * h + 1][r];
                            if (at & 1) {
                                a[r] = product_upper<true>(product_lower<true>(p0, w0), p1, w1);
                                b[r] = rest_upper<true>(rest_lower<true>(p0, w0, a[r]), p1, w1, a[r]);
                            } else {
                                a[r] = product_upper<false>(product_lower<false>(p0, w0), p1, w1);
                                b[r] = rest_upper<false>(rest_lower<false>(p0, w0, a[r]), p1, w1, a[r]);
                            }
                        }
                        // the compiler does not see vector instructions in asm statements: the distance a matrix instruction may want
                        asm("s_nop 1" : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(b[0]), "+v"(b[1]), "+v"(b[2]), "+v"(b[3]));
                        ps[ct][h] = words_to_half8(a[0], a[1], a[2], a[3]);
                        rest[ct][h] = words_to_half8(b[0], b[1], b[2], b[3]);
                        pbacc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eights, ps[ct][h], pbacc[ct], 0, 0, 0);
                        pbacc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eights, rest[ct][h], pbacc[ct], 0, 0, 0);
                    }
                if (kPairs && g % 2 == 1 && g + 1 < GV) read_pair(g + 1);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = 4 * g + k;
                    const int2_t w = words[c % 2];
                    if (c + 2 < 4 * GV) words[c % 2] = read_codes(c + 2);
                    __builtin_amdgcn_sched_barrier(0);
                    const half8_t a0 = code_operand((uint32_t)w.x), a1 = code_operand((uint32_t)w.y);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        acc[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, ps[ct][0], acc[ct][c], 0, 0, 0);
                        acc[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, ps[ct][1], acc[ct][c], 0, 0, 0);
                        acc[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, rest[ct][0], acc[ct][c], 0, 0, 0);
                        acc[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, rest[ct][1], acc[ct][c], 0, 0, 0);
                    }
                }
            }
            if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                issue_rest(buf);
            }
            buf = buf + 1 == S::RING ? 0 : buf + 1;
        }

        // ---- the rows' sums of this wave: lane (col, qk) holds elements 16 c + 4 qk .. + 3 of row 16 ct + col.  What is worked out
        // from the lane here is worked out from an opaque copy of it, or it would be kept in registers through the tile loop.
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        const int col = tid % 16, qk = tid % kWave / 16;
        auto sums = [&](int ct, int c) __attribute__((always_inline)) {
            float4_t o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = fmaf(acc[ct][c][r], kCodeScaleA, pbacc[ct][c / 4]);
            return o;
        };
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            l_run[ct] = xor32_sum(xor16_sum(l_run[ct]));
#pragma unroll
            for (int g = 0; g < GV; ++g) pbacc[ct][g] = xor32_sum(xor16_sum(pbacc[ct][g] * (qk == 0 ? -kCodeScaleA : qk == 1 ? 0.0f : qk == 2 ? 1.0f : 8.0f)));
        }
        auto finish_quad = [&](int64_t row, int e, float m, float l, float4_t o) __attribute__((always_inline)) {
            if (u.whole_row) {
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                const half2_t a = half2_t{(half_t)(o[0] * inv), (half_t)(o[1] * inv)}, b = half2_t{(half_t)(o[2] * inv), (half_t)(o[3] * inv)};
                *reinterpret_cast<uint2 *>(p.out + row * DV + e) = make_uint2(half2_to_bits(a), half2_to_bits(b));
            } else {
                const int64_t rec = row * p.slots + (u.which == 0 ? u.slot : p.slots - 1 - u.slot);
                *reinterpret_cast<float4_t *>(p.part_acc + rec * DV + e) = o;
                if (e == 0) *reinterpret_cast<float2 *>(p.part_ml + rec * 2) = make_float2(m, l);
            }
        };
        if (solo) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if (16 * ct + col >= u.rows) continue;
                int agent;
                const int64_t row = row_index(p, u, 16 * ct + col, agent);
#pragma unroll
                for (int c = 0; c < 4 * GV; ++c) finish_quad(row, 16 * c + 4 * qk, m_run[ct], l_run[ct], sums(ct, c));
            }
            return;
        }
        // the four waves of the workgroup join theirs, in wave order, by way of the tile buffers (nothing is on its way to them)
        float *const mine_lds = reinterpret_cast<float *>(region);
        wave_lds_sync();
        if (mine > 0) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if (16 * ct + col >= u.rows) continue;
#pragma unroll
                for (int c = 0; c < 4 * GV; ++c)
                    *reinterpret_cast<float4_t *>(mine_lds + (16 * ct + col) * S::ROW_PITCH + 16 * c + 4 * qk) = sums(ct, c);
            }
        }
        if (qk == 0) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                ml_lds[wave][16 * ct + col][0] = m_run[ct];
                ml_lds[wave][16 * ct + col][1] = mine > 0 ? l_run[ct] : 0.0f;
            }
        }
        __syncthreads();
        // a thread takes the same four elements of every STRIDE-th row, two rows at a time
        constexpr int QUADS = DV / 4, STRIDE = kThreads / QUADS;
        const int e = 4 * (tid % QUADS);
        for (int r0 = tid / QUADS; r0 < u.rows; r0 += 2 * STRIDE) {
            float4_t part[2][kWaves];
            float ml[2][kWaves][2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int r = min(r0 + k * STRIDE, u.rows - 1);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    part[k][w] = *reinterpret_cast<const float4_t *>(tiles_lds + w * S::WAVE_BYTES + 4 * (r * S::ROW_PITCH + e));
                    ml[k][w][0] = ml_lds[w][r][0];
                    ml[k][w][1] = ml_lds[w][r][1];
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int r = r0 + k * STRIDE;
                if (r >= u.rows) break;
                float m = kNegBig, l = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    if (ml[k][w][1] > 0.0f) m = fmaxf(m, ml[k][w][0]);
                float4_t o = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    // what a wave without tiles left in its buffer is no number to multiply
                    const float weight = ml[k][w][1] > 0.0f ? __builtin_amdgcn_exp2f(ml[k][w][0] - m) : 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] += weight > 0.0f ? weight * part[k][w][i] : 0.0f;
                    l = fmaf(weight, ml[k][w][1], l);
                }
                int agent;
                finish_quad(row_index(p, u, r, agent), e, m, l, o);
            }
        }
        __syncthreads(); // the tile buffers are free again
    };

    for (int x = (int)begin; x < x1;) {
        const Part u = locate(p, plan, x, x1, per, round, worker);
        if (CTP > 1 && u.rows > kCols) run_part(Int<CTP>(), u);
        else run_part(Int<1>(), u);
        x += u.counted;
    }
}

// Joins the records of every (layer, agent, query head): the prefix's, then those of the agent's own tokens.  A workgroup owns a row;
// a thread four elements of every PARTS-th record, kBatch of them asked for together; the threads' sums are joined in order.  Rows
// that the attention launch finished itself are left alone; rows that see no token become zeros.
constexpr int kBatch = 4;

template <int DV>
__global__ __launch_bounds__(kThreads) void prefix_merge_kernel(const float *__restrict__ part_acc, const float *__restrict__ part_ml,
                                                                const int32_t *__restrict__ plan, uint16_t *__restrict__ out,
                                                                int num_agents, int q_heads, int kv_heads, int slots, int row_tile)
{
    constexpr int QUADS = DV / 4, PARTS = kThreads / QUADS;
    __shared__ float4_t s_acc[PARTS][QUADS];
    __shared__ float s_ml[PARTS][2];
    const int64_t row = blockIdx.x;
    const int quad = threadIdx.x % QUADS, part = threadIdx.x / QUADS;
    const int qh = (int)(row % q_heads), agent = (int)(row / q_heads % num_agents), li = (int)(row / q_heads / num_agents);
    const int n_rep = q_heads / kv_heads, kvh = qh / n_rep;
    const int per = plan[0], head_tiles = plan[1], group_tiles = plan[2], round = plan[3];
    const int own0 = plan[kHeader + agent], own_tiles = plan[kHeader + num_agents + agent], shared = plan[kHeader + 2 * num_agents + agent];
    const int group0 = plan[kHeader + 3 * num_agents + agent], first_agent = plan[kHeader + 4 * num_agents + agent];
    const int base = (li * kv_heads + kvh) * head_tiles;
    auto records_of = [&](int u0, int tiles) { return tiles > 0 ? (u0 + rounded_up(tiles, round) - 1) / per - u0 / per + 1 : 0; };
    const int n_prefix = records_of(base + group0 + ((agent - first_agent) * n_rep + qh - kvh * n_rep) / row_tile * rounded_up(shared, round), shared);
    const int n_own = records_of(base + group_tiles + own0, own_tiles);
    if (shared == 0 && n_own == 1) return;
    const int records = n_prefix + n_own;
    const int64_t rec0 = row * slots;
    float m = kNegBig, l = 0.0f;
    float4_t o = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = part; s0 < records; s0 += PARTS * kBatch) {
        float mm[kBatch], ll[kBatch];
        float4_t a[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int at = s0 + k * PARTS, s = min(at, records - 1);
            const int64_t rec = rec0 + (s < n_prefix ? s : slots - 1 - (s - n_prefix));
            const float2 t = *reinterpret_cast<const float2 *>(part_ml + rec * 2);
            mm[k] = t.x;
            ll[k] = at < records ? t.y : 0.0f;
            a[k] = *reinterpret_cast<const float4_t *>(part_acc + rec * DV + 4 * quad);
        }
        float m_new = m;
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (ll[k] > 0.0f) m_new = fmaxf(m_new, mm[k]);
        const float keep = __builtin_amdgcn_exp2f(m - m_new);
        l *= keep;
        o *= keep;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (!(ll[k] > 0.0f)) continue;
            const float weight = __builtin_amdgcn_exp2f(mm[k] - m_new);
            l = fmaf(weight, ll[k], l);
            o += weight * a[k];
        }
        m = m_new;
    }
    s_acc[part][quad] = o;
    if (quad == 0) {
        s_ml[part][0] = m;
        s_ml[part][1] = l;
    }
    __syncthreads();
    if (part > 0) return;
    const int parts = min(PARTS, max(records, 1)); // that have any
    m = kNegBig;
    for (int k = 0; k < parts; ++k)
        if (s_ml[k][1] > 0.0f) m = fmaxf(m, s_ml[k][0]);
    l = 0.0f;
    o = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < parts; ++k) {
        if (!(s_ml[k][1] > 0.0f)) continue;
        const float weight = __builtin_amdgcn_exp2f(s_ml[k][0] - m);
        l = fmaf(weight, s_ml[k][1], l);
        o += weight * s_acc[k][quad];
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    const half2_t lo = half2_t{(half_t)(o[0] * inv), (half_t)(o[1] * inv)}, hi = half2_t{(half_t)(o[2] * inv), (half_t)(o[3] * inv)};
    *reinterpret_cast<uint2 *>(out + row * DV + 4 * quad) = make_uint2(half2_to_bits(lo), half2_to_bits(hi));
}

template <int DK, int DV, int CTP>
hipError_t launch_t(const PrefixParams &p, bool bf, int compute_units, hipStream_t stream)
{
    const dim3 grid((unsigned)(compute_units * Shape<DK, DV>::WAVES_PER_SIMD));
    if (bf) hipLaunchKernelGGL((prefix_attention_kernel<DK, DV, CTP, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((prefix_attention_kernel<DK, DV, CTP, false>), grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

template <int DK, int DV, int CTP>
hipError_t launch_columns(int ct, const PrefixParams &p, bool bf, int compute_units, hipStream_t stream)
{
    if constexpr (CTP > 1)
        if (ct < CTP) return launch_columns<DK, DV, CTP - 1>(ct, p, bf, compute_units, stream);
    return launch_t<DK, DV, CTP>(p, bf, compute_units, stream);
}

// Column tiles of a prefix unit: the rows of an average group in as few units as pay, all alike.  Three column tiles of 64-wide
// heads, two of wider ones.  Three or four of 128-wide heads take two layers of 128 rows behind 16,384 tokens from 82.0 to 96.6 and
// 99.7 us (four layers of 40 rows behind 4,096 from 36.8 to 35.1 and 35.6): in the plan a tile counts for one however many rows it has.
int column_tiles(const q4kv_spec &s, int num_agents, int num_groups)
{
    if (num_groups == 0) return 1;
    const int rows = s.num_q_heads / s.num_kv_heads * ((num_agents + num_groups - 1) / num_groups);
    const int tiles = (rows + kCols - 1) / kCols, most = s.v_dim == 64 ? 3 : 2, units = (tiles + most - 1) / most;
    return (tiles + units - 1) / units;
}

// Records per row: a worker's range is at least kSoloTiles (a wave's) or kWaves tiles (a workgroup's) long, and no shorter than an
// even share of all tiles, to which a row's prefix and own tiles, T together and no more than max_seq_len has, contribute T for every
// layer and KV head.  Each of the two may begin and end inside a range: two records more.
int record_slots(const q4kv_spec &s, int max_seq_len, int layers, int workgroups)
{
    const int64_t tiles = (max_seq_len + kWave - 1) / kWave, units = (int64_t)layers * s.num_kv_heads;
    const int64_t shared = std::min<int64_t>(tiles / kWaves, workgroups / units);
    const int64_t solo = std::min<int64_t>(tiles / kSoloTiles, (int64_t)workgroups * kWaves / units);
    return (int)std::max(shared, solo) + 4;
}

int prefix_workgroups(int compute_units) { return compute_units; }

} // namespace

int prefix_max_agents() { return kMaxAgents; }

bool prefix_supported(const q4kv_spec &s)
{
    if (s.v_aliases_k || s.num_q_heads / s.num_kv_heads > kCols) return false;
    return (s.k_dim == s.v_dim && (s.k_dim == 64 || s.k_dim == 128 || s.k_dim == 256)) || (s.k_dim == 192 && s.v_dim == 128);
}

int64_t prefix_tiles(const q4kv_spec &s, int num_agents, int num_groups, int max_seq_len, int layers)
{
    const int row_tile = kCols * column_tiles(s, num_agents, num_groups), n_rep = s.num_q_heads / s.num_kv_heads;
    const int64_t row_tiles = ((int64_t)num_agents * n_rep + row_tile - 1) / row_tile + num_groups;
    return (int64_t)layers * s.num_kv_heads * (num_agents + row_tiles) * ((max_seq_len + kWave - 1) / kWave);
}

size_t prefix_workspace_bytes(const q4kv_spec &s, int num_agents, int max_seq_len, int layers, int compute_units, size_t &acc_at, size_t &ml_at)
{
    const int slots = record_slots(s, max_seq_len, layers, prefix_workgroups(compute_units));
    const size_t records = (size_t)layers * num_agents * s.num_q_heads * slots;
    acc_at = ((size_t)plan_ints(num_agents) * sizeof(int32_t) + 255) / 256 * 256;
    ml_at = acc_at + records * s.v_dim * sizeof(float);
    return ml_at + records * 2 * sizeof(float);
}

hipError_t launch_prefix_attention(const PrefixArgs &a, hipStream_t stream)
{
    const q4kv_spec &s = *a.spec;
    PrefixParams p;
    p.k_codes = a.k->codes; p.k_scale = a.k->scale; p.k_bias = a.k->bias;
    p.v_codes = a.v->codes; p.v_scale = a.v->scale; p.v_bias = a.v->bias;
    p.q = a.q; p.out = a.out;
    p.block_table = a.block_table; p.seq_len = a.seq_len; p.group_begin = a.group_begin; p.prefix_len = a.prefix_len;
    size_t acc_at, ml_at;
    prefix_workspace_bytes(s, a.num_agents, a.max_seq_len, a.layers, a.compute_units, acc_at, ml_at);
    p.plan = static_cast<int32_t *>(a.workspace);
    p.part_acc = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + acc_at);
    p.part_ml = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + ml_at);
    p.num_agents = a.num_agents; p.num_groups = a.num_groups; p.max_blocks = a.max_blocks; p.num_blocks = a.k->num_blocks;
    p.kv_heads = s.num_kv_heads; p.q_heads = s.num_q_heads; p.n_rep = s.num_q_heads / s.num_kv_heads;
    p.layer_begin = a.layer_begin; p.layers = a.layers; p.max_seq_len = a.max_seq_len;
    p.slots = record_slots(s, a.max_seq_len, a.layers, prefix_workgroups(a.compute_units));
    const int ct = column_tiles(s, a.num_agents, a.num_groups);
    p.row_tile = kCols * ct;
    p.score_scale = a.sm_scale * kLog2e;
    p.inv_n_rep = 1.0f / (float)p.n_rep;
    const bool bf = s.param_format == Q4KV_PARAMS_BF16;
    hipError_t e = hipErrorInvalidValue;
    if (s.k_dim == 256) e = launch_columns<256, 256, 2>(ct, p, bf, a.compute_units, stream);
    else if (s.k_dim == 192) e = launch_columns<192, 128, 2>(ct, p, bf, a.compute_units, stream);
    else if (s.k_dim == 128) e = launch_columns<128, 128, 2>(ct, p, bf, a.compute_units, stream);
    else if (s.k_dim == 64) e = launch_columns<64, 64, 3>(ct, p, bf, a.compute_units, stream);
    if (e != hipSuccess) return e;
    const auto merge = s.v_dim == 256 ? prefix_merge_kernel<256> : s.v_dim == 128 ? prefix_merge_kernel<128> : prefix_merge_kernel<64>;
    hipLaunchKernelGGL(merge, dim3((unsigned)((int64_t)a.layers * a.num_agents * s.num_q_heads)), dim3(kThreads), 0, stream, p.part_acc, p.part_ml,
                       p.plan, p.out, a.num_agents, s.num_q_heads, s.num_kv_heads, p.slots, p.row_tile);
    return hipGetLastError();
}

} // namespace q4kv
