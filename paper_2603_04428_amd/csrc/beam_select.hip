// The choice of a beam search's step: for row r (a beam) of a group and token t
//     total(r, t) = score(r) + x(r, t) - log sum_u exp x(r, u)
// and the num_out largest totals of each group, equal ones in the order of row, then logit, then token.
//
// One pass over the logits.  A wave takes a span of one row and leaves a record: the span's sum of exp(x - ref), ref, and its
// num_out largest elements in order.  A second kernel, one workgroup per group, adds the sums up, forms the totals of what the
// records list and takes the best.  Two launches, no atomics on memory, and the same order of every sum on every run.
//
// What bounds it is memory for large batches (every logit is read once) and the trips to memory of two launches for small ones.
#include <type_traits>

#include "q4_device.h"
#include "q4kv_internal.h"

namespace q4kv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kList = 192;     // candidates a wave can hold: what it keeps (64 at most) and two appends of up to 64
constexpr int kMergeList = 1536;
constexpr int kUnroll = 4;     // 16-byte loads per lane in flight

struct SpanRecord {
    double sum; // of exp(x - ref) over the span; ref
    float ref;
    int32_t pad;
};

struct SelectParams {
    const void *logits;
    int64_t row_stride;
    const float *score;
    const int32_t *end_token, *group_begin;
    SpanRecord *records;  // [rows][spans]
    uint64_t *keys;       // [rows][spans][num_out]: value and place, largest first, 0 where there are no more
    double *row_log;      // [rows]: logarithm of the row's sum of exponentials
    int32_t *parent, *token;
    float *total;
    int32_t rows, vocab, spans, span_len, groups, num_out;
};

// binary32 as unsigned integers of the same order, and back
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o)
{
    return __builtin_bit_cast(float, o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t ordered64(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return u ^ ((uint64_t)((int64_t)u >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double unordered64(uint64_t o)
{
    return __builtin_bit_cast(double, o & 0x8000000000000000ull ? o ^ 0x8000000000000000ull : ~o);
}

// A candidate: its value, then (equal values) the lower token first.  Never 0: tokens are below 2^31.
__device__ __forceinline__ uint64_t candidate(float x, int32_t token)
{
    return (uint64_t)ordered(x + 0.0f) << 32 | (uint32_t)~token; // + 0: both zeros are one value
}

// The type of the logits: elements of a 16-byte load, and those as binary32.
typedef uint32_t words_t __attribute__((ext_vector_type(4)));
template <int FORMAT>
struct Logits {
    static constexpr int kPer = FORMAT == 2 ? 4 : 8, kBytes = 16 / kPer;
    struct __attribute__((packed, aligned(kBytes))) Loose { words_t w; }; // rows may begin at any element
    static __device__ __forceinline__ words_t load(const char *row, int i) { return reinterpret_cast<const Loose *>(row + (int64_t)i * kBytes)->w; }
    // the same where the row may end inside: -inf from `end` on (end > 0)
    static __device__ __forceinline__ words_t load_to(const char *row, int i, int end)
    {
        typedef std::conditional_t<FORMAT == 2, uint32_t, uint16_t> bits_t;
        constexpr uint32_t banned = FORMAT == 2 ? 0xff800000u : FORMAT == 1 ? 0xff80u : 0xfc00u;
        uint32_t e[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            e[j] = reinterpret_cast<const bits_t *>(row)[min(i + j, end - 1)];
            if (i + j >= end) e[j] = banned;
        }
        if constexpr (FORMAT == 2) return words_t{e[0], e[1], e[2], e[3]};
        else return words_t{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
    }
    static __device__ __forceinline__ void widen(const words_t &w, float *x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = w[i]; // a value of its own: a bit cast of a vector's element takes the vector's first
            if constexpr (FORMAT == 2) {
                x[i] = __builtin_bit_cast(float, v);
            } else if constexpr (FORMAT == 1) {
                x[2 * i] = __builtin_bit_cast(float, v << 16);
                x[2 * i + 1] = __builtin_bit_cast(float, v & 0xffff0000u);
            } else {
                const half2_t h = bits_to_half2(v);
                x[2 * i] = (float)h.x;
                x[2 * i + 1] = (float)h.y;
            }
        }
    }
};

constexpr float kLowest = -3.40282347e38f, kInf = __builtin_inff();

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c)); // the builtins quiet each operand first
    return r;
}

// exp(x - ref): the difference first (exact for neighbouring values of 16-bit types), then log2 e in two terms, so that the
// constant's own rounding (1.3e-8 of the exponent) does not shift every term of a sum the same way
__device__ __forceinline__ float exp_from(float x, float ref)
{
    const float d = x - ref;
    return __builtin_amdgcn_exp2f(__builtin_fmaf(d, 1.925963033500e-8f, d * 1.442695022f));
}

// The `keep` largest of n <= kList candidates in LDS, in order, at the front of the list (one wave; every lane calls).
__device__ __forceinline__ int keep_best(uint64_t *list, int n, int keep)
{
    const int lane = threadIdx.x & 63;
    constexpr int PER = kList / kWave;
    uint64_t mine[PER];
    int rank[PER];
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        mine[i] = i * kWave + lane < n ? list[i * kWave + lane] : 0;
        rank[i] = 0;
    }
    if (n <= kWave) {
#pragma unroll 4
        for (int j = 0; j < n; ++j) rank[0] += list[j] > mine[0];
    } else {
#pragma unroll 2
        for (int j = 0; j < n; ++j) {
            const uint64_t other = list[j];
#pragma unroll
            for (int i = 0; i < PER; ++i) rank[i] += other > mine[i];
        }
    }
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (i * kWave + lane < n && rank[i] < keep) list[rank[i]] = mine[i]; // candidates differ, so their ranks do
    wave_lds_sync();
    return min(n, keep);
}

// A value above `floor` that at least `keep` lanes reach with their `mine`, and few more do: halving of the range between the
// lanes' extremes until the count is between keep and twice that.  At least `keep` lanes are above the floor.
__device__ __forceinline__ float reached_by(float mine, float floor, float top, int keep)
{
    const float lowest = -wave_max(-mine);
    uint32_t lo = max(ordered(floor) + 1, ordered(lowest)), hi = ordered(top); // enough lanes reach lo, none is above hi
    while (lo < hi) { // 32 rounds at most
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        const int n = __popcll(__ballot(mine >= unordered(mid)));
        if (n >= keep) {
            lo = mid;
            if (n <= 2 * keep) break;
        } else {
            hi = mid - 1;
        }
    }
    return unordered(lo);
}

// Element `at` of N values in registers (N a power of two).
template <int N>
__device__ __forceinline__ float element(const float *x, int at)
{
    if constexpr (N == 1) {
        return x[0];
    } else {
        const float a = element<N / 2>(x, at), b = element<N / 2>(x + N / 2, at);
        return at & (N / 2) ? b : a;
    }
}

// A span of a row: its candidates, in order, in `list`; the sum of exp(x - ref) and ref.  clean: NaN and +inf are replaced while
// reading.  Without it they show in the maximum and the sum, and the answer is false: the span is to be done again.
template <int FORMAT>
__device__ __forceinline__ bool scan_span(const char *row, int begin, int end, int keep, bool clean, uint64_t *list, int &listed,
                                          double &sum_out, float &ref_out)
{
    typedef Logits<FORMAT> L;
    constexpr int PER = L::kPer, HELD = kUnroll * PER, STEP = kWave * HELD;
    const int lane = threadIdx.x & 63;
    float ref = kLowest, threshold = kLowest; // candidates are at or above the threshold
    double sum = 0.0;
    int n = 0;
    words_t next[kUnroll] = {};
    for (int at = begin - STEP; at < end; at += STEP) {
        // the values that were asked for a step ago, and the next ones asked for
        float x[HELD];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) L::widen(next[u], x + u * PER);
        const int ahead = at + STEP + lane * PER;
        if (at + 2 * STEP <= end) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) next[u] = L::load(row, ahead + u * kWave * PER);
        } else if (at + STEP < end) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) next[u] = L::load_to(row, ahead + u * kWave * PER, end);
        }
        if (at < begin) continue;
        if (clean) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) x[i] = x[i] != x[i] ? -kInf : fminf(x[i], -kLowest);
        }
        float mine = x[0];
#pragma unroll
        for (int i = 1; i + 1 < HELD; i += 2) mine = max3(x[i], x[i + 1], mine);
        mine = fmaxf(mine, x[HELD - 1]);
        // The reference is the maximum of the first step; it moves only where an exponential could grow large.
        float highest = 0.0f;
        if (at == begin || __any(mine > ref + 40.0f)) {
            highest = fmaxf(wave_max(mine), kLowest);
            if (at != begin) sum *= __builtin_amdgcn_exp2f((ref - highest) * 1.442695022f);
            ref = highest;
        }
        float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < HELD; ++i) part[i & 3] += exp_from(x[i], ref);
        sum += (double)((part[0] + part[1]) + (part[2] + part[3]));
        const uint64_t over = __ballot(mine >= threshold);
        if (over == 0) continue;
        // `keep` lanes and more with a candidate: this step alone has so many elements at or above what `keep` of its lanes reach
        if (__popcll(over) >= keep) threshold = reached_by(mine, unordered(ordered(threshold) - 1), wave_max(mine), keep);
        // bit i: x[i] is no less than the threshold, by the sign of the difference (either zero less -0 is +0)
        if (threshold == 0.0f) threshold = -0.0f;
        uint32_t bits = 0;
#pragma unroll
        for (int i = HELD - 1; i >= 0; --i) bits = __builtin_amdgcn_alignbit(bits, __builtin_bit_cast(uint32_t, x[i] - threshold), 31);
        bits = ~bits & (uint32_t)((1ull << HELD) - 1);
        while (true) {
            const uint64_t mask = __ballot(bits != 0);
            if (mask == 0) break;
            if (n > kList - kWave) {
                n = keep_best(list, n, keep);
                if (n == keep) threshold = fmaxf(threshold, unordered((uint32_t)(list[keep - 1] >> 32)));
            }
            const int i = bits ? __ffs(bits) - 1 : 0;
            const float v = element<HELD>(x, i);
            const bool take = bits && v >= threshold;
            const uint64_t taken = __ballot(take);
            if (take) {
                const int place = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(taken >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)taken, 0));
                list[place] = candidate(v, at + (i / PER * kWave + lane) * PER + i % PER);
            }
            n += __popcll(taken);
            bits &= bits - 1;
        }
        // later steps have higher tokens: what only equals the last one kept does not come in any more
        if (at + STEP < end && n >= keep) {
            n = keep_best(list, n, keep);
            threshold = fmaxf(threshold, unordered((uint32_t)(list[keep - 1] >> 32) + 1));
        }
    }
    listed = keep_best(list, n, keep);
    ref_out = ref;
    sum = row_sum<kWave>(sum);
    if (!clean && !(sum < (double)kInf && ref < kInf)) return false; // a NaN or +inf among them
    // The largest elements dominate the sum of a peaked row: theirs are taken again in binary64.
    double fix = 0.0;
    if (lane < listed) {
        const float v = unordered((uint32_t)(list[lane] >> 32));
        fix = exp((double)v - (double)ref) - (double)exp_from(v, ref);
    }
    sum_out = sum + row_sum<kWave>(fix);
    return true;
}

__device__ __forceinline__ bool dead(float score) { return !(score > -kInf); }

template <int FORMAT>
__global__ __launch_bounds__(kThreads, 4) void beam_scan_kernel(SelectParams p)
{
    __shared__ uint64_t s_list[kWaves][kList];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * kWaves + wave; // waves are on their own: no barrier
    const int r = (int)(unit / p.spans), span = (int)(unit - (int64_t)r * p.spans);
    if (r >= p.rows) return;
    if (dead(p.score[r]) || (p.end_token && p.end_token[r] >= 0)) return;
    const int begin = span * p.span_len, end = p.vocab - begin < p.span_len ? p.vocab : begin + p.span_len;
    const char *row = static_cast<const char *>(p.logits) + (int64_t)r * p.row_stride * Logits<FORMAT>::kBytes;
    uint64_t *list = s_list[wave];
    int n;
    double sum;
    float ref;
    for (bool clean = false; !scan_span<FORMAT>(row, begin, end, p.num_out, clean, list, n, sum, ref);) clean = true; // twice at most
    if (lane == 0) p.records[unit] = SpanRecord{sum, ref, 0};
    if (lane < p.num_out) p.keys[unit * p.num_out + lane] = lane < n ? list[lane] : 0;
}

// A continuation in the merge: its total, then the lower row, then the row's own order (where a logit is so large that totals
// next to it are equal, the larger logit is still the better one).
struct Choice {
    uint64_t total, key;
    uint32_t row;
};
__device__ __forceinline__ bool better(const Choice &a, const Choice &b)
{
    return a.total > b.total || (a.total == b.total && (a.row < b.row || (a.row == b.row && a.key > b.key)));
}

struct MergeList {
    uint64_t total[kMergeList], key[kMergeList];
    uint32_t row[kMergeList];
    __device__ __forceinline__ Choice at(int i) const { return Choice{total[i], key[i], row[i]}; }
    __device__ __forceinline__ void set(int i, const Choice &c)
    {
        total[i] = c.total;
        key[i] = c.key;
        row[i] = c.row;
    }
};

// As keep_best, for a workgroup's list; `room`: LDS for what is kept.
__device__ __forceinline__ int keep_best_choices(MergeList &list, Choice *room, int n, int keep)
{
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const Choice mine = list.at(i);
        int ahead = 0, equal = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) {
            const uint64_t other = list.total[j];
            ahead += other > mine.total;
            equal += other == mine.total;
        }
        if (equal > 1)
#pragma unroll 1
            for (int j = 0; j < n; ++j) ahead += list.total[j] == mine.total && better(list.at(j), mine);
        if (ahead < keep) room[ahead] = mine;
    }
    __syncthreads();
    const int kept = min(n, keep);
    if ((int)threadIdx.x < kept) list.set(threadIdx.x, room[threadIdx.x]);
    __syncthreads();
    return kept;
}

// Where a thread is in the merge: a record (a span's elements in order, the next kAhead of them in registers), or a finished row.
constexpr int kAhead = 4;
struct Walk {
    const uint64_t *keys;
    uint64_t ahead[kAhead];
    double score, row_log;
    int32_t row, end;
    bool on;
};

__device__ __forceinline__ Walk walk_at(const SelectParams &p, int lo, int64_t i, int64_t records)
{
    Walk w;
    w.on = i < records;
    w.keys = nullptr;
    w.score = w.row_log = 0.0;
    w.row = lo;
    w.end = -1;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) w.ahead[j] = 0;
    if (w.on) {
        const int span = (int)(i % p.spans);
        w.row = lo + (int)(i / p.spans);
        w.keys = p.keys + ((int64_t)w.row * p.spans + span) * p.num_out;
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (j < p.num_out) w.ahead[j] = w.keys[j];
        const float score = p.score[w.row];
        if (p.end_token) w.end = p.end_token[w.row];
        w.score = (double)score;
        w.on = !dead(score) && (w.end < 0 || span == 0);
        if (w.end >= 0) w.ahead[0] = (uint32_t)~w.end; // its one continuation; the rest is never looked at
    }
    return w;
}

__device__ __forceinline__ Choice choice_of(const Walk &w, uint64_t key)
{
    const double total = w.end >= 0 ? w.score : w.score + ((double)unordered((uint32_t)(key >> 32)) - w.row_log);
    return Choice{ordered64(total), key, (uint32_t)w.row};
}

__global__ __launch_bounds__(kThreads) void beam_merge_kernel(SelectParams p)
{
    __shared__ MergeList s_list;
    __shared__ Choice s_room[Q4KV_MAX_BEAM_OUT];
    __shared__ int s_n;
    __shared__ float s_reached[kWaves];
    const int g = blockIdx.x, t = threadIdx.x, keep = p.num_out;
    const int lo = min(max(p.group_begin[g], 0), p.rows), hi = min(max(p.group_begin[g + 1], 0), p.rows);
    const int64_t records = (int64_t)max(hi - lo, 0) * p.spans;
    Walk w = walk_at(p, lo, t, records); // of the first records; asked for ahead of the rows' sums
    if (t == 0) s_n = 0;
    // logarithms of the rows' sums: as many lanes to a row as it has spans, up to a wave
    int lanes = 1;
    while (lanes < p.spans && lanes < kWave) lanes <<= 1;
    for (int r = lo + t / lanes; r - t / lanes < hi; r += kThreads / lanes) {
        const SpanRecord *rec = p.records + (int64_t)r * p.spans;
        const bool on = r < hi && !dead(p.score[r]) && !(p.end_token && p.end_token[r] >= 0);
        const int first = t & (lanes - 1);
        float ref = kLowest;
        if (on)
            for (int i = first; i < p.spans; i += lanes) ref = fmaxf(ref, rec[i].ref);
        for (int off = 1; off < lanes; off <<= 1) ref = fmaxf(ref, __shfl_xor(ref, off));
        double sum = 0.0;
        if (on)
            for (int i = first; i < p.spans; i += lanes) sum += rec[i].sum * exp((double)rec[i].ref - (double)ref);
        for (int off = 1; off < lanes; off <<= 1) sum += __shfl_xor(sum, off);
        if (on && first == 0) p.row_log[r] = (double)ref + log(sum); // -inf for a row without any, which is never used
    }
    __syncthreads();
    if (w.on && w.end < 0) w.row_log = p.row_log[w.row];
    // What `keep` lanes of a wave reach with the first element of their records is reached by the group's best `keep`.
    float reached = -kInf;
    {
        float mine = w.on && w.ahead[0] ? (float)unordered64(choice_of(w, w.ahead[0]).total) : -kInf;
        if (__popcll(__ballot(mine > -kInf)) >= keep) reached = reached_by(mine, -kInf, wave_max(mine), keep);
        if ((t & 63) == 0) s_reached[t >> 6] = reached;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) reached = fmaxf(reached, s_reached[i]);
    // Every thread walks down its record until its next element is no better than the worst kept.
    int n = 0;
    Choice worst = {};
    bool full = false;
    for (int64_t base = 0; base < records; base += kThreads) {
        if (base > 0) {
            w = walk_at(p, lo, base + t, records);
            if (w.on && w.end < 0) w.row_log = p.row_log[w.row];
        }
        for (int next = 0;; next += kAhead) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) { // at most kAhead * kThreads in a round
                const Choice c = choice_of(w, w.ahead[j]);
                w.on = w.on && w.ahead[j] != 0 && (float)unordered64(c.total) >= reached && !(full && !better(c, worst));
                if (w.on) s_list.set(atomicAdd(&s_n, 1), c);
                if (w.end >= 0) w.on = false;
            }
            const bool more = __syncthreads_or(w.on && next + kAhead < keep);
            n = s_n;
            __syncthreads(); // everybody has the same n before the next push
            if (n > kMergeList - kAhead * kThreads || (more && !full && n >= keep)) {
                n = keep_best_choices(s_list, s_room, n, keep);
                if (t == 0) s_n = n;
                full = n == keep;
                if (full) worst = s_list.at(keep - 1);
                __syncthreads();
            }
            if (!more) break;
#pragma unroll
            for (int j = 0; j < kAhead; ++j) w.ahead[j] = w.on && next + kAhead + j < keep ? w.keys[next + kAhead + j] : 0;
        }
    }
    n = keep_best_choices(s_list, s_room, n, keep);
    for (int i = t; i < keep; i += kThreads) {
        const int64_t at = (int64_t)g * keep + i;
        const bool in = i < n;
        p.parent[at] = in ? (int32_t)s_list.row[i] : -1;
        p.token[at] = in ? (int32_t)~(uint32_t)s_list.key[i] : -1;
        p.total[at] = in ? (float)unordered64(s_list.total[i]) : -kInf;
    }
}

// Elements of a span: whole steps of a wave, so many that about kWavesPerCu waves per compute unit share the call's rows.
constexpr int kWavesPerCu = 8, kMaxSteps = 8;
int span_length(int format, int vocab, int rows, int compute_units)
{
    const int64_t step = (int64_t)kWave * kUnroll * (format == 2 ? 4 : 8);
    const int64_t steps = ((int64_t)vocab + step - 1) / step * rows / ((int64_t)compute_units * kWavesPerCu);
    return (int)(step * (steps < 1 ? 1 : steps > kMaxSteps ? kMaxSteps : steps));
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

} // namespace

int beam_select_spans(int format, int vocab, int rows, int compute_units)
{
    const int len = span_length(format, vocab, rows, compute_units);
    return (int)(((int64_t)vocab + len - 1) / len);
}

size_t beam_select_workspace_bytes(int format, int vocab, int rows, int num_out, int compute_units)
{
    const size_t units = (size_t)rows * beam_select_spans(format, vocab, rows, compute_units);
    return up(units * sizeof(SpanRecord)) + up((size_t)rows * sizeof(double)) + up(units * num_out * sizeof(uint64_t));
}

hipError_t launch_beam_select(const BeamSelectArgs &a, hipStream_t stream)
{
    SelectParams p;
    p.logits = a.logits;
    p.row_stride = a.row_stride;
    p.score = a.score;
    p.end_token = a.end_token;
    p.group_begin = a.group_begin;
    p.rows = a.rows;
    p.vocab = a.vocab;
    p.span_len = span_length(a.format, a.vocab, a.rows, a.compute_units);
    p.spans = beam_select_spans(a.format, a.vocab, a.rows, a.compute_units);
    p.groups = a.groups;
    p.num_out = a.num_out;
    p.parent = a.parent;
    p.token = a.token;
    p.total = a.total;
    const int64_t units = (int64_t)p.rows * p.spans;
    char *at = static_cast<char *>(a.workspace);
    p.records = reinterpret_cast<SpanRecord *>(at);
    at += up((size_t)units * sizeof(SpanRecord));
    p.row_log = reinterpret_cast<double *>(at);
    at += up((size_t)p.rows * sizeof(double));
    p.keys = reinterpret_cast<uint64_t *>(at);
    if (units > 0) {
        const dim3 grid((unsigned)((units + kWaves - 1) / kWaves));
        if (a.format == 0)
            hipLaunchKernelGGL(beam_scan_kernel<0>, grid, dim3(kThreads), 0, stream, p);
        else if (a.format == 1)
            hipLaunchKernelGGL(beam_scan_kernel<1>, grid, dim3(kThreads), 0, stream, p);
        else
            hipLaunchKernelGGL(beam_scan_kernel<2>, grid, dim3(kThreads), 0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(beam_merge_kernel, dim3((unsigned)p.groups), dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

} // namespace q4kv
