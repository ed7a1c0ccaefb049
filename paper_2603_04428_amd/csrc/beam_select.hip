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
constexpr int kRowLogs = 64; // rows of a group whose logarithms are kept in LDS
constexpr int kHeld = 32;      // elements of a step per lane

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

// exp(x - ref) as 2^(x c - ref c), one fused multiply-add in front of the exponential.  log2 e in binary32 is 1.93e-8 too small,
// which would shift every term of a sum the same way (15 below the reference by 2e-7): in 5 of 32 places the next larger number
// stands for it, 1e-7 too large, so that what is left on average is 6e-10.  ref c is rounded; the terms are 2^-shift too large
// then, the same for all places of one constant.
constexpr float kLog2e[2] = {1.442695022f, 1.442695141f};
constexpr double kLog2 = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

// exp r for |r| <= 0.35 to 3e-13: the first eleven terms of its series
__device__ __forceinline__ double exp_series(double r)
{
    double y = 1.0 / 3628800.0;
#pragma unroll
    for (int n = 9; n >= 0; --n) {
        constexpr double inverse[10] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880};
        y = __builtin_fma(y, r, inverse[n]);
    }
    return y;
}
// exp d for d <= 1, -inf as well, to 1e-12: 2^n times the series of what is left of d
__device__ __forceinline__ double exp_wide(double d)
{
    d = fmax(d, -1000.0);
    const double n = __builtin_rint(d * kLog2);
    return __builtin_amdgcn_ldexp(exp_series(__builtin_fma(-n, kLn2, d)), (int)n);
}
// log v, v > 0: the instruction's binary32 logarithm, and one step of Newton's method on exp
__device__ __forceinline__ double log_wide(double v)
{
    const int e = __builtin_amdgcn_frexp_exp(v);
    const double m = __builtin_amdgcn_ldexp(v, -e); // [0.5, 1)
    const double y = (double)(__builtin_amdgcn_logf((float)m) * 0.693147181f); // -0.7 .. 0, to 1e-7
    return (y + __builtin_fma(m, exp_wide(-y), -1.0)) + e * kLn2;
}
struct Reference {
    float ref, minus[2]; // -ref c
    __device__ __forceinline__ void set(float r)
    {
        ref = r;
        minus[0] = -(r * kLog2e[0]);
        minus[1] = -(r * kLog2e[1]);
    }
    template <int WHICH>
    __device__ __forceinline__ float exp(float x) const
    {
        return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e[WHICH], minus[WHICH]));
    }
    // what the sum of such terms has to be multiplied with
    __device__ __forceinline__ double unshift(int which) const
    {
        return exp_series(-kLn2 * ((double)ref * (double)kLog2e[which] + (double)minus[which]));
    }
    // the rounding of ref c is a small part of one: below 2^20 it is 2^-4 or less
    __device__ __forceinline__ bool usable() const { return fabsf(minus[0]) < 0x1p20f; }
};

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
        const int lo = (int)(uint32_t)mine[0], hi = (int)(mine[0] >> 32);
        for (int j = 0; j < n; ++j)
            rank[0] += ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, j) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, j)) > mine[0];
    } else {
#pragma unroll 4
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

// A value that at least `keep` lanes reach with their `mine`, and few more do.  For up to eight the lanes are cut into eight (four)
// groups: every group has a lane that reaches the lowest of the groups' maxima.  Where that lets many lanes through, and for more
// than eight, by halving the range up to the largest until the count is between keep and twice that.
__device__ __forceinline__ float reached_by(float mine, int keep)
{
    float low;
    if (keep <= 8) {
        float v = mine;
        v = fmaxf(v, Q4KV_DPP(v, v, 0xB1, 0xF));                 // quad_perm [1,0,3,2]
        v = fmaxf(v, Q4KV_DPP(v, v, 0x4E, 0xF));                 // quad_perm [2,3,0,1]
        v = fmaxf(v, Q4KV_DPP(v, v, 0x141, 0xF));                // row_half_mirror: groups of eight lanes
        const float w = Q4KV_DPP(v, v, 0x140, 0xF);              // row_mirror: the other eight of a row
        v = keep <= 4 ? fmaxf(v, w) : fminf(v, w);
        low = -xor32_max(xor16_max(-v));
        if (__popcll(__ballot(mine >= low)) <= 2 * keep + 8) return low;
    } else {
        low = -wave_max(-mine);
    }
    uint32_t lo = ordered(low), hi = ordered(wave_max(mine)); // enough lanes reach lo, none is above hi
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

__device__ __forceinline__ bool dead(float score) { return !(score > -kInf); }

// A span of a row: its candidates, in order, in `list`; the sum of exp(x - ref) and ref.  A lane has UNROLL loads of a step.
// CLEAN: NaN and +inf are replaced while reading.  Without it they show in the maximum and the sum, and the answer is false: the
// span is to be done again (so it is where the largest logit is beyond 700,000 on either side of zero).
template <int FORMAT, bool CLEAN, int UNROLL, typename Skip>
__device__ __forceinline__ bool scan_span(const char *row, int begin, int end, int keep, Skip skip, uint64_t *list, int &listed, double &sum_out,
                                          float &ref_out)
{
    typedef Logits<FORMAT> L;
    constexpr int PER = L::kPer, STEP = kWave * UNROLL * PER;
    // places of the larger constant: 5 of a lane's 32
    constexpr auto upper = [](int u, int e) { return PER == 8 ? e == 0 || (u == 0 && e == 4) : e == 0 && u < 5; };
    static_assert(CLEAN || UNROLL * PER == 32, "places of the larger constant");
    const int lane = threadIdx.x & 63;
    Reference at_ref;
    at_ref.set(0.0f);
    float threshold = kLowest; // candidates are at or above the threshold
    double sum[2] = {0.0, 0.0};
    int n = 0;
    bool unset = true;
    auto widen = [](const words_t &w, float (&x)[PER]) {
        L::widen(w, x);
        if constexpr (CLEAN) {
#pragma unroll
            for (int e = 0; e < PER; ++e) x[e] = x[e] != x[e] ? -kInf : fminf(x[e], -kLowest);
        }
    };
    words_t next[UNROLL] = {};
    for (int at = begin - STEP; at < end; at += STEP) {
        // the values that were asked for a step ago, and the next ones asked for
        words_t now[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) now[u] = next[u];
        const int ahead = at + STEP + lane * PER;
        if (at + 2 * STEP <= end) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) next[u] = L::load(row, ahead + u * kWave * PER);
        } else if (at + STEP < end) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) next[u] = L::load_to(row, ahead + u * kWave * PER, end);
        }
        if (at < begin) {
            if (skip()) break; // asked for while the first values are on their way
            continue;
        }
        float top[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if constexpr (FORMAT == 0 && !CLEAN) {
                const half2_t h = bits_to_half2(pk_max(pk_max(now[u][0], now[u][1]), pk_max(now[u][2], now[u][3])));
                top[u] = fmaxf((float)h.x, (float)h.y);
            } else {
                float x[PER];
                widen(now[u], x);
                top[u] = max3(x[0], x[1], x[2]);
#pragma unroll
                for (int e = 3; e + 1 < PER; e += 2) top[u] = max3(x[e], x[e + 1], top[u]);
                top[u] = fmaxf(top[u], x[PER - 1]);
            }
        }
        float mine = top[0];
#pragma unroll
        for (int u = 1; u < UNROLL; ++u) mine = fmaxf(mine, top[u]);
        // The reference is the maximum of the first step that has a value; it moves only where an exponential could grow large.
        if (unset || __any(mine > at_ref.ref + 40.0f)) {
            const float highest = wave_max(mine);
            if (highest > -kInf) {
                const float scale = unset ? 0.0f : __builtin_amdgcn_exp2f((at_ref.ref - highest) * kLog2e[0]);
                sum[0] *= scale;
                sum[1] *= scale;
                at_ref.set(highest);
                unset = false;
            }
        }
        float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float x[PER];
            widen(now[u], x);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if (CLEAN) part[1] += __builtin_amdgcn_exp2f((x[e] - at_ref.ref) * kLog2e[0]);
                else if (upper(u, e)) part[0] += at_ref.exp<1>(x[e]);
                else part[1 + (u * PER + e) % 3] += at_ref.exp<0>(x[e]);
            }
        }
        sum[0] += (double)(part[1] + part[2] + part[3]);
        if (!CLEAN) sum[1] += (double)part[0];
        const uint64_t over = __ballot(mine >= threshold);
        if (over == 0) continue;
        // `keep` lanes and more with a candidate: this step alone has so many elements at or above what `keep` of its lanes reach
        if (__popcll(over) >= keep) threshold = fmaxf(threshold, reached_by(mine, keep));
        uint32_t granules = 0;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) granules |= __any(top[u] >= threshold) ? 1u << u : 0u;
        while (granules) {
            const int u = __ffs(granules) - 1;
            granules &= granules - 1;
            words_t w = now[0];
#pragma unroll
            for (int k = 1; k < UNROLL; ++k)
                if (u == k) w = now[k];
            float x[PER];
            widen(w, x);
            // bit e: x[e] is no less than the threshold, by the sign of the difference (either zero less -0 is +0)
            if (threshold == 0.0f) threshold = -0.0f;
            uint32_t bits = 0;
#pragma unroll
            for (int e = PER - 1; e >= 0; --e) bits = __builtin_amdgcn_alignbit(bits, __builtin_bit_cast(uint32_t, x[e] - threshold), 31);
            bits = ~bits & ((1u << PER) - 1);
            while (true) {
                const uint64_t mask = __ballot(bits != 0);
                if (mask == 0) break;
                if (n > kList - kWave) {
                    n = keep_best(list, n, keep);
                    if (n == keep) threshold = fmaxf(threshold, unordered((uint32_t)(list[keep - 1] >> 32)));
                }
                const int e = bits ? __ffs(bits) - 1 : 0;
                const float v = element<PER>(x, e);
                const bool take = bits && v >= threshold;
                const uint64_t taken = __ballot(take);
                if (take) {
                    const int place = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(taken >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)taken, 0));
                    list[place] = candidate(v, at + (u * kWave + lane) * PER + e);
                }
                n += __popcll(taken);
                bits &= bits - 1;
            }
        }
        // Later steps have higher tokens: what only equals the last one kept does not come in any more.  The list is put in order
        // for that after the first of them, and then whenever it has grown to twice what is kept.
        if (at + STEP < end && n >= keep && (at == begin || n >= 2 * keep)) {
            n = keep_best(list, n, keep);
            threshold = fmaxf(threshold, unordered((uint32_t)(list[keep - 1] >> 32) + 1));
        }
    }
    listed = keep_best(list, n, keep);
    ref_out = unset ? kLowest : at_ref.ref;
    const double shift[2] = {CLEAN ? 1.0 : at_ref.unshift(0), CLEAN ? 1.0 : at_ref.unshift(1)};
    const double all = row_sum<kWave>(sum[0] * shift[0] + sum[1] * shift[1]);
    if (!CLEAN && !(all < (double)kInf && at_ref.usable())) return false; // a NaN or +inf among them, or a far reference
    // The largest elements dominate the sum of a peaked row: theirs are taken again in binary64.
    double fix = 0.0;
    if (lane < listed) {
        const float v = unordered((uint32_t)(list[lane] >> 32));
        const int o = ((int)~(uint32_t)list[lane] - begin) % STEP;
        fix = exp_wide((double)v - (double)at_ref.ref);
        if (CLEAN) fix -= (double)__builtin_amdgcn_exp2f((v - at_ref.ref) * kLog2e[0]);
        else if (upper(o / (kWave * PER), o % PER)) fix -= (double)at_ref.exp<1>(v) * shift[1];
        else fix -= (double)at_ref.exp<0>(v) * shift[0];
    }
    sum_out = unset ? 0.0 : all + row_sum<kWave>(fix);
    return true;
}

template <int FORMAT>
__global__ __launch_bounds__(kThreads, FORMAT == 2 ? 3 : 4) void beam_scan_kernel(SelectParams p)
{
    __shared__ uint64_t s_list[kWaves][kList];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * kWaves + wave; // waves are on their own: no barrier
    const int r = (int)(unit / p.spans), span = (int)(unit - (int64_t)r * p.spans);
    if (r >= p.rows) return;
    const int begin = span * p.span_len, end = p.vocab - begin < p.span_len ? p.vocab : begin + p.span_len;
    const char *row = static_cast<const char *>(p.logits) + (int64_t)r * p.row_stride * Logits<FORMAT>::kBytes;
    uint64_t *list = s_list[wave];
    int n;
    double sum;
    float ref;
    const float score = p.score[r];
    const int32_t finished = p.end_token ? p.end_token[r] : -1;
    const auto skip = [=] { return dead(score) || finished >= 0; }; // a row that is not read: its records are not looked at
    if (!scan_span<FORMAT, false, FORMAT == 2 ? 8 : 4>(row, begin, end, p.num_out, skip, list, n, sum, ref))
        scan_span<FORMAT, true, 1>(row, begin, end, p.num_out, skip, list, n, sum, ref);
    if (skip()) return;
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
    __shared__ double s_log[kRowLogs];
    __shared__ int s_n;
    __shared__ float s_reached[kWaves];
    const int g = blockIdx.x, t = threadIdx.x, keep = p.num_out;
    const int lo = min(max(p.group_begin[g], 0), p.rows), hi = min(max(p.group_begin[g + 1], 0), p.rows);
    const int64_t records = (int64_t)max(hi - lo, 0) * p.spans;
    Walk w = walk_at(p, lo, t, records); // of the first records; asked for ahead of the rows' sums
    if (t == 0) s_n = 0;
    // logarithms of the rows' sums: as many lanes to a row as it has spans, up to a wave.  Records of rows that were not read hold
    // anything; what comes of them is never used.
    int lanes = 1;
    while (lanes < p.spans && lanes < kWave) lanes <<= 1;
    const int first = t & (lanes - 1);
    for (int r = lo + t / lanes; r - t / lanes < hi; r += kThreads / lanes) {
        const SpanRecord *rec = p.records + (int64_t)r * p.spans;
        const SpanRecord mine = r < hi && first < p.spans ? rec[first] : SpanRecord{0.0, kLowest, 0};
        float ref = mine.ref;
        if (r < hi)
            for (int i = first + lanes; i < p.spans; i += lanes) ref = fmaxf(ref, rec[i].ref);
        for (int off = 1; off < lanes; off <<= 1) ref = fmaxf(ref, __shfl_xor(ref, off));
        double sum = mine.sum * exp_wide((double)mine.ref - (double)ref);
        if (r < hi)
            for (int i = first + lanes; i < p.spans; i += lanes) sum += rec[i].sum * exp_wide((double)rec[i].ref - (double)ref);
        for (int off = 1; off < lanes; off <<= 1) sum += __shfl_xor(sum, off);
        if (r < hi && first == 0) {
            const double row_log = (double)ref + log_wide(sum);
            if (r - lo < kRowLogs) s_log[r - lo] = row_log;
            else p.row_log[r] = row_log;
        }
    }
    __syncthreads();
    auto log_of = [&](int r) { return r - lo < kRowLogs ? s_log[r - lo] : p.row_log[r]; };
    if (w.on && w.end < 0) w.row_log = log_of(w.row);
    // What `keep` lanes of a wave reach with the first element of their records is reached by the group's best `keep`.
    float reached = -kInf;
    {
        float mine = w.on && w.ahead[0] ? (float)unordered64(choice_of(w, w.ahead[0]).total) : -kInf;
        reached = reached_by(mine, keep);
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
            if (w.on && w.end < 0) w.row_log = log_of(w.row);
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
int span_length(int vocab, int rows, int compute_units)
{
    const int64_t step = (int64_t)kWave * kHeld;
    const int64_t steps = ((int64_t)vocab + step - 1) / step * rows / ((int64_t)compute_units * kWavesPerCu);
    return (int)(step * (steps < 1 ? 1 : steps > kMaxSteps ? kMaxSteps : steps));
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

} // namespace

int beam_select_spans(int vocab, int rows, int compute_units)
{
    const int len = span_length(vocab, rows, compute_units);
    return (int)(((int64_t)vocab + len - 1) / len);
}

size_t beam_select_workspace_bytes(int vocab, int rows, int num_out, int compute_units)
{
    const size_t units = (size_t)rows * beam_select_spans(vocab, rows, compute_units);
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
    p.span_len = span_length(a.vocab, a.rows, a.compute_units);
    p.spans = beam_select_spans(a.vocab, a.rows, a.compute_units);
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
