// The choice of a beam search's step: for row r (a beam) of a group and token t
//     total(r, t) = score(r) + x(r, t) - log sum_u exp x(r, u)
// and the num_out largest totals of each group, equal ones in the order of row, then logit, then token.
//
// One pass over the logits.  A wave takes a span of one row and leaves a record: the span's sum of exp(x - ref), ref, and its
// num_out largest elements in order.  A second kernel, one workgroup per group, adds the sums up, forms the totals of what the
// records list and takes the best.  Two launches, no atomics on memory, and the same order of every sum on every run.
//
// While a wave streams its span it does no more than a maximum and an exponential per element (5.2 instructions of a
// bfloat16 one, and by the counters one slot more for the exponential) and notes each lane's maximum of every step.  Those maxima
// then say how large an element has to be to count, and which lanes of which steps have one: their 64 bytes are read again.
// Candidates kept while streaming took 1.4 times the vector instructions, the spans' ends included.
//
// What bounds it, for large batches: 247 live rows of 262,144 bfloat16 logits (129 MB) take 28 us, 4.6 TB/s.  Reading alone is 21 us of
// that (a kernel that only reads: 6.2 to 6.3 TB/s), issue 16 (9.8 million quad-cycles of the vector units), and neither is behind the
// other: all waves are on the chip at once (they begin within 0.4 us of each other and end between 16 and 29), stream at the same time,
// and then are at their ends at the same time, with 106 of their 272 vector instructions a step and a trip to memory for each step
// that is read again.  Elsewhere it is the chain of each wave (a trip to memory, 32 elements a lane, the best of them: 4 us) and of the
// merge (three trips, logarithms, threshold, ranks: 4 us), both of them with instruction fetch in them, and two launches.  Four rows
// of 32,000 binary16 5.4 + 4.6 us, 72 rows of 50,001 binary32 in 16 groups with 16 out 10.5 + 8.4, ten live rows of 80 of 128,000 with 8 out
// 11.0 + 7.0.
#include "q4_device.h"
#include "q4kv_internal.h"

namespace q4kv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kList = 192;     // candidates a wave can hold: what it keeps (64 at most) and two appends of up to 64
constexpr int kRowsHeld = 64; // rows of a group that the merge keeps in LDS
constexpr int kHeld = 32;      // elements of a step per lane
constexpr int kMaxSteps = 8;   // steps of a span

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
    uint64_t *keys;       // [rows][num_out][spans]: value and place, a span's largest first, 0 where there are no more
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
    static constexpr uint32_t kBanned = FORMAT == 2 ? 0xff800000u : FORMAT == 1 ? 0xff80ff80u : 0xfc00fc00u;
    // the same, -inf where that would read beyond `end`
    static __device__ __forceinline__ words_t load_to(const char *row, int i, int end)
    {
        return i + kPer <= end ? load(row, i) : words_t{kBanned, kBanned, kBanned, kBanned};
    }
    static __device__ __forceinline__ float one(const char *row, int i)
    {
        if constexpr (FORMAT == 2) return reinterpret_cast<const float *>(row)[i];
        const uint16_t b = reinterpret_cast<const uint16_t *>(row)[i];
        return FORMAT == 1 ? bf16_bits_to_float(b) : half_bits_to_float(b);
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
// exp d for d up to some 9 (an element over its span's reference), -inf as well, to 1e-12: 2^n times the series of what is left of d
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
__device__ __forceinline__ double lane_value(double v, int lane)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
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
        for (int j0 = 0; j0 < n; j0 += 4) // those from n on are 0, which is ahead of none
#pragma unroll
            for (int j = j0; j < j0 + 4; ++j)
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

// A value that at least `keep` (up to eight) lanes reach with their `mine`: the lanes are cut into eight (four) groups, and every group
// has a lane that reaches the lowest of the groups' maxima.
__device__ __forceinline__ float reached_by_groups(float mine, int keep)
{
    float v = mine;
    v = fmaxf(v, Q4KV_DPP(v, v, 0xB1, 0xF));                 // quad_perm [1,0,3,2]
    v = fmaxf(v, Q4KV_DPP(v, v, 0x4E, 0xF));                 // quad_perm [2,3,0,1]
    v = fmaxf(v, Q4KV_DPP(v, v, 0x141, 0xF));                // row_half_mirror: groups of eight lanes
    const float w = Q4KV_DPP(v, v, 0x140, 0xF);              // row_mirror: the other eight of a row
    v = keep <= 4 ? fmaxf(v, w) : fminf(v, w);
    return -xor32_max(xor16_max(-v));
}

// A value that at least `keep` of the wave's N * 64 values reach, and few more do: halving of the range from `low` (which so many
// reach, or which is -inf) to their largest until the count is between keep and twice that.
template <int N>
__device__ __forceinline__ float reached_by_halving(const float (&v)[N], float low, float high, int keep)
{
    uint32_t lo = ordered(low), hi = ordered(high);
#pragma unroll 1
    while (lo < hi) { // 32 rounds at most
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        const float m = unordered(mid);
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__ballot(v[i] >= m));
        if (n >= keep) {
            lo = mid;
            if (n <= 2 * keep) break;
        } else {
            hi = mid - 1;
        }
    }
    return unordered(lo);
}

// Word `at` of N words in registers (N a power of two).
template <int N>
__device__ __forceinline__ uint32_t word_of(const uint32_t *x, int at)
{
    if constexpr (N == 1) {
        return x[0];
    } else {
        const uint32_t a = word_of<N / 2>(x, at), b = word_of<N / 2>(x + N / 2, at);
        return at & (N / 2) ? b : a;
    }
}

__device__ __forceinline__ bool dead(float score) { return !(score > -kInf); }

// A span of a row: its candidates, in order, in `list`; the sum of exp(x - ref) and ref.  tops: LDS, [kMaxSteps][64].
// CLEAN: NaN and +inf are replaced while reading.  Without it they show in the maximum and the sum, and the answer is false: the
// span is to be done again (so it is where the largest logit is beyond 700,000 on either side of zero).
template <int FORMAT, bool CLEAN>
__device__ __forceinline__ bool scan_span(const char *row, int begin, int end, int keep, float *tops, uint64_t *list, int &listed,
                                          double &sum_out, float &ref_out)
{
    typedef Logits<FORMAT> L;
    constexpr int PER = L::kPer, UNROLL = kHeld / PER, STEP = kWave * kHeld;
    // places of the larger constant: 5 of a lane's 32
    constexpr auto upper = [](int u, int e) { return PER == 8 ? e == 0 || (u == 0 && e == 4) : e == 0 && u < 5; };
    const int lane = threadIdx.x & 63;
    auto clean = [](float x) { return !CLEAN ? x : x != x ? -kInf : fminf(x, -kLowest); };
    auto widen = [&](const words_t &w, float (&x)[PER]) {
        L::widen(w, x);
#pragma unroll
        for (int e = 0; e < PER; ++e) x[e] = clean(x[e]);
    };
    Reference at_ref;
    at_ref.set(0.0f);
    bool unset = true;
    int set_at = begin; // the step whose maximum the reference is
    double sum[2] = {0.0, 0.0};
    const int left = (end - begin) % PER, whole = end - left; // what does not fill a load is one element of `left` lanes more, in the first step
    words_t now[UNROLL] = {}, next[UNROLL] = {};
    float largest = -kInf, rest = -kInf;
    for (int at = begin - STEP; at < end; at += STEP) {
        // the values that were asked for a step ago, and the next ones asked for
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) now[u] = next[u];
        const int ahead = at + STEP + lane * PER;
        if (at + 2 * STEP <= whole) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) next[u] = L::load(row, ahead + u * kWave * PER);
        } else {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) next[u] = L::load_to(row, ahead + u * kWave * PER, whole);
        }
        if (at < begin) {
            if (lane < left) rest = clean(L::one(row, whole + lane));
            continue;
        }
        float extra = at == begin ? rest : -kInf, mine = extra;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if constexpr (FORMAT == 0 && !CLEAN) {
                const half2_t h = bits_to_half2(pk_max(pk_max(now[u][0], now[u][1]), pk_max(now[u][2], now[u][3])));
                mine = max3(mine, (float)h.x, (float)h.y);
            } else {
                float x[PER];
                widen(now[u], x);
#pragma unroll
                for (int e = 0; e < PER; e += 2) mine = max3(x[e], x[e + 1], mine);
            }
        }
        tops[(at - begin) / STEP * kWave + lane] = mine;
        largest = fmaxf(largest, mine);
        // The reference is the maximum of the first step that has a value; it moves where a step's is well above it (exponents are
        // good to 2^-24 of their size).
        if (unset || __any(mine > at_ref.ref + 8.0f)) {
            const float highest = wave_max(mine);
            if (highest > -kInf) {
                const Reference was = at_ref;
                at_ref.set(highest);
                if (__builtin_expect(!unset, 0)) {
                    // What is there may be nearly all of the sum (many elements just below the limit).  Terms 2^(x c - was c) become
                    // terms 2^(x c - ref c) with the products as they are rounded: so one factor at the end is right for all of them.
                    // Odd lanes look at the second constant.
                    const double moved = lane & 1 ? (double)at_ref.minus[1] - (double)was.minus[1] : (double)at_ref.minus[0] - (double)was.minus[0];
                    const double scale = exp_wide(CLEAN ? (double)was.ref - (double)highest : kLn2 * moved);
                    sum[0] *= lane_value(scale, 0);
                    sum[1] *= lane_value(scale, 1);
                }
                unset = false;
                set_at = at;
            }
        }
        auto term = [&](float x) { return CLEAN ? __builtin_amdgcn_exp2f((x - at_ref.ref) * kLog2e[0]) : at_ref.exp<0>(x); };
        float part[4] = {0.0f, term(extra), 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float x[PER];
            widen(now[u], x);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if (!CLEAN && upper(u, e)) part[0] += at_ref.exp<1>(x[e]);
                else part[1 + (u * PER + e) % 3] += term(x[e]);
            }
        }
        sum[0] += (double)(part[1] + part[2] + part[3]);
        if (!CLEAN) sum[1] += (double)part[0];
    }
    ref_out = unset ? kLowest : at_ref.ref;
    const double shift[2] = {CLEAN ? 1.0 : at_ref.unshift(0), CLEAN ? 1.0 : at_ref.unshift(1)};
    const double all = row_sum<kWave>(sum[0] * shift[0] + sum[1] * shift[1]);
    if (!CLEAN && !(all < (double)kInf && at_ref.usable())) return false; // a NaN or +inf among them, or a far reference
    // Elements below `threshold` are not among the best: as many lanes (or steps of lanes) have a larger one.
    const int steps = (end - begin + STEP - 1) / STEP;
    wave_lds_sync();
    float top[kMaxSteps];
#pragma unroll
    for (int k = 0; k < kMaxSteps; ++k) top[k] = k < steps ? tops[k * kWave + lane] : -kInf;
    float threshold = keep <= 8 ? reached_by_groups(largest, keep) : -wave_max(-largest);
    if (keep > 8 || __popcll(__ballot(largest >= threshold)) > 2 * keep + 8)
        threshold = reached_by_halving(top, threshold, wave_max(largest), keep);
    threshold = fmaxf(threshold, kLowest);
    uint32_t flagged = 0; // steps in which the lane has an element to look at
#pragma unroll
    for (int k = 0; k < kMaxSteps; ++k) flagged |= (uint32_t)(top[k] >= threshold) << k;
    int n = 0;
    uint64_t worst = 0; // of the list once it has been full
    auto push = [&](bool take, float v, int token) {
        if (n > kList - kWave) {
            n = keep_best(list, n, keep);
            if (n == keep) worst = list[keep - 1];
        }
        const uint64_t key = candidate(v, token);
        take = take && key > worst;
        const uint64_t taken = __ballot(take);
        if (take) list[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(taken >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)taken, 0))] = key;
        n += __popcll(taken);
    };
    float v = rest;
    int token = whole + lane, step = 0;
    uint32_t bits = 0;
    bool take = rest >= threshold;
    while (true) {
        if (__any(take)) push(take, v, token);
        // the next element of the lane, in this step or the next flagged one
        if (!__any(bits != 0)) {
            if (!__any(flagged != 0)) break;
            const bool mine = flagged != 0;
            step = mine ? __ffs(flagged) - 1 : 0;
            flagged &= flagged - 1;
            const int at = begin + step * STEP + lane * PER;
            if (steps > 1 && mine) {
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) now[u] = L::load_to(row, at + u * kWave * PER, whole);
            }
            // bit u * PER + e: the element is no less than the threshold, by the sign of the difference (either zero less -0 is +0)
            const float less = threshold == 0.0f ? -0.0f : threshold;
#pragma unroll
            for (int u = UNROLL - 1; u >= 0; --u) {
                float x[PER];
                widen(now[u], x);
#pragma unroll
                for (int e = PER - 1; e >= 0; --e) bits = __builtin_amdgcn_alignbit(bits, __builtin_bit_cast(uint32_t, x[e] - less), 31);
            }
            bits = mine ? ~bits : 0u;
        }
        take = bits != 0;
        const int i = take ? __ffs(bits) - 1 : 0, u = i / PER;
        bits &= bits - 1;
        uint32_t words[kHeld * 4 / PER];
#pragma unroll
        for (int k = 0; k < UNROLL * 4; ++k) words[k] = now[k / 4][k % 4];
        const uint32_t word = word_of<UNROLL * 4>(words, FORMAT == 2 ? i : i >> 1);
        if constexpr (FORMAT == 2) v = __builtin_bit_cast(float, word);
        else if constexpr (FORMAT == 1) v = __builtin_bit_cast(float, i & 1 ? word & 0xffff0000u : word << 16);
        else v = half_bits_to_float((uint16_t)(i & 1 ? word >> 16 : word & 0xffffu));
        v = clean(v);
        token = begin + step * STEP + (u * kWave + lane) * PER + i % PER;
    }
    listed = keep_best(list, n, keep);
    // The largest elements dominate the sum of a peaked row: theirs are taken again in binary64, in the place of the terms that
    // they were summed as.  (Those that an earlier reference made are not these terms, and stay.)
    double fix = 0.0;
    const int t = lane < listed ? (int)~(uint32_t)list[lane] : 0;
    if (lane < listed && (t < whole ? t : begin) >= set_at) {
        const float x = unordered((uint32_t)(list[lane] >> 32));
        const int o = (t - begin) % STEP;
        fix = exp_wide((double)x - (double)at_ref.ref);
        if (CLEAN) fix -= (double)__builtin_amdgcn_exp2f((x - at_ref.ref) * kLog2e[0]);
        else if (t < whole && upper(o / (kWave * PER), o % PER)) fix -= (double)at_ref.exp<1>(x) * shift[1];
        else fix -= (double)at_ref.exp<0>(x) * shift[0];
    }
    sum_out = unset ? 0.0 : all + row_sum<kWave>(fix);
    return true;
}

template <int FORMAT>
__global__ __launch_bounds__(kThreads, FORMAT == 2 ? 3 : 4) void beam_scan_kernel(SelectParams p)
{
    __shared__ uint64_t s_list[kWaves][kList];
    __shared__ float s_tops[kWaves][kMaxSteps * kWave];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * kWaves + wave; // waves are on their own: no barrier
    const int r = (int)(unit / p.spans), span = (int)(unit - (int64_t)r * p.spans);
    if (r >= p.rows) return;
    const int begin = span * p.span_len, end = p.vocab - begin < p.span_len ? p.vocab : begin + p.span_len;
    const char *row = static_cast<const char *>(p.logits) + (int64_t)r * p.row_stride * Logits<FORMAT>::kBytes;
    uint64_t *list = s_list[wave];
    int n = 0;
    double sum = 0.0;
    float ref = kLowest;
    const float score = p.score[r];
    const int32_t finished = p.end_token ? p.end_token[r] : -1;
    // Nothing of such a row is read, and its records are not looked at.  (Asking for the first values ahead of this is 0.2 us less
    // where all rows live, and read 9 MB in vain where a first step's ten of eighty do: 10.1 us for 6.)
    if (dead(score) || finished >= 0) return;
    if (!scan_span<FORMAT, false>(row, begin, end, p.num_out, s_tops[wave], list, n, sum, ref))
        scan_span<FORMAT, true>(row, begin, end, p.num_out, s_tops[wave], list, n, sum, ref);
    if (lane == 0) p.records[unit] = SpanRecord{sum, ref, 0};
    if (lane < p.num_out) p.keys[((int64_t)r * p.num_out + lane) * p.spans + span] = lane < n ? list[lane] : 0;
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

template <int SIZE>
struct MergeList {
    uint64_t total[SIZE], key[SIZE];
    uint32_t row[SIZE];
    __device__ __forceinline__ Choice at(int i) const { return Choice{total[i], key[i], row[i]}; }
    __device__ __forceinline__ void set(int i, const Choice &c)
    {
        total[i] = c.total;
        key[i] = c.key;
        row[i] = c.row;
    }
};

// How many of the list's n entries are better than one, counted by THREADS / 64 neighbouring lanes per entry, 64 entries at a time.
template <int THREADS, int SIZE>
__device__ __forceinline__ int rank_of(const MergeList<SIZE> &list, int n, const Choice &mine)
{
    constexpr int SHARE = THREADS / kWave;
    static_assert(SHARE == 4 || SHARE == 16, "lanes of a quad or a row");
    int ahead = 0;
#pragma unroll 2
    for (int j = threadIdx.x % SHARE; j < n; j += SHARE) { // no branch: the reads of several entries overlap
        const Choice other = list.at(j);
        ahead += (other.total > mine.total) |
                 ((other.total == mine.total) & ((other.row < mine.row) | ((other.row == mine.row) & (other.key > mine.key))));
    }
    ahead += __builtin_amdgcn_mov_dpp(ahead, 0xB1, 0xF, 0xF, true); // quad_perm [1,0,3,2]
    ahead += __builtin_amdgcn_mov_dpp(ahead, 0x4E, 0xF, 0xF, true); // quad_perm [2,3,0,1]
    if constexpr (SHARE == 16) {
        ahead += __builtin_amdgcn_mov_dpp(ahead, 0x141, 0xF, 0xF, true); // row_half_mirror
        ahead += __builtin_amdgcn_mov_dpp(ahead, 0x140, 0xF, 0xF, true); // row_mirror
    }
    return ahead;
}

// As keep_best, for a workgroup's list; `room`: LDS for what is kept.
template <int THREADS, int SIZE>
__device__ __forceinline__ int keep_best_choices(MergeList<SIZE> &list, Choice *room, int n, int keep)
{
    constexpr int SHARE = THREADS / kWave;
    __syncthreads();
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += kWave) {
        const int i = i0 + threadIdx.x / SHARE;
        const Choice mine = list.at(min(i, n - 1));
        const int rank = rank_of<THREADS>(list, n, mine);
        if (i < n && rank < keep && threadIdx.x % SHARE == 0) room[rank] = mine;
    }
    __syncthreads();
    const int kept = min(n, keep);
    if ((int)threadIdx.x < kept) list.set(threadIdx.x, room[threadIdx.x]);
    __syncthreads();
    return kept;
}

// maximum over the 16 lanes of a row, in all of them
__device__ __forceinline__ float row16_max(float v)
{
    v = fmaxf(v, Q4KV_DPP(v, v, 0xB1, 0xF));  // quad_perm [1,0,3,2]
    v = fmaxf(v, Q4KV_DPP(v, v, 0x4E, 0xF));  // quad_perm [2,3,0,1]
    v = fmaxf(v, Q4KV_DPP(v, v, 0x141, 0xF)); // row_half_mirror
    return fmaxf(v, Q4KV_DPP(v, v, 0x140, 0xF)); // row_mirror
}

// One group's choice out of what its rows' records list: chunks of kThreads * kTaken elements, of which those come into a list
// that reach what `keep` of the chunk reach.  A chain of trips to memory (bounds, records, outputs) and of instructions
// that every wave runs once; hence no loop is unrolled that does not have to be.
constexpr int kTaken = 4, kRecordsHeld = 4;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void beam_merge_kernel(SelectParams p)
{
    constexpr int kThreads = THREADS, kWaves = THREADS / kWave, kSize = (kTaken + 2) * THREADS;
    struct Row {
        double score, log; // of the sum of its exponentials
        int32_t end;       // its end token, or kOpen, or kDead
    };
    constexpr int32_t kOpen = -1, kDead = -2;
    __shared__ MergeList<kSize> s_list;
    __shared__ Choice s_room[Q4KV_MAX_BEAM_OUT];
    __shared__ Row s_row[kRowsHeld];
    __shared__ int s_n;
    __shared__ float s_low[kWaves], s_most[kWaves];
    __shared__ int s_count[3][kWaves];
    const int g = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6, keep = p.num_out;
    const int lo = min(max(p.group_begin[g], 0), p.rows), hi = min(max(p.group_begin[g + 1], 0), p.rows);
    const int per_row = p.spans * keep; // elements of a row's records: at most 2^20 spans
    const int64_t elements = (int64_t)max(hi - lo, 0) * per_row;
    const uint64_t *keys = p.keys + (int64_t)lo * per_row;
    uint64_t key[kTaken];
#pragma unroll
    for (int e = 0; e < kTaken; ++e) key[e] = e * kThreads + t < elements ? keys[e * kThreads + t] : 0; // asked for ahead of the rows' sums
    if (t == 0) s_n = 0;
    // Logarithms of the rows' sums, 16 lanes to a row.  Records of rows that were not read hold anything; what comes of them is
    // never used.
#pragma unroll 1
    for (int r = lo + t / 16; r - t / 16 < hi; r += kThreads / 16) {
        const SpanRecord *rec = p.records + (int64_t)r * p.spans;
        const int spans = r < hi ? p.spans : 0;
        const float score = spans ? p.score[r] : 0.0f;
        const int32_t end = spans && p.end_token ? p.end_token[r] : -1;
        SpanRecord held[kRecordsHeld];
#pragma unroll
        for (int k = 0; k < kRecordsHeld; ++k) held[k] = (t & 15) + 16 * k < spans ? rec[(t & 15) + 16 * k] : SpanRecord{0.0, kLowest, 0};
        float ref = kLowest;
#pragma unroll
        for (int k = 0; k < kRecordsHeld; ++k) ref = fmaxf(ref, held[k].ref);
#pragma unroll 1
        for (int i = (t & 15) + 16 * kRecordsHeld; i < spans; i += 16) ref = fmaxf(ref, rec[i].ref);
        ref = row16_max(ref);
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < kRecordsHeld; ++k) sum += held[k].sum * exp_wide((double)held[k].ref - (double)ref);
#pragma unroll 1
        for (int i = (t & 15) + 16 * kRecordsHeld; i < spans; i += 16) sum += rec[i].sum * exp_wide((double)rec[i].ref - (double)ref);
        const double row_log = (double)ref + log_wide(row_sum<16>(sum));
        if (spans && (t & 15) == 0) {
            if (r - lo < kRowsHeld) s_row[r - lo] = Row{(double)score, row_log, dead(score) ? kDead : end >= 0 ? end : kOpen};
            else p.row_log[r] = row_log;
        }
    }
    __syncthreads();
    auto row_at = [&](int r) {
        if (r - lo < kRowsHeld) return s_row[r - lo];
        const float score = p.score[r];
        const int32_t end = p.end_token ? p.end_token[r] : -1;
        return Row{(double)score, p.row_log[r], dead(score) ? kDead : end >= 0 ? end : kOpen};
    };
    int n = 0;
    float reached = -kInf;
    Choice worst = {};
    bool full = false;
    const float one_row = 1.0f / (float)per_row;
#pragma unroll 1
    for (int64_t base = 0; base < elements; base += kThreads * kTaken) {
        const int first_row = lo + (int)(base / per_row);
        const uint32_t offset = (uint32_t)(base % per_row) + t;
        Choice c[kTaken];
        float total[kTaken], low = kInf, most = -kInf;
        int valid = 0;
#pragma unroll
        for (int e = 0; e < kTaken; ++e) {
            // `at` is below per_row + kTaken * THREADS, so at most that many rows further on, 4,096: a quotient of that size is off by
            // less than 2^-10 in binary32, and one off at most as an integer
            const uint32_t at = offset + e * kThreads;
            uint32_t row = (uint32_t)((float)at * one_row);
            if (at < row * per_row) --row;
            else if (at - row * per_row >= (uint32_t)per_row) ++row;
            const bool first = at == row * per_row, in = base + e * kThreads + t < elements;
            total[e] = -kInf;
            c[e] = Choice{0, key[e], (uint32_t)first_row + row};
            if (in && (key[e] != 0 || first)) {
                const Row r = row_at(first_row + (int)row);
                double v = r.score + ((double)unordered((uint32_t)(key[e] >> 32)) - r.log);
                bool on = r.end == kOpen && key[e] != 0;
                if (r.end >= 0) { // finished: its one continuation, in the place of the first element
                    on = first;
                    c[e].key = (uint32_t)~r.end;
                    v = r.score;
                }
                c[e].total = ordered64(v);
                if (on) total[e] = fmaxf((float)v, kLowest);
            }
            valid += __popcll(__ballot(total[e] > -kInf));
            most = fmaxf(most, total[e]);
            if (total[e] > -kInf) low = fminf(low, total[e]);
        }
        // the next chunk's are on their way while this one's are looked at
#pragma unroll
        for (int e = 0; e < kTaken; ++e) {
            const int64_t at = base + (kTaken + e) * kThreads + t;
            key[e] = at < elements ? keys[at] : 0;
        }
        low = -wave_max(-low);
        most = wave_max(most);
        if (lane == 0) {
            s_low[wave] = low;
            s_most[wave] = most;
            s_count[2][wave] = valid;
        }
        __syncthreads();
        valid = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            low = fminf(low, s_low[i]);
            most = fmaxf(most, s_most[i]);
            valid += s_count[2][i];
        }
        if (valid >= keep) { // halving as in reached_by_halving, by all waves together
            uint32_t under = ordered(low), above = ordered(most);
            int slot = 0;
#pragma unroll 1
            while (under < above) {
                const uint32_t mid = under + (above - under + 1) / 2;
                const float m = unordered(mid);
                int count = 0;
#pragma unroll
                for (int e = 0; e < kTaken; ++e) count += __popcll(__ballot(total[e] >= m));
                if (lane == 0) s_count[slot][wave] = count;
                __syncthreads(); // the other slot's counts have been read by all when this one's are written again
                count = 0;
#pragma unroll
                for (int i = 0; i < kWaves; ++i) count += s_count[slot][i];
                slot ^= 1;
                if (count >= keep) {
                    under = mid;
                    if (count <= 2 * keep) break;
                } else {
                    above = mid - 1;
                }
            }
            reached = fmaxf(reached, unordered(under));
        }
        int mine = 0, place[kTaken];
#pragma unroll
        for (int e = 0; e < kTaken; ++e) {
            const bool on = total[e] > -kInf && total[e] >= reached && !(full && !better(c[e], worst));
            const uint64_t mask = __ballot(on);
            place[e] = on ? mine + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)) : -1;
            mine += __popcll(mask);
        }
        if (mine > 0) {
            int first = 0;
            if (lane == 0) first = atomicAdd(&s_n, mine);
            first = __builtin_amdgcn_readfirstlane(first);
#pragma unroll
            for (int e = 0; e < kTaken; ++e)
                if (place[e] >= 0) s_list.set(first + place[e], c[e]);
        }
        __syncthreads();
        n = s_n;
        __syncthreads(); // everybody has the same n before the next append
        if (n > kSize - kTaken * kThreads || (n > 2 * keep + kWave && base + kThreads * kTaken < elements)) {
            n = keep_best_choices<kThreads>(s_list, s_room, n, keep);
            if (t == 0) s_n = n;
            full = n == keep;
            if (full) worst = s_list.at(keep - 1);
            __syncthreads();
        }
    }
    if (n > kWave) n = keep_best_choices<kThreads>(s_list, s_room, n, keep);
    // the last ones, and behind them the places that stay empty
    constexpr int SHARE = kThreads / kWave;
    const int i = t / SHARE;
    const Choice c = s_list.at(i);
    const int rank = rank_of<kThreads>(s_list, n, c), place = i < n ? rank : i;
    if (place < keep && t % SHARE == 0) {
        const int64_t at = (int64_t)g * keep + place;
        p.parent[at] = i < n ? (int32_t)c.row : -1;
        p.token[at] = i < n ? (int32_t)~(uint32_t)c.key : -1;
        p.total[at] = i < n ? (float)unordered64(c.total) : -kInf;
    }
}

// Elements of a span: whole steps of a wave, so many that about kWavesPerCu waves per compute unit share the call's rows, and that
// a wave has four times as many maxima as it keeps elements.  Measured, a call of 256 rows of 262,144 with at most 4 / 8 / 16 steps a
// span 40.9 / 39.2 / 39.9 us, 64 rows of 128,000 19.3 / 19.4 / 19.7; with 16 waves wanted per compute unit spans are shorter and the merge has more
// records: ten of 80 rows of 128,000 alive 10.1 + 8.9 us for 11.0 + 7.3.  24 rows of 32,000 with 64 out take as long with
// one step a span as with four, 80 us; what helps there is the wider merge below.
constexpr int kWavesPerCu = 8;
int span_length(int vocab, int rows, int num_out, int compute_units)
{
    const int64_t step = (int64_t)kWave * kHeld;
    const int64_t steps = ((int64_t)vocab + step - 1) / step * rows / ((int64_t)compute_units * kWavesPerCu);
    const int64_t least = (num_out + 15) / 16;
    return (int)(step * (steps < least ? least : steps > kMaxSteps ? kMaxSteps : steps));
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

} // namespace

int beam_select_spans(int vocab, int rows, int num_out, int compute_units)
{
    const int len = span_length(vocab, rows, num_out, compute_units);
    return (int)(((int64_t)vocab + len - 1) / len);
}

size_t beam_select_workspace_bytes(int vocab, int rows, int num_out, int compute_units)
{
    const size_t units = (size_t)rows * beam_select_spans(vocab, rows, num_out, compute_units);
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
    p.span_len = span_length(a.vocab, a.rows, a.num_out, a.compute_units);
    p.spans = beam_select_spans(a.vocab, a.rows, a.num_out, a.compute_units);
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
    // A workgroup of 1,024 where a group's records list more than a chunk of 256 threads: 8 rows of 63 spans with 8 out 8.0 us for
    // 7.3, of 25 with 16 out 15.9 for 9.8; a whole call of 24 rows with 64 out 77 for 37.
    if (units * p.num_out > (int64_t)p.groups * kThreads * kTaken)
        hipLaunchKernelGGL(beam_merge_kernel<1024>, dim3((unsigned)p.groups), dim3(1024), 0, stream, p);
    else
        hipLaunchKernelGGL(beam_merge_kernel<kThreads>, dim3((unsigned)p.groups), dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

} // namespace q4kv
