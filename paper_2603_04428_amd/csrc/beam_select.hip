// The choice of a beam search's step: for row r (a beam) of a group and token t
//     total(r, t) = score(r) + x(r, t) - log sum_u exp x(r, u)
// and the num_out largest totals of each group, equal ones in the order of row, then logit, then token.
//
// One pass over the logits.  A wave takes a span of one row and leaves a record: the span's sum of exp(x - ref), ref, and its
// num_out largest elements in order.  A second kernel, one workgroup per group, adds the sums up, forms the totals of what the
// records list and takes the best.  Two launches, no atomics on memory, and the same order of every sum on every run.
//
// What bounds it is memory for large batches (every logit is read once) and the trips to memory of two launches for small ones.
#include "q4_device.h"
#include "q4kv_internal.h"

namespace q4kv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kList = 192;     // candidates a wave can hold: what it keeps (64 at most) and two appends of up to 64
constexpr int kMergeList = 1024;
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
template <int FORMAT>
struct Logits {
    static constexpr int kPer = FORMAT == 2 ? 4 : 8;
    typedef uint32_t words_t __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(FORMAT == 2 ? 4 : 2))) Loose { words_t w; }; // rows may begin at any element
    static __device__ __forceinline__ words_t load(const void *row, int64_t i)
    {
        return reinterpret_cast<const Loose *>(static_cast<const char *>(row) + i * (16 / kPer))->w;
    }
    static __device__ __forceinline__ float one(const void *row, int64_t i)
    {
        if constexpr (FORMAT == 2) return static_cast<const float *>(row)[i];
        const uint16_t b = static_cast<const uint16_t *>(row)[i];
        return FORMAT == 1 ? bf16_bits_to_float(b) : half_bits_to_float(b);
    }
    static __device__ __forceinline__ void widen(words_t w, float (&x)[kPer])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (FORMAT == 2) {
                const uint32_t bits = w[i]; // a value of its own: the cast of a vector's element takes the first one
                x[i] = __builtin_bit_cast(float, bits);
            } else if constexpr (FORMAT == 1) {
                x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
                x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
            } else {
                const half2_t h = bits_to_half2(w[i]);
                x[2 * i] = (float)h.x;
                x[2 * i + 1] = (float)h.y;
            }
        }
    }
};

constexpr float kLowest = -3.40282347e38f, kInf = __builtin_inff();

// exp(x - ref): log2 e in two terms, so that the constant's own rounding (1.3e-8 of the exponent) does not shift every term of a
// sum the same way
__device__ __forceinline__ float exp_from(float x, float ref)
{
    const float d = x - ref;
    return __builtin_amdgcn_exp2f(__builtin_fmaf(d, 1.925963033500e-8f, d * 1.442695022f));
}

__device__ __forceinline__ double wave_sum_double(double v)
{
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off);
    return v;
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
        for (int j = 0; j < n; ++j) rank[0] += list[j] > mine[0];
    } else {
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

// A value that at least `keep` lanes reach with their `mine`, and few more do (keep lanes or more are above `floor`): halving
// of the range between the lanes' extremes until the count is between keep and twice that.
__device__ __forceinline__ float reached_by(float mine, float floor, float top, int keep)
{
    uint32_t lo = ordered(floor) + 1, hi = ordered(top); // lo is reached by enough lanes, what is above hi by none
    for (int i = 0; i < 32 && lo < hi; ++i) {
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

// CLEAN: NaN and +inf are replaced while reading.  Without it they show in the wave's maximum and sum, and the span is done again.
template <int FORMAT, bool CLEAN>
__device__ __forceinline__ bool scan_span(const SelectParams &p, const void *row, int begin, int end, uint64_t *list, int &listed,
                                          double &sum_out, float &ref_out)
{
    typedef Logits<FORMAT> L;
    constexpr int PER = L::kPer, STEP = kWave * kUnroll * PER;
    const int lane = threadIdx.x & 63, keep = p.num_out;
    float ref = kLowest, threshold = kLowest; // candidates are at or above the threshold
    double sum = 0.0;
    int n = 0;
    bool first = true;
    typename L::words_t next[kUnroll];
    auto load = [&](int at) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int i = at + (u * kWave + lane) * PER;
            if (i + PER <= end) {
                next[u] = L::load(row, i);
            } else { // the end of the span inside a load: element by element, -inf behind it
                uint32_t bits[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    if constexpr (FORMAT == 2) {
                        bits[w] = i + w < end ? static_cast<const uint32_t *>(row)[i + w] : 0xff800000u;
                    } else {
                        const uint32_t banned = FORMAT == 1 ? 0xff80u : 0xfc00u;
                        const uint16_t *h = static_cast<const uint16_t *>(row);
                        bits[w] = i + 2 * w < end ? h[i + 2 * w] : banned;
                        bits[w] |= (i + 2 * w + 1 < end ? h[i + 2 * w + 1] : banned) << 16;
                    }
                }
                next[u] = typename L::words_t{bits[0], bits[1], bits[2], bits[3]};
            }
        }
    };
    load(begin);
    for (int at = begin; at < end; at += STEP) {
        float x[kUnroll][PER], top[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            L::widen(next[u], x[u]);
            if constexpr (CLEAN) {
#pragma unroll
                for (int i = 0; i < PER; ++i) x[u][i] = x[u][i] != x[u][i] ? -kInf : fminf(x[u][i], -kLowest);
            }
        }
        if (at + STEP < end) load(at + STEP);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            top[u] = x[u][0];
#pragma unroll
            for (int i = 1; i < PER; ++i) top[u] = fmaxf(top[u], x[u][i]);
        }
        float mine = top[0];
#pragma unroll
        for (int u = 1; u < kUnroll; ++u) mine = fmaxf(mine, top[u]);
        // The reference is the maximum of the first step; it moves only where an exponential could grow large.
        if (first || __any(mine > ref + 40.0f)) {
            const float highest = fmaxf(wave_max(mine), kLowest);
            if (!first) sum *= __builtin_amdgcn_exp2f((ref - highest) * 1.442695022f);
            ref = highest;
            first = false;
        }
        float part = 0.0f;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < PER; ++i) s += exp_from(x[u][i], ref);
            part += s;
        }
        sum += (double)part;
        // candidates
        const uint64_t over = __ballot(mine >= threshold);
        if (over == 0) continue;
        if (__popcll(over) >= keep) {
            // this step alone has `keep` elements at or above what `keep` of its lanes reach
            const float t = reached_by(mine, unordered(ordered(threshold) - 1), wave_max(mine), keep);
            threshold = fmaxf(threshold, t);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (!__any(top[u] >= threshold)) continue;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const bool take = x[u][i] >= threshold;
                const uint64_t mask = __ballot(take);
                if (mask == 0) continue;
                if (n > kList - kWave) {
                    n = keep_best(list, n, keep);
                    if (n == keep) threshold = fmaxf(threshold, unordered((uint32_t)(list[keep - 1] >> 32)));
                }
                if (take) {
                    const int place = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
                    list[place] = candidate(x[u][i], at + (u * kWave + lane) * PER + i);
                }
                n += __popcll(mask);
            }
        }
        // later steps have higher tokens: what only equals the last one kept does not come in any more
        if (at + STEP < end && n >= keep) {
            n = keep_best(list, n, keep);
            threshold = fmaxf(threshold, unordered((uint32_t)(list[keep - 1] >> 32) + 1));
        }
    }
    n = keep_best(list, n, keep);
    listed = n;
    ref_out = ref;
    sum = wave_sum_double(sum);
    if (!CLEAN && !(sum < (double)kInf && ref < kInf)) return false; // a NaN or +inf among them
    // The largest elements dominate the sum of a peaked row: theirs are taken again in binary64.
    double fix = 0.0;
    if (lane < n) {
        const float v = unordered((uint32_t)(list[lane] >> 32));
        fix = exp((double)v - (double)ref) - (double)exp_from(v, ref);
    }
    sum_out = sum + wave_sum_double(fix);
    return true;
}

__device__ __forceinline__ bool dead(float score) { return !(score > -kInf); }

template <int FORMAT>
__global__ __launch_bounds__(kThreads) void beam_scan_kernel(SelectParams p)
{
    __shared__ uint64_t s_list[kWaves][kList];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * kWaves + wave; // waves are on their own: no barrier
    const int r = (int)(unit / p.spans), span = (int)(unit - (int64_t)r * p.spans);
    if (r >= p.rows) return;
    if (dead(p.score[r]) || (p.end_token && p.end_token[r] >= 0)) return;
    const int begin = span * p.span_len, end = p.vocab - begin < p.span_len ? p.vocab : begin + p.span_len;
    const char *row = static_cast<const char *>(p.logits) + (int64_t)r * p.row_stride * (16 / Logits<FORMAT>::kPer);
    uint64_t *list = s_list[wave];
    int n;
    double sum;
    float ref;
    if (!scan_span<FORMAT, false>(p, row, begin, end, list, n, sum, ref)) scan_span<FORMAT, true>(p, row, begin, end, list, n, sum, ref);
    if (lane == 0) p.records[unit] = SpanRecord{sum, ref, 0};
    if (lane < p.num_out) p.keys[unit * p.num_out + lane] = lane < n ? list[lane] : 0;
}

// A continuation in the merge: its total, then the lower row, then the row's own order (where a logit is so large that totals
// next to it are equal, the larger logit is still the better one).
struct Choice {
    uint64_t total, key;
    uint32_t row, pad;
};
__device__ __forceinline__ bool better(const Choice &a, const Choice &b)
{
    return a.total > b.total || (a.total == b.total && (a.row < b.row || (a.row == b.row && a.key > b.key)));
}

__device__ __forceinline__ int keep_best_choices(Choice *list, int n, int keep)
{
    constexpr int PER = kMergeList / kThreads;
    Choice mine[PER];
    int rank[PER];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int at = i * kThreads + threadIdx.x;
        rank[i] = at < n ? 0 : keep;
        if (at < n) {
            mine[i] = list[at];
            for (int j = 0; j < n; ++j) rank[i] += better(list[j], mine[i]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (rank[i] < keep) list[rank[i]] = mine[i];
    __syncthreads();
    return min(n, keep);
}

__global__ __launch_bounds__(kThreads) void beam_merge_kernel(SelectParams p)
{
    __shared__ Choice s_list[kMergeList];
    __shared__ int s_n;
    const int g = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6, keep = p.num_out;
    const int lo = min(max(p.group_begin[g], 0), p.rows), hi = min(max(p.group_begin[g + 1], 0), p.rows);
    if (t == 0) s_n = 0;
    // logarithms of the rows' sums, a wave each
    for (int r = lo + wave; r < hi; r += kWaves) {
        const float score = p.score[r];
        if (dead(score) || (p.end_token && p.end_token[r] >= 0)) continue;
        const SpanRecord *rec = p.records + (int64_t)r * p.spans;
        float ref = kLowest;
        for (int i = lane; i < p.spans; i += kWave) ref = fmaxf(ref, rec[i].ref);
        ref = wave_max(ref);
        double sum = 0.0;
        for (int i = lane; i < p.spans; i += kWave) sum += rec[i].sum * exp((double)rec[i].ref - (double)ref);
        sum = wave_sum_double(sum);
        if (lane == 0) p.row_log[r] = (double)ref + log(sum); // a row without any: never used
    }
    __threadfence_block();
    __syncthreads();
    // Every thread walks down one record (a span's elements in order) until its next element is no better than the worst kept.
    const int64_t records = (int64_t)max(hi - lo, 0) * p.spans;
    int n = 0;
    Choice worst = {};
    bool full = false;
    for (int64_t base = 0; base < records; base += kThreads) {
        const int64_t i = base + t;
        bool on = i < records, finished = false;
        int r = lo, next = 0;
        float score = 0.0f;
        double row_log = 0.0;
        const uint64_t *keys = nullptr;
        if (on) {
            r = lo + (int)(i / p.spans);
            score = p.score[r];
            on = !dead(score);
            finished = on && p.end_token && p.end_token[r] >= 0;
            if (finished) on = i % p.spans == 0;
            else if (on) row_log = p.row_log[r];
            keys = p.keys + ((int64_t)r * p.spans + i % p.spans) * keep;
        }
        while (true) {
            Choice c = {};
            if (on) {
                if (finished) {
                    c = Choice{ordered64((double)score), (uint32_t)~p.end_token[r], (uint32_t)r, 0};
                    on = next == 0;
                } else {
                    const uint64_t key = next < keep ? keys[next] : 0;
                    on = key != 0;
                    c = Choice{ordered64((double)score + ((double)unordered((uint32_t)(key >> 32)) - row_log)), key, (uint32_t)r, 0};
                }
                ++next;
                on = on && !(full && !better(c, worst));
            }
            if (!__syncthreads_or(on)) break;
            if (on) s_list[atomicAdd(&s_n, 1)] = c; // at most kThreads in a round
            __syncthreads();
            n = s_n;
            if (n > kMergeList - kThreads || (!full && n >= keep)) {
                n = keep_best_choices(s_list, n, keep);
                if (t == 0) s_n = n;
                full = n == keep;
                if (full) worst = s_list[keep - 1];
                __syncthreads();
            }
        }
    }
    n = keep_best_choices(s_list, n, keep);
    for (int i = t; i < keep; i += kThreads) {
        const int64_t at = (int64_t)g * keep + i;
        const bool in = i < n;
        p.parent[at] = in ? (int32_t)s_list[i].row : -1;
        p.token[at] = in ? (int32_t)~(uint32_t)s_list[i].key : -1;
        p.total[at] = in ? (float)unordered64(s_list[i].total) : -kInf;
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
