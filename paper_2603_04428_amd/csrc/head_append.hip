// From a layer's projections to its queries and cache rows in one pass (Sec. 3.4, the first half of update_and_fetch, with
// what a model does to a head in front of it): per head of Q and K
//     y_i = x_i w_i / sqrt(mean_{i < norm_dim} x_i^2 + eps)        for i < norm_dim, y_i = x_i behind it or without weights
//     (y_i, y_j) -> (y_i c - y_j s, y_j c + y_i s)                 for the pairs (i, j) of the rotated span, c and s of the
//                                                                  token's position from the caller's tables
// rounded once to binary16; Q goes out, K and the rows of V (as they are) are quantized into the agents' blocks as q4kv_append
// does.  Done in three passes (norm and rotate Q, the same for K, append) the rows of K travel twice more.
//
// What bounds it is memory: 2 bytes in per element of Q, K and V, 2 out for Q and 0.5625 for K and V.  A lane takes 8
// consecutive elements (16 bytes), a row of up to 512 elements LPR lanes, a wider one two passes of a wave; a row of 192 leaves
// a quarter of its 32 lanes idle, one of 576 44 % of its places (three passes of 32 lanes take 240 registers and longer: 23.2 us for
// 21.7 in replayed graphs).  Measured (kernel trace): 512 tokens of ten agents, 16 + 8 + 8 256-wide heads, 42 us for 138 MB; 301 of five,
// latent rows, 23 us for 58 MB; one token of ten 5 us.
//
// All arithmetic in front of the rounding is binary64: codes come from roundings, so a result on the other side of a border
// moves a cache value by a whole scale (a fifteenth of its group's range), and with binary32 about one element in 2,000 is
// rounded differently.  The vector ALUs do binary64 multiply-adds at the rate of binary32 ones.  Products of a weight and a
// table entry have 48 bits and are exact; they are taken once per (lane, token) and serve all heads the lane visits.
#include "q4_device.h"
#include "q4kv_internal.h"
#include "quantize_octet.h"

namespace q4kv {
namespace {

constexpr int kThreads = 256;

struct HeadSection { // Q, K or V
    const uint16_t *x;
    int64_t token_stride;  // elements from a token's row to the next token's
    const float *weight;   // [layers in call][norm_dim] or null
    int heads, dim, splits; // splits: workgroups that share the heads
};

struct HeadAppendParams {
    HeadSection sec[3];
    uint16_t *q_out;
    uint32_t *codes[2];
    uint16_t *scale[2], *bias[2];
    const float *cos, *sin;
    const int32_t *block_table, *seq_len_before, *positions;
    double eps, inv_norm_dim;
    int norm_dim, rot_begin, rot_dim, neighbours, table_len;
    int agents, chunk, max_blocks, num_blocks, layer_begin;
    int tokens_log2; // tokens of a workgroup's rows
    uint32_t token_chunks;
};

// binary64 to binary16 in one rounding: what lies below the upper word's 20 fraction bits is folded into the last of them
// (round to odd), the rest is exact in binary32, and only the conversion to binary16 rounds
__device__ __forceinline__ half_t half_once(double d)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, d);
    const uint32_t hi = (uint32_t)(u >> 32) | min((uint32_t)u, 1u);
    return (half_t)(float)__builtin_bit_cast(double, (uint64_t)hi << 32);
}

template <bool IN_BF>
__device__ __forceinline__ void widen(const uint4 &raw, float (&x)[8])
{
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = IN_BF ? __builtin_bit_cast(float, w[i] << 16) : half_bits_to_float((uint16_t)(w[i] & 0xffffu));
        x[2 * i + 1] = IN_BF ? __builtin_bit_cast(float, w[i] & 0xffff0000u) : half_bits_to_float((uint16_t)(w[i] >> 16));
    }
}

// Sum over the LPR lanes of a row, in all of them: exchanges inside 16 lanes as data-parallel-primitive moves, the rest as swaps
// of half rows.
template <int CTRL>
__device__ __forceinline__ double dpp_add(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
    return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int LPR>
__device__ __forceinline__ double row_sum(double v)
{
    v = dpp_add<0xB1>(v);  // quad_perm [1,0,3,2]
    v = dpp_add<0x4E>(v);  // quad_perm [2,3,0,1]
    v = dpp_add<0x141>(v); // row_half_mirror
    if constexpr (LPR >= 16) v = dpp_add<0x140>(v); // row_mirror
    if constexpr (LPR >= 32) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
        v = __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
    }
    if constexpr (LPR >= 64) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
        v = __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
    }
    return v;
}

// 1 / sqrt(v): the instruction is good to 2^-23 or better, two Newton steps to a few 2^-53.  A row of zeros without an eps stays zeros.
__device__ __forceinline__ double inverse_root(double v)
{
    if (!(v > 0.0)) return 0.0;
    double r = __builtin_amdgcn_rsq(v);
    r = __builtin_fma(r * 0.5, __builtin_fma(-v * r, r, 1.0), r);
    return __builtin_fma(r * 0.5, __builtin_fma(-v * r, r, 1.0), r);
}

// LPR: lanes of a row (a power of two); CPL: passes over a row.  BF: type of the stored parameters, IN_BF: of the projections.
// SPLIT: the norm ends inside the rotated span, so that of some pairs only one half is normed.
template <int LPR, int CPL, bool BF, bool IN_BF, bool SPLIT>
__global__ __launch_bounds__(kThreads) void head_append_kernel(HeadAppendParams p)
{
    constexpr int ROWS = kThreads / LPR; // rows of a workgroup: 2^tokens_log2 tokens of as many heads as that leaves
    const int in_row = threadIdx.x % LPR, row = threadIdx.x / LPR;
    const int a = blockIdx.y, li = blockIdx.z;
    int split = (int)(blockIdx.x / p.token_chunks), which = 0;
    const uint32_t token_chunk = blockIdx.x - (uint32_t)split * p.token_chunks;
    while (split >= p.sec[which].splits) split -= p.sec[which++].splits; // the splits of all sections are the grid's extent
    const HeadSection s = p.sec[which];
    const int tokens = 1 << p.tokens_log2, heads_step = ROWS >> p.tokens_log2;
    const int c = (int)token_chunk * tokens + (row & (tokens - 1));
    if (c >= p.chunk) return; // the whole row leaves

    const int t = p.seq_len_before[a] + c;
    const int pos = p.positions ? p.positions[(int64_t)a * p.chunk + c] : t;
    if (p.rot_dim > 0 && (pos < 0 || pos >= p.table_len)) return;
    int64_t dst0 = -1; // row of head 0 in the pool
    if (which > 0) {
        const int bi = t / kBlockTokens;
        if (t < 0 || bi >= p.max_blocks) return;
        const int blk = p.block_table[(int64_t)a * p.max_blocks + bi];
        if (blk < 0 || blk >= p.num_blocks) return;
        dst0 = (((int64_t)(p.layer_begin + li) * p.num_blocks + blk) * s.heads) * kBlockTokens + t % kBlockTokens;
    }
    const int64_t token = ((int64_t)li * p.agents + a) * p.chunk + c;
    const uint16_t *src = s.x + token * s.token_stride;
    const bool normed = which < 2 && s.weight != nullptr;
    const bool prepared = which < 2 && (normed || p.rot_dim > 0); // else rows go as they are

    // what a chunk of eight elements is multiplied with: y = (x ca + x' cb) f, x' its partners in the rotation (itself and zero
    // where it is not rotated), f = 1 / rms under the norm
    double ca[CPL][8], cb[CPL][8];
    int partner[CPL];       // element the partners begin at
    bool front[CPL], partner_front[CPL]; // under the norm
    const bool pairs_inside = p.neighbours != 0;
    if (prepared) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            const int d = 8 * (in_row + LPR * i), r = d - p.rot_begin;
            front[i] = partner_front[i] = normed && d < p.norm_dim;
            partner[i] = d < s.dim ? d : 0;
            float w[8], wp[8], cs[8], sn[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = wp[e] = cs[e] = 1.0f;
                sn[e] = 0.0f;
            }
            const float *weight = s.weight + (int64_t)li * p.norm_dim;
            if (front[i]) __builtin_memcpy(w, __builtin_assume_aligned(weight + d, 16), 32);
            if (d < s.dim && r >= 0 && r < p.rot_dim) {
                const int half_span = p.rot_dim / 2;
                const float *cos = p.cos + (int64_t)pos * half_span, *sin = p.sin + (int64_t)pos * half_span;
                if (pairs_inside) {
                    float c4[4], s4[4];
                    __builtin_memcpy(c4, __builtin_assume_aligned(cos + r / 2, 16), 16);
                    __builtin_memcpy(s4, __builtin_assume_aligned(sin + r / 2, 16), 16);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        cs[e] = c4[e / 2];
                        sn[e] = (e & 1) ? s4[e / 2] : -s4[e / 2];
                        wp[e] = w[e ^ 1];
                    }
                } else {
                    const bool upper = r >= half_span;
                    const int at = upper ? r - half_span : r;
                    partner[i] = upper ? d - half_span : d + half_span;
                    partner_front[i] = normed && partner[i] < p.norm_dim;
                    __builtin_memcpy(cs, __builtin_assume_aligned(cos + at, 16), 32);
                    __builtin_memcpy(sn, __builtin_assume_aligned(sin + at, 16), 32);
                    if (partner_front[i]) __builtin_memcpy(wp, __builtin_assume_aligned(weight + partner[i], 16), 32);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sn[e] = upper ? sn[e] : -sn[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ca[i][e] = (double)w[e] * (double)cs[e];
                cb[i][e] = (double)wp[e] * (double)sn[e];
            }
        }
    }

    const int G = s.dim / kGroup;
    const int h0 = split * heads_step + (row >> p.tokens_log2), step = s.splits * heads_step;
    uint4 raw[CPL], other[CPL]; // of the head in hand; the next one's are asked for as soon as these have been taken apart
    auto load = [&](int h) {
        const uint16_t *x_row = src + (int64_t)h * s.dim;
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            const int d = 8 * (in_row + LPR * i);
            raw[i] = make_uint4(0, 0, 0, 0);
            if (d < s.dim) raw[i] = *reinterpret_cast<const uint4 *>(x_row + d);
            if (prepared && !pairs_inside) other[i] = *reinterpret_cast<const uint4 *>(x_row + partner[i]);
        }
    };
    auto finish = [&](int h, int i, const uint4 &y8) { // eight prepared elements: out, or into the cache
        const int chunk = in_row + LPR * i;
        if (8 * chunk >= s.dim) return; // whole octets: dim is a multiple of 64
        if (which == 0) {
            *reinterpret_cast<uint4 *>(p.q_out + (token * s.heads + h) * s.dim + 8 * chunk) = y8;
        } else {
            const int sub = threadIdx.x & 7, pool = which - 1;
            uint16_t sb, bb;
            const uint32_t word = quantize_octet<BF>(y8, sub, &sb, &bb);
            const int64_t dst = dst0 + (int64_t)h * kBlockTokens;
            p.codes[pool][dst * (s.dim / 8) + chunk] = word;
            if (sub < 2) (sub == 0 ? p.scale[pool] : p.bias[pool])[dst * G + chunk / 8] = sub == 0 ? sb : bb;
        }
    };
    if (h0 < s.heads) load(h0);
    if (!prepared) {
        for (int h = h0; h < s.heads; h += step) {
            uint4 now[CPL];
#pragma unroll
            for (int i = 0; i < CPL; ++i) now[i] = raw[i];
            if (h + step < s.heads) load(h + step);
#pragma unroll
            for (int i = 0; i < CPL; ++i) {
                if constexpr (IN_BF) {
                    float x[8];
                    widen<true>(now[i], x);
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = half2_to_bits(half2_t{(half_t)x[2 * e], (half_t)x[2 * e + 1]});
                    now[i] = make_uint4(o[0], o[1], o[2], o[3]);
                }
                finish(h, i, now[i]);
            }
        }
        return;
    }
    for (int h = h0; h < s.heads; h += step) {
        float x[CPL][8], xp[CPL][8];
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            widen<IN_BF>(raw[i], x[i]);
            if (pairs_inside) {
#pragma unroll
                for (int e = 0; e < 8; ++e) xp[i][e] = x[i][e ^ 1];
            } else {
                widen<IN_BF>(other[i], xp[i]);
            }
        }
        if (h + step < s.heads) load(h + step);
        double x64[CPL][8];
#pragma unroll
        for (int i = 0; i < CPL; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) x64[i][e] = (double)x[i][e];
        double inv = 1.0;
        if (normed) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < CPL; ++i) {
                double part = 0.0;
#pragma unroll
                for (int e = 0; e < 8; ++e) part = __builtin_fma(x64[i][e], x64[i][e], part);
                sum += front[i] ? part : 0.0;
            }
            inv = inverse_root(__builtin_fma(row_sum<LPR>(sum), p.inv_norm_dim, p.eps));
        }
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            const double f = front[i] ? inv : 1.0;
            const double g = partner_front[i] ? inv : 1.0;
            half_t o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double v = (double)xp[i][e];
                // where only one half of a pair is under the norm each factor goes to its own term: either may be zero
                if constexpr (SPLIT) o[e] = half_once(__builtin_fma(v * g, cb[i][e], x64[i][e] * f * ca[i][e]));
                else o[e] = half_once(__builtin_fma(v, cb[i][e], x64[i][e] * ca[i][e]) * f);
            }
            uint32_t out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = half2_to_bits(half2_t{o[2 * e], o[2 * e + 1]});
            finish(h, i, make_uint4(out[0], out[1], out[2], out[3]));
        }
    }
}

template <int LPR, int CPL, bool BF, bool IN_BF>
auto kernel_of(bool split)
{
    return split ? head_append_kernel<LPR, CPL, BF, IN_BF, true> : head_append_kernel<LPR, CPL, BF, IN_BF, false>;
}
template <int LPR, int CPL>
hipError_t launch_rows(const HeadAppendParams &p, bool bf, bool in_bf, bool split, dim3 grid, hipStream_t stream)
{
    const auto kernel = bf ? (in_bf ? kernel_of<LPR, CPL, true, true>(split) : kernel_of<LPR, CPL, true, false>(split))
                           : (in_bf ? kernel_of<LPR, CPL, false, true>(split) : kernel_of<LPR, CPL, false, false>(split));
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

} // namespace

int head_append_max_dim() { return 1024; }

hipError_t launch_head_append(const HeadAppendArgs &a, hipStream_t stream)
{
    const q4kv_spec &s = *a.spec;
    HeadAppendParams p;
    p.sec[0] = HeadSection{static_cast<const uint16_t *>(a.q), a.q_stride, a.form->q_weight, s.num_q_heads, s.k_dim, 1};
    p.sec[1] = HeadSection{static_cast<const uint16_t *>(a.k_new), a.k_stride, a.form->k_weight, s.num_kv_heads, s.k_dim, 1};
    p.sec[2] = HeadSection{static_cast<const uint16_t *>(a.v_new), a.v_stride, nullptr, a.v ? s.num_kv_heads : 0, s.v_dim, a.v ? 1 : 0};
    p.q_out = a.q_out;
    const q4kv_pool *const pools[2] = {a.k, a.v ? a.v : a.k};
    for (int i = 0; i < 2; ++i) {
        p.codes[i] = pools[i]->codes;
        p.scale[i] = pools[i]->scale;
        p.bias[i] = pools[i]->bias;
    }
    p.cos = a.form->cos_table;
    p.sin = a.form->sin_table;
    p.block_table = a.block_table;
    p.seq_len_before = a.seq_len_before;
    p.positions = a.positions;
    p.eps = a.form->eps;
    p.inv_norm_dim = a.form->norm_dim > 0 ? 1.0 / a.form->norm_dim : 0.0;
    p.norm_dim = a.form->norm_dim;
    p.rot_begin = a.form->rot_begin;
    p.rot_dim = a.form->rot_dim;
    p.neighbours = a.form->neighbours;
    p.table_len = a.form->table_len;
    p.agents = a.num_agents;
    p.chunk = a.chunk_len;
    p.max_blocks = a.max_blocks;
    p.num_blocks = a.k->num_blocks;
    p.layer_begin = a.layer_begin;
    const int layers = a.layer_end - a.layer_begin;
    const int dim = a.v && s.v_dim > s.k_dim ? s.v_dim : s.k_dim;
    const int lanes = dim <= 64 ? 8 : dim <= 128 ? 16 : dim <= 256 ? 32 : 64;
    const int rows = kThreads / lanes;
    p.tokens_log2 = 0;
    while ((1 << p.tokens_log2) < rows && (1 << p.tokens_log2) < a.chunk_len) ++p.tokens_log2;
    const int tokens = 1 << p.tokens_log2, heads_step = rows / tokens;
    p.token_chunks = (uint32_t)((a.chunk_len + tokens - 1) / tokens);
    // A lane visits up to eight heads of its token, with the same weights and table entries in its registers (a wave spends about 500
    // instructions on them, and 120 to 280 on a head), as long as Q, K and V each keep three workgroups per compute unit.  Measured
    // (us a call, 16 / 8 / 4 / 3 / 2 workgroups): 512 tokens of ten agents, 256-wide 56.3 / 42.3 / 38.3 / 38.2 / 39.1; 301 of five, latent rows
    // 33.6 / 24.9 / 21.2 / 21.3 / 23.5; 700 of eight, 64-wide, three layers 20.2 / 15.9 / 15.5 / 15.5 / 18.3; 300 of three, 192 + 128 17.3 / 16.8 /
    // 16.8 / 13.8 / 13.8; 2,000 of one, 128-wide, two layers 35.5 / 28.5 / 25.6 / 22.5 / 22.6.
    const int64_t columns = (int64_t)p.token_chunks * a.num_agents * layers;
    int total = 0;
    for (HeadSection &sec : p.sec) {
        if (sec.heads == 0) continue;
        const int steps = (sec.heads + heads_step - 1) / heads_step;
        int per = 1;
        while (per < 8 && per * 2 <= steps && columns * (steps / (per * 2)) >= 3 * (int64_t)a.compute_units) per *= 2;
        sec.splits = (steps + per - 1) / per;
        total += sec.splits;
    }
    const dim3 grid(p.token_chunks * (unsigned)total, (unsigned)a.num_agents, (unsigned)layers);
    const bool bf = s.param_format == Q4KV_PARAMS_BF16, in_bf = a.in_format == Q4KV_PARAMS_BF16;
    const q4kv_head_form &f = *a.form;
    const bool split = (f.q_weight || f.k_weight) && !f.neighbours && f.norm_dim > f.rot_begin && f.norm_dim < f.rot_begin + f.rot_dim;
    if (dim <= 64) return launch_rows<8, 1>(p, bf, in_bf, split, grid, stream);
    if (dim <= 128) return launch_rows<16, 1>(p, bf, in_bf, split, grid, stream);
    if (dim <= 256) return launch_rows<32, 1>(p, bf, in_bf, split, grid, stream);
    if (dim <= 512) return launch_rows<64, 1>(p, bf, in_bf, split, grid, stream);
    return launch_rows<64, 2>(p, bf, in_bf, split, grid, stream);
}

} // namespace q4kv
