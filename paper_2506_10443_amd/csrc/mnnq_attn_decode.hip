// Attention of one or a few tokens over the 8-bit cache (mnnq_attn_decode).
//
// For a sequence and key head the queries of the group's heads and of all tokens are the rows of one product, 16 at a
// time: S = K Q^T with tokens down and rows across (v_mfma_f32_16x16x32_f16), O^T = V^T P^T.  Tokens-down puts a row's scores
// into the lanes of one column, where the next product wants its probabilities: the four scores of a lane in two tiles of 16
// tokens are its eight values of P^T as they stand.
//   * Codes become halves exactly; bfloat16 queries become halves scaled by a power of two per row so that the greatest is in
//     [2^14, 2^15), exact down to 2^-31 of it, below that to 2^-39 of it; ranges, scale and that power are one factor per row and
//     block applied to the fp32 sums.
//   * V's range goes into P: p r / U, U the greatest range so far (the accumulators are rescaled when it grows).  Probabilities
//     stay below 2^14 instead of 1, so that a half holds them down to 2^-32 of the greatest, 2^-28 with the least r / U.  Where a wave
//     meets ranges 16 times below U, or U comes to 16 times its first, a great range says nothing about a row: it may have no attention
//     there, codes of zero, or end before.  P then stays as it is, under a power of two per row and half step, and r / U multiplies the
//     fp32 products.
// A wave takes 32 tokens at a time, with the codes of its next 32 in flight; the waves of a workgroup share a part of the
// sequence and join through LDS, the parts are joined by a second kernel.
//
// 2 D bytes per token and key head are read once and 4 D rows operations done with them, at most a few dozen per byte: HBM bounds long
// caches, a chain of launch, ramp and join short ones.  One token (both kernels): 131072 tokens of 4 key heads, 134 MB, 33.6 us, 29 of
// them the first kernel at 4.6 TB/s (its loads alone 25.5); 32 ragged sequences, 178 MB, 45.3; 1001 tokens 8.6.  Ranges far apart: 131072
// tokens 41.2, in blocks of 16 tokens 50.1.  Loads go to registers, not through LDS: each code is used by one lane.
#include "mnnq_attn.h"
#include "mnnq_forms.h"

#include <type_traits>

namespace mnnq {

namespace {

constexpr int kWaves = 4;
constexpr int kStep = 32;                        // tokens of a wave's step
constexpr float kTopBits = 8.0f;                 // a probability at the running maximum is 2^8
constexpr float kSlack = 6.0f;                   // the running maximum follows when it is 2^6 behind
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kLeastNormal = 1.17549435e-38f;
constexpr float kNear = 1.0f / 16;               // the least r / U that goes into P
constexpr int kOutOfRange = 0x7ffffff0;          // a byte offset beyond every piece: loads give 0

struct DecodeArgs {
    mnnq_kv_cache c;
    Rows q, out;
    float* means;                                // [sequences, kv_heads, rows, parts, DP] where there is more than one part
    float2* stats;                               // [sequences, kv_heads, rows, parts]: maximum (log2; -inf: no key) and sum
    float* scores;                               // [sequences, kv_heads, rows, scores_stride] where weights are asked for
    float* weights;
    int64_t tokens, scores_stride, weights_stride;
    int bound, part_len, parts;
    int group, rows;                             // rows: group * tokens
    float scale_log2;
    bool bf16;
};

__device__ __forceinline__ int length_of(const DecodeArgs& a, int64_t s)
{
    const int n = a.c.lengths[s];
    return n < 0 ? 0 : n > a.bound ? a.bound : n;
}

// Maximum over the four lanes of a column (l, l + 16, l + 32, l + 48), the same in all of them.
__device__ __forceinline__ float column_max(float v)
{
    const u2v a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const u2v b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// N 16-byte pieces of a bfloat16 query row per lane as halves times 2^up, up such that the row's greatest is in [2^14, 2^15).
template <int N>
__device__ __forceinline__ int scale_query(const u4v (&raw)[N], half8v (&out)[N])
{
    typedef unsigned short us2v __attribute__((ext_vector_type(2)));
    us2v two = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) two = __builtin_elementwise_max(two, __builtin_bit_cast(us2v, raw[i][j] & 0x7fff7fffu));
    uint32_t top = max((uint32_t)two.x, (uint32_t)two.y);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const int up = max(-126, min(126, 14 + 127 - (int)(top >> 7)));      // (the exponent's bits)
    const float mul = __uint_as_float((uint32_t)(up + 127) << 23);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const half2v h = __builtin_bit_cast(half2v, pack16(__uint_as_float(raw[i][j] << 16) * mul,
                                                               __uint_as_float(raw[i][j] & 0xffff0000u) * mul, false));
            out[i][2 * j] = h.x, out[i][2 * j + 1] = h.y;
        }
    return up;
}

template <int DP, int KF, int VF, int MT>
__global__ __launch_bounds__(64 * kWaves, DP == 256 ? 1 : 2) void decode_kernel(DecodeArgs a, const int32_t* __restrict__ tables,
                                                              const float* __restrict__ k_ranges,
                                                              const float* __restrict__ v_ranges)
{
    constexpr int KC = DP / 64;                  // 16-byte pieces of a K row per lane
    constexpr int VB = DP / 16;                  // bytes of a V row per lane
    constexpr int VW = VB / 4;
    constexpr int ND = DP / 16;                  // matrix instructions of O^T per row tile
    constexpr int DH = DP < 512 / kWaves ? DP : 512 / kWaves;      // values of a row that the waves join at a time
    constexpr int kStride = kWaves * kStep;
    __shared__ __align__(16) float red[kWaves][16 * (DH + 4)];
    __shared__ float red_m[kWaves][16], red_l[kWaves][16];

    const mnnq_kv_cache& c = a.c;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int D = c.head_dim, B = c.block_tokens;
    const int64_t s = blockIdx.z;
    const int kvh = blockIdx.y % c.kv_heads, row0 = (blockIdx.y / c.kv_heads) * 16 * MT;
    const int block_shift = __builtin_ctz(B);
    const int p0 = blockIdx.x * a.part_len;
    int p = p0 + wave * kStep;

    // Entries of the table are fetched two steps ahead, the length beside the first ones (an entry behind the last token is
    // of no use, and does no harm).
    const int32_t* table = tables + s * c.table_blocks;
    const int last_entry = (int)c.table_blocks - 1;
    struct Entries {
        int at[2];
    };
    auto find = [&](int p) {
        const int n = p >> block_shift, m = (p + 16) >> block_shift;
        return Entries{{table[n < last_entry ? n : last_entry], table[m < last_entry ? m : last_entry]}};
    };
    Entries ahead = find(p);
    const int len = length_of(a, s);
    if (p0 >= len && a.parts > 1) return;        // (one part: rows of zeros are stored)
    const int p1 = p0 + a.part_len < len ? p0 + a.part_len : len;

    // The codes of a step: two tiles of 16 tokens; there: 0 where the cache has no such block, and behind the last token, where the
    // table's entry may name a block of anybody's or nobody's.
    struct Codes {
        bool there[2];
        u4v k[2][KC];
        uint32_t v[8][VW];
        float kr[2], vr[2];
    };
    int k_off[KC], v_off[4];
#pragma unroll
    for (int j = 0; j < KC; ++j) k_off[j] = 64 * j + 16 * g < D ? col * D + 16 * g + 64 * j : kOutOfRange;
#pragma unroll
    for (int j = 0; j < 4; ++j) v_off[j] = VB * col < D ? (4 * g + j) * D + VB * col : kOutOfRange;
    auto load = [&](int p, const Entries& b, Codes& x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = p + 16 * i;
            const bool known = (uint32_t)b.at[i] < (uint32_t)c.blocks;
            x.there[i] = known & (at < p1);
            const int64_t slot = (int64_t)(known ? b.at[i] : 0) * c.kv_heads + kvh;
            // (rows behind the last token may hold anything, NaN codes among it: they are beyond the piece and come as zeros)
            const int left = p1 - at < 16 ? p1 - at : 16;
            const int bytes = x.there[i] ? left * D : 0;
            const int64_t from = (slot * B + (at & (B - 1))) * D;
            const __amdgpu_buffer_rsrc_t rk = rsrc(static_cast<const uint8_t*>(c.k_codes) + from, bytes);
            const __amdgpu_buffer_rsrc_t rv = rsrc(static_cast<const uint8_t*>(c.v_codes) + from, bytes);
#pragma unroll
            for (int j = 0; j < KC; ++j) x.k[i][j] = __builtin_bit_cast(u4v, __builtin_amdgcn_raw_buffer_load_b128(rk, k_off[j], 0, 0));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (VW == 1) {
                    x.v[4 * i + j][0] = __builtin_amdgcn_raw_buffer_load_b32(rv, v_off[j], 0, 0);
                } else if constexpr (VW == 2) {
                    const u2v w = __builtin_bit_cast(u2v, __builtin_amdgcn_raw_buffer_load_b64(rv, v_off[j], 0, 0));
                    x.v[4 * i + j][0] = w.x, x.v[4 * i + j][1] = w.y;
                } else {
                    const u4v w = __builtin_bit_cast(u4v, __builtin_amdgcn_raw_buffer_load_b128(rv, v_off[j], 0, 0));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.v[4 * i + j][e] = w[e];
                }
            }
            x.kr[i] = k_ranges[slot];
            x.vr[i] = v_ranges[slot];
        }
    };
    // What the scalar loads of the step before brought is taken before new ones are requested: they return in any order, so that
    // a wait for one is a wait for all.
    auto arrived = [&](Codes& x, Entries& b) {
        asm volatile("" : "+s"(x.kr[0]), "+s"(x.kr[1]), "+s"(x.vr[0]), "+s"(x.vr[1]), "+s"(b.at[0]), "+s"(b.at[1]));
    };

    Codes x0, x1;
    if (p < p1) load(p, ahead, x0);
    ahead = find(p + kStride);

    // queries, their power of two, and how far each row sees
    half8v qf[MT][2 * KC];
    float factor[MT];
    int limit[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int r = row0 + m * 16 + col;
        const bool there = r < a.rows;
        const int t = there ? r / a.group : 0;
        const int h = kvh * a.group + (there ? r - t * a.group : 0);
        limit[m] = there ? len - (int)a.tokens + t + 1 : 0;
        const uint16_t* src = a.q.data + (s * a.tokens + t) * a.q.token + h * a.q.head;
        u4v raw[2 * KC];
#pragma unroll
        for (int i = 0; i < 2 * KC; ++i) {
            const int d = 64 * (i / 2) + 16 * g + 8 * (i & 1);
            raw[i] = u4v{0, 0, 0, 0};
            if (there && d < D) raw[i] = *reinterpret_cast<const u4v*>(src + d);
        }
        factor[m] = a.scale_log2;
        if (a.bf16) {
            factor[m] *= __uint_as_float((uint32_t)(127 - scale_query(raw, qf[m])) << 23);
        } else {
#pragma unroll
            for (int i = 0; i < 2 * KC; ++i) qf[m][i] = __builtin_bit_cast(half8v, raw[i]);
        }
    }
    const int lowest_limit = len - (int)a.tokens + 1;             // tokens below it are seen by every row

    f4v o[MT][ND];
    float mx[MT], l[MT];
    int earliest = p1;                           // first token of the wave's, in sixteens, that is there
    float unit = 0.0f, inv_unit = 0.0f;          // U and 1 / U
    float first_unit = __builtin_inff();         // the first U
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        mx[m] = kLowest;
        l[m] = 0.0f;
#pragma unroll
        for (int i = 0; i < ND; ++i) o[m][i] = f4v{0, 0, 0, 0};
    }

    // V: a byte of four tokens each, twice
    auto values_of = [&](const Codes& x, int w, int b) {
        half8v vf;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            half2v lo, hi;
            byte_to_half<VF>(x.v[4 * i][w], x.v[4 * i + 1][w], x.v[4 * i + 2][w], x.v[4 * i + 3][w], b, lo, hi);
            vf[4 * i] = lo.x, vf[4 * i + 1] = lo.y, vf[4 * i + 2] = hi.x, vf[4 * i + 3] = hi.y;
        }
        return vf;
    };
    // A step's products with V, ranges far apart: a pass for each half step, one for both where they share a range.  P: -0 where hidden.
    auto add_apart = [&](Codes& x, const float (&pr)[MT][8], float v0, float v1) {
        const bool both = v0 == v1;
#pragma nounroll
        for (int half = 0; half < (both ? 1 : 2); ++half) {
            const float v = half ? v1 : v0;
            if (v == 0.0f) continue;
            const bool number = v < __builtin_inff();
            half8v ph[MT];
            float back[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                float mine[8], top = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    mine[i] = both || i / 4 == half ? pr[m][i] : -0.0f;
                    top = fmaxf(top, mine[i]);
                }
                // the row's greatest to [2^13, 2^14); a range that is no number, to the rows that see it, as it is
                const uint32_t up = min(267u - (__float_as_uint(column_max(top)) >> 23), 253u);
                const float mul = number ? __uint_as_float(up << 23) : v;
                back[m] = number ? v * inv_unit * __uint_as_float((254u - up) << 23) : 1.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) mine[i] = __float_as_uint(mine[i]) >> 31 ? 0.0f : mine[i] * mul;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const half2v h = __builtin_bit_cast(half2v, pack16(mine[2 * e], mine[2 * e + 1], false));
                    ph[m][2 * e] = h.x, ph[m][2 * e + 1] = h.y;
                }
            }
            // (the codes as new ones: their halves are not kept over the passes, which would take more registers than there are)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int w = 0; w < VW; ++w) asm volatile("" : "+v"(x.v[i][w]));
#pragma unroll
            for (int w = 0; w < VW; ++w)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const half8v vf = values_of(x, w, b);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        o[m][4 * w + b] += __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, ph[m], f4v{0, 0, 0, 0}, 0, 0, 0) * back[m];
                }
        }
    };

    // A step whose ranges call for the other form hides all of its tokens and ends the loop: a branch out of it costs more (131072
    // tokens, 33.9 us: 34.4 with one behind the scores, 36 with one in front of them).
    int end = p1;
    auto step = [&](int p, Codes& x, auto apart) {
        f4v sc[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 2; ++i) sc[m][i] = f4v{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < KC; ++j) {
                const half8v k0 = codes_to_half8<KF>(x.k[i][j][0], x.k[i][j][1]);
                const half8v k1 = codes_to_half8<KF>(x.k[i][j][2], x.k[i][j][3]);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    sc[m][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf[m][2 * j], sc[m][i], 0, 0, 0);
                    sc[m][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf[m][2 * j + 1], sc[m][i], 0, 0, 0);
                }
            }
        const float k0 = x.there[0] ? x.kr[0] : 0.0f, k1 = x.there[1] ? x.kr[1] : 0.0f;
        // (a range that is not finite is that of undefined values, which only rows that see them may get)
        const float v0 = x.there[0] ? x.vr[0] : 0.0f, v1 = x.there[1] ? x.vr[1] : 0.0f;
        float less_unit = 1.0f;                  // what the accumulators take of U's growth
        if (!(fmaxf(v0, v1) <= unit && fminf(v0, v1) >= unit * kNear)) {
            // (a zero, and what is no number, have no say)
            const bool n0 = v0 > 0.0f && v0 < __builtin_inff(), n1 = v1 > 0.0f && v1 < __builtin_inff();
            const float vmax = fmaxf(n0 ? v0 : 0.0f, n1 ? v1 : 0.0f), now = fmaxf(vmax, unit), low = now * kNear;
            if (!decltype(apart)::value && ((n0 && v0 < low) || (n1 && v1 < low) || first_unit < low)) {
                end = p;
            } else if (vmax > unit) {
                first_unit = fminf(first_unit, vmax);
                const float before = unit;
                unit = fmaxf(vmax, kLeastNormal);
                inv_unit = 1.0f / unit;
                less_unit = before * inv_unit;
            }
        }
        const float ratio[2] = {v0 * inv_unit, v1 * inv_unit};
        earliest = min(earliest, x.there[0] ? p : x.there[1] ? p + 16 : p1);
        const bool masked = p + kStep > lowest_limit || p + kStep > end || !x.there[0] || !x.there[1];
        half8v pf[MT];
        float all_pr[MT][8];                     // (ranges apart)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            uint32_t hidden = 0;
            if (masked)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int t = p + 16 * (i / 4) + 4 * g + (i & 3);
                    if (t >= limit[m] || t >= end || !x.there[i / 4]) {
                        hidden |= 1u << i;
                        sc[m][i / 4][i & 3] = -__builtin_inff();
                    }
                }
            // (the factor is positive, or 0 or NaN with a range that is)
            const float f[2] = {factor[m] * (k0 * (1.0f / code_top<KF>())), factor[m] * (k1 * (1.0f / code_top<KF>()))};
            float top = kLowest;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                top = fmaxf(top, f[i] * fmaxf(fmaxf(sc[m][i][0], sc[m][i][1]), fmaxf(sc[m][i][2], sc[m][i][3])));
            if (a.scores && row0 + m * 16 + col < a.rows) {
                float* to = a.scores + ((s * c.kv_heads + kvh) * a.rows + row0 + m * 16 + col) * a.scores_stride + p + 4 * g;
#pragma unroll
                for (int i = 0; i < 2; ++i) *reinterpret_cast<f4v*>(to + 16 * i) = sc[m][i] * f[i];      // (what is hidden is not looked at)
            }
            top = column_max(top);
            const bool follow = __ballot(top > mx[m] + kSlack) != 0;
            if (follow || less_unit != 1.0f) {
                const float now = top > mx[m] + kSlack ? top : mx[m];        // (each row by itself)
                const float down = __builtin_amdgcn_exp2f(mx[m] - now);
                mx[m] = now;
                l[m] *= down;
#pragma unroll
                for (int i = 0; i < ND; ++i) o[m][i] *= down * less_unit;
            }
            const float less = kTopBits - mx[m];
            float pr[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[m][i / 4][i & 3], f[i / 4], less));
            if (masked)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (hidden >> i & 1) pr[i] = 0.0f;
            l[m] += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
            if constexpr (decltype(apart)::value) {
#pragma unroll
                for (int i = 0; i < 8; ++i) all_pr[m][i] = hidden >> i & 1 ? -0.0f : pr[i];
                continue;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) pr[i] *= ratio[i / 4];
            if (masked)                              // (a ratio that is no number is not theirs)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (hidden >> i & 1) pr[i] = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const half2v h = __builtin_bit_cast(half2v, pack16(pr[2 * e], pr[2 * e + 1], false));
                pf[m][2 * e] = h.x, pf[m][2 * e + 1] = h.y;
            }
        }
        if constexpr (decltype(apart)::value) {
            add_apart(x, all_pr, v0, v1);
            return;
        }
#pragma unroll
        for (int w = 0; w < VW; ++w)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const half8v vf = values_of(x, w, b);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    o[m][4 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[m], o[m][4 * w + b], 0, 0, 0);
            }
    };

    for (; p < end; p += 2 * kStride) {
        const int q = p + kStride;
        arrived(x0, ahead);
        if (q < p1) load(q, ahead, x1);
        ahead = find(q + kStride);
        step(p, x0, std::false_type{});
        if (q >= end) break;
        arrived(x1, ahead);
        if (q + kStride < p1) load(q + kStride, ahead, x0);
        ahead = find(q + 2 * kStride);
        step(q, x1, std::false_type{});
    }
    // (a step's codes when it needs them, so that its products have the registers)
    p = end, end = p1;
    if (__builtin_expect(p < p1, 0))
        for (; p < p1; p += kStride) {
            load(p, find(p), x0);
            step(p, x0, std::true_type{});
        }

    // Join the waves: lane (g, col) holds of row col the values d = VB (4 g + v) + i, v = 0..3.
    const int row = threadIdx.x / (4 * kWaves), at = threadIdx.x % (4 * kWaves);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float sum = l[m];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (m > 0) __syncthreads();
        // (a row without a key has a maximum of -inf; one that sees keys of -inf only the lowest number, and 0 / 0 in the end)
        if (g == 0) red_m[wave][col] = earliest < p1 && earliest < limit[m] ? mx[m] : -__builtin_inff(), red_l[wave][col] = sum;
        __syncthreads();
        float top = red_m[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, red_m[w][col]);
        const float base = fmaxf(top, kLowest);
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all += red_l[w][col] * __builtin_amdgcn_exp2f(red_m[w][col] - base);
        // The sum is divided out before the range comes in: a mean is no greater than what it is of, a sum may pass binary32.  (1 / all by
        // the instruction, to one unit of fp32; a range that the quotient would bring below the normal numbers goes to the sums.)
        const bool divide = a.parts > 1 ? all > 0.0f || all != all : top >= kLowest;      // (of several parts another may have what is divided by)
        float f = __builtin_amdgcn_exp2f(mx[m] - base) * (divide ? __builtin_amdgcn_rcpf(all) : 0.0f);
        const float range = unit * (1.0f / code_top<VF>());
        if (unit < 0x1p-60f) {
#pragma unroll
            for (int i = 0; i < ND; ++i) o[m][i] *= range;
        } else {
            f *= range;
        }
        const int r = row0 + m * 16 + row;
        const int64_t rows = (s * c.kv_heads + kvh) * a.rows;
        const int t = r / a.group, h = kvh * a.group + r - t * a.group;
        if (a.stats && threadIdx.x < 16 && row0 + m * 16 + col < a.rows)
            a.stats[(rows + row0 + m * 16 + col) * a.parts + blockIdx.x] = float2{top, all};
#pragma unroll
        for (int first = 0; first < DP; first += DH) {
            if (first > 0) __syncthreads();
            // (a row's pieces of 4 VB values: in one half or quarter each)
            if (4 * g * VB / DH == first / DH)
#pragma unroll
                for (int i = 0; i < ND; ++i)
#pragma unroll
                    for (int v = 0; v < 4; ++v) red[wave][col * (DH + 4) + VB * (4 * g + v) + i - first] = o[m][i][v] * f;
            __syncthreads();
            constexpr int N = DH / (4 * kWaves);
            const int d = first + at * N;
            float val[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                val[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) val[i] += red[w][row * (DH + 4) + at * N + i];
            }
            if (r >= a.rows || d >= D) continue;     // (head_dim is a multiple of a thread's values)
            if (a.parts > 1) {
                float* to = a.means + ((rows + r) * a.parts + blockIdx.x) * DP + d;
#pragma unroll
                for (int i = 0; i < N; ++i) to[i] = val[i];
            } else {
                uint16_t* to = a.out.data + (s * a.tokens + t) * a.out.token + h * a.out.head + d;
#pragma unroll
                for (int i = 0; i < N; i += 2)
                    *reinterpret_cast<uint32_t*>(to + i) = pack16(val[i], val[i + 1], a.bf16);
            }
        }
    }
}

constexpr int kJoinThreads = 256;
constexpr int kMaxParts = 1024;
constexpr int kEarly = 4;                        // means that a thread of a join requests before it knows the length
constexpr int kRowsAtOnce = 64;                  // rows whose statistics a workgroup holds

// Behind the parts.  Workgroups below a.rows (where there are several parts): one row's parts joined.  The others: attention
// given to kJoinThreads tokens.
template <int DP>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(DecodeArgs a)
{
    constexpr int PER = DP / 4;                  // threads of a part: four values each
    constexpr int TEAMS = kJoinThreads / PER;
    __shared__ float f[kMaxParts];
    __shared__ float wave_top[kJoinThreads / 64], wave_sum[kJoinThreads / 64];
    __shared__ f4v red[TEAMS][PER];
    __shared__ float row_top[kRowsAtOnce], row_inv[kRowsAtOnce];
    __shared__ int row_limit[kRowsAtOnce];       // the row sees the tokens below
    const mnnq_kv_cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int kvh = blockIdx.y;
    const int64_t s = blockIdx.z;
    const int joins = a.parts > 1 ? a.rows : 0;
    if ((int)blockIdx.x < joins) {
        // The length and the first of the means are requested together; what lies in parts behind the length is not looked at.
        const int r = blockIdx.x, team = tid / PER, d = tid % PER;
        const int64_t first = ((s * c.kv_heads + kvh) * a.rows + r) * a.parts;
        const f4v* from = reinterpret_cast<const f4v*>(a.means + first * DP) + d;
        f4v early[kEarly];
#pragma unroll
        for (int i = 0; i < kEarly; ++i) {
            const int part = i * TEAMS + team;
            early[i] = from[(int64_t)(part < a.parts ? part : 0) * PER];
        }
        const float2 mine = a.stats[first + (tid < a.parts ? tid : 0)];
        const int n = (length_of(a, s) + a.part_len - 1) / a.part_len;
        float top = tid < n ? mine.x : -__builtin_inff();
        for (int i = tid + kJoinThreads; i < n; i += kJoinThreads) top = fmaxf(top, a.stats[first + i].x);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        if (lane == 0) wave_top[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kJoinThreads / 64; ++w) top = fmaxf(top, wave_top[w]);
        const float base = fmaxf(top, kLowest);
        float l = 0.0f;
        for (int i = tid; i < n; i += kJoinThreads) {
            const float2 st = i == tid ? mine : a.stats[first + i];
            f[i] = st.y * __builtin_amdgcn_exp2f(st.x - base);
            l += f[i];
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) l += __shfl_xor(l, m);
        if (lane == 0) wave_sum[wave] = l;
        __syncthreads();
        l = 0.0f;
#pragma unroll
        for (int w = 0; w < kJoinThreads / 64; ++w) l += wave_sum[w];
        const float inv = top >= kLowest ? __builtin_amdgcn_rcpf(l) : 0.0f;
        f4v v = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kEarly; ++i)
            if (i * TEAMS + team < n) v += early[i] * (f[i * TEAMS + team] * inv);
#pragma unroll 8
        for (int i = kEarly * TEAMS + team; i < n; i += TEAMS) v += from[(int64_t)i * PER] * (f[i] * inv);
        red[team][d] = v;
        __syncthreads();
        if (team == 0 && 4 * d < c.head_dim) {
#pragma unroll
            for (int i = 1; i < TEAMS; ++i) v += red[i][d];
            const int t = r / a.group, h = kvh * a.group + r - t * a.group;
            uint16_t* to = a.out.data + (s * a.tokens + t) * a.out.token + h * a.out.head;
            *reinterpret_cast<u2v*>(to + 4 * d) = u2v{pack16(v.x, v.y, a.bf16), pack16(v.z, v.w, a.bf16)};
        }
        return;
    }
    const int len = length_of(a, s), n = (len + a.part_len - 1) / a.part_len;
    const int t0 = ((int)blockIdx.x - joins) * kJoinThreads, t = t0 + tid;
    if (t0 >= len) return;
    const int32_t block = t < len ? c.block_table[s * c.table_blocks + (t >> __builtin_ctz(c.block_tokens))] : -1;
    const int64_t row0 = (s * c.kv_heads + kvh) * a.rows;
    float sum = 0.0f;
    for (int first = 0; first < a.rows; first += kRowsAtOnce) {
        const int rows = a.rows - first < kRowsAtOnce ? a.rows - first : kRowsAtOnce;
        __syncthreads();
        // sixteen lanes per row
        for (int r = tid / 16; r < rows; r += kJoinThreads / 16) {
            const int limit = len - (int)a.tokens + (first + r) / a.group + 1;
            const float2* st = a.stats + (row0 + first + r) * a.parts;
            const int i0 = tid & 15;
            const float2 mine = i0 < n ? st[i0] : float2{-__builtin_inff(), 0.0f};
            float top = mine.x;
            for (int i = i0 + 16; i < n; i += 16) top = fmaxf(top, st[i].x);
#pragma unroll
            for (int m = 1; m < 16; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
            const float base = fmaxf(top, kLowest);
            float l = mine.y * __builtin_amdgcn_exp2f(mine.x - base);
            for (int i = i0 + 16; i < n; i += 16) l += st[i].y * __builtin_amdgcn_exp2f(st[i].x - base);
#pragma unroll
            for (int m = 1; m < 16; m <<= 1) l += __shfl_xor(l, m);
            if (i0 == 0) {
                row_top[r] = top - kTopBits;
                row_inv[r] = 1.0f / l;
                row_limit[r] = limit;
            }
        }
        __syncthreads();
        if (t < len) {
            const float* from = a.scores + (row0 + first) * a.scores_stride + t;
#pragma unroll 8
            for (int r = 0; r < rows; ++r) {
                const float p = __builtin_amdgcn_exp2f(from[r * a.scores_stride] - row_top[r]) * row_inv[r];
                sum += t < row_limit[r] ? p : 0.0f;      // (by its place: a row that is no number would give NaN also to what it does not see)
            }
        }
    }
    if ((uint32_t)block < (uint32_t)c.blocks) a.weights[(s * c.kv_heads + kvh) * a.weights_stride + t] += sum;
}

struct Plan {
    int DP, MT;
    int64_t chunks;
    int part_len, parts;
};

Plan plan_of(const mnnq_kv_cache& c, int64_t tokens, int heads, int64_t bound)
{
    Plan p;
    p.DP = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
    const int64_t rows = heads / c.kv_heads * tokens;
    p.MT = rows > 16 ? 2 : 1;
    p.chunks = (rows + 16 * p.MT - 1) / (16 * p.MT);
    const int64_t base = c.sequences * c.kv_heads * p.chunks;
    // One sequence: a workgroup per CU, of 128 tokens at least.  Several, of lengths that only the device knows: five per CU, so that
    // what the short ones leave idle is little, of 256 tokens at least (256 wide, where a CU holds one: one).  Measured in us, 256 / 512 /
    // 768 workgroups: 16384 tokens of 8 key heads 13.9 / 14.8 / 14.8, 131072 of 4 33.3 / 33.6 / 34.0; 4 sequences of 8000, 256 wide,
    // 21.4 / 28.3 / 28.4.  768 / 1280 / 2048: 32 ragged sequences of up to 6045 49.8 / 45.0 / 59.2, 24 of up to 8000 54.4 / 47.6 / 47.9,
    // 64 of up to 4000, 4 key heads, 37.7 / 34.3 / 45.3, 8 of 8000 32.7 / 32.5 / 35.4.  (Parts sized on the device from the lengths
    // themselves: 45.5, 45.5, 33.8, 35.3, and 1.5 more for one sequence: its chain is longer.)  Least tokens 128 / 256: 1001 tokens of 4
    // key heads 8.4 / 9.5; 8 sequences with weights 19.8 / 18.0.
    const int64_t most = (c.sequences > 1 && p.DP < 256 ? 1280 : 256) / base, least = c.sequences > 1 ? 256 : 128;
    const int64_t want = most > 0 ? most : 1;
    int64_t part = (bound + want - 1) / want;
    if (part < least) part = least;
    // One part, without the second kernel: up to 512 tokens (300 tokens 7.7 against 8.6 us), and two workgroups per CU that are not
    // long (64 sequences of 1000 tokens, 8 key heads, 28.9 against 35.7).
    if (bound <= 512 || (base >= 512 && bound <= 2048)) part = bound;
    const int64_t whole = kWaves * kStep;
    part = (part + whole - 1) / whole * whole;
    if (part * kMaxParts < bound) part = (bound + kMaxParts * whole - 1) / (kMaxParts * whole) * whole;
    p.part_len = (int)part;
    p.parts = (int)((bound + part - 1) / part);
    return p;
}

// Where the workspace's arrays begin, and its size.
struct Space {
    size_t stats, scores, total;
};

Space space_of(const mnnq_kv_cache& c, const Plan& p, int64_t rows, int64_t bound, bool weights)
{
    const auto round16 = [](size_t n) { return (n + 15) / 16 * 16; };
    const size_t all = (size_t)(c.sequences * c.kv_heads * rows);
    Space s{0, 0, 0};
    s.stats = p.parts > 1 ? all * p.parts * p.DP * sizeof(float) : 0;
    s.scores = s.stats + (p.parts > 1 || weights ? round16(all * p.parts * sizeof(float2)) : 0);
    s.total = s.scores + (weights ? all * ((bound + kStep - 1) / kStep * kStep) * sizeof(float) : 0);
    return s;
}

template <int DP, int KF, int VF>
void launch_tiles(const DecodeArgs& a, const Plan& p, hipStream_t st)
{
    const dim3 grid((unsigned)p.parts, (unsigned)(a.c.kv_heads * p.chunks), (unsigned)a.c.sequences);
    const int32_t* table = a.c.block_table;
    const float *kr = a.c.k_range, *vr = a.c.v_range;
    if (p.MT == 1) decode_kernel<DP, KF, VF, 1><<<grid, 64 * kWaves, 0, st>>>(a, table, kr, vr);
    else decode_kernel<DP, KF, VF, 2><<<grid, 64 * kWaves, 0, st>>>(a, table, kr, vr);
}

template <int DP>
int launch_width(const DecodeArgs& a, const Plan& p, hipStream_t st)
{
    const bool k8 = a.c.k_form == MNNQ_KV_FP8, v8 = a.c.v_form == MNNQ_KV_FP8;
    if (k8 && v8) launch_tiles<DP, MNNQ_KV_FP8, MNNQ_KV_FP8>(a, p, st);
    else if (k8) launch_tiles<DP, MNNQ_KV_FP8, MNNQ_KV_INT8>(a, p, st);
    else if (v8) launch_tiles<DP, MNNQ_KV_INT8, MNNQ_KV_FP8>(a, p, st);
    else launch_tiles<DP, MNNQ_KV_INT8, MNNQ_KV_INT8>(a, p, st);
    MNNQ_HIP_TRY(hipGetLastError());
    const int64_t joins = p.parts > 1 ? a.rows : 0, given = a.weights ? (a.bound + kJoinThreads - 1) / kJoinThreads : 0;
    if (joins + given > 0) {
        join_kernel<DP><<<dim3((unsigned)(joins + given), (unsigned)a.c.kv_heads, (unsigned)a.c.sequences), kJoinThreads, 0, st>>>(a);
        MNNQ_HIP_TRY(hipGetLastError());
    }
    return MNNQ_OK;
}

}  // namespace

size_t attn_decode_ws_bytes(const mnnq_kv_cache& c, int64_t tokens, int heads, int64_t bound, bool weights)
{
    return space_of(c, plan_of(c, tokens, heads, bound), heads / c.kv_heads * tokens, bound, weights).total;
}

int launch_attn_decode(const mnnq_kv_cache& c, bool bf16, int64_t tokens, int heads, int64_t bound, float scale,
                       const Rows& q, const Rows& out, float* weights, int64_t weights_stride, void* workspace,
                       hipStream_t st)
{
    const Plan p = plan_of(c, tokens, heads, bound);
    DecodeArgs a{};
    a.c = c;
    a.q = q;
    a.out = out;
    a.weights = weights;
    a.weights_stride = weights_stride;
    a.tokens = tokens;
    a.bound = (int)bound;
    a.part_len = p.part_len;
    a.parts = p.parts;
    a.scores_stride = (bound + kStep - 1) / kStep * kStep;
    a.group = heads / c.kv_heads;
    a.rows = (int)(a.group * tokens);
    a.scale_log2 = scale * kLog2e;
    a.bf16 = bf16;
    const Space sp = space_of(c, p, a.rows, bound, weights != nullptr);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.means = p.parts > 1 ? reinterpret_cast<float*>(ws) : nullptr;
    a.stats = p.parts > 1 || weights ? reinterpret_cast<float2*>(ws + sp.stats) : nullptr;
    a.scores = weights ? reinterpret_cast<float*>(ws + sp.scores) : nullptr;
    return p.DP == 64 ? launch_width<64>(a, p, st) : p.DP == 128 ? launch_width<128>(a, p, st) : launch_width<256>(a, p, st);
}

}  // namespace mnnq
