// Attention of one or a few tokens over the 8-bit cache (mnnq_attn_decode).
//
// For a sequence and key head the queries of the group's heads and of all tokens are the rows of one product, 16 at a
// time: S = K Q^T with tokens down and rows across (v_mfma_f32_16x16x32_f16), O^T = V^T P^T.  Tokens-down puts a row's scores
// into the lanes of one column, where the next product wants its probabilities: the four scores of a lane in two tiles of 16
// tokens are its eight values of P^T as they stand.
//   * Codes become halves exactly; queries become halves scaled by a power of two per row so that the greatest is in
//     [2^14, 2^15) - exact down to 2^-39 of it for bfloat16 too - and ranges, scale and that power are one factor per row and
//     block applied to the fp32 sums.
//   * V's range goes into P: p r / U, U the greatest range so far (the accumulators are rescaled when it grows).  Probabilities
//     are kept under 2^14 instead of 1 so that a half holds them down to 2^-38.
// A wave takes 32 tokens at a time, with the codes of its next 32 in flight; four waves of a workgroup share a part of the
// sequence and join through LDS, the parts are joined by a second kernel.
#include "mnnq_attn.h"

namespace mnnq {

namespace {

constexpr int kWaves = 4;
constexpr int kStep = 32;                        // tokens of a wave's step
constexpr float kTopBits = 13.0f;                // probabilities are p 2^13 where the running maximum is the row's
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -3.402823466e38f;

struct DecodeArgs {
    mnnq_kv_cache c;
    Rows q, out;
    float* part;                                 // partial results, NULL with one part
    float* scores;                               // [sequences, heads, tokens, bound] where weights are asked for
    int64_t tokens, bound, part_len, parts;
    int heads, group, rows;                      // rows: group * tokens
    float scale_log2;
    bool bf16;
};

// Partial result of a part and row: DP sums, then the maximum and the sum of the probabilities.
__host__ __device__ inline int64_t part_floats(int DP) { return DP + 2; }

template <int DP, int KF, int VF, int MT>
__global__ __launch_bounds__(64 * kWaves) void decode_kernel(DecodeArgs a, const int32_t* __restrict__ tables,
                                                               const float* __restrict__ k_ranges,
                                                               const float* __restrict__ v_ranges)
{
    constexpr int KC = DP / 64;                  // 16-byte pieces of a K row per lane
    constexpr int VB = DP / 16;                  // bytes of a V row per lane
    constexpr int VW = VB / 4;
    constexpr int ND = DP / 16;                  // matrix instructions of O^T per row tile
    constexpr int DH = DP < 128 ? DP : 128;      // values of a row that the waves join at a time
    __shared__ __align__(16) float red[kWaves][16 * (DH + 4)];
    __shared__ float red_m[kWaves][16], red_l[kWaves][16];

    const mnnq_kv_cache& c = a.c;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int D = c.head_dim, B = c.block_tokens;
    const int64_t s = blockIdx.z;
    const int kvh = blockIdx.y % c.kv_heads, row0 = (blockIdx.y / c.kv_heads) * 16 * MT;
    int64_t len = c.lengths[s];
    len = len < 0 ? 0 : len > a.bound ? a.bound : len;
    const int64_t p0 = blockIdx.x * a.part_len;
    if (p0 >= len && !(p0 == 0 && a.parts == 1)) return;        // (one part: rows of zeros are stored)
    const int64_t p1 = p0 + a.part_len < len ? p0 + a.part_len : len;
    const int32_t* table = tables + s * c.table_blocks;
    const int block_shift = __builtin_ctz(B);

    // queries, their power of two, and how far each row sees
    half8v qf[MT][2 * KC];
    float factor[MT];
    int64_t limit[MT];
    int64_t lowest_limit = len;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int r = row0 + m * 16 + col;
        const bool there = r < a.rows;
        const int t = there ? r / a.group : 0;
        const int h = kvh * a.group + (there ? r - t * a.group : 0);
        limit[m] = there ? len - a.tokens + t + 1 : 0;
        const uint16_t* src = a.q.data + (s * a.tokens + t) * a.q.token + h * a.q.head;
        u4v raw[2 * KC];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2 * KC; ++i) {
            const int d = 64 * (i / 2) + 16 * g + 8 * (i & 1);
            raw[i] = there && d < D ? *reinterpret_cast<const u4v*>(src + d) : u4v{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max(top, max(raw[i][j] & 0x7fffu, (raw[i][j] >> 16) & 0x7fffu));
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        // exponent e with 2^e <= greatest < 2^(e+1)
        const int e = (int)(__float_as_uint(value16(top, a.bf16)) >> 23) - 127;
        const int up = max(-126, min(126, 14 - e));
        const float mul = __uint_as_float((uint32_t)(up + 127) << 23);
        factor[m] = a.scale_log2 * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
        for (int i = 0; i < 2 * KC; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                qf[m][i][2 * j] = (_Float16)(value16(raw[i][j] & 0xffffu, a.bf16) * mul);
                qf[m][i][2 * j + 1] = (_Float16)(value16(raw[i][j] >> 16, a.bf16) * mul);
            }
        }
    }
    lowest_limit = len - a.tokens + 1;           // tokens below it are seen by every row

    f4v o[MT][ND];
    float mx[MT], l[MT];
    float unit = 0.0f;                           // U
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        mx[m] = kLowest;
        l[m] = 0.0f;
#pragma unroll
        for (int i = 0; i < ND; ++i) o[m][i] = f4v{0, 0, 0, 0};
    }

    struct Codes {
        u4v k[2][KC];
        uint32_t v[8][VW];
        int64_t block[2];
    };
    // block of the 16 tokens from p on; -1: none of ours
    auto block_at = [&](int64_t p) -> int64_t {
        if (p >= p1) return -1;
        const int64_t b = __builtin_amdgcn_readfirstlane(table[p >> block_shift]);
        return b >= 0 && b < c.blocks ? b : -1;
    };
    auto load = [&](int64_t p, Codes& x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t at = p + 16 * i;
            x.block[i] = block_at(at);
            const int64_t block = x.block[i] < 0 ? 0 : x.block[i];
            const int64_t base = ((block * c.kv_heads + kvh) * B + (at & (B - 1))) * D;
            const uint8_t* kp = static_cast<const uint8_t*>(c.k_codes) + base + col * D + 16 * g;
            const uint8_t* vp = static_cast<const uint8_t*>(c.v_codes) + base + 4 * g * D + VB * col;
#pragma unroll
            for (int j = 0; j < KC; ++j)
                x.k[i][j] = x.block[i] >= 0 && 64 * j + 16 * g < D ? *reinterpret_cast<const u4v*>(kp + 64 * j)
                                                                   : u4v{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in = x.block[i] >= 0 && VB * col < D;
                if (VW == 1) {
                    x.v[4 * i + j][0] = in ? *reinterpret_cast<const uint32_t*>(vp + j * D) : 0;
                } else if (VW == 2) {
                    const u2v w = in ? *reinterpret_cast<const u2v*>(vp + j * D) : u2v{0, 0};
                    x.v[4 * i + j][0] = w.x, x.v[4 * i + j][1 % VW] = w.y;
                } else {
                    const u4v w = in ? *reinterpret_cast<const u4v*>(vp + j * D) : u4v{0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.v[4 * i + j][e % VW] = w[e];
                }
            }
        }
    };

    Codes next;
    int64_t p = p0 + wave * kStep;
    if (p < p1) load(p, next);
    for (; p < p1; p += kWaves * kStep) {
        Codes x = next;
        if (p + kWaves * kStep < p1) load(p + kWaves * kStep, next);
        float kr[2], vr[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t at = (x.block[i] < 0 ? 0 : x.block[i]) * c.kv_heads + kvh;
            kr[i] = x.block[i] < 0 ? 0.0f : k_ranges[at] * (1.0f / code_top<KF>());
            vr[i] = x.block[i] < 0 ? 0.0f : v_ranges[at];
        }
        // scores
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
        const bool masked = p + kStep > lowest_limit || p + kStep > p1 || x.block[0] < 0 || x.block[1] < 0;
        // (a range that is not finite is that of undefined values, which only rows that see them may get)
        const float vmax = fmaxf(vr[0] < __builtin_inff() ? vr[0] : 0.0f, vr[1] < __builtin_inff() ? vr[1] : 0.0f);
        if (vmax > unit) {
            const float down = unit / fmaxf(vmax, 1.17549435e-38f);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < ND; ++i) o[m][i] *= down;
            unit = fmaxf(vmax, 1.17549435e-38f);
        }
        const float inv_unit = unit > 0.0f ? 1.0f / unit : 0.0f;
        half8v pf[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float top = kLowest;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float f = factor[m] * kr[i];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sc[m][i][e] *= f;
                    if (masked) {
                        const int64_t t = p + 16 * i + 4 * g + e;
                        if (t >= limit[m] || t >= p1 || x.block[i] < 0) sc[m][i][e] = -__builtin_inff();
                    }
                    top = fmaxf(top, sc[m][i][e]);
                }
            }
            if (a.scores && row0 + m * 16 + col < a.rows) {
                const int r = row0 + m * 16 + col;
                float* to = a.scores + ((s * c.kv_heads + kvh) * a.rows + r) * a.bound;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t t = p + 16 * i + 4 * g + e;
                        if (t < p1) to[t] = sc[m][i][e];
                    }
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(mx[m], top);
            if (__ballot(now > mx[m])) {
                const float down = __builtin_amdgcn_exp2f(mx[m] - now);
                mx[m] = now;
                l[m] *= down;
#pragma unroll
                for (int i = 0; i < ND; ++i) o[m][i] *= down;
            }
            float pr[8];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    pr[4 * i + e] = __builtin_amdgcn_exp2f(sc[m][i][e] - mx[m] + kTopBits);
                    l[m] += pr[4 * i + e];
                    pr[4 * i + e] *= vr[i] * inv_unit;
                    if (masked && sc[m][i][e] == -__builtin_inff()) pr[4 * i + e] = 0.0f;
                }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t two = pack16(pr[2 * e], pr[2 * e + 1], false);
                const half2v h = __builtin_bit_cast(half2v, two);
                pf[m][2 * e] = h.x, pf[m][2 * e + 1] = h.y;
            }
        }
        // what lies behind the last token may be anything, NaN codes among it
        if (p + kStep > p1) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (p + 16 * (j / 4) + 4 * g + (j & 3) >= p1)
#pragma unroll
                    for (int e = 0; e < VW; ++e) x.v[j][e] = 0;
        }
        // V: bytes of four tokens of a lane turned to four tokens of a byte
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            uint32_t t[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t a0 = x.v[4 * i][w], a1 = x.v[4 * i + 1][w], a2 = x.v[4 * i + 2][w], a3 = x.v[4 * i + 3][w];
                const uint32_t l01 = __builtin_amdgcn_perm(a1, a0, 0x05010400u), h01 = __builtin_amdgcn_perm(a1, a0, 0x07030602u);
                const uint32_t l23 = __builtin_amdgcn_perm(a3, a2, 0x05010400u), h23 = __builtin_amdgcn_perm(a3, a2, 0x07030602u);
                t[i][0] = __builtin_amdgcn_perm(l23, l01, 0x05040100u);
                t[i][1] = __builtin_amdgcn_perm(l23, l01, 0x07060302u);
                t[i][2] = __builtin_amdgcn_perm(h23, h01, 0x05040100u);
                t[i][3] = __builtin_amdgcn_perm(h23, h01, 0x07060302u);
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const half8v vf = codes_to_half8<VF>(t[0][b], t[1][b]);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    o[m][4 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[m], o[m][4 * w + b], 0, 0, 0);
            }
        }
    }

    // Join the waves: lane (g, col) holds of row col the values d = VB (4 g + v) + i, v = 0..3.
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float sum = l[m];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (m > 0) __syncthreads();
        if (g == 0) red_m[wave][col] = mx[m];
        if (g == 0) red_l[wave][col] = sum;
        __syncthreads();
        float top = red_m[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, red_m[w][col]);
        const float f = __builtin_amdgcn_exp2f(mx[m] - top) * unit * (1.0f / code_top<VF>());
        // thread: row tid / 16, DH / 16 values at a time
        const int row = threadIdx.x >> 4;
        const int r = row0 + m * 16 + row;
        float rt = red_m[0][row];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) rt = fmaxf(rt, red_m[w][row]);
        float rl = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) rl += red_l[w][row] * __builtin_amdgcn_exp2f(red_m[w][row] - rt);
        const float inv = rl > 0.0f || rl != rl ? 1.0f / rl : 0.0f;
        const int64_t stat = ((s * c.kv_heads + kvh) * a.rows + r) * a.parts + blockIdx.x;
        const int t = r / a.group, h = kvh * a.group + r - t * a.group;
        if (a.part && r < a.rows && (threadIdx.x & 15) == 0) {
            a.part[stat * part_floats(DP) + DP] = rt;
            a.part[stat * part_floats(DP) + DP + 1] = rl;
        }
#pragma unroll
        for (int first = 0; first < DP; first += DH) {
            if (first > 0) __syncthreads();
            if (DP == DH || (4 * g * VB) / DH == first / DH)
#pragma unroll
                for (int i = 0; i < ND; ++i)
#pragma unroll
                    for (int v = 0; v < 4; ++v) red[wave][col * (DH + 4) + VB * (4 * g + v) + i - first] = o[m][i][v] * f;
            __syncthreads();
            const int d0 = (threadIdx.x & 15) * (DH / 16);
            float val[DH / 16];
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) {
                val[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) val[i] += red[w][row * (DH + 4) + d0 + i];
            }
            if (r >= a.rows) continue;
            // (head_dim is a multiple of 16, so of the values of a thread)
            if (first + d0 < D) {
                if (a.parts > 1) {
                    float* to = a.part + stat * part_floats(DP) + first + d0;
#pragma unroll
                    for (int i = 0; i < DH / 16; ++i) to[i] = val[i];
                } else {
                    uint16_t* to = a.out.data + (s * a.tokens + t) * a.out.token + h * a.out.head + first + d0;
#pragma unroll
                    for (int i = 0; i < DH / 16; i += 2)
                        *reinterpret_cast<uint32_t*>(to + i) = pack16(val[i] * inv, val[i + 1] * inv, a.bf16);
                }
            }
        }
    }
}

// Joins the parts of a row: one workgroup per row, a thread per two values and every fourth... of the parts.
template <int DP>
__global__ __launch_bounds__(256) void join_kernel(DecodeArgs a)
{
    constexpr int PER = DP / 2;                  // threads of a part: two values each
    constexpr int TEAMS = 256 / PER;
    __shared__ float red[TEAMS][DP];
    const mnnq_kv_cache& c = a.c;
    const int tid = threadIdx.x, team = tid / PER, d = (tid % PER) * 2;
    const int r = blockIdx.x, kvh = blockIdx.y;
    const int64_t s = blockIdx.z;
    int64_t len = c.lengths[s];
    len = len < 0 ? 0 : len > a.bound ? a.bound : len;
    const int n = (int)((len + a.part_len - 1) / a.part_len);
    const float* part = a.part + ((s * c.kv_heads + kvh) * a.rows + r) * a.parts * part_floats(DP);
    float top = kLowest;
    for (int i = 0; i < n; ++i) top = fmaxf(top, part[i * part_floats(DP) + DP]);
    float l = 0.0f, v0 = 0.0f, v1 = 0.0f;
    for (int i = 0; i < n; ++i) {
        const float* p = part + i * part_floats(DP);
        const float f = __builtin_amdgcn_exp2f(p[DP] - top);
        l += p[DP + 1] * f;
        if (i % TEAMS == team) {
            v0 += p[d] * f;
            v1 += p[d + 1] * f;
        }
    }
    red[team][d] = v0, red[team][d + 1] = v1;
    __syncthreads();
    if (team == 0 && d < c.head_dim) {
#pragma unroll
        for (int i = 1; i < TEAMS; ++i) v0 += red[i][d], v1 += red[i][d + 1];
        const int t = r / a.group, h = kvh * a.group + r - t * a.group;
        const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
        uint16_t* to = a.out.data + (s * a.tokens + t) * a.out.token + h * a.out.head;
        *reinterpret_cast<uint32_t*>(to + d) = pack16(v0 * inv, v1 * inv, a.bf16);
    }
}

// Adds the attention given to every token: a thread per token, the rows' maxima and sums from the scores' parts.
__global__ __launch_bounds__(256) void weights_kernel(DecodeArgs a, float* weights, int64_t stride, int DP)
{
    const mnnq_kv_cache& c = a.c;
    const int64_t s = blockIdx.z;
    const int kvh = blockIdx.y;
    int64_t len = c.lengths[s];
    len = len < 0 ? 0 : len > a.bound ? a.bound : len;
    const int64_t t = blockIdx.x * 256 + threadIdx.x;
    if (blockIdx.x * 256 >= len) return;
    const int n = (int)((len + a.part_len - 1) / a.part_len);
    float sum = 0.0f;
    for (int r = 0; r < a.rows; ++r) {
        const int64_t row = (s * c.kv_heads + kvh) * a.rows + r;
        const float* part = a.part + row * a.parts * part_floats(DP);
        float top = kLowest, l = 0.0f;
        for (int i = 0; i < n; ++i) top = fmaxf(top, part[i * part_floats(DP) + DP]);
        for (int i = 0; i < n; ++i) l += part[i * part_floats(DP) + DP + 1] * __builtin_amdgcn_exp2f(part[i * part_floats(DP) + DP] - top);
        if (t < len && !(l <= 0.0f)) sum += __builtin_amdgcn_exp2f(a.scores[row * a.bound + t] - top + kTopBits) / l;
    }
    if (t < len) weights[(s * c.kv_heads + kvh) * stride + t] += sum;
}

struct Plan {
    int DP, MT;
    int64_t chunks, part_len, parts;
};

Plan plan_of(const mnnq_kv_cache& c, int64_t tokens, int heads, int64_t bound, bool weights)
{
    Plan p;
    p.DP = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
    const int64_t rows = heads / c.kv_heads * tokens;
    p.MT = rows > 16 ? 2 : 1;
    p.chunks = (rows + 16 * p.MT - 1) / (16 * p.MT);
    const int64_t base = c.sequences * c.kv_heads * p.chunks;
    const int64_t want = 2048 / base > 1 ? 2048 / base : 1;
    int64_t len = (bound + want - 1) / want;
    len = (len + kWaves * kStep - 1) / (kWaves * kStep) * (kWaves * kStep);
    p.part_len = len;
    p.parts = (bound + len - 1) / len;
    return p;
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

size_t part_bytes(const mnnq_kv_cache& c, const Plan& p, int64_t rows, bool weights)
{
    if (p.parts == 1 && !weights) return 0;
    return round16((size_t)(c.sequences * c.kv_heads * rows * p.parts * part_floats(p.DP)) * 4);
}

template <int DP, int KF, int VF>
void launch_mt(const DecodeArgs& a, const Plan& p, hipStream_t st)
{
    const dim3 grid((unsigned)p.parts, (unsigned)(a.c.kv_heads * p.chunks), (unsigned)a.c.sequences);
    if (p.MT == 1) decode_kernel<DP, KF, VF, 1><<<grid, 64 * kWaves, 0, st>>>(a, a.c.block_table, a.c.k_range, a.c.v_range);
    else decode_kernel<DP, KF, VF, 2><<<grid, 64 * kWaves, 0, st>>>(a, a.c.block_table, a.c.k_range, a.c.v_range);
}

template <int DP>
void launch_forms(const DecodeArgs& a, const Plan& p, hipStream_t st)
{
    const bool k8 = a.c.k_form == MNNQ_KV_FP8, v8 = a.c.v_form == MNNQ_KV_FP8;
    if (k8 && v8) launch_mt<DP, MNNQ_KV_FP8, MNNQ_KV_FP8>(a, p, st);
    else if (k8) launch_mt<DP, MNNQ_KV_FP8, MNNQ_KV_INT8>(a, p, st);
    else if (v8) launch_mt<DP, MNNQ_KV_INT8, MNNQ_KV_FP8>(a, p, st);
    else launch_mt<DP, MNNQ_KV_INT8, MNNQ_KV_INT8>(a, p, st);
}

}  // namespace

size_t attn_decode_ws_bytes(const mnnq_kv_cache& c, int64_t tokens, int heads, int64_t bound, bool weights)
{
    const Plan p = plan_of(c, tokens, heads, bound, weights);
    const int64_t rows = heads / c.kv_heads * tokens;
    return part_bytes(c, p, rows, weights) + (weights ? round16((size_t)(c.sequences * c.kv_heads * rows * bound) * 4) : 0);
}

int launch_attn_decode(const mnnq_kv_cache& c, bool bf16, int64_t tokens, int heads, int64_t bound, float scale,
                       const Rows& q, const Rows& out, float* weights, int64_t weights_stride, void* workspace,
                       hipStream_t st)
{
    const Plan p = plan_of(c, tokens, heads, bound, weights != nullptr);
    DecodeArgs a;
    a.c = c;
    a.q = q;
    a.out = out;
    a.tokens = tokens;
    a.bound = bound;
    a.part_len = p.part_len;
    a.parts = p.parts;
    a.heads = heads;
    a.group = heads / c.kv_heads;
    a.rows = (int)(a.group * tokens);
    a.scale_log2 = scale * kLog2e;
    a.bf16 = bf16;
    a.part = p.parts > 1 || weights ? static_cast<float*>(workspace) : nullptr;
    a.scores = weights ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + part_bytes(c, p, a.rows, true)) : nullptr;
    if (p.DP == 64) launch_forms<64>(a, p, st);
    else if (p.DP == 128) launch_forms<128>(a, p, st);
    else launch_forms<256>(a, p, st);
    MNNQ_HIP_TRY(hipGetLastError());
    if (p.parts > 1) {
        const dim3 grid((unsigned)a.rows, (unsigned)c.kv_heads, (unsigned)c.sequences);
        if (p.DP == 64) join_kernel<64><<<grid, 256, 0, st>>>(a);
        else if (p.DP == 128) join_kernel<128><<<grid, 256, 0, st>>>(a);
        else join_kernel<256><<<grid, 256, 0, st>>>(a);
        MNNQ_HIP_TRY(hipGetLastError());
    }
    if (weights) {
        const dim3 grid((unsigned)((bound + 255) / 256), (unsigned)c.kv_heads, (unsigned)c.sequences);
        weights_kernel<<<grid, 256, 0, st>>>(a, weights, weights_stride, p.DP);
        MNNQ_HIP_TRY(hipGetLastError());
    }
    return MNNQ_OK;
}

}  // namespace mnnq
