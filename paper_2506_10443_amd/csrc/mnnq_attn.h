// Shared parts of the attention calls: what the launchers are given, 16-bit types, codes of the cache.
#pragma once

#include "mnnq_common.h"

namespace mnnq {

// Rows of 16-bit values: distances in elements from one token's, one head's row to the next one's.
struct Rows {
    uint16_t* data;
    int64_t token, head;
};

// A sequence's rows among `total`: what the array of starts says, clamped to the rows that exist.
struct Span {
    int64_t begin, count;
};

int launch_attn_prefill(bool bf16, int64_t sequences, const int32_t* q_start, const int32_t* k_start, int64_t q_tokens,
                        int64_t k_tokens, int heads, int kv_heads, int head_dim, float scale, const Rows& q, const Rows& k,
                        const Rows& v, const Rows& out, hipStream_t st);
int launch_kv_append(const mnnq_kv_cache& c, bool bf16, const int32_t* start, int64_t tokens, const Rows& k, const Rows& v,
                     hipStream_t st);
// bound: the most tokens of a sequence that are looked at.
size_t attn_decode_ws_bytes(const mnnq_kv_cache& c, int64_t tokens, int heads, int64_t bound, bool weights);
int launch_attn_decode(const mnnq_kv_cache& c, bool bf16, int64_t tokens, int heads, int64_t bound, float scale,
                       const Rows& q, const Rows& out, float* weights, int64_t weights_stride, void* workspace,
                       hipStream_t st);
int launch_kv_evict(const mnnq_kv_cache& c, const float* weights, int64_t weights_stride, int64_t keep, int64_t recent,
                    const int32_t* new_table, int64_t new_table_blocks, int32_t* kept, int32_t* new_lengths,
                    float* new_weights, int64_t new_weights_stride, hipStream_t st);

#if defined(__HIPCC__)

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float f2v __attribute__((ext_vector_type(2)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ Span span_of(const int32_t* start, int64_t s, int64_t total)
{
    const int64_t a = start[s], b = start[s + 1];
    const int64_t lo = a < 0 ? 0 : a > total ? total : a, hi = b < lo ? lo : b > total ? total : b;
    return {lo, hi - lo};
}

// Two floats as two 16-bit values of the call's type, rounded to nearest even.
__device__ __forceinline__ uint32_t pack16(float a, float b, bool bf16)
{
    const f2v v = {a, b};
    return bf16 ? __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf2v))
                : __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2v));
}

// The float that 16 bits stand for.
__device__ __forceinline__ float value16(uint32_t bits, bool bf16)
{
    return bf16 ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

template <int FORM>
__device__ constexpr float code_top() { return FORM == MNNQ_KV_FP8 ? 448.0f : 127.0f; }

// Four codes as exact halves.  int8: a byte u under the high byte 0x64 is the half 1024 + u.
template <int FORM>
__device__ __forceinline__ void codes_to_half(uint32_t w, half2v& lo, half2v& hi)
{
    if (FORM == MNNQ_KV_FP8) {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
    } else {
        const uint32_t u = w ^ 0x80808080u;
        const half2v mid = {(_Float16)1152.0f, (_Float16)1152.0f};
        lo = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - mid;
        hi = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - mid;
    }
}

// Eight codes (two dwords) as an operand of the matrix instruction.
template <int FORM>
__device__ __forceinline__ half8v codes_to_half8(uint32_t w0, uint32_t w1)
{
    half2v a, b, c, d;
    codes_to_half<FORM>(w0, a, b);
    codes_to_half<FORM>(w1, c, d);
    return half8v{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// Byte b (0..3) of four dwords as exact halves.
template <int FORM>
__device__ __forceinline__ void byte_to_half(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, int b, half2v& lo, half2v& hi)
{
    if (FORM == MNNQ_KV_FP8) {
        const uint32_t pair = (uint32_t)(0x0c0c0000 | (4 + b) << 8 | b);
        const uint32_t w = __builtin_amdgcn_perm(w1, w0, pair), v = __builtin_amdgcn_perm(w3, w2, pair);
        lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.0f, false);
    } else {
        // (a byte c under a byte of zeros, with the bits of 0x6480 turned over, is the half 1024 + 128 + c)
        const uint32_t pair = (uint32_t)(0x0c000c00 | (4 + b) << 16 | b);
        const half2v mid = {(_Float16)1152.0f, (_Float16)1152.0f};
        lo = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(w1, w0, pair) ^ 0x64806480u) - mid;
        hi = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(w3, w2, pair) ^ 0x64806480u) - mid;
    }
}

// The four codes of a dword as numbers, exact.
template <int FORM>
__device__ __forceinline__ void codes_to_float(uint32_t w, float (&v)[4])
{
    half2v lo, hi;
    codes_to_half<FORM>(w, lo, hi);
    v[0] = (float)lo.x, v[1] = (float)lo.y, v[2] = (float)hi.x, v[3] = (float)hi.y;
}

// The last of 0 .. n - 1 for which `holds`, given that it does for none behind one that it does not for; 0 if for none.  All lanes of a wave
// ask at once, 64 places at a time: one load's latency for up to 64 sequences where a search by halves has six
// (200 prompts of 20 tokens, 12 heads, 34.6 -> 31.5 us; 64 of 64, 28 heads, 32.7 -> 31.6).
template <typename Holds>
__device__ __forceinline__ int64_t last_of(int64_t n, Holds holds)
{
    const int lane = __lane_id();
    int64_t at = 0;
    while (n > 1) {
        const int64_t stride = (n + 63) >> 6, mine = lane * stride;
        const uint64_t yes = __ballot(mine < n && holds(at + (mine < n ? mine : 0))) | 1;
        const int64_t steps = (63 - __builtin_clzll(yes)) * stride;
        at += steps;
        n = n - steps < stride ? n - steps : stride;
    }
    return at;
}

// Four numbers within the codes' range as codes, ties to even.
template <int FORM>
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d)
{
    if (FORM == MNNQ_KV_FP8) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
    }
    // (adding 1.5 * 2^23 rounds to an integer, whose low byte is that of the sum's bits)
    constexpr float kMagic = 12582912.0f;
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b + kMagic), __float_as_uint(a + kMagic), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d + kMagic), __float_as_uint(c + kMagic), 0x04000c0cu);
    return lo | hi;
}

#endif

}  // namespace mnnq
