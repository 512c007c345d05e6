// Causal attention over packed prompts (mnnq_attn_prefill).
//
// A wave owns 32 queries of one head, a workgroup of NW waves 32 NW consecutive ones; keys and values come in tiles of 64 tokens
// through LDS.  S^T = K Q^T and O^T = V^T P^T on the 32 x 32 x 16 matrix instructions: a query is a column, so its statistics
// belong to two lanes (l, l + 32) and the scores that a lane holds of it are the probabilities that the second product wants of that
// lane - tokens 4 h + {0..3} and 8 + 4 h + {0..3} of every 16, h = l / 32, an order that V's transposing LDS reads follow.
#include "mnnq_attn.h"
#include "mnnq_forms.h"

namespace mnnq {

namespace {

#define MNNQ_LDS(p) ((__attribute__((address_space(3))) void*)(p))

constexpr int kTile = 64;                        // keys of a tile
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -3.402823466e38f;
constexpr int kOutOfRange = 0x7ffffff0;          // a byte offset beyond every tile: loads give 0

struct PrefillArgs {
    Rows q, k, v, out;
    const int32_t* q_start;
    const int32_t* k_start;
    int64_t sequences, q_tokens, k_tokens, tiles;
    int heads, kv_heads, D;
    float scale_log2;
};

template <bool BF16>
struct Type;
template <>
struct Type<true> {
    typedef bf8v V8;
    static __device__ __forceinline__ f16v mfma(V8 a, V8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static constexpr float kLift = 0.0f;
};
template <>
struct Type<false> {
    typedef half8v V8;
    static __device__ __forceinline__ f16v mfma(V8 a, V8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static constexpr float kLift = 6.0f;         // probabilities up to 2^14 (with kSlack) instead of 2^8: halves reach further down
};
constexpr float kSlack = 8.0f;                   // the running maximum follows when it is 2^8 behind

typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));

// 16 bytes per lane from base + off, zeros where that is not below `bytes`, to at + 16 lane.
__device__ __forceinline__ void load_to_lds(const void* base, int64_t bytes, uint8_t* at, int off)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(base, bytes), MNNQ_LDS(at), 16, off, 0, 0, 0);
}

// Whether a tile of V holds an infinity or a NaN (the same answer in all lanes of the wave).
template <int DP, bool BF16>
__device__ __forceinline__ bool holds_no_number(const uint8_t* tile, int lane)
{
    typedef unsigned short us2v __attribute__((ext_vector_type(2)));
    us2v top = {0, 0};
#pragma unroll 4
    for (int i = 0; i < kTile * DP * 2 / 1024; ++i) {
        const u4v w = *reinterpret_cast<const u4v*>(tile + (i * 64 + lane) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(us2v, w[j] & 0x7fff7fffu));
    }
    constexpr unsigned short kFirst = BF16 ? 0x7f80 : 0x7c00;       // the infinity's bits
    return __ballot(top.x >= kFirst || top.y >= kFirst) != 0;
}

template <int DP, bool BF16, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 2 : 1) void prefill_kernel(PrefillArgs a)
{
    using T = Type<BF16>;
    typedef typename T::V8 V8;
    constexpr int BM = 32 * NW;
    constexpr int CH = DP / 8;                   // 16-byte units of a row
    constexpr int kTileBytes = kTile * DP * 2;
    constexpr int kLoads = kTileBytes / 1024 / NW;
    extern __shared__ __align__(16) uint8_t lds[];   // K0 K1 V0 V1

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    // tile of queries and head
    const int64_t tile_id = a.tiles - 1 - blockIdx.x / a.heads;
    const int head = blockIdx.x % a.heads, kvh = head / (a.heads / a.kv_heads);
    int64_t s = 0;
    {   // sequence s owns the tiles from q_start[s] / BM + s on: n queries fill at most n / BM + 1
        int64_t lo = 0, hi = a.sequences - 1;
        while (lo < hi) {
            const int64_t mid = (lo + hi + 1) >> 1;
            const int64_t at = a.q_start[mid], in = at < 0 ? 0 : at > a.q_tokens ? a.q_tokens : at;
            if (in / BM + mid <= tile_id) lo = mid;
            else hi = mid - 1;
        }
        s = lo;
    }
    const Span qs = span_of(a.q_start, s, a.q_tokens), ks = span_of(a.k_start, s, a.k_tokens);
    const int64_t q0 = (tile_id - (qs.begin / BM + s)) * BM;
    if (q0 < 0 || q0 >= qs.count) return;
    const int64_t shift = ks.count - qs.count;   // query i sees the keys up to i + shift
    const int64_t q_end = q0 + BM < qs.count ? q0 + BM : qs.count;
    int64_t n_keys = q_end + shift;              // seen by the last query here
    n_keys = n_keys < 0 ? 0 : n_keys;
    const int n_tiles = (int)((n_keys + kTile - 1) / kTile);
    const int64_t mine = q0 + wave * 32 + col;   // this lane's query
    const bool there = mine < qs.count;
    const int64_t limit = there ? mine + shift + 1 : 0;      // keys below it are seen
    const int64_t wave_low = q0 + wave * 32 + shift + 1;     // seen by all queries of the wave
    const int64_t wave_high = q0 + wave * 32 + 32 + shift;   // by the last one

    // queries
    V8 qf[DP / 16];
    {
        const uint16_t* src = a.q.data + (qs.begin + (there ? mine : q0)) * a.q.token + head * a.q.head + 8 * half;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            u4v w = {0, 0, 0, 0};
            if (there && 16 * i + 8 * half < a.D) w = *reinterpret_cast<const u4v*>(src + 16 * i);
            qf[i] = __builtin_bit_cast(V8, w);
        }
    }

    // Direct loads: unit u of a tile's row lies at place u ^ (row's pattern), chosen for each operand so that the lanes which an
    // LDS read serves together touch every bank once.
    auto k_pattern = [](int row) { return DP == 64 ? (row >> 1) & 7 : row & 15; };
    auto v_pattern = [](int row) { return DP == 64 ? ((row >> 1) & 1) << 2 : (row & 3) << 2; };
    const uint16_t* k_base = a.k.data + ks.begin * a.k.token + kvh * a.k.head;
    const uint16_t* v_base = a.v.data + ks.begin * a.v.token + kvh * a.v.head;
    int k_off[kLoads], v_off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int unit = (wave * kLoads + i) * 64 + lane, row = unit / CH, at = unit % CH;
        const int ku = at ^ k_pattern(row), vu = at ^ v_pattern(row);
        k_off[i] = ku * 8 < a.D ? (int)(row * a.k.token + ku * 8) * 2 : kOutOfRange;
        v_off[i] = vu * 8 < a.D ? (int)(row * a.v.token + vu * 8) * 2 : kOutOfRange;
    }
    auto tile_bytes = [&](int64_t token, int64_t first) {
        const int64_t rows = ks.count - first < kTile ? ks.count - first : kTile;
        return ((rows - 1) * token + a.D) * 2;
    };
    auto issue = [&](int t, int slot) {
        const int64_t first = (int64_t)t * kTile;
        const uint16_t* kp = k_base + first * a.k.token;
        const uint16_t* vp = v_base + first * a.v.token;
        const int64_t kn = tile_bytes(a.k.token, first), vn = tile_bytes(a.v.token, first);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            load_to_lds(kp, kn, lds + slot * kTileBytes + (wave * kLoads + i) * 1024, k_off[i]);
            load_to_lds(vp, vn, lds + (2 + slot) * kTileBytes + (wave * kLoads + i) * 1024, v_off[i]);
        }
    };

    f16v o[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] = f16v{};
    float mx = kLowest, l = 0.0f;                // mx: of the scores times scale_log2; l: of this lane's tokens

    if (n_tiles > 0) issue(0, 0);
    for (int t = 0; t < n_tiles; ++t) {
        const int slot = t & 1;
        __builtin_amdgcn_s_waitcnt(0x0070);      // vmcnt(0) lgkmcnt(0): the tile is here, the one before is read
        __builtin_amdgcn_s_barrier();
        if (t + 1 < n_tiles) issue(t + 1, slot ^ 1);
        const int64_t first = (int64_t)t * kTile;
        if (first >= wave_high) continue;        // no query of this wave sees the tile
        const uint8_t* kt = lds + slot * kTileBytes;
        const uint8_t* vt = lds + (2 + slot) * kTileBytes;
        f16v sc[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sc[j] = f16v{};
            const int row = 32 * j + col;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                const V8 kf = *reinterpret_cast<const V8*>(kt + row * DP * 2 + (((2 * i + half) ^ k_pattern(row)) << 4));
                sc[j] = T::mfma(kf, qf[i], sc[j]);
            }
        }
        const bool masked = first + kTile > wave_low;
        if (masked) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (first + 32 * j + 8 * (e / 4) + 4 * half + e % 4 >= limit) sc[j][e] = -__builtin_inff();
        }
        float top = sc[0][0];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[j][e]);
        top = fmaxf(top, __shfl_xor(top, 32)) * a.scale_log2;
        // the maximum follows only when it is far behind: probabilities stay below 2^kSlack
        if (__ballot(top > mx + kSlack)) {
            const float now = fmaxf(mx, top);
            const float down = __builtin_amdgcn_exp2f(mx - now);
            mx = now;
            l *= down;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) o[i] *= down;
        }
        const float less = T::kLift - mx;
        V8 pf[4];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                u4v w;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j][e + 2 * x], a.scale_log2, less));
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j][e + 2 * x + 1], a.scale_log2, less));
                    l += p0;
                    l += p1;
                    w[x] = pack16(p0, p1, BF16);
                }
                pf[2 * j + e / 8] = __builtin_bit_cast(V8, w);
            }
        // four tokens of a row of V^T per read: the 16 lanes of a group address 4 tokens x 16 values
        auto read_v = [&](int ks16, int i) {
            const int row = 16 * ks16 + 4 * half + ((lane & 15) >> 2);
            const int unit = 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            const uint8_t* at = vt + row * DP * 2 + ((unit ^ v_pattern(row)) << 4) + (lane & 1) * 8;
            const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v*)at);
            const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v*)(at + 8 * DP * 2));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if (masked && holds_no_number<DP, BF16>(vt, lane)) {
            // 0 * inf: a product over all keys would carry what a query must not see into its row.  The numbers first; then the
            // others token by token, and only the columns that see the token take the result.
            constexpr short kFirst = BF16 ? 0x7f80 : 0x7c00;
#pragma unroll
            for (int ks16 = 0; ks16 < 4; ++ks16)
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    s8v x = read_v(ks16, i);
                    x = (x & 0x7fff) >= kFirst ? 0 : x;
                    o[i] = T::mfma(__builtin_bit_cast(V8, x), pf[ks16], o[i]);
                }
#pragma nounroll
            for (int j = 0; j < kTile; ++j) {
                const int e = (j & 3) + 4 * ((j >> 3) & 1);
                const bool seen = first + j < limit;
                V8 pj = pf[0];
                pj = j >= 16 ? pf[1] : pj;
                pj = j >= 32 ? pf[2] : pj;
                pj = j >= 48 ? pf[3] : pj;
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    s8v one = read_v(j >> 4, i);
                    one = (one & 0x7fff) >= kFirst ? one : 0;
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        if (x != e || half != ((j >> 2) & 1)) one[x] = 0;
                    const f16v with = T::mfma(__builtin_bit_cast(V8, one), pj, o[i]);
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[i][x] = seen ? with[x] : o[i][x];
                }
            }
            continue;
        }
#pragma unroll
        for (int ks16 = 0; ks16 < 4; ++ks16)
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) o[i] = T::mfma(__builtin_bit_cast(V8, read_v(ks16, i)), pf[ks16], o[i]);
    }

    l += __shfl_xor(l, 32);
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    if (!there) return;
    uint16_t* to = a.out.data + (qs.begin + mine) * a.out.token + head * a.out.head + 4 * half;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int d = 32 * i + 2 * e;
            if (d < a.D) {
                const u2v w = {pack16(o[i][e] * inv, o[i][e + 1] * inv, BF16), pack16(o[i][e + 2] * inv, o[i][e + 3] * inv, BF16)};
                *reinterpret_cast<u2v*>(to + d) = w;
            }
        }
}

template <int DP, bool BF16, int NW>
int launch_waves(PrefillArgs& a, hipStream_t st)
{
    constexpr size_t kLds = 4 * (size_t)kTile * DP * 2;
    static thread_local int allowed = -1;
    if (int e = allow_large_lds(prefill_kernel<DP, BF16, NW>, kLds, allowed)) return e;
    a.tiles = a.q_tokens / (32 * NW) + a.sequences;
    prefill_kernel<DP, BF16, NW><<<dim3((unsigned)(a.tiles * a.heads)), 64 * NW, kLds, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    return MNNQ_OK;
}

template <int DP, bool BF16>
int launch_type(PrefillArgs& a, hipStream_t st)
{
    return launch_waves<DP, BF16, 4>(a, st);
}

template <int DP>
int launch_width(bool bf16, PrefillArgs& a, hipStream_t st)
{
    return bf16 ? launch_type<DP, true>(a, st) : launch_type<DP, false>(a, st);
}

}  // namespace

int launch_attn_prefill(bool bf16, int64_t sequences, const int32_t* q_start, const int32_t* k_start, int64_t q_tokens,
                        int64_t k_tokens, int heads, int kv_heads, int head_dim, float scale, const Rows& q, const Rows& k,
                        const Rows& v, const Rows& out, hipStream_t st)
{
    PrefillArgs a{q, k, v, out, q_start, k_start, sequences, q_tokens, k_tokens, 0, heads, kv_heads, head_dim, scale * kLog2e};
    return head_dim <= 64 ? launch_width<64>(bf16, a, st)
         : head_dim <= 128 ? launch_width<128>(bf16, a, st) : launch_width<256>(bf16, a, st);
}

}  // namespace mnnq
