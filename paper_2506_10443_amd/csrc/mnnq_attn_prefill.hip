// Causal attention over packed prompts (mnnq_attn_prefill).
//
// A wave owns 32 queries of one head, a workgroup of NW waves 32 NW consecutive ones; keys and values come in tiles of 64 tokens
// through LDS.  S^T = K Q^T and O^T = V^T P^T on the 32 x 32 x 16 matrix instructions: a query is a column, so its statistics
// belong to two lanes (l, l + 32) and the scores that a lane holds of it are the probabilities that the second product wants of that
// lane - tokens 4 h + {0..3} and 8 + 4 h + {0..3} of every 16, h = l / 32, an order that V's transposing LDS reads follow.
#include "mnnq_attn.h"
#include "mnnq_forms.h"

#include <type_traits>

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
    static constexpr float kLift = -16.0f;       // probabilities from 2^-16 down: sums of the greatest values stay numbers
    // l + the two values of a dword, which are summed as the second product uses them: rounded.  One instruction in place of two
    // additions (packed prompts of up to 1500 tokens, 28 heads, 64 -> 58 us).
    static __device__ __forceinline__ float add_pair(uint32_t two, float l)
    {
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2v, two), bf2v{(__bf16)1.0f, (__bf16)1.0f}, l, false);
    }
};
template <>
struct Type<false> {
    typedef half8v V8;
    static __device__ __forceinline__ f16v mfma(V8 a, V8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float add_pair(uint32_t two, float l)
    {
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, two), half2v{(_Float16)1.0f, (_Float16)1.0f}, l, false);
    }
    static constexpr float kLift = 6.0f;         // probabilities up to 2^14 (with kSlack) instead of 2^8: halves reach further down
};
constexpr float kSlack = 8.0f;                   // the running maximum follows when it is 2^8 behind

typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));

// All but the youngest N of this wave's direct loads are in LDS; its LDS reads are done; they are, and everybody's.
template <int N = 0>
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

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

// Two transposing reads.  (The compiler would wait in front of them for every direct load in flight, also for those of other tiles;
// pointers that alias nothing else here leave the waits to landed().)
__device__ __forceinline__ s8v read_transposed(const uint8_t* __restrict__ a, const uint8_t* __restrict__ b, const int* __restrict__)
{
    const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v*)a);
    const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v*)b);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Order of a stretch of code: LDS reads, AHEAD of the matrix instructions they feed, EACH behind one, for N / 2 of N.
template <int AHEAD, int EACH, int N>
__device__ __forceinline__ void pace()
{
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (i < N / 2) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
    }
}

// What a workgroup works on: BM queries of a head and the keys they see.
struct Work {
    Span q, k;
    int64_t q0;                                  // first query, in the sequence
    int64_t shift;                               // query i sees the keys up to i + shift
    int head, kvh;
    int tiles, full;                             // tiles of keys that some query sees; that all queries see all of
};

template <int BM>
__device__ __forceinline__ bool find_work(const PrefillArgs& a, Work& w)
{
    // Long rows first.  Workgroup b runs on XCD b % 8: where that fits, the heads that share keys are on one XCD (8192 tokens of 32
    // heads, 8 key heads: 0.28 instead of 1.05 GB past the L2s, in the same time).
    const int64_t tile_id = a.tiles - 1 - blockIdx.x / a.heads;
    w.head = blockIdx.x % a.heads;
    if (a.heads % kXcdCount == 0) w.head = w.head % kXcdCount * (a.heads / kXcdCount) + w.head / kXcdCount;
    w.kvh = w.head / (a.heads / a.kv_heads);
    // Sequence s owns the tiles from q_start[s] / BM + s on: n queries fill at most n / BM + 1.
    const int64_t lo = last_of(a.sequences, [&](int64_t s) {
        const int64_t at = a.q_start[s], in = at < 0 ? 0 : at > a.q_tokens ? a.q_tokens : at;
        return in / BM + s <= tile_id;
    });
    w.q = span_of(a.q_start, lo, a.q_tokens);
    w.k = span_of(a.k_start, lo, a.k_tokens);
    w.q0 = (tile_id - (w.q.begin / BM + lo)) * BM;
    if (w.q0 < 0 || w.q0 >= w.q.count) return false;
    w.shift = w.k.count - w.q.count;
    const int64_t q_end = w.q0 + BM < w.q.count ? w.q0 + BM : w.q.count;
    const int64_t keys = q_end + w.shift < 0 ? 0 : q_end + w.shift;
    w.tiles = (int)((keys + kTile - 1) / kTile);
    const int64_t by_all = w.q0 + w.shift + 1 < 0 ? 0 : (w.q0 + w.shift + 1) / kTile;
    w.full = by_all < w.tiles ? (int)by_all : w.tiles;
    return true;
}

// Place of a row's 16-byte unit u in LDS: u ^ pattern, chosen for each operand so that the lanes which an LDS read serves together
// touch every bank once.
template <int DP>
__device__ __forceinline__ int k_pattern(int row) { return DP == 64 ? (row >> 1) & 7 : row & 15; }
template <int DP>
__device__ __forceinline__ int v_pattern(int row) { return DP == 64 ? ((row >> 1) & 1) << 2 : (row & 3) << 2; }

// Direct loads of tiles of keys or values by WAVES waves, each its own part of the rows.
template <int DP, int WAVES>
struct Loader {
    static constexpr int kLoads = kTile * DP * 2 / 1024 / WAVES;
    const uint16_t* base;
    int64_t token, rows;
    int D, wave;
    int off[kLoads];

    template <typename Pattern>
    __device__ __forceinline__ Loader(const Rows& x, const Span& span, int head, int D, int wave, int lane, Pattern pattern)
        : base(x.data + span.begin * x.token + head * x.head), token(x.token), rows(span.count), D(D), wave(wave)
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int unit = (wave * kLoads + i) * 64 + lane, row = unit / (DP / 8), u = (unit % (DP / 8)) ^ pattern(row);
            off[i] = u * 8 < D ? (int)(row * token + u * 8) * 2 : kOutOfRange;
        }
    }
    __device__ __forceinline__ void load(int t, uint8_t* to) const
    {
        const int64_t first = (int64_t)t * kTile, left = rows - first < kTile ? rows - first : kTile;
        const uint16_t* from = base + first * token;
        const int64_t bytes = ((left - 1) * token + D) * 2;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_to_lds(from, bytes, to + (wave * kLoads + i) * 1024, off[i]);
    }
};

// A wave's 32 queries: lane (half, col) holds of query col the scores of keys 8 i + 4 half + {0..3} of a tile and the results
// d = 8 i + 4 half + {0..3}.  DP: width of a row in LDS, DU: the part of it that products are made of (4096
// tokens, 80 wide, 32 heads: 96 of 128 takes 120 us, all of it 136; 192 wide, 16 heads: 192 of 256 takes 143, all of it 185).
template <int DP, int DU, bool BF16>
struct Queries {
    using T = Type<BF16>;
    typedef typename T::V8 V8;
    int lane, col, half;
    int64_t limit;                               // this lane's query sees the keys below
    float scale;                                 // of the scores, log2
    bool there;
    V8 qf[DU / 16];
    f16v o[DU / 32];
    float mx, l;                                 // maximum of the scores times scale; sum over this lane's keys

    __device__ __forceinline__ Queries(const PrefillArgs& a, const Work& w, int lane, int64_t first)
        : lane(lane), col(lane & 31), half(lane >> 5), scale(a.scale_log2), mx(kLowest), l(0.0f)
    {
        const int64_t mine = first + col;
        there = mine < w.q.count;
        limit = there ? mine + w.shift + 1 : 0;
        const uint16_t* src = a.q.data + (w.q.begin + (there ? mine : 0)) * a.q.token + w.head * a.q.head + 8 * half;
#pragma unroll
        for (int i = 0; i < DU / 16; ++i) {
            u4v x = {0, 0, 0, 0};
            if (there && 16 * i + 8 * half < a.D) x = *reinterpret_cast<const u4v*>(src + 16 * i);
            qf[i] = __builtin_bit_cast(V8, x);
        }
#pragma unroll
        for (int i = 0; i < DU / 32; ++i) o[i] = f16v{};
    }

    // S^T = K Q^T of a tile.
    __device__ __forceinline__ void scores(const uint8_t* kt, f16v (&sc)[2]) const
    {
        V8 kf[2][DU / 16];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < DU / 16; ++i) {
                const int row = 32 * j + col;
                kf[j][i] = *reinterpret_cast<const V8*>(kt + row * DP * 2 + (((2 * i + half) ^ k_pattern<DP>(row)) << 4));
            }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sc[j] = f16v{};
#pragma unroll
            for (int i = 0; i < DU / 16; ++i) sc[j] = T::mfma(kf[j][i], qf[i], sc[j]);
        }
    }

    // Probabilities of the tile that begins with key `first`.
    template <bool MASKED>
    __device__ __forceinline__ void probabilities(f16v (&sc)[2], int64_t first, V8 (&pf)[4])
    {
        if (MASKED) {
            const int left = (int)(limit - first < kTile ? limit - first : kTile);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * j + 8 * (e / 4) + 4 * half + e % 4 >= left) sc[j][e] = -__builtin_inff();
        }
        float top = sc[0][0];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[j][e]);
        const u2v other = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(other[0]), __uint_as_float(other[1])) * scale;
        // the maximum follows only when it is far behind: probabilities stay below 2^kSlack
        if (__ballot(top > mx + kSlack)) {
            const float now = top > mx + kSlack ? top : mx;      // (each row by itself: its bits do not depend on the others)
            const float down = __builtin_amdgcn_exp2f(mx - now);
            mx = now;
            l *= down;
#pragma unroll
            for (int i = 0; i < DU / 32; ++i) o[i] *= down;
        }
        const float less = T::kLift - mx;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                u4v w;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j][e + 2 * x], scale, less));
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j][e + 2 * x + 1], scale, less));
                    w[x] = pack16(p0, p1, BF16);
                    l = T::add_pair(w[x], l);
                }
                pf[2 * j + e / 8] = __builtin_bit_cast(V8, w);
            }
    }

    // Four keys of a row of V^T per read: the 16 lanes of a group address 4 keys x 16 values.
    __device__ __forceinline__ s8v read_v(const uint8_t* vt, int ks16, int i) const
    {
        const int row = 16 * ks16 + 4 * half + ((lane & 15) >> 2);
        const int unit = 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        const uint8_t* at = vt + row * DP * 2 + ((unit ^ v_pattern<DP>(row)) << 4) + (lane & 1) * 8;
        return read_transposed(at, at + 8 * DP * 2, nullptr);
    }

    // O^T += V^T P^T of the tile that begins with key `first`.
    template <bool MASKED>
    __device__ __forceinline__ void values(const uint8_t* vt, const V8 (&pf)[4], int64_t first)
    {
        if (MASKED && holds_no_number<DP, BF16>(vt, lane)) {
            // 0 * inf: a product over all keys would carry what a query must not see into its row.  The numbers first; then the
            // others key by key, and only the columns that see the key take the result.
            constexpr short kFirst = BF16 ? 0x7f80 : 0x7c00;
#pragma unroll
            for (int ks16 = 0; ks16 < 4; ++ks16)
#pragma unroll
                for (int i = 0; i < DU / 32; ++i) {
                    s8v x = read_v(vt, ks16, i);
                    x = (x & 0x7fff) >= kFirst ? 0 : x;
                    o[i] = T::mfma(__builtin_bit_cast(V8, x), pf[ks16], o[i]);
                }
            const V8 p0 = pf[0], p1 = pf[1], p2 = pf[2], p3 = pf[3];
#pragma unroll
            for (int i = 0; i < DU / 32; ++i)
#pragma nounroll
                for (int j = 0; j < kTile; ++j) {
                    const V8 pj = j < 32 ? (j < 16 ? p0 : p1) : (j < 48 ? p2 : p3);
                    // (the key's value: element e of the lanes of one half)
                    const int e = half == ((j >> 2) & 1) ? (j & 3) + 4 * ((j >> 3) & 1) : -1;
                    s8v one = read_v(vt, j >> 4, i);
#pragma unroll
                    for (int x = 0; x < 8; ++x) one[x] = x == e && (one[x] & 0x7fff) >= kFirst ? one[x] : 0;
                    const f16v with = T::mfma(__builtin_bit_cast(V8, one), pj, o[i]);
                    const bool seen = first + j < limit;
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[i][x] = seen ? with[x] : o[i][x];
                }
            return;
        }
#pragma unroll
        for (int ks16 = 0; ks16 < 4; ++ks16)
#pragma unroll
            for (int i = 0; i < DU / 32; ++i) o[i] = T::mfma(__builtin_bit_cast(V8, read_v(vt, ks16, i)), pf[ks16], o[i]);
    }

    // 1 / sum.  A row that sees keys and has a sum of zero has scores of -inf only: 0 / 0, and not the zeros of a row that sees none.
    __device__ __forceinline__ float inverse(float sum) const { return limit > 0 ? 1.0f / sum : 0.0f; }

    __device__ __forceinline__ void store(const PrefillArgs& a, const Work& w, int64_t first)
    {
        const float inv = inverse(l + __shfl_xor(l, 32));
        if (!there) return;
#pragma unroll
        for (int i = 0; i < DU / 32; ++i) store_block(a, w, first, i, o[i], inv);
    }

    // Results 32 i .. 32 i + 31 of the query, times inv.
    __device__ __forceinline__ void store_block(const PrefillArgs& a, const Work& w, int64_t first, int i, const f16v& x, float inv) const
    {
        uint16_t* to = a.out.data + (w.q.begin + first + col) * a.out.token + w.head * a.out.head + 4 * half;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int d = 32 * i + 2 * e;
            if (d < a.D)
                *reinterpret_cast<u2v*>(to + d) = u2v{pack16(x[e] * inv, x[e + 1] * inv, BF16),
                                                      pack16(x[e + 2] * inv, x[e + 3] * inv, BF16)};
        }
    }
};

// NW 32-query blocks, KS waves on each with every KS-th tile of keys, the next tile in flight while one is worked on; the KS join through
// LDS.  KS = 1: two tiles of K and V in LDS, 64 KB at 128 wide, so that a CU holds two workgroups, whose waves share the matrix cores and
// the vector units; KS = 2: one workgroup, for half as many steps.  4 D operations per visible pair and head, and as many
// instructions on scores as matrix ones: what bounds it is the two of them by turns.  One prompt of 8192, 32 heads on 8, 128 wide:
// 515-548 us, 1.00-1.07 PFLOP/s, matrix cores busy half of the cycles and vector issue a little less; a large matrix product
// reaches 1.39.  Packed prompts of up to 1500 tokens, 28 heads on 4: 57 us.  64 queries a wave (half the LDS reads) spills:
// 589-637; eight waves in two halves that take turns at the matrix cores: no faster.
template <int DP, int DU, bool BF16, int NW, int KS>
__global__ __launch_bounds__(64 * NW * KS, DP == 256 ? 1 : 2) void prefill_kernel(PrefillArgs a)
{
    static_assert(KS == 1 || KS == 2);
    constexpr int kTileBytes = kTile * DP * 2, NV = DU / 32;
    extern __shared__ __align__(16) uint8_t lds[];   // of each part K0 K1 V0 V1; then sums and statistics
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = wave % NW, part = wave / NW;
    Work w;
    if (!find_work<32 * NW>(a, w)) return;
    const int64_t first = w.q0 + block * 32;
    uint8_t* const mine = lds + part * 4 * kTileBytes;
    const Loader<DP, NW> keys(a.k, w.k, w.kvh, a.D, block, lane, k_pattern<DP>);
    const Loader<DP, NW> vals(a.v, w.k, w.kvh, a.D, block, lane, v_pattern<DP>);
    auto issue = [&](int r) {                    // tile r KS + part
        if (r * KS + part >= w.tiles) return;
        keys.load(r * KS + part, mine + (r & 1) * kTileBytes);
        vals.load(r * KS + part, mine + (2 + (r & 1)) * kTileBytes);
    };
    issue(0);
    Queries<DP, DU, BF16> q(a, w, lane, first);
    auto tile = [&](int r, auto masked) {
        f16v sc[2];
        typename Type<BF16>::V8 pf[4];
        const int64_t key = (int64_t)(r * KS + part) * kTile;
        q.scores(mine + (r & 1) * kTileBytes, sc);
        pace<DU / 16, 1, DU / 8>();
        q.template probabilities<decltype(masked)::value>(sc, key, pf);
        q.template values<decltype(masked)::value>(mine + (2 + (r & 1)) * kTileBytes, pf, key);
        if (!decltype(masked)::value) pace<DU / 8, 2, DU / 8>();
    };
    auto arrived = [&](int r) {
        landed();
        meet();
        issue(r + 1);
    };
    const int rounds = (w.tiles + KS - 1) / KS, full = w.full / KS;
    int r = 0;
    for (; r < full; ++r) {
        arrived(r);
        tile(r, std::false_type{});
    }
    for (; r < rounds; ++r) {
        arrived(r);
        const int t = r * KS + part;             // (where no query of this wave sees it: nothing)
        if (t < w.tiles && (int64_t)t * kTile < first + 32 + w.shift) tile(r, std::true_type{});
    }
    if constexpr (KS == 1) {
        q.store(a, w, first);
        return;
    }
    // Join: results 32 i .. are summed and stored by part i % KS.
    float* const sums = reinterpret_cast<float*>(lds);
    constexpr int kSlots = (NV + 1) / 2;         // results that a wave leaves to the other one, at most
    float* const stats = sums + NW * KS * kSlots * 16 * 64;
    const float l = q.l + __shfl_xor(q.l, 32);
    meet();
    if (q.half == 0) stats[wave * 64 + q.col] = q.mx, stats[wave * 64 + 32 + q.col] = l;
    meet();
    const float* const of = stats + block * 64 + q.col;
    float top = of[0], sum = 0.0f;
#pragma unroll
    for (int x = 1; x < KS; ++x) top = fmaxf(top, of[x * NW * 64]);
#pragma unroll
    for (int x = 0; x < KS; ++x) sum += of[x * NW * 64 + 32] * __builtin_amdgcn_exp2f(of[x * NW * 64] - top);
    const float down = __builtin_amdgcn_exp2f(q.mx - top);
    const float inv = q.inverse(sum);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        q.o[i] *= down;
        if (i % KS != part)
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[((wave * kSlots + i / 2) * 16 + e) * 64 + lane] = q.o[i][e];
    }
    meet();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i % KS != part) continue;
        const int other = block + (1 - part) * NW;
#pragma unroll
        for (int e = 0; e < 16; ++e) q.o[i][e] += sums[((other * kSlots + i / 2) * 16 + e) * 64 + lane];
        if (q.there) q.store_block(a, w, first, i, q.o[i], inv);
    }
}

// NW waves on the same 32 queries, each with every NW-th tile of keys and room for one tile of its own: for calls with so few queries
// that tiles of queries leave CUs idle.  A wave requests its next keys when it has read the ones before, values likewise; the waves
// join through LDS.  No barrier before the join: a wave waits for its own loads only.  Bound by that chain (load, scores, statistics,
// values, once per NW tiles): 512 tokens, 12 heads on 2, 9.1 us with four waves; of it about 3 is what any launch takes.
template <int DP, int DU, bool BF16, int NW>
__global__ __launch_bounds__(64 * NW, 1) void prefill_split_kernel(PrefillArgs a)
{
    constexpr int kTileBytes = kTile * DP * 2, NV = DU / 32;
    extern __shared__ __align__(16) uint8_t lds[];   // K and V of wave 0, of wave 1, ...; then the waves' sums and statistics
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Work w;
    if (!find_work<32>(a, w)) return;
    uint8_t* const kt = lds + wave * 2 * kTileBytes;
    uint8_t* const vt = kt + kTileBytes;
    const Loader<DP, 1> keys(a.k, w.k, w.kvh, a.D, 0, lane, k_pattern<DP>);
    const Loader<DP, 1> vals(a.v, w.k, w.kvh, a.D, 0, lane, v_pattern<DP>);
    if (wave < w.tiles) keys.load(wave, kt), vals.load(wave, vt);
    Queries<DP, DU, BF16> q(a, w, lane, w.q0);
    auto tile = [&](int t, auto masked) {
        f16v sc[2];
        typename Type<BF16>::V8 pf[4];
        landed<Loader<DP, 1>::kLoads>();             // (all but the values behind them)
        q.scores(kt, sc);
        read();
        const bool more = t + NW < w.tiles;
        if (more) keys.load(t + NW, kt);
        q.template probabilities<decltype(masked)::value>(sc, (int64_t)t * kTile, pf);
        if (more) landed<Loader<DP, 1>::kLoads>();
        else landed<0>();
        q.template values<decltype(masked)::value>(vt, pf, (int64_t)t * kTile);
        read();
        if (more) vals.load(t + NW, vt);
    };
    int t = wave;
    for (; t < w.full; t += NW) tile(t, std::false_type{});
    for (; t < w.tiles; t += NW) tile(t, std::true_type{});

    // Join: block i of the results (d = 32 i ..) is summed and stored by wave i % NW.
    float* const sums = reinterpret_cast<float*>(lds);
    float* const stats = sums + NW * DP * 32;
    meet();
    const float l = q.l + __shfl_xor(q.l, 32);
    if (q.half == 0) stats[wave * 64 + q.col] = q.mx, stats[wave * 64 + 32 + q.col] = l;
    meet();
    float top = stats[q.col], sum = 0.0f;
#pragma unroll
    for (int x = 1; x < NW; ++x) top = fmaxf(top, stats[x * 64 + q.col]);
#pragma unroll
    for (int x = 0; x < NW; ++x) sum += stats[x * 64 + 32 + q.col] * __builtin_amdgcn_exp2f(stats[x * 64 + q.col] - top);
    const float down = __builtin_amdgcn_exp2f(q.mx - top);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[((wave * NV + i) * 16 + e) * 64 + lane] = q.o[i][e] * down;
    meet();
    const float inv = q.inverse(sum);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i % NW != wave) continue;
        f16v o = {};
#pragma unroll
        for (int x = 0; x < NW; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] += sums[((x * NV + i) * 16 + e) * 64 + lane];
        if (q.there) q.store_block(a, w, w.q0, i, o, inv);
    }
}

template <int DP, int DU, bool BF16, int NW, int KS>
int launch_waves(PrefillArgs& a, hipStream_t st)
{
    constexpr size_t kLds = KS * 4 * (size_t)kTile * DP * 2;
    static thread_local int allowed = -1;
    if (int e = allow_large_lds(prefill_kernel<DP, DU, BF16, NW, KS>, kLds, allowed)) return e;
    a.tiles = a.q_tokens / (32 * NW) + a.sequences;
    prefill_kernel<DP, DU, BF16, NW, KS><<<dim3((unsigned)(a.tiles * a.heads)), 64 * NW * KS, kLds, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    return MNNQ_OK;
}

template <int DP, int DU, bool BF16, int NW>
int launch_split(PrefillArgs& a, hipStream_t st)
{
    constexpr size_t kTiles = NW * 2 * (size_t)kTile * DP * 2, kJoin = NW * (DP * 32 + 64) * sizeof(float);
    constexpr size_t kLds = kTiles > kJoin ? kTiles : kJoin;
    static thread_local int allowed = -1;
    if (int e = allow_large_lds(prefill_split_kernel<DP, DU, BF16, NW>, kLds, allowed)) return e;
    a.tiles = a.q_tokens / 32 + a.sequences;
    prefill_split_kernel<DP, DU, BF16, NW><<<dim3((unsigned)(a.tiles * a.heads)), 64 * NW, kLds, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    return MNNQ_OK;
}

template <int DP, int DU, bool BF16>
int launch_type(PrefillArgs& a, hipStream_t st)
{
    // By the number of 32-query blocks there may be.  Up to one per CU: four waves share a block's keys; up to four: two; else four
    // waves have a block each and share tiles of keys.  Measured in us, 4 waves a block / 2 / a block each: 204 blocks (512 tokens, 12
    // heads) 9.4 / 10.7 / 16.7; 84 (64 queries behind 2048 keys, 28 heads) 20.5 / 25.4 / 39.9; 476 16.4 / 12.7 / 18.1; 924 34.5 /
    // 23.2 / 28.4; 2080 93.9 / 65.6 / 52.3; 2296 (twenty of 100) 58.8 / 35.1 / 28.3.  (256 wide, LDS holds the tiles of two.)
    const int64_t blocks = (a.q_tokens / 32 + a.sequences) * a.heads;
    // Between one and two 128-query tiles per CU whose keys are many: those tiles, two waves on each 32 queries.  Us, against the other
    // forms: 1200 tokens, 28 heads, 25.9 / 30.0; 1536, 32 heads, 34.3 / 37.5; 4096, 12 heads, 70 / 87; 8192, 8 heads, 146 / 179 (64 wide 89 /
    // 110); one per CU: 8192, 4 heads, 110 / 96; more than two: 2500, 28 heads, 69 / 63; few keys: nine of 128, 32 heads, 21.8 / 13.8.
    const int64_t wide = ((a.q_tokens + 127) / 128 + a.sequences - 1) * a.heads;
    if constexpr (DP < 256) {
        if (blocks <= 256) return launch_split<DP, DU, BF16, 4>(a, st);
        if (wide > 256 && wide <= 512 && a.k_tokens >= 1024 * a.sequences) return launch_waves<DP, DU, BF16, 4, 2>(a, st);
    }
    if (blocks <= 1152) return launch_split<DP, DU, BF16, 2>(a, st);
    return launch_waves<DP, DU, BF16, 4, 1>(a, st);
}

template <int DP, int DU>
int launch_width(bool bf16, PrefillArgs& a, hipStream_t st)
{
    return bf16 ? launch_type<DP, DU, true>(a, st) : launch_type<DP, DU, false>(a, st);
}

}  // namespace

int launch_attn_prefill(bool bf16, int64_t sequences, const int32_t* q_start, const int32_t* k_start, int64_t q_tokens,
                        int64_t k_tokens, int heads, int kv_heads, int head_dim, float scale, const Rows& q, const Rows& k,
                        const Rows& v, const Rows& out, hipStream_t st)
{
    PrefillArgs a{q, k, v, out, q_start, k_start, sequences, q_tokens, k_tokens, 0, heads, kv_heads, head_dim, scale * kLog2e};
    return head_dim <= 64 ? launch_width<64, 64>(bf16, a, st)
         : head_dim <= 96 ? launch_width<128, 96>(bf16, a, st)
         : head_dim <= 128 ? launch_width<128, 128>(bf16, a, st)
         : head_dim <= 192 ? launch_width<256, 192>(bf16, a, st) : launch_width<256, 256>(bf16, a, st);
}

}  // namespace mnnq
