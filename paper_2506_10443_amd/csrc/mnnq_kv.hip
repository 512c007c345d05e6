// The 8-bit key / value cache: appending rows (mnnq_kv_append) and dropping tokens (mnnq_kv_evict).
//
// A code c of a block and head with range r stands for c r / TOP, TOP = 127 (int8) or 448 (e4m3).  A new value x becomes
// round(x TOP / r), an older code whose block's range grows round(c r / r').  Both products are exact in binary32 (11
// significant bits times 7, or 4 times 11), and the quotient of two such numbers is never nearer to a tie than a correctly rounded
// division can tell without being one: the codes are those of the definition in exact arithmetic.
#include "mnnq_attn.h"

namespace mnnq {

namespace {

// ---- append

struct AppendArgs {
    mnnq_kv_cache c;
    Rows k, v;
    const int32_t* start;       // NULL: `each` rows per sequence
    int64_t tokens, each;
    int64_t pieces_each;        // blocks that `each` rows can touch
    bool bf16;
};

// Piece `p` of the grid: a block of a sequence that new rows go to.  false: nothing to do.
struct Piece {
    int64_t row;                // of the first new token in this block
    int first, count;           // its slot in the block; new tokens in it
    int64_t block;
};

__device__ __forceinline__ bool find_piece(const AppendArgs& a, int64_t p, Piece& out)
{
    const mnnq_kv_cache& c = a.c;
    int64_t s, begin, n, j;
    if (!a.start) {
        s = p / a.pieces_each;
        j = p - s * a.pieces_each;
        begin = s * a.each;
        n = a.each;
    } else {
        // Sequence s owns the pieces from start[s] / block + 2 s on: n tokens touch at most n / block + 2 blocks.
        const int64_t total = a.tokens;
        auto base = [&](int64_t i) {
            const int64_t at = a.start[i];
            return (at < 0 ? 0 : at > total ? total : at) / c.block_tokens + 2 * i;
        };
        s = last_of(c.sequences, [&](int64_t i) { return base(i) <= p; });
        j = p - base(s);
        const Span span = span_of(a.start, s, total);
        begin = span.begin;
        n = span.count;
    }
    const int64_t room = c.table_blocks * c.block_tokens;
    int64_t len = c.lengths[s];
    len = len < 0 ? 0 : len > room ? room : len;
    const int64_t b = len / c.block_tokens + j;
    int64_t from = b * c.block_tokens, to = from + c.block_tokens;
    const int64_t first = from > len ? from : len;
    const int64_t last = len + n < room ? len + n : room;
    to = to < last ? to : last;
    if (j < 0 || first >= to) return false;
    const int64_t block = c.block_table[s * c.table_blocks + b];
    if (block < 0 || block >= c.blocks) return false;
    out = {begin + first - len, (int)(first - from), (int)(to - first), block};
    return true;
}

// Quotients n / range, correctly rounded, three operations each: q = n inv, q + (n - q range) inv with inv = 1 / range correctly
// rounded (Markstein's theorem; a range is a number of 11 bits at most, not one of all ones).  Range and numerators are scaled by a power of
// two that brings the range to [1, 2), or as near as one such factor can, so that nothing on the way leaves the normal numbers.
struct Divisor {
    float scale, range, inv;
    __device__ __forceinline__ explicit Divisor(float r)
    {
        const int e = (int)((__float_as_uint(r) >> 23) & 255u) - 127;
        const int up = min(-e, 118);            // (2^118 * 448 is still a number)
        scale = __uint_as_float((uint32_t)max(up + 127, 1) << 23);
        range = r * scale;
        inv = 1.0f / range;
    }
    // n: a numerator times `scale`
    __device__ __forceinline__ float operator()(float n) const
    {
        const float q = n * inv;
        return __builtin_fmaf(__builtin_fmaf(-range, q, n), inv, q);
    }
};

// Codes of a range that is no number are zeros: a code without a number would reach tokens' rows that do not see it, as 0 * NaN.
__device__ __forceinline__ bool a_number(uint32_t range) { return range < 0x7f800000u; }

// Sixteen codes of a range `before` as codes of the divisor's range.
template <int FORM>
__device__ __forceinline__ uint4 recode16(uint4 w, float before, const Divisor& by)
{
    const float from = before * by.scale;
    uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float c[4];
        codes_to_float<FORM>(d[j], c);
        d[j] = codes_of<FORM>(by(c[0] * from), by(c[1] * from), by(c[2] * from), by(c[3] * from));
    }
    return uint4{d[0], d[1], d[2], d[3]};
}

// Eight values as codes of the divisor's range.
template <int FORM, bool BF16>
__device__ __forceinline__ uint2 encode8(const uint4& x, const Divisor& by)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    const float up = by.scale * code_top<FORM>();
    uint32_t out[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            y[j] = by(value16(j & 1 ? w[2 * i + j / 2] >> 16 : w[2 * i + j / 2] & 0xffffu, BF16) * up);
        out[i] = codes_of<FORM>(y[0], y[1], y[2], y[3]);
    }
    return uint2{out[0], out[1]};
}

// R: 16-byte pieces of the new rows that a thread holds, THREADS * R at least in all.
template <int FORM, int THREADS, int R>
__device__ __forceinline__ void append_piece(const AppendArgs& a, const Piece& p, const Rows& x, uint8_t* codes, float* ranges,
                                             int head)
{
    typedef unsigned short us2v __attribute__((ext_vector_type(2)));
    __shared__ uint32_t wave_top[THREADS / 64];
    const int tid = threadIdx.x, D = a.c.head_dim, per_row = D / 8;
    const uint16_t* src = x.data + p.row * x.token + head * x.head;
    const int64_t slot = p.block * a.c.kv_heads + head;
    uint8_t* dst = codes + slot * a.c.block_tokens * D;
    const float before = p.first > 0 ? ranges[slot] : 0.0f;
    uint4 w[R];
    int to[R];                                   // the piece's place among the codes; -1: none
    int row = tid / per_row, ch = tid - row * per_row;
    const int row_step = THREADS / per_row, ch_step = THREADS - row_step * per_row;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        to[i] = row < p.count ? (p.first + row) * D + ch * 8 : -1;
        w[i] = uint4{0, 0, 0, 0};
        if (row < p.count) w[i] = *reinterpret_cast<const uint4*>(src + row * x.token + ch * 8);
        row += row_step, ch += ch_step;
        if (ch >= per_row) ch -= per_row, ++row;
    }
    // greatest magnitude: of the bits without the sign, as integers (a NaN is above every number)
    us2v two = {0, 0};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) two = __builtin_elementwise_max(two, __builtin_bit_cast(us2v, v[j] & 0x7fff7fffu));
    }
    uint32_t top = max((uint32_t)two.x, (uint32_t)two.y);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    if (THREADS > 64) {
        if ((tid & 63) == 0) wave_top[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) top = max(top, wave_top[i]);
    }
    // (as integers too: magnitudes, and a NaN stays one)
    const float range = __uint_as_float(max(__float_as_uint(value16(top, a.bf16)), __float_as_uint(before) & 0x7fffffffu));
    const Divisor by(range);
    const bool number = a_number(__float_as_uint(range));
    if (p.first > 0 && __float_as_uint(range) != __float_as_uint(before))
        for (int i = tid; i < p.first * D / 16; i += THREADS) {
            uint4* at = reinterpret_cast<uint4*>(dst + i * 16);
            *at = number ? recode16<FORM>(*at, before, by) : uint4{0, 0, 0, 0};
        }
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (to[i] >= 0) {
            uint2 q = {0, 0};
            if (number && __float_as_uint(range) != 0)
                q = a.bf16 ? encode8<FORM, true>(w[i], by) : encode8<FORM, false>(w[i], by);
            *reinterpret_cast<uint2*>(dst + to[i]) = q;
        }
    if (tid == 0) ranges[slot] = range;
}

// One workgroup per block that rows go to, head, and K or V: range, older codes and new rows are that block's alone, so nothing is
// shared and nothing is atomic.  The new rows stay in registers between the range and the codes (2 bytes read and 1 written per
// number): a prompt of 8192 rows, 8 heads, 128 wide, 50 MB, 11.1 us = 4.5 TB/s; one row 3.4, a launch and two dependent loads.
template <int THREADS, int R>
__global__ __launch_bounds__(THREADS) void append_kernel(AppendArgs a)
{
    Piece p;
    if (!find_piece(a, blockIdx.x, p)) return;
    const int head = blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const Rows& x = is_v ? a.v : a.k;
    uint8_t* codes = static_cast<uint8_t*>(is_v ? a.c.v_codes : a.c.k_codes);
    float* ranges = is_v ? a.c.v_range : a.c.k_range;
    if ((is_v ? a.c.v_form : a.c.k_form) == MNNQ_KV_FP8) append_piece<MNNQ_KV_FP8, THREADS, R>(a, p, x, codes, ranges, head);
    else append_piece<MNNQ_KV_INT8, THREADS, R>(a, p, x, codes, ranges, head);
}

// ---- evict

struct EvictArgs {
    mnnq_kv_cache c;
    const float* weights;
    int64_t weights_stride, keep, recent;
    const int32_t* new_table;
    int64_t new_table_blocks;
    int32_t* kept;
    int32_t* new_lengths;
    float* new_weights;
    int64_t new_weights_stride;
};

__device__ __forceinline__ int64_t evict_length(const EvictArgs& a, int64_t s)
{
    const int64_t room = a.c.table_blocks * a.c.block_tokens;
    int64_t len = a.c.lengths[s];
    len = len > room ? room : len;
    return len < 0 ? 0 : len;
}

// Whether the cache has the block of a sequence's token.
__device__ __forceinline__ bool token_there(const EvictArgs& a, int64_t s, int token)
{
    return (uint32_t)a.c.block_table[s * a.c.table_blocks + (token >> __builtin_ctz(a.c.block_tokens))] < (uint32_t)a.c.blocks;
}

__device__ __forceinline__ int lanes_below(uint64_t mask)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Floats in the order of their values as unsigned integers; NaN above all, both zeros the same.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t b = __float_as_uint(w + 0.0f);
    if (w != w) return 0xffffffffu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The weight again (a zero without its sign, a NaN as one of them).
__device__ __forceinline__ float weight_of(uint32_t key)
{
    return __uint_as_float(key == 0xffffffffu ? 0x7fc00000u : key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// Of a token: zero behind the weights.
__device__ __forceinline__ float weight_at(const EvictArgs& a, int64_t row, int token)
{
    return token < a.weights_stride ? a.weights[row * a.weights_stride + token] : 0.0f;
}

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kDigits[3] = {11, 11, 10};         // bits of a key that a pass settles, from the top

struct SelectSpace {
    int hist[2048];
    __align__(16) int wave_sum[kSelectWaves], wave_equal[kSelectWaves], wave_above[kSelectWaves];
    uint32_t digit;
    int need, old;
};

// One workgroup per sequence and key head: the key of the last token that is kept by a radix search of three passes over the
// keys, then the kept tokens in order.  Wave w has the tokens from w * per_wave on, 64 at a time; R: keys that a thread holds (0: they
// are read again in every pass).  Comparing keys pairwise or sorting them would cost more than the three counts of n; one
// workgroup, since each pass waits for the one before: 4097 tokens 11.9 us, 16 x 8 rows of up to 16315 16.3, both the chain of
// barriers and additions to LDS counters, at under a tenth of the rate of memory.
// `missing` of the tokens are in blocks that the cache does not have, which are masked everywhere and kept nowhere: GAPS.
// raw: the weights of a thread's R tokens.
template <int R, bool GAPS>
__device__ __forceinline__ void select_row(const EvictArgs& a, SelectSpace& sh, int64_t s, int head, int len, int missing,
                                           const float (&raw)[R > 0 ? R : 1])
{
    static_assert(!(R > 0 && GAPS));
    constexpr int kUnroll = R > 0 ? R : 1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t room = a.new_table_blocks * a.c.block_tokens, most_kept = a.keep < room ? a.keep : room;
    const int n = len - missing < most_kept ? len - missing : (int)most_kept;
    const int64_t row = s * a.c.kv_heads + head;
    int32_t* kept = a.kept + row * a.keep;
    float* nw = a.new_weights + row * a.new_weights_stride;
    const int last = a.recent < n ? (int)a.recent : n;       // kept as the newest
    int old = len - last;                                    // the others compete
    if (GAPS) {                                              // (those of the last that are there, counted from the end)
        if (wave == 0) {
            int found = 0;
            old = len;
            while (found < last && old > 0) {                // (there are at least n)
                const int token = old - 64 + lane;
                uint64_t some = __ballot(token >= 0 && token_there(a, s, token >= 0 ? token : 0));
                found += __popcll(some);
                for (; found > last; --found) some &= some - 1;
                old = found < last ? old - 64 : old - 64 + __builtin_ctzll(some);
            }
            if (lane == 0) sh.old = old < 0 ? 0 : old;
        }
        __syncthreads();
        old = sh.old;
    }
    const int competing = len - missing - last;
    const int places = n - last;                             // for this many places
    const int steps = (len + kSelectThreads - 1) / kSelectThreads, first = wave * steps * 64 + lane;
    const int most = R > 0 ? R : steps;                      // (a bound that loops over held keys are unrolled by)
    // (0: no token that competes; the keys of numbers and NaN are above it)
    auto key_at = [&](int j) {
        const int token = first + j * 64;
        return token < old && (!GAPS || token_there(a, s, token)) ? weight_key(weight_at(a, row, token)) : 0u;
    };
    uint32_t held[kUnroll];
    if (R > 0)
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) held[j] = j < steps && first + j * 64 < old ? weight_key(raw[j]) : 0u;
    auto key_of = [&](int j) { return R > 0 ? held[R > 0 ? j : 0] : key_at(j); };

    // prefix: the settled bits of the last kept key; need: places left for keys that have them.  All keys are above 0, none above
    // the greatest.
    uint32_t prefix = places > 0 ? 0u : 0xffffffffu;
    int need = 0;
    if (places > 0 && places < competing) {
        need = places;
        int shift = 32;
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = kDigits[pass], above = shift;
            shift -= bits;
            if (pass > 0) {                      // (for the first one they are zero)
                for (int i = tid; i < 2048; i += kSelectThreads) sh.hist[i] = 0;
                __syncthreads();
            }
            const uint32_t settled = pass == 0 ? 0u : prefix >> above, mask = (1u << bits) - 1;
#pragma unroll kUnroll
            for (int j = 0; j < most; ++j) {
                if (j >= steps) continue;
                const uint32_t key = key_of(j);
                if (key && (pass == 0 || key >> above == settled)) atomicAdd(&sh.hist[key >> shift & mask], 1);
            }
            __syncthreads();
            // from the top: thread t has bins 2047 - 2 t and 2046 - 2 t
            const int b0 = sh.hist[2047 - 2 * tid], b1 = sh.hist[2046 - 2 * tid];
            int sum = b0 + b1;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const int other = __shfl_up(sum, m);
                if (lane >= m) sum += other;
            }
            if (lane == 63) sh.wave_sum[wave] = sum;
            __syncthreads();
            int before = sum - b0 - b1;
#pragma unroll
            for (int x = 0; x < kSelectWaves; ++x) before += x < wave ? sh.wave_sum[x] : 0;
            if (before < need && before + b0 + b1 >= need) {
                const bool second = before + b0 < need;
                sh.digit = 2047 - 2 * tid - (second ? 1 : 0);
                sh.need = need - before - (second ? b0 : 0);
            }
            __syncthreads();
            prefix |= sh.digit << shift;
            need = sh.need;
        }
    }
    // Kept: the keys above the prefix, of those that equal it the first `need`, and the newest tokens behind them.
    int n_above = 0, n_equal = 0;
#pragma unroll kUnroll
    for (int j = 0; j < most; ++j) {
        if (j >= steps) continue;
        n_above += __popcll(__ballot(key_of(j) > prefix));
        n_equal += __popcll(__ballot(key_of(j) == prefix));
    }
    if (lane == 0) sh.wave_above[wave] = n_above, sh.wave_equal[wave] = n_equal;
    __syncthreads();
    int at = 0, equal_before = 0;
#pragma unroll
    for (int x = 0; x < kSelectWaves; ++x)
        if (x < wave) at += sh.wave_above[x], equal_before += sh.wave_equal[x];
    at += equal_before < need ? equal_before : need;
    at = __builtin_amdgcn_readfirstlane(at), equal_before = __builtin_amdgcn_readfirstlane(equal_before);
#pragma unroll kUnroll
    for (int j = 0; j < most; ++j) {
        if (j >= steps) continue;
        const uint32_t key = key_of(j);
        bool take = key > prefix;
        const uint64_t eq = __ballot(key == prefix);
        if (eq && equal_before < need) take |= key == prefix && equal_before + lanes_below(eq) < need;
        const uint64_t tk = __ballot(take);
        const int to = at + lanes_below(tk);
        if (take && to < n) {
            kept[to] = first + j * 64;
            nw[to] = weight_of(key);
        }
        equal_before += __popcll(eq);
        at += __popcll(tk);
    }
    if (!GAPS) {
        for (int i = tid; i < last; i += kSelectThreads) {
            kept[places + i] = old + i;
            nw[places + i] = weight_of(weight_key(weight_at(a, row, old + i)));
        }
    } else if (wave == 0) {
        int to = places;
        for (int token = old + lane; token - lane < len; token += 64) {
            const bool there = token < len && token_there(a, s, token < len ? token : 0);
            const uint64_t some = __ballot(there);
            const int place = to + lanes_below(some);
            if (there && place < n) {
                kept[place] = token;
                nw[place] = weight_of(weight_key(weight_at(a, row, token)));
            }
            to += __popcll(some);
        }
    }
    for (int64_t i = n + tid; i < a.keep; i += kSelectThreads) kept[i] = -1;
    for (int64_t i = n + tid; i < a.new_weights_stride; i += kSelectThreads) nw[i] = 0.0f;
    if (head == 0 && tid == 0) a.new_lengths[s] = n;
}

template <int R>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictArgs a)
{
    __shared__ SelectSpace sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = a.c.block_tokens;
    const int64_t s = blockIdx.y;
    const int head = blockIdx.x, len = (int)evict_length(a, s);
    const int steps = (len + kSelectThreads - 1) / kSelectThreads;
    // (weights and table are requested together)
    float raw[R > 0 ? R : 1];
    if (R > 0)
#pragma unroll
        for (int j = 0; j < R; ++j)
            raw[j] = j < steps ? weight_at(a, s * a.c.kv_heads + head, wave * steps * 64 + j * 64 + lane) : 0.0f;
    int missing = 0;
    for (int64_t first = (int64_t)tid * B; first < len; first += (int64_t)kSelectThreads * B)
        if (!token_there(a, s, (int)first)) missing += len - (int)first < B ? len - (int)first : B;
    if (__ballot(missing != 0))
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) missing += __shfl_xor(missing, m);
    if (lane == 0) sh.wave_sum[wave] = missing;
    for (int i = tid; i < 2048; i += kSelectThreads) sh.hist[i] = 0;
    __syncthreads();
    missing = 0;
#pragma unroll
    for (int x = 0; x < kSelectWaves; ++x) missing += sh.wave_sum[x];
    // (R is chosen by the room that weights and table have, whichever is less: a sequence may be longer than its weights)
    const float none[1] = {0.0f};
    if (missing > 0) select_row<0, true>(a, sh, s, head, len, missing, none);
    else if (R > 0 && steps > R) select_row<0, false>(a, sh, s, head, len, 0, none);
    else select_row<R, false>(a, sh, s, head, len, 0, raw);
}

constexpr int kMoveThreads = 256;
constexpr int kMovePieces = 4;                   // 16-byte pieces of K, and of V, that a thread has in flight

// One workgroup per new block and key head.  Ranges first (the greatest of the tokens' old ones), then the codes, moved as they are
// where old and new range agree.  A copy bounds it: 16 sequences x 8 heads of up to 4096 kept tokens, 128 wide, 243 MB read
// and written, 45-54 us = 4.5-5.3 TB/s.
template <int KF, int VF>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(EvictArgs a)
{
    __shared__ int64_t from[128];
    __shared__ float range_of[2][128];
    const int tid = threadIdx.x, lane = tid & 63, D = a.c.head_dim, B = a.c.block_tokens;
    const int64_t s = blockIdx.z, b = blockIdx.x;
    const int head = blockIdx.y;
    const int32_t* kept = a.kept + (s * a.c.kv_heads + head) * a.keep + b * B;
    // (the length, the new block and the first of the places are requested together)
    const int32_t early = tid < B && b * B + tid < a.keep ? kept[tid] : -1;
    const int64_t to = a.new_table[s * a.new_table_blocks + b];
    const int64_t left = a.new_lengths[s] - b * B;
    if (left <= 0 || to < 0 || to >= a.c.blocks) return;
    const int count = (int)(left < B ? left : B);
    // where each token lies (in a block that the cache has: the others were not kept), and its ranges
    if (tid < count) {
        const int64_t at = (int64_t)a.c.block_table[s * a.c.table_blocks + early / B] * a.c.kv_heads + head;
        from[tid] = (at * B + early % B) * D;
        range_of[0][tid] = a.c.k_range[at];
        range_of[1][tid] = a.c.v_range[at];
    }
    __syncthreads();
    // (magnitudes as integers; a NaN stays one)
    uint32_t top[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        top[x] = lane < count ? __float_as_uint(range_of[x][lane]) & 0x7fffffffu : 0u;
        if (lane + 64 < count) top[x] = max(top[x], __float_as_uint(range_of[x][lane + 64]) & 0x7fffffffu);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top[x] = max(top[x], (uint32_t)__shfl_xor((int)top[x], m));
    }
    uint8_t* const codes[2] = {static_cast<uint8_t*>(a.c.k_codes), static_cast<uint8_t*>(a.c.v_codes)};
    const int64_t slot = to * a.c.kv_heads + head;
    const Divisor by_k(__uint_as_float(top[0])), by_v(__uint_as_float(top[1]));
    const int per_row = D / 16, pieces = count * per_row;
    for (int base = tid; base < pieces; base += kMoveThreads * kMovePieces) {
        uint4 k[kMovePieces], v[kMovePieces];
        int r[kMovePieces];
#pragma unroll
        for (int i = 0; i < kMovePieces; ++i) {
            const int at = base + i * kMoveThreads;
            r[i] = at < pieces ? at / per_row : -1;
            k[i] = v[i] = uint4{0, 0, 0, 0};
            if (r[i] >= 0) {
                const int64_t source = from[r[i]] + (at - r[i] * per_row) * 16;
                k[i] = *reinterpret_cast<const uint4*>(codes[0] + source);
                v[i] = *reinterpret_cast<const uint4*>(codes[1] + source);
            }
        }
#pragma unroll
        for (int i = 0; i < kMovePieces; ++i) {
            if (r[i] < 0) continue;
            const float kb = range_of[0][r[i]], vb = range_of[1][r[i]];
            if (__float_as_uint(kb) != top[0]) k[i] = a_number(top[0]) ? recode16<KF>(k[i], kb, by_k) : uint4{0, 0, 0, 0};
            if (__float_as_uint(vb) != top[1]) v[i] = a_number(top[1]) ? recode16<VF>(v[i], vb, by_v) : uint4{0, 0, 0, 0};
            const int64_t place = slot * B * D + (int64_t)(base + i * kMoveThreads) * 16;
            *reinterpret_cast<uint4*>(codes[0] + place) = k[i];
            *reinterpret_cast<uint4*>(codes[1] + place) = v[i];
        }
    }
    if (tid == 0) {
        a.c.k_range[slot] = __uint_as_float(top[0]);
        a.c.v_range[slot] = __uint_as_float(top[1]);
    }
}

}  // namespace

int launch_kv_append(const mnnq_kv_cache& c, bool bf16, const int32_t* start, int64_t tokens, const Rows& k, const Rows& v,
                     hipStream_t st)
{
    AppendArgs a{c, k, v, start, tokens, 0, 0, bf16};
    int64_t pieces;
    if (start) {
        pieces = tokens / c.block_tokens + 2 * c.sequences;
    } else {
        a.each = tokens / c.sequences;
        a.pieces_each = (a.each + c.block_tokens - 2) / c.block_tokens + 1;
        pieces = a.pieces_each * c.sequences;
    }
    const dim3 grid((unsigned)pieces, (unsigned)(2 * c.kv_heads));
    // the most 16-byte pieces of a block, head and kind that come at once
    const int64_t rows = !start && a.each < c.block_tokens ? a.each : c.block_tokens, most = rows * (c.head_dim / 8);
    if (most <= 64) append_kernel<64, 1><<<grid, 64, 0, st>>>(a);
    else if (most <= 1024) append_kernel<256, 4><<<grid, 256, 0, st>>>(a);
    else append_kernel<256, 16><<<grid, 256, 0, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    return MNNQ_OK;
}

int launch_kv_evict(const mnnq_kv_cache& c, const float* weights, int64_t weights_stride, int64_t keep, int64_t recent,
                    const int32_t* new_table, int64_t new_table_blocks, int32_t* kept, int32_t* new_lengths,
                    float* new_weights, int64_t new_weights_stride, hipStream_t st)
{
    const EvictArgs a{c,    weights,     weights_stride, keep,        recent,            new_table, new_table_blocks,
                      kept, new_lengths, new_weights,    new_weights_stride};
    const dim3 rows((unsigned)c.kv_heads, (unsigned)c.sequences);
    const int64_t room = c.table_blocks * c.block_tokens, most = room < weights_stride ? room : weights_stride;
    if (most <= 4 * kSelectThreads) select_kernel<4><<<rows, kSelectThreads, 0, st>>>(a);
    else if (most <= 16 * kSelectThreads) select_kernel<16><<<rows, kSelectThreads, 0, st>>>(a);
    else select_kernel<0><<<rows, kSelectThreads, 0, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    const int64_t needed = (keep + c.block_tokens - 1) / c.block_tokens;
    const dim3 grid((unsigned)(new_table_blocks < needed ? new_table_blocks : needed), (unsigned)c.kv_heads, (unsigned)c.sequences);
    const bool k8 = c.k_form == MNNQ_KV_FP8, v8 = c.v_form == MNNQ_KV_FP8;
    if (k8 && v8) move_kernel<MNNQ_KV_FP8, MNNQ_KV_FP8><<<grid, kMoveThreads, 0, st>>>(a);
    else if (k8) move_kernel<MNNQ_KV_FP8, MNNQ_KV_INT8><<<grid, kMoveThreads, 0, st>>>(a);
    else if (v8) move_kernel<MNNQ_KV_INT8, MNNQ_KV_FP8><<<grid, kMoveThreads, 0, st>>>(a);
    else move_kernel<MNNQ_KV_INT8, MNNQ_KV_INT8><<<grid, kMoveThreads, 0, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    return MNNQ_OK;
}

}  // namespace mnnq
