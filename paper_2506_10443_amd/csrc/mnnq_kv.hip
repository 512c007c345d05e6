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
        int64_t lo = 0, hi = c.sequences - 1;
        const int64_t total = a.tokens;
        auto base = [&](int64_t i) {
            const int64_t at = a.start[i];
            return (at < 0 ? 0 : at > total ? total : at) / c.block_tokens + 2 * i;
        };
        while (lo < hi) {
            const int64_t mid = (lo + hi + 1) >> 1;
            if (base(mid) <= p) lo = mid;
            else hi = mid - 1;
        }
        s = lo;
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

// A power of two that keeps a product with TOP finite (bfloat16 goes to 3.4e38); what it takes below the normal numbers has
// codes of zero against such a range.
__device__ __forceinline__ float headroom(float range) { return range > 0x1p100f ? 0x1p-64f : 1.0f; }

// Sixteen codes of a range `before` as codes of the range `range`.
template <int FORM>
__device__ __forceinline__ uint4 recode16(uint4 w, float before, float range)
{
    const float room = headroom(range), from = before * room, to = range * room;
    uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float c[4];
        codes_to_float<FORM>(d[j], c);
        d[j] = codes_of<FORM>(c[0] * from / to, c[1] * from / to, c[2] * from / to, c[3] * from / to);
    }
    return uint4{d[0], d[1], d[2], d[3]};
}

template <int FORM>
__device__ __forceinline__ uint2 encode8(uint4 x, float range, bool bf16)
{
    const float room = headroom(range), to = range * room;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t out[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t bits = j & 1 ? w[2 * i + j / 2] >> 16 : w[2 * i + j / 2] & 0xffffu;
            y[j] = value16(bits, bf16) * room * code_top<FORM>() / to;
        }
        out[i] = codes_of<FORM>(y[0], y[1], y[2], y[3]);
    }
    return uint2{out[0], out[1]};
}

template <int FORM, int THREADS>
__device__ void append_piece(const AppendArgs& a, const Piece& p, const Rows& x, uint8_t* codes, float* ranges, int head)
{
    __shared__ uint32_t wave_top[THREADS / 64];
    const int tid = threadIdx.x, D = a.c.head_dim, per_row = D / 8;
    const int chunks = p.count * per_row;
    const uint16_t* src = x.data + p.row * x.token + head * x.head;
    const int64_t slot = p.block * a.c.kv_heads + head;
    uint8_t* dst = codes + slot * a.c.block_tokens * D;
    const float before = p.first > 0 ? ranges[slot] : 0.0f;
    // greatest magnitude: of the bits without the sign, as integers (a NaN is above every number)
    uint32_t top = 0;
    for (int i = tid; i < chunks; i += THREADS) {
        const int row = i / per_row, ch = i - row * per_row;
        const uint4 w = *reinterpret_cast<const uint4*>(src + row * x.token + ch * 8);
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = v[j] & 0x7fffu, hi = (v[j] >> 16) & 0x7fffu;
            top = max(top, max(lo, hi));
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    if (THREADS > 64) {
        if ((tid & 63) == 0) wave_top[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) top = max(top, wave_top[w]);
    }
    const float fresh = value16(top, a.bf16);
    // (as integers too: magnitudes, and a NaN stays one)
    const float range = __uint_as_float(max(__float_as_uint(fresh), __float_as_uint(before) & 0x7fffffffu));
    if (p.first > 0 && __float_as_uint(range) != __float_as_uint(before)) {
        for (int i = tid; i < p.first * D / 16; i += THREADS) {
            uint4* at = reinterpret_cast<uint4*>(dst + i * 16);
            *at = recode16<FORM>(*at, before, range);
        }
    }
    for (int i = tid; i < chunks; i += THREADS) {
        const int row = i / per_row, ch = i - row * per_row;
        const uint4 w = *reinterpret_cast<const uint4*>(src + row * x.token + ch * 8);
        const uint2 q = range > 0.0f || range != range ? encode8<FORM>(w, range, a.bf16) : uint2{0, 0};
        *reinterpret_cast<uint2*>(dst + (p.first + row) * D + ch * 8) = q;
    }
    if (tid == 0) ranges[slot] = range;
}

// One workgroup per block that rows go to, head, and K or V.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void append_kernel(AppendArgs a)
{
    Piece p;
    if (!find_piece(a, blockIdx.x, p)) return;
    const int head = blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const Rows& x = is_v ? a.v : a.k;
    uint8_t* codes = static_cast<uint8_t*>(is_v ? a.c.v_codes : a.c.k_codes);
    float* ranges = is_v ? a.c.v_range : a.c.k_range;
    if ((is_v ? a.c.v_form : a.c.k_form) == MNNQ_KV_FP8) append_piece<MNNQ_KV_FP8, THREADS>(a, p, x, codes, ranges, head);
    else append_piece<MNNQ_KV_INT8, THREADS>(a, p, x, codes, ranges, head);
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
    len = len > a.weights_stride ? a.weights_stride : len;
    return len < 0 ? 0 : len;
}

__device__ __forceinline__ int64_t evict_kept(const EvictArgs& a, int64_t len)
{
    const int64_t room = a.new_table_blocks * a.c.block_tokens;
    const int64_t n = len < a.keep ? len : a.keep;
    return n < room ? n : room;
}

// Floats in the order of their values as unsigned integers; NaN above all, both zeros the same.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t b = __float_as_uint(w + 0.0f);
    if (w != w) return 0xffffffffu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kSelectThreads = 1024;

// One workgroup per sequence and key head: the key of the last token that is kept by a radix search of four passes, then the
// kept tokens in order.
__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictArgs a)
{
    __shared__ int hist[256];
    __shared__ int wave_sum[2][kSelectThreads / 64];
    __shared__ uint32_t sh_prefix;
    __shared__ int sh_need;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int head = blockIdx.x;
    const int64_t s = blockIdx.y;
    const int64_t len = evict_length(a, s), n = evict_kept(a, len);
    const int64_t row = s * a.c.kv_heads + head;
    const float* w = a.weights + row * a.weights_stride;
    int32_t* kept = a.kept + row * a.keep;
    float* nw = a.new_weights + row * a.new_weights_stride;
    const int64_t last = a.recent < n ? a.recent : n;        // kept as the newest
    const int64_t old = len - last;                          // the others compete
    int need = (int)(n - last);                              // for this many places
    uint32_t prefix = 0;
    if (need > 0 && need < old) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int64_t i = tid; i < old; i += kSelectThreads) {
                const uint32_t key = weight_key(w[i]);
                if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255], 1);
            }
            __syncthreads();
            if (tid == 0) {
                int left = need, b = 255;
                while (b > 0 && hist[b] < left) left -= hist[b--];
                sh_prefix = prefix | (uint32_t)b << shift;
                sh_need = left;
            }
            __syncthreads();
            prefix = sh_prefix;
            need = sh_need;                                  // places left for keys with this prefix
            __syncthreads();
        }
    }
    // above the prefix: kept; equal to it: the first `need`; all of them where there are places for all.
    const bool all = n - last >= old, none = n - last <= 0;
    int64_t done = 0;
    int equal_before = 0;
    for (int64_t base = 0; base < len; base += kSelectThreads) {
        const int64_t i = base + tid;
        const uint32_t key = i < old ? weight_key(w[i]) : 0;
        const bool competes = i < old && !none;
        const bool equal = competes && !all && key == prefix;
        const uint64_t eq = __ballot(equal);
        if (lane == 0) wave_sum[0][wave] = __popcll(eq);
        __syncthreads();
        int rank = equal_before + __popcll(eq & (((uint64_t)1 << lane) - 1));
        int eq_total = 0;
        for (int j = 0; j < kSelectThreads / 64; ++j) {
            if (j < wave) rank += wave_sum[0][j];
            eq_total += wave_sum[0][j];
        }
        equal_before += eq_total;
        const bool take = (i >= old && i < len) || (competes && (all || key > prefix)) || (equal && rank < need);
        const uint64_t tk = __ballot(take);
        if (lane == 0) wave_sum[1][wave] = __popcll(tk);
        __syncthreads();
        int64_t at = done + __popcll(tk & (((uint64_t)1 << lane) - 1));
        for (int j = 0; j < kSelectThreads / 64; ++j) {
            if (j < wave) at += wave_sum[1][j];
            done += wave_sum[1][j];
        }
        if (take && at < n) {
            kept[at] = (int32_t)i;
            nw[at] = w[i];
        }
    }
    for (int64_t i = n + tid; i < a.keep; i += kSelectThreads) kept[i] = -1;
    for (int64_t i = n + tid; i < a.new_weights_stride; i += kSelectThreads) nw[i] = 0.0f;
    if (head == 0 && tid == 0) a.new_lengths[s] = (int32_t)n;
}

constexpr int kMoveThreads = 256;

template <int FORM>
__device__ void move_block(const EvictArgs& a, const int32_t* kept, int count, int64_t s, int head, int64_t to, uint8_t* codes,
                           float* ranges, int64_t* from, float* range_of, float& sh_top)
{
    const int tid = threadIdx.x, D = a.c.head_dim, B = a.c.block_tokens;
    // where each token lies, and its range
    for (int i = tid; i < count; i += kMoveThreads) {
        const int64_t t = kept[i];
        const int64_t block = a.c.block_table[s * a.c.table_blocks + t / B];
        const bool there = block >= 0 && block < a.c.blocks;
        const int64_t at = block * a.c.kv_heads + head;
        from[i] = there ? (at * B + t % B) * D : -1;
        range_of[i] = there ? ranges[at] : 0.0f;
    }
    __syncthreads();
    if (tid < 64) {
        uint32_t top = 0;
        for (int i = tid; i < count; i += 64) top = max(top, __float_as_uint(range_of[i]) & 0x7fffffffu);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        if (tid == 0) sh_top = __uint_as_float(top);
    }
    __syncthreads();
    const float range = sh_top;
    uint8_t* dst = codes + (to * a.c.kv_heads + head) * B * D;
    const int per_row = D / 16;
    for (int i = tid; i < count * per_row; i += kMoveThreads) {
        const int r = i / per_row;
        uint4 w = {0, 0, 0, 0};
        if (from[r] >= 0) w = *reinterpret_cast<const uint4*>(codes + from[r] + (i - r * per_row) * 16);
        const float before = range_of[r];
        if (__float_as_uint(before) != __float_as_uint(range)) w = recode16<FORM>(w, before, range);
        *reinterpret_cast<uint4*>(dst + i * 16) = w;
    }
    if (tid == 0) ranges[to * a.c.kv_heads + head] = range;
}

// One workgroup per new block, key head, and K or V.
__global__ __launch_bounds__(kMoveThreads) void move_kernel(EvictArgs a)
{
    __shared__ int64_t from[128];
    __shared__ float range_of[128];
    __shared__ float sh_top;
    const int64_t s = blockIdx.z, b = blockIdx.x;
    const int head = blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const int64_t n = evict_kept(a, evict_length(a, s));
    const int64_t first = b * a.c.block_tokens;
    if (first >= n) return;
    const int count = (int)(n - first < a.c.block_tokens ? n - first : a.c.block_tokens);
    const int64_t to = a.new_table[s * a.new_table_blocks + b];
    if (to < 0 || to >= a.c.blocks) return;
    const int32_t* kept = a.kept + (s * a.c.kv_heads + head) * a.keep + first;
    uint8_t* codes = static_cast<uint8_t*>(is_v ? a.c.v_codes : a.c.k_codes);
    float* ranges = is_v ? a.c.v_range : a.c.k_range;
    if ((is_v ? a.c.v_form : a.c.k_form) == MNNQ_KV_FP8)
        move_block<MNNQ_KV_FP8>(a, kept, count, s, head, to, codes, ranges, from, range_of, sh_top);
    else
        move_block<MNNQ_KV_INT8>(a, kept, count, s, head, to, codes, ranges, from, range_of, sh_top);
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
    if (!start && a.each == 1) append_kernel<64><<<grid, 64, 0, st>>>(a);
    else append_kernel<256><<<grid, 256, 0, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    return MNNQ_OK;
}

int launch_kv_evict(const mnnq_kv_cache& c, const float* weights, int64_t weights_stride, int64_t keep, int64_t recent,
                    const int32_t* new_table, int64_t new_table_blocks, int32_t* kept, int32_t* new_lengths,
                    float* new_weights, int64_t new_weights_stride, hipStream_t st)
{
    const EvictArgs a{c,    weights,     weights_stride, keep,        recent,            new_table, new_table_blocks,
                      kept, new_lengths, new_weights,    new_weights_stride};
    select_kernel<<<dim3((unsigned)c.kv_heads, (unsigned)c.sequences), kSelectThreads, 0, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    const int64_t room = new_table_blocks, most = (keep + c.block_tokens - 1) / c.block_tokens;
    const dim3 grid((unsigned)(room < most ? room : most), (unsigned)(2 * c.kv_heads), (unsigned)c.sequences);
    move_kernel<<<grid, kMoveThreads, 0, st>>>(a);
    MNNQ_HIP_TRY(hipGetLastError());
    return MNNQ_OK;
}

}  // namespace mnnq
