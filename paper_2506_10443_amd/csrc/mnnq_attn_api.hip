// C-ABI entry points of the attention calls: argument checks (all before the first HIP call), then the launchers.
#include <math.h>

#include "mnnq_attn.h"

namespace mnnq {

namespace {

constexpr int64_t kMaxGridYZ = 65535;
constexpr int64_t kMaxRows = (int64_t)1 << 31;           // tokens are indexed by int32 arrays
constexpr int64_t kMaxTokens = (int64_t)1 << 30;         // of a sequence in a cache
constexpr int64_t kMaxGridX = (int64_t)1 << 24;          // workgroups of 256 in x: 2^32 work items at most
constexpr int64_t kMaxStride = (int64_t)1 << 23;         // 64 rows within 32-bit byte offsets

inline bool misaligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

int check_type(int type) { return type == MNNQ_F16 || type == MNNQ_BF16 ? MNNQ_OK : MNNQ_ERR_UNSUPPORTED; }

int check_heads(int heads, int kv_heads, int head_dim)
{
    if (heads <= 0 || kv_heads <= 0 || head_dim <= 0 || heads % kv_heads != 0) return MNNQ_ERR_SHAPE;
    if (head_dim % 16 != 0 || head_dim > 256 || heads > 4096) return MNNQ_ERR_UNSUPPORTED;
    return MNNQ_OK;
}

// Rows that are not empty: distances that keep 16-byte loads aligned.
int check_rows(int64_t token, int64_t head)
{
    if (token < 0 || head < 0) return MNNQ_ERR_SHAPE;
    if (token % 8 != 0 || head % 8 != 0) return MNNQ_ERR_ALIGN;
    if (token > kMaxStride) return MNNQ_ERR_UNSUPPORTED;
    return MNNQ_OK;
}

Rows rows(const void* p, int64_t token, int64_t head)
{
    return Rows{static_cast<uint16_t*>(const_cast<void*>(p)), token, head};
}

int check_cache(const mnnq_kv_cache* c)
{
    if (!c || !c->k_codes || !c->v_codes || !c->k_range || !c->v_range || !c->block_table || !c->lengths) return MNNQ_ERR_NULL;
    if (c->blocks <= 0 || c->sequences <= 0 || c->table_blocks <= 0) return MNNQ_ERR_SHAPE;
    if (int s = check_heads(c->kv_heads, c->kv_heads, c->head_dim)) return s;
    if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128)
        return MNNQ_ERR_UNSUPPORTED;
    if ((c->k_form != MNNQ_KV_INT8 && c->k_form != MNNQ_KV_FP8) || (c->v_form != MNNQ_KV_INT8 && c->v_form != MNNQ_KV_FP8))
        return MNNQ_ERR_UNSUPPORTED;
    if (c->blocks > kMaxRows || c->sequences > kMaxGridYZ || c->table_blocks > kMaxTokens / c->block_tokens)
        return MNNQ_ERR_UNSUPPORTED;
    if (misaligned(c->k_codes, 16) || misaligned(c->v_codes, 16) || misaligned(c->k_range, 4) || misaligned(c->v_range, 4) ||
        misaligned(c->block_table, 4) || misaligned(c->lengths, 4))
        return MNNQ_ERR_ALIGN;
    return MNNQ_OK;
}

// The most tokens of a sequence that a decode call looks at.
int64_t decode_bound(const mnnq_kv_cache& c, int64_t max_length)
{
    const int64_t room = c.table_blocks * c.block_tokens;
    return max_length > 0 && max_length < room ? max_length : room;
}

int check_decode(const mnnq_kv_cache* c, int64_t tokens, int heads, int64_t max_length)
{
    if (int s = check_cache(c)) return s;
    if (int s = check_heads(heads, c->kv_heads, c->head_dim)) return s;
    if (tokens <= 0 || max_length < 0) return MNNQ_ERR_SHAPE;
    // a row index fits 31 bits, the row tiles of a call the grid
    if (tokens > 65535 || heads / c->kv_heads * tokens > 65535 || (heads / c->kv_heads * tokens + 15) / 16 * c->kv_heads > kMaxGridYZ)
        return MNNQ_ERR_UNSUPPORTED;
    return MNNQ_OK;
}

}  // namespace

}  // namespace mnnq

using namespace mnnq;

extern "C" {

int mnnq_attn_prefill(int type, int64_t sequences, const int32_t* q_start, const int32_t* k_start, int64_t q_tokens,
                      int64_t k_tokens, int heads, int kv_heads, int head_dim, float scale, const void* q, int64_t q_token,
                      int64_t q_head, const void* k, int64_t k_token, int64_t k_head, const void* v, int64_t v_token,
                      int64_t v_head, void* out, int64_t out_token, int64_t out_head, void* stream)
{
    if (!q_start || !k_start || (q_tokens > 0 && (!q || !out)) || (k_tokens > 0 && (!k || !v))) return MNNQ_ERR_NULL;
    if (int s = check_type(type)) return s;
    if (sequences <= 0 || q_tokens < 0 || k_tokens < 0 || !(scale > 0.0f) || !isfinite(scale)) return MNNQ_ERR_SHAPE;
    if (int s = check_heads(heads, kv_heads, head_dim)) return s;
    if (sequences >= kMaxRows || q_tokens >= kMaxRows || k_tokens >= kMaxRows) return MNNQ_ERR_UNSUPPORTED;
    if (q_tokens / 128 + sequences >= kMaxGridX / heads) return MNNQ_ERR_UNSUPPORTED;       // workgroups of a launch
    const int64_t strides[4][2] = {{q_token, q_head}, {k_token, k_head}, {v_token, v_head}, {out_token, out_head}};
    for (const auto& r : strides)
        if (int s = check_rows(r[0], r[1])) return s;
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16) || misaligned(q_start, 4) ||
        misaligned(k_start, 4))
        return MNNQ_ERR_ALIGN;
    if (q_tokens == 0) return MNNQ_OK;
    return launch_attn_prefill(type == MNNQ_BF16, sequences, q_start, k_start, q_tokens, k_tokens, heads, kv_heads, head_dim,
                               scale, rows(q, q_token, q_head), rows(k, k_token, k_head), rows(v, v_token, v_head),
                               rows(out, out_token, out_head), static_cast<hipStream_t>(stream));
}

int mnnq_kv_append(const mnnq_kv_cache* cache, int type, const int32_t* start, int64_t tokens, const void* k,
                   int64_t k_token, int64_t k_head, const void* v, int64_t v_token, int64_t v_head, void* stream)
{
    if (int s = check_cache(cache)) return s;
    if (tokens > 0 && (!k || !v)) return MNNQ_ERR_NULL;
    if (int s = check_type(type)) return s;
    if (tokens < 0 || (!start && tokens % cache->sequences != 0)) return MNNQ_ERR_SHAPE;
    if (tokens >= kMaxRows || tokens / cache->block_tokens + 2 * cache->sequences >= kMaxGridX) return MNNQ_ERR_UNSUPPORTED;
    if (int s = check_rows(k_token, k_head)) return s;
    if (int s = check_rows(v_token, v_head)) return s;
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(start, 4)) return MNNQ_ERR_ALIGN;
    if (tokens == 0) return MNNQ_OK;
    return launch_kv_append(*cache, type == MNNQ_BF16, start, tokens, rows(k, k_token, k_head), rows(v, v_token, v_head),
                            static_cast<hipStream_t>(stream));
}

size_t mnnq_attn_decode_workspace_size(const mnnq_kv_cache* cache, int64_t tokens, int heads, int64_t max_length,
                                       int with_weights)
{
    if (check_decode(cache, tokens, heads, max_length)) return 0;
    return attn_decode_ws_bytes(*cache, tokens, heads, decode_bound(*cache, max_length), with_weights != 0);
}

int mnnq_attn_decode(const mnnq_kv_cache* cache, int type, int64_t tokens, int heads, int64_t max_length, float scale,
                     const void* q, int64_t q_token, int64_t q_head, void* out, int64_t out_token, int64_t out_head,
                     float* weights, int64_t weights_stride, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !out) return MNNQ_ERR_NULL;
    if (int s = check_decode(cache, tokens, heads, max_length)) return s;
    if (int s = check_type(type)) return s;
    if (!(scale > 0.0f) || !isfinite(scale)) return MNNQ_ERR_SHAPE;
    if (int s = check_rows(q_token, q_head)) return s;
    if (int s = check_rows(out_token, out_head)) return s;
    const int64_t bound = decode_bound(*cache, max_length);
    if (weights && weights_stride < bound) return MNNQ_ERR_SIZE;
    if (misaligned(q, 16) || misaligned(out, 16) || misaligned(weights, 4) || misaligned(workspace, 16)) return MNNQ_ERR_ALIGN;
    const size_t need = attn_decode_ws_bytes(*cache, tokens, heads, bound, weights != nullptr);
    if (need > 0 && !workspace) return MNNQ_ERR_NULL;
    if (need > 0 && workspace_bytes < need) return MNNQ_ERR_SIZE;
    return launch_attn_decode(*cache, type == MNNQ_BF16, tokens, heads, bound, scale, rows(q, q_token, q_head),
                              rows(out, out_token, out_head), weights, weights_stride, workspace,
                              static_cast<hipStream_t>(stream));
}

int mnnq_kv_evict(const mnnq_kv_cache* cache, const float* weights, int64_t weights_stride, int64_t keep, int64_t recent,
                  const int32_t* new_table, int64_t new_table_blocks, int32_t* kept, int32_t* new_lengths,
                  float* new_weights, int64_t new_weights_stride, void* stream)
{
    if (int s = check_cache(cache)) return s;
    if (!weights || !new_table || !kept || !new_lengths || !new_weights) return MNNQ_ERR_NULL;
    if (keep <= 0 || recent < 0 || recent > keep || weights_stride <= 0 || new_table_blocks <= 0) return MNNQ_ERR_SHAPE;
    if (new_weights_stride < keep) return MNNQ_ERR_SIZE;
    if (keep > kMaxTokens || keep / cache->block_tokens >= kMaxGridX || new_table_blocks > kMaxTokens / cache->block_tokens)
        return MNNQ_ERR_UNSUPPORTED;
    if (misaligned(weights, 4) || misaligned(new_table, 4) || misaligned(kept, 4) || misaligned(new_lengths, 4) ||
        misaligned(new_weights, 4))
        return MNNQ_ERR_ALIGN;
    // in place, one workgroup would write what another still reads
    if (new_table == cache->block_table || new_lengths == cache->lengths || new_weights == weights) return MNNQ_ERR_UNSUPPORTED;
    return launch_kv_evict(*cache, weights, weights_stride, keep, recent, new_table, new_table_blocks, kept, new_lengths,
                           new_weights, new_weights_stride, static_cast<hipStream_t>(stream));
}

}  // extern "C"
