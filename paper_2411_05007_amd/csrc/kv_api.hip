// C-ABI entry points of the paged 8-bit cache of keys and values: argument checks and launches.
#include <hip/hip_runtime.h>

#include "../../include/svdq.h"
#include "kernels.h"
#include "layout.h"

namespace {

constexpr int kMaxTokens = 1 << 30;      // of a sequence: positions and key indices are 32-bit with room to add a tile
constexpr int kMaxGridY = 65535;
constexpr int64_t kMostStride = 1 << 25;

int check_shape(const svdq_kv_shape &s) {
    if (s.kv_heads <= 0 || s.head_dim <= 0 || s.page_tokens <= 0) return SVDQ_EINVAL;
    if (s.head_dim != 64 && s.head_dim != 128 && s.head_dim != 256) return SVDQ_EUNSUPPORTED;
    if (s.page_tokens < 32 || s.page_tokens > 1024 || (s.page_tokens & (s.page_tokens - 1))) return SVDQ_EUNSUPPORTED;
    return s.kv_heads > kMaxGridY ? SVDQ_EUNSUPPORTED : SVDQ_OK;
}
int check_cache(const svdq_kv_cache_dev *c) {
    if (!c) return SVDQ_EINVAL;
    const int st = check_shape(c->shape);
    if (st != SVDQ_OK) return st;
    if (c->pages <= 0 || !c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return SVDQ_EINVAL;
    return (((uintptr_t)c->k_codes | (uintptr_t)c->v_codes) & 15) ? SVDQ_EINVAL : SVDQ_OK;
}
int check_tables(const int32_t *cu, const int32_t *len, const int32_t *table, int sequences, int width, int total, int page_tokens) {
    if (sequences < 0 || width < 0 || total < 0) return SVDQ_EINVAL;
    if (sequences == 0 || total == 0) return SVDQ_OK;
    if (!cu || !len || !table || width == 0) return SVDQ_EINVAL;
    if (((uintptr_t)cu | (uintptr_t)len | (uintptr_t)table) & 3) return SVDQ_EINVAL;
    if (sequences > kMaxGridY || (long long)width * page_tokens > kMaxTokens) return SVDQ_EUNSUPPORTED;
    return SVDQ_OK;
}
int check_rope(const svdq_kv_rope *r, int dim) {
    if (!r) return SVDQ_OK;
    if (!r->table || ((uintptr_t)r->table & 15) || r->positions <= 0 || r->dims <= 0 || r->dims > dim || r->dims % 16 != 0) return SVDQ_EINVAL;
    return SVDQ_OK;
}
int check_rows(const svdq_kv_rows *r) {
    if (!r || !r->data || ((uintptr_t)r->data & 15)) return SVDQ_EINVAL;
    if (r->token_stride % 8 != 0 || r->head_stride % 8 != 0 || r->token_stride < 0 || r->head_stride < 0) return SVDQ_EINVAL;
    return r->token_stride > kMostStride ? SVDQ_EUNSUPPORTED : SVDQ_OK;      // (the rows of a block are addressed with 32 bits from its first)
}
svdq::KvCache cache_of(const svdq_kv_cache_dev *c) {
    svdq::KvCache k{};
    k.k = static_cast<uint8_t *>(c->k_codes);
    k.v = static_cast<uint8_t *>(c->v_codes);
    k.ks = static_cast<uint8_t *>(c->k_scales);
    k.vs = static_cast<uint8_t *>(c->v_scales);
    k.pages = c->pages;
    k.heads = c->shape.kv_heads;
    k.dim = c->shape.head_dim;
    k.page_shift = __builtin_ctz((unsigned)c->shape.page_tokens);
    return k;
}
svdq::KvBatch batch_of(const svdq_kv_batch *b) { return svdq::KvBatch{b->cu_new, b->kv_len, b->block_table, b->sequences, b->table_width, b->new_tokens}; }
svdq::KvRope rope_of(const svdq_kv_rope *r) {
    return r ? svdq::KvRope{r->table, r->positions, r->dims, r->interleaved != 0} : svdq::KvRope{nullptr, 0, 0, 0};
}
svdq::KvRows rows_of(const svdq_kv_rows *r) { return svdq::KvRows{static_cast<const uint16_t *>(r->data), r->token_stride, r->head_stride}; }
int done(hipError_t e) { return e == hipSuccess ? SVDQ_OK : svdq::record_hip_error(e); }

}  // namespace

extern "C" {

int svdq_kv_cache_sizes(const svdq_kv_shape *shape, int pages, svdq_kv_sizes *out) {
    if (!shape || !out || pages <= 0) return SVDQ_EINVAL;
    const int st = check_shape(*shape);
    if (st != SVDQ_OK) return st;
    out->codes = (size_t)pages * shape->kv_heads * shape->page_tokens * shape->head_dim;
    out->scales = (size_t)pages * shape->kv_heads * (shape->page_tokens / 32);
    return SVDQ_OK;
}

int svdq_kv_append(const svdq_kv_cache_dev *cache, const svdq_kv_batch *batch, const svdq_kv_rope *rope, const svdq_kv_rows *k,
                   const svdq_kv_rows *v, void *hip_stream) {
    int st = check_cache(cache);
    if (st != SVDQ_OK) return st;
    if (!batch) return SVDQ_EINVAL;
    st = check_tables(batch->cu_new, batch->kv_len, batch->block_table, batch->sequences, batch->table_width, batch->new_tokens, cache->shape.page_tokens);
    if (st != SVDQ_OK) return st;
    if ((st = check_rope(rope, cache->shape.head_dim)) != SVDQ_OK) return st;
    if (batch->sequences == 0 || batch->new_tokens == 0) return SVDQ_OK;
    if ((st = check_rows(k)) != SVDQ_OK || (st = check_rows(v)) != SVDQ_OK) return st;
    const svdq::KvAppendParams p{cache_of(cache), batch_of(batch), rope_of(rope), rows_of(k), rows_of(v)};
    return done(svdq::launch_kv_append(p, static_cast<hipStream_t>(hip_stream)));
}

size_t svdq_kv_attention_workspace_bytes(const svdq_kv_shape *shape, int q_heads, int sequences, int max_new, int max_len) {
    if (!shape || check_shape(*shape) != SVDQ_OK || q_heads <= 0 || q_heads % shape->kv_heads != 0 || sequences < 0 || max_new < 0 || max_len < 0 || max_len > kMaxTokens)
        return 0;
    return svdq::kv_workspace_bytes(sequences, shape->kv_heads, q_heads / shape->kv_heads, shape->head_dim, max_new, max_len);
}

int svdq_kv_attention(const svdq_kv_cache_dev *cache, const svdq_kv_batch *batch, const svdq_kv_rope *rope, const svdq_kv_rows *q, int q_heads,
                      float scale, int causal, int window, void *out, void *workspace, size_t workspace_bytes, void *hip_stream) {
    int st = check_cache(cache);
    if (st != SVDQ_OK) return st;
    const svdq_kv_shape &s = cache->shape;
    if (!batch || q_heads <= 0 || q_heads % s.kv_heads != 0 || window < 0 || batch->max_new < 0 || batch->max_len < 0) return SVDQ_EINVAL;
    st = check_tables(batch->cu_new, batch->kv_len, batch->block_table, batch->sequences, batch->table_width, batch->new_tokens, s.page_tokens);
    if (st != SVDQ_OK) return st;
    if ((st = check_rope(rope, s.head_dim)) != SVDQ_OK) return st;
    if (batch->sequences == 0 || batch->new_tokens == 0) return SVDQ_OK;
    if ((st = check_rows(q)) != SVDQ_OK) return st;
    if (!out || ((uintptr_t)out & 15) || !workspace || ((uintptr_t)workspace & 255)) return SVDQ_EINVAL;
    if (batch->max_len > kMaxTokens || (long long)batch->new_tokens * (q_heads / s.kv_heads) > 0x7fffffffll - (1 << 20)) return SVDQ_EUNSUPPORTED;
    const svdq::KvPlan plan = svdq::plan_kv_attention(batch->sequences, s.kv_heads, q_heads / s.kv_heads, s.head_dim, batch->max_new, batch->max_len, causal ? window : 0,
                                                          batch->new_tokens);
    if (plan.few && (long long)batch->sequences * plan.row_tiles > kMaxGridY) return SVDQ_EUNSUPPORTED;
    // (the size that the query gives, of which a call with fewer tokens or a window may need less: what is refused does not hang on those)
    if (workspace_bytes < svdq::kv_workspace_bytes(batch->sequences, s.kv_heads, q_heads / s.kv_heads, s.head_dim, batch->max_new, batch->max_len)) return SVDQ_ENOSPACE;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    svdq::KvAttentionParams p{};
    p.cache = cache_of(cache);
    p.batch = batch_of(batch);
    p.rope = rope_of(rope);
    p.q = rows_of(q);
    p.out = static_cast<uint16_t *>(out);
    p.q_heads = q_heads;
    p.group = q_heads / s.kv_heads;
    p.scale = scale * 1.4426950408889634f;      // exp(x) = exp2(x log2(e))
    p.causal = causal != 0;
    p.window = window;
    p.tile_rows = plan.tile_rows;
    p.parts = plan.parts;
    p.row_tiles = plan.row_tiles;
    p.row_cap = plan.row_cap;
    p.chunk_blocks = plan.chunk_blocks;
    p.chunks = plan.chunks;
    p.partial = reinterpret_cast<float *>(ws);
    p.part_ml = reinterpret_cast<float *>(ws + plan.ml_off);
    p.least_rows = plan.few ? svdq::kKvFewRows + 1 : 0;
    p.most_rows = plan.many ? svdq::kKvFewRows : 0x7fffffff;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (plan.many) {
        const long long items = (long long)batch->new_tokens * p.group / plan.tile_rows + batch->sequences;
        if (items * s.kv_heads > 0x7fffffffll) return SVDQ_EUNSUPPORTED;
        const hipError_t e = svdq::launch_kv_attention_tile(p, stream);
        if (e != hipSuccess) return done(e);
    }
    if (!plan.few || plan.row_tiles == 0) return SVDQ_OK;
    // (behind the other kernel: where that one's parts are added, it is for every token of the batch, and what it makes of those without parts is written over here)
    p.partial = reinterpret_cast<float *>(ws + plan.few_off);
    p.arrived = reinterpret_cast<unsigned long long *>(ws + plan.words_off);
    return done(svdq::launch_kv_attention_rows(p, stream));
}

int svdq_kv_gather(const svdq_kv_cache_dev *cache, const int32_t *first_token, const int32_t *cu_rows, const int32_t *block_table, int sequences,
                   int table_width, int rows, void *out_k, void *out_v, void *hip_stream) {
    int st = check_cache(cache);
    if (st != SVDQ_OK) return st;
    st = check_tables(cu_rows, first_token, block_table, sequences, table_width, rows, cache->shape.page_tokens);
    if (st != SVDQ_OK) return st;
    if (sequences == 0 || rows == 0 || (!out_k && !out_v)) return SVDQ_OK;
    if (((uintptr_t)out_k | (uintptr_t)out_v) & 15) return SVDQ_EINVAL;
    const svdq::KvGatherParams p{cache_of(cache), svdq::KvBatch{cu_rows, first_token, block_table, sequences, table_width, rows}, static_cast<uint16_t *>(out_k),
                                 static_cast<uint16_t *>(out_v)};
    return done(svdq::launch_kv_gather(p, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
