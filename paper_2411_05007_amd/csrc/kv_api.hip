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
int check_norm(const svdq_kv_norm *n) {
    if (!n) return SVDQ_OK;
    if (((uintptr_t)n->q_weight | (uintptr_t)n->k_weight | (uintptr_t)n->q_first | (uintptr_t)n->k_first) & 15) return SVDQ_EINVAL;
    return n->first_tokens < 0 || !(n->eps >= 1e-30f && n->eps <= 3.4028235e38f) ? SVDQ_EINVAL : SVDQ_OK;
}
svdq::KvNorm norm_of(const svdq_kv_norm *n, const float *weight, const float *first, int dim) {
    return svdq::KvNorm{weight, first, n->per_head ? dim : 0, n->first_tokens, n->eps, 1};
}
svdq::KvRows rows_of(const svdq_kv_rows *r) { return svdq::KvRows{static_cast<const uint16_t *>(r->data), r->token_stride, r->head_stride}; }
int check_pool(const svdq_kv_pool_dev *p) {
    if (!p || !p->refs || ((uintptr_t)p->refs & 3) || p->pages <= 0 || p->page_tokens <= 0) return SVDQ_EINVAL;
    return p->page_tokens < 32 || p->page_tokens > 1024 || (p->page_tokens & (p->page_tokens - 1)) ? SVDQ_EUNSUPPORTED : SVDQ_OK;
}
svdq::KvPool pool_of(const svdq_kv_pool_dev *p) { return svdq::KvPool{p->refs, p->pages, __builtin_ctz((unsigned)p->page_tokens)}; }
// a table of `sequences` rows that is written
int check_table(const int32_t *table, int sequences, int width, int page_tokens) {
    if (sequences < 0 || width < 0) return SVDQ_EINVAL;
    if (sequences == 0) return SVDQ_OK;
    if (!table || ((uintptr_t)table & 3) || width == 0) return SVDQ_EINVAL;
    return sequences > kMaxGridY || (long long)width * page_tokens > kMaxTokens ? SVDQ_EUNSUPPORTED : SVDQ_OK;
}
bool overlap(const void *a, size_t a_bytes, const void *b, size_t b_bytes) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + b_bytes && y < x + a_bytes;
}
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
    return svdq_kv_append_normed(cache, batch, nullptr, rope, k, v, hip_stream);
}

int svdq_kv_append_normed(const svdq_kv_cache_dev *cache, const svdq_kv_batch *batch, const svdq_kv_norm *norm, const svdq_kv_rope *rope, const svdq_kv_rows *k,
                          const svdq_kv_rows *v, void *hip_stream) {
    int st = check_cache(cache);
    if (st != SVDQ_OK) return st;
    if (!batch) return SVDQ_EINVAL;
    st = check_tables(batch->cu_new, batch->kv_len, batch->block_table, batch->sequences, batch->table_width, batch->new_tokens, cache->shape.page_tokens);
    if (st != SVDQ_OK) return st;
    if ((st = check_rope(rope, cache->shape.head_dim)) != SVDQ_OK) return st;
    if ((st = check_norm(norm)) != SVDQ_OK) return st;
    if (batch->sequences == 0 || batch->new_tokens == 0) return SVDQ_OK;
    if ((st = check_rows(k)) != SVDQ_OK || (st = check_rows(v)) != SVDQ_OK) return st;
    svdq::KvAppendParams p{cache_of(cache), batch_of(batch), rope_of(rope), rows_of(k), rows_of(v), {}};
    if (norm) p.norm = norm_of(norm, norm->k_weight, norm->k_first, cache->shape.head_dim);
    return done(svdq::launch_kv_append(p, static_cast<hipStream_t>(hip_stream)));
}

size_t svdq_kv_attention_workspace_bytes(const svdq_kv_shape *shape, int q_heads, int sequences, int max_new, int max_len) {
    if (!shape || check_shape(*shape) != SVDQ_OK || q_heads <= 0 || q_heads % shape->kv_heads != 0 || sequences < 0 || max_new < 0 || max_len < 0 || max_len > kMaxTokens)
        return 0;
    return svdq::kv_workspace_bytes(sequences, shape->kv_heads, q_heads / shape->kv_heads, shape->head_dim, max_new, max_len);
}

int svdq_kv_attention(const svdq_kv_cache_dev *cache, const svdq_kv_batch *batch, const svdq_kv_rope *rope, const svdq_kv_rows *q, int q_heads,
                      float scale, int causal, int window, void *out, void *workspace, size_t workspace_bytes, void *hip_stream) {
    return svdq_kv_attention_normed(cache, batch, nullptr, rope, q, q_heads, scale, causal, window, 0, out, workspace, workspace_bytes, hip_stream);
}

int svdq_kv_attention_normed(const svdq_kv_cache_dev *cache, const svdq_kv_batch *batch, const svdq_kv_norm *norm, const svdq_kv_rope *rope, const svdq_kv_rows *q,
                             int q_heads, float scale, int causal, int window, int sinks, void *out, void *workspace, size_t workspace_bytes, void *hip_stream) {
    int st = check_cache(cache);
    if (st != SVDQ_OK) return st;
    const svdq_kv_shape &s = cache->shape;
    if (!batch || q_heads <= 0 || q_heads % s.kv_heads != 0 || window < 0 || sinks < 0 || batch->max_new < 0 || batch->max_len < 0) return SVDQ_EINVAL;
    st = check_tables(batch->cu_new, batch->kv_len, batch->block_table, batch->sequences, batch->table_width, batch->new_tokens, s.page_tokens);
    if (st != SVDQ_OK) return st;
    if ((st = check_rope(rope, s.head_dim)) != SVDQ_OK || (st = check_norm(norm)) != SVDQ_OK) return st;
    if (batch->sequences == 0 || batch->new_tokens == 0) return SVDQ_OK;
    if ((st = check_rows(q)) != SVDQ_OK) return st;
    if (!out || ((uintptr_t)out & 15) || !workspace || ((uintptr_t)workspace & 255)) return SVDQ_EINVAL;
    if (batch->max_len > kMaxTokens || (long long)batch->new_tokens * (q_heads / s.kv_heads) > 0x7fffffffll - (1 << 20)) return SVDQ_EUNSUPPORTED;
    if (!causal || window == 0) sinks = 0;
    if (sinks > kMaxTokens) sinks = kMaxTokens;
    // (keys that a row sees: whole blocks of the first ones, where a window is)
    const long long wide = causal ? (long long)window + ((sinks + 31) & ~31) : 0;
    const svdq::KvPlan plan = svdq::plan_kv_attention(batch->sequences, s.kv_heads, q_heads / s.kv_heads, s.head_dim, batch->max_new, batch->max_len,
                                                      wide > 0x7fffffffll ? 0x7fffffff : (int)wide, batch->new_tokens, norm || sinks > 0);
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
    p.sinks = sinks;
    if (norm) p.norm = norm_of(norm, norm->q_weight, norm->q_first, s.head_dim);
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

int svdq_kv_pages_release(const svdq_kv_pool_dev *pool, int32_t *block_table, const int32_t *first_token, const int32_t *end_token, int sequences, int table_width,
                          void *hip_stream) {
    int st = check_pool(pool);
    if (st != SVDQ_OK || (st = check_table(block_table, sequences, table_width, pool->page_tokens)) != SVDQ_OK) return st;
    if (((uintptr_t)first_token | (uintptr_t)end_token) & 3) return SVDQ_EINVAL;
    if (sequences == 0) return SVDQ_OK;
    return done(svdq::launch_kv_release(pool_of(pool), block_table, first_token, end_token, sequences, table_width, static_cast<hipStream_t>(hip_stream)));
}

int svdq_kv_pages_fork(const svdq_kv_pool_dev *pool, const int32_t *from_table, const int32_t *from_len, int from_sequences, int from_width, const int32_t *parent,
                       int32_t *to_table, int32_t *to_len, int sequences, int to_width, void *hip_stream) {
    int st = check_pool(pool);
    if (st != SVDQ_OK || (st = check_table(from_table, from_sequences, from_width, pool->page_tokens)) != SVDQ_OK ||
        (st = check_table(to_table, sequences, to_width, pool->page_tokens)) != SVDQ_OK)
        return st;
    if (sequences == 0) return SVDQ_OK;
    if (!parent || !to_len || (from_sequences > 0 && !from_len) || (((uintptr_t)from_len | (uintptr_t)parent | (uintptr_t)to_len) & 3)) return SVDQ_EINVAL;
    // (rows are read while others are written)
    const size_t from_bytes = (size_t)from_sequences * from_width * 4, to_bytes = (size_t)sequences * to_width * 4;
    const size_t each = (size_t)sequences * 4;
    if (overlap(from_table, from_bytes, to_table, to_bytes) || overlap(from_len, (size_t)from_sequences * 4, to_len, each)) return SVDQ_EINVAL;
    if (overlap(parent, each, to_len, each) || overlap(parent, each, to_table, to_bytes)) return SVDQ_EINVAL;
    const svdq::KvForkParams p{pool_of(pool), from_table, from_len, parent, to_table, to_len, from_sequences, from_width, sequences, to_width};
    return done(svdq::launch_kv_fork(p, static_cast<hipStream_t>(hip_stream)));
}

size_t svdq_kv_pages_reserve_workspace_bytes(const svdq_kv_pool_dev *pool, int sequences, int table_width) {
    if (!pool || pool->pages <= 0 || sequences < 0 || table_width < 0) return 0;
    return svdq::plan_kv_reserve(pool->pages, sequences, table_width).total;
}

int svdq_kv_pages_reserve(const svdq_kv_pool_dev *pool, const svdq_kv_cache_dev *cache, const svdq_kv_batch *batch, int32_t *copies, int32_t *missing, void *workspace,
                          size_t workspace_bytes, void *hip_stream) {
    int st = check_pool(pool);
    if (st != SVDQ_OK || (cache && (st = check_cache(cache)) != SVDQ_OK)) return st;
    if (!batch || (cache && (cache->pages < pool->pages || cache->shape.page_tokens != pool->page_tokens))) return SVDQ_EINVAL;
    if ((st = check_tables(batch->cu_new, batch->kv_len, batch->block_table, batch->sequences, batch->table_width, batch->new_tokens, pool->page_tokens)) != SVDQ_OK) return st;
    if (((uintptr_t)copies | (uintptr_t)missing) & 3) return SVDQ_EINVAL;
    if (batch->sequences > 0 && (!batch->cu_new || !batch->kv_len || !batch->block_table || batch->table_width == 0 || !workspace || ((uintptr_t)workspace & 255))) return SVDQ_EINVAL;
    if (batch->sequences > kMaxGridY) return SVDQ_EUNSUPPORTED;
    if (batch->sequences == 0 && !missing) return SVDQ_OK;
    const svdq::KvReservePlan plan = svdq::plan_kv_reserve(pool->pages, batch->sequences, batch->table_width);
    if (batch->sequences > 0 && workspace_bytes < plan.total) return SVDQ_ENOSPACE;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    svdq::KvReserveParams p{};
    p.pool = pool_of(pool);
    if (cache) p.cache = cache_of(cache);
    p.batch = batch_of(batch);
    p.copies = copies;
    p.missing = missing;
    p.free_words = reinterpret_cast<unsigned long long *>(ws);
    p.slice_free = reinterpret_cast<int32_t *>(ws + plan.slice_off);
    p.lack_count = reinterpret_cast<int32_t *>(ws + plan.count_off);
    p.shared = reinterpret_cast<int32_t *>(ws + plan.shared_off);
    p.lacks = reinterpret_cast<unsigned long long *>(ws + plan.lacks_off);
    p.slices = plan.slices;
    p.words = plan.words;
    return done(svdq::launch_kv_reserve(p, static_cast<hipStream_t>(hip_stream)));
}

int svdq_kv_copy_pages(const svdq_kv_cache_dev *to, const svdq_kv_cache_dev *from, const int32_t *copies, int count, void *hip_stream) {
    int st = check_cache(to);
    if (st != SVDQ_OK || (st = check_cache(from)) != SVDQ_OK) return st;
    if (to->shape.kv_heads != from->shape.kv_heads || to->shape.head_dim != from->shape.head_dim || to->shape.page_tokens != from->shape.page_tokens) return SVDQ_EINVAL;
    if (count < 0 || (count > 0 && (!copies || ((uintptr_t)copies & 3)))) return SVDQ_EINVAL;
    if (count == 0) return SVDQ_OK;
    return done(svdq::launch_kv_copy_pages(cache_of(to), cache_of(from), copies, count, static_cast<hipStream_t>(hip_stream)));
}

size_t svdq_kv_compact_workspace_bytes(const svdq_kv_shape *shape, int sequences, int moves) {
    if (!shape || check_shape(*shape) != SVDQ_OK || sequences < 0 || moves < 0) return 0;
    const size_t blocks = svdq::kv_compact_items(moves, sequences) * shape->kv_heads;
    return blocks == 0 ? 256 : blocks * 64 * shape->head_dim + (2 * blocks + 255) / 256 * 256;
}

int svdq_kv_compact(const svdq_kv_cache_dev *to, const svdq_kv_cache_dev *from, const svdq_kv_moves *moves, const svdq_kv_rope *rope, void *workspace,
                    size_t workspace_bytes, void *hip_stream) {
    int st = check_cache(to);
    if (st != SVDQ_OK || (st = check_cache(from)) != SVDQ_OK) return st;
    if (!moves || to->shape.kv_heads != from->shape.kv_heads || to->shape.head_dim != from->shape.head_dim) return SVDQ_EINVAL;
    if ((st = check_tables(moves->cu_moves, moves->to_first, moves->to_table, moves->sequences, moves->to_width, moves->moves, to->shape.page_tokens)) != SVDQ_OK) return st;
    if ((st = check_tables(moves->cu_moves, moves->from_token, moves->from_table, moves->sequences, moves->from_width, moves->moves, from->shape.page_tokens)) != SVDQ_OK) return st;
    if ((st = check_rope(rope, to->shape.head_dim)) != SVDQ_OK) return st;
    if (moves->sequences > kMaxGridY) return SVDQ_EUNSUPPORTED;
    if (workspace) {
        if ((uintptr_t)workspace & 255) return SVDQ_EINVAL;
        if (workspace_bytes < svdq_kv_compact_workspace_bytes(&to->shape, moves->sequences, moves->moves)) return SVDQ_ENOSPACE;
    }
    if (moves->sequences == 0 || moves->moves == 0) return SVDQ_OK;
    svdq::KvCompactParams p{};
    p.to = cache_of(to);
    p.from = cache_of(from);
    p.batch = svdq::KvBatch{moves->cu_moves, moves->to_first, moves->to_table, moves->sequences, moves->to_width, moves->moves};
    p.from_token = moves->from_token;
    p.from_table = moves->from_table;
    p.from_width = moves->from_width;
    p.per_head = moves->per_head != 0;
    p.rope = rope_of(rope);
    p.stage = static_cast<uint8_t *>(workspace);
    if (workspace) p.stage_bytes = p.stage + svdq::kv_compact_items(moves->moves, moves->sequences) * to->shape.kv_heads * 64 * to->shape.head_dim;
    return done(svdq::launch_kv_compact(p, static_cast<hipStream_t>(hip_stream)));
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
