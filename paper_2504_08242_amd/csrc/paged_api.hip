// Entry points of the paged-cache operators: argument validation, dispatch.  No device memory is allocated here.
#include "paged.h"

namespace {

using jup::set_error;

constexpr int32_t kMostIndexed = 1 << 30;  // entries that a kernel goes through in steps of a workgroup, in 32 bits

bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Empty string when the pool is usable, otherwise the reason.
const char* check_pool(const jup_paged_pool_t* p) {
    if (!p) return "pool is NULL";
    if (p->dtype != JUP_F32 && p->dtype != JUP_BF16) return "the pool's dtype must be JUP_F32 or JUP_BF16";
    if (p->n_blocks <= 0 || p->n_kv_heads <= 0 || p->head_dim <= 0) return "sizes of the pool must be positive";
    if (p->page_size < 8 || p->page_size > jup::kMaxPageSize || (p->page_size & (p->page_size - 1)))
        return "page_size must be a power of two, 8 .. 65536";
    if ((int64_t)p->n_blocks * p->page_size > INT32_MAX) return "n_blocks * page_size exceeds 2^31 - 1";
    if (!p->k || !p->v) return "k and v of the pool must not be NULL";
    if (p->block_stride < 0 || p->head_stride < 0 || p->slot_stride < 0) return "strides must not be negative";
    if (p->dtype == JUP_BF16) {
        if (p->head_dim != 128) return "JUP_BF16 requires head_dim == 128";
        if (off16(p->k) || off16(p->v)) return "k and v of the pool must be 16-byte aligned";
        if ((p->block_stride | p->head_stride | p->slot_stride) & 7) return "strides of a JUP_BF16 pool must be multiples of 8";
        // (a page's rows are addressed by 32-bit byte offsets)
        if (p->slot_stride * 2 > (1 << 26)) return "slot_stride of a JUP_BF16 pool must not exceed 2^25";
    } else if (p->head_dim > 256 || (p->head_dim & 1)) {
        return "head_dim must be even and at most 256";
    }
    return "";
}

bool bad_rows(int dtype, const void* p, int64_t row_stride, int64_t head_stride) {
    return row_stride < 0 || head_stride < 0 || (dtype == JUP_BF16 && (off16(p) || ((row_stride | head_stride) & 7)));
}

jup_status_t launched(const char* me, hipError_t e) {
    return e == hipSuccess ? JUP_OK : set_error(JUP_EDEVICE, "%s: %s", me, hipGetErrorString(e));
}

const char* check_workspace(const void* p, size_t bytes) {
    if (!p || ((uintptr_t)p % jup::kAlign)) return "workspace must be non-NULL and 256-byte aligned";
    if (bytes < jup_paged_workspace_bytes()) return "workspace is smaller than jup_paged_workspace_bytes()";
    return "";
}

jup_status_t check_attention(const char* me, const jup_paged_pool_t* pool, const jup_paged_attention_t* a) {
    const char* why = check_pool(pool);
    if (*why) return set_error(JUP_EINVAL, "%s: %s", me, why);
    if (!a) return set_error(JUP_EINVAL, "%s: args is NULL", me);
    if (a->n_seqs < 0 || a->n_seqs > JUP_PAGED_MAX_SEQS)
        return set_error(JUP_EINVAL, "%s: n_seqs=%d is outside 0..%d", me, a->n_seqs, JUP_PAGED_MAX_SEQS);
    if (a->n_rows < 0 || a->max_new < 0) return set_error(JUP_EINVAL, "%s: n_rows and max_new must not be negative", me);
    if (a->n_heads <= 0 || a->n_heads % pool->n_kv_heads)
        return set_error(JUP_EINVAL, "%s: n_heads=%d must be a positive multiple of n_kv_heads=%d", me, a->n_heads, pool->n_kv_heads);
    if ((int64_t)a->n_rows * a->n_heads > INT32_MAX) return set_error(JUP_EINVAL, "%s: n_rows * n_heads exceeds 2^31 - 1", me);
    if (a->table_width < 0 || (int64_t)a->table_width * pool->page_size > INT32_MAX - 255)
        return set_error(JUP_EINVAL, "%s: table_width=%d is negative, or table_width * page_size exceeds 2^31 - 256", me, a->table_width);
    if (a->table_stride < a->table_width) return set_error(JUP_EINVAL, "%s: table_stride is shorter than table_width", me);
    if (!(a->scale > 0.0f) || a->scale > 1e38f) return set_error(JUP_EINVAL, "%s: scale must be positive and at most 1e38", me);
    if (a->n_rows == 0 || a->n_seqs == 0) return JUP_OK;
    if (!a->q || !a->out || !a->row_start || !a->lengths || (a->table_width > 0 && !a->table))
        return set_error(JUP_EINVAL, "%s: the rows, row_start, lengths and table must not be NULL", me);
    if (bad_rows(pool->dtype, a->q, a->q_row_stride, a->q_head_stride) || bad_rows(pool->dtype, a->out, a->out_row_stride, a->out_head_stride))
        return set_error(JUP_EINVAL, "%s: strides must not be negative; JUP_BF16: tensors 16-byte aligned, strides multiples of 8", me);
    if (pool->dtype == JUP_BF16 && *(why = check_workspace(a->workspace, a->workspace_bytes))) return set_error(JUP_EINVAL, "%s: %s", me, why);
    return JUP_OK;
}

}  // namespace

extern "C" {

jup_status_t jup_paged_extend(const jup_paged_extend_t* a, void* stream) {
    const char* me = "jup_paged_extend";
    if (!a) return set_error(JUP_EINVAL, "%s: args is NULL", me);
    if (a->n_seqs < 0 || a->n_seqs > JUP_PAGED_MAX_SEQS)
        return set_error(JUP_EINVAL, "%s: n_seqs=%d is outside 0..%d", me, a->n_seqs, JUP_PAGED_MAX_SEQS);
    if (a->page_size < 8 || a->page_size > jup::kMaxPageSize || (a->page_size & (a->page_size - 1)))
        return set_error(JUP_EINVAL, "%s: page_size=%d must be a power of two, 8 .. 65536", me, a->page_size);
    if (a->table_width < 0 || (int64_t)a->table_width * a->page_size > INT32_MAX - 255)
        return set_error(JUP_EINVAL, "%s: table_width=%d is negative, or table_width * page_size exceeds 2^31 - 256", me, a->table_width);
    if (a->table_stride < a->table_width) return set_error(JUP_EINVAL, "%s: table_stride is shorter than table_width", me);
    if (a->n_free < 0 || a->n_free > kMostIndexed) return set_error(JUP_EINVAL, "%s: n_free=%d is outside 0..2^30", me, a->n_free);
    if (a->max_rows < 0) return set_error(JUP_EINVAL, "%s: max_rows=%d is negative", me, a->max_rows);
    if (!a->free_count || !a->row_start || !a->new_free_count || !a->status)
        return set_error(JUP_EINVAL, "%s: free_count, row_start, new_free_count and status must not be NULL", me);
    if (a->n_free > 0 && !a->free_blocks) return set_error(JUP_EINVAL, "%s: free_blocks is NULL", me);
    if (a->max_rows > 0 && (!a->positions || !a->slots)) return set_error(JUP_EINVAL, "%s: positions and slots must not be NULL", me);
    if (a->n_seqs > 0 && (!a->lengths || !a->n_new || !a->owned || !a->new_lengths || !a->new_owned || (a->table_width > 0 && !a->table)))
        return set_error(JUP_EINVAL, "%s: lengths, n_new, owned, table, new_lengths and new_owned must not be NULL", me);
    return launched(me, jup::launch_paged_extend(*a, (hipStream_t)stream));
}

jup_status_t jup_paged_append(const jup_paged_pool_t* pool, const jup_paged_append_t* a, void* stream) {
    const char* me = "jup_paged_append";
    const char* why = check_pool(pool);
    if (*why) return set_error(JUP_EINVAL, "%s: %s", me, why);
    if (!a) return set_error(JUP_EINVAL, "%s: args is NULL", me);
    if (a->n_rows < 0) return set_error(JUP_EINVAL, "%s: n_rows=%d is negative", me, a->n_rows);
    if (!(a->rope_theta >= 0.0f) || a->rope_theta > 3e38f) return set_error(JUP_EINVAL, "%s: rope_theta must be 0 or positive and finite", me);
    if (a->rope_theta == 0.0f && (a->q || a->q_out)) return set_error(JUP_EINVAL, "%s: q goes with a rotation (rope_theta is 0)", me);
    if (!a->q != !a->q_out) return set_error(JUP_EINVAL, "%s: q and q_out go together", me);
    if (a->q && a->n_heads <= 0) return set_error(JUP_EINVAL, "%s: n_heads must be positive", me);
    if (a->n_rows == 0) return JUP_OK;
    if (!a->k || !a->v || !a->slots) return set_error(JUP_EINVAL, "%s: k, v and slots must not be NULL", me);
    if (a->rope_theta > 0.0f && !a->positions) return set_error(JUP_EINVAL, "%s: positions is NULL", me);
    if (bad_rows(pool->dtype, a->k, a->k_row_stride, a->k_head_stride) || bad_rows(pool->dtype, a->v, a->v_row_stride, a->v_head_stride) ||
        (a->q && (bad_rows(pool->dtype, a->q, a->q_row_stride, a->q_head_stride) || bad_rows(pool->dtype, a->q_out, a->q_out_row_stride, a->q_out_head_stride))))
        return set_error(JUP_EINVAL, "%s: strides must not be negative; JUP_BF16: tensors 16-byte aligned, strides multiples of 8", me);
    return launched(me, jup::launch_paged_append(*pool, *a, (hipStream_t)stream));
}

jup_status_t jup_paged_attention(const jup_paged_pool_t* pool, const jup_paged_attention_t* a, void* stream) {
    const char* me = "jup_paged_attention";
    const jup_status_t rc = check_attention(me, pool, a);
    if (rc != JUP_OK || a->n_rows == 0 || a->n_seqs == 0) return rc;
    return launched(me, jup::launch_paged_attention(*pool, *a, (hipStream_t)stream));
}

jup_status_t jup_stage_prefill_paged(jup_stage_t* stage, const void* hidden_in, int32_t n_rows, const jup_paged_batch_t* b,
                                     void* hidden_out, void* stream) {
    const char* me = "jup_stage_prefill_paged";
    if (!stage) return set_error(JUP_EINVAL, "%s: stage is NULL", me);
    if (!b) return set_error(JUP_EINVAL, "%s: batch is NULL", me);
    const jup_stage_config_t& c = stage->cfg;
    if (n_rows < 0) return set_error(JUP_EINVAL, "%s: n_rows=%d is negative", me, n_rows);
    if (n_rows > stage->max_chunk_tokens)
        return set_error(JUP_ECAP, "%s: n_rows=%d exceeds the stage's max_chunk_tokens=%d", me, n_rows, stage->max_chunk_tokens);
    jup::PagedStep step{};
    step.pool = b->pool;
    step.layer_stride = b->layer_stride;
    step.positions = b->positions;
    step.slots = b->slots;
    jup_paged_attention_t& a = step.attention;
    a.n_seqs = b->n_seqs; a.n_rows = n_rows; a.n_heads = c.n_heads; a.max_new = b->max_new; a.table_width = b->table_width;
    a.table_stride = b->table_stride; a.row_start = b->row_start; a.lengths = b->lengths; a.table = b->table;
    a.scale = 1.0f / sqrtf((float)c.head_dim); a.workspace = b->workspace; a.workspace_bytes = b->workspace_bytes;
    a.q = hidden_in; a.out = hidden_out;  // (stand for the stage's own: given or not, aligned or not)
    const jup_status_t rc = check_attention(me, &b->pool, &a);
    if (rc != JUP_OK) return rc;
    if (b->pool.n_kv_heads != c.n_heads || b->pool.head_dim != c.head_dim || (b->pool.dtype == JUP_F32) != (c.dtype == JUP_F32))
        return set_error(JUP_EINVAL, "%s: the pool was made for another configuration", me);
    if (b->layer_stride < 0 || (c.dtype != JUP_F32 && (b->layer_stride & 7)))
        return set_error(JUP_EINVAL, "%s: layer_stride must not be negative, and a multiple of 8 in a JUP_BF16 pool", me);
    if (n_rows == 0) return JUP_OK;
    if (b->n_seqs == 0) return set_error(JUP_EINVAL, "%s: rows without requests", me);
    if (!b->positions || !b->slots) return set_error(JUP_EINVAL, "%s: positions and slots must not be NULL", me);
    hipStream_t s = (hipStream_t)stream;
    return launched(me, c.dtype == JUP_F32
                            ? jup::f32_forward(*stage, (const float*)hidden_in, n_rows, 0, jup::KvView{}, (float*)hidden_out, s, nullptr, &step)
                            : jup::bf16_forward(*stage, hidden_in, n_rows, 0, jup::KvView{}, hidden_out, s, nullptr, nullptr, nullptr, &step));
}

jup_status_t jup_verify_drafts(const jup_verify_drafts_t* a, void* stream) {
    const char* me = "jup_verify_drafts";
    if (!a) return set_error(JUP_EINVAL, "%s: args is NULL", me);
    if (a->n_seqs < 0 || a->n_seqs > JUP_PAGED_MAX_SEQS)
        return set_error(JUP_EINVAL, "%s: n_seqs=%d is outside 0..%d", me, a->n_seqs, JUP_PAGED_MAX_SEQS);
    if (a->n_rows < 0 || a->n_rows > kMostIndexed) return set_error(JUP_EINVAL, "%s: n_rows=%d is outside 0..2^30", me, a->n_rows);
    if (a->vocab <= 0 || a->vocab > (1 << 30)) return set_error(JUP_EINVAL, "%s: vocab=%d is outside 1..2^30", me, a->vocab);
    if (a->probs_dtype != JUP_F32 && a->probs_dtype != JUP_BF16) return set_error(JUP_EINVAL, "%s: probs_dtype must be JUP_F32 or JUP_BF16", me);
    if (a->target_row_stride < 0 || a->draft_row_stride < 0) return set_error(JUP_EINVAL, "%s: strides must not be negative", me);
    if (!a->lengths != !a->new_lengths) return set_error(JUP_EINVAL, "%s: lengths and new_lengths go together", me);
    if (const char* why = check_workspace(a->workspace, a->workspace_bytes); *why) return set_error(JUP_EINVAL, "%s: %s", me, why);
    if (a->n_seqs == 0) return JUP_OK;
    if (!a->row_start || !a->u_sample || !a->n_accepted || !a->next_token)
        return set_error(JUP_EINVAL, "%s: row_start, u_sample, n_accepted and next_token must not be NULL", me);
    if (a->n_rows > 0 && (!a->tokens || !a->target_probs || !a->u_accept))
        return set_error(JUP_EINVAL, "%s: tokens, target_probs and u_accept must not be NULL", me);
    return launched(me, jup::launch_verify_drafts(*a, (hipStream_t)stream));
}

}  // extern "C"
