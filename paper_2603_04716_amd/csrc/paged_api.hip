// C-ABI entry points of the paged key/value cache: argument checks and launches, no state.
#include <math.h>
#include <string.h>

#include "paged.h"

using namespace pd;

static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// The cache and the sequences of a call, checked; view is set on success.
static pd_status check_call(const char *who, const pd_paged_kv *kv, const pd_paged_seqs *q, PagedView *view, int *kind)
{
    if (!kv || !q || !kv->k || !kv->v || (q->n_seqs > 0 && q->n_rows > 0 && (!q->lens || !q->page_table))) {
        set_error("%s: NULL argument", who);
        return PD_ERR_INVALID_ARG;
    }
    if ((kv->dtype != PD_F32 && kv->dtype != PD_BF16) || (kv->e4m3 && kv->dtype != PD_BF16)) {
        set_error("%s: rows are fp32 or bf16, and bf16 beside E4M3 pages", who);
        return PD_ERR_DTYPE;
    }
    if (kv->e4m3 && (!kv->k_scales || !kv->v_scales)) {
        set_error("%s: E4M3 pages need scales", who);
        return PD_ERR_INVALID_ARG;
    }
    if (!aligned16(kv->k) || !aligned16(kv->v)) {
        set_error("%s: pages must be 16-byte aligned", who);
        return PD_ERR_INVALID_ARG;
    }
    const int ps = kv->page_size;
    if ((kv->head_dim != 64 && kv->head_dim != 128) || (ps != 16 && ps != 32 && ps != 64 && ps != 128) || kv->n_pages < 1 ||
        kv->n_kv_heads < 1 || kv->n_kv_heads > 1024) {
        set_error("%s: needs head_dim 64 or 128, page_size 16, 32, 64 or 128, n_pages >= 1 and 1 .. 1024 kv heads (%d, %d, %d, %d)",
                  who, kv->head_dim, ps, kv->n_pages, kv->n_kv_heads);
        return PD_ERR_SHAPE;
    }
    if (q->n_seqs < 0 || q->n_seqs > kPagedMaxSeqs || q->n_rows < 0 || q->n_rows > (1 << 24)) {
        set_error("%s: n_seqs outside 0 .. %d or n_rows outside 0 .. 2^24 (%d, %d)", who, kPagedMaxSeqs, q->n_seqs, q->n_rows);
        return PD_ERR_INVALID_ARG;
    }
    if (q->table_width < 1 || (int64_t)q->table_width * ps > (1 << 30) || (!q->row_starts && q->n_rows < q->n_seqs)) {
        set_error("%s: table_width %d outside 1 .. 2^30 / page_size, or fewer rows than sequences without row_starts", who, q->table_width);
        return PD_ERR_SHAPE;
    }
    *kind = kv->e4m3 ? PAGED_E4M3 : kv->dtype == PD_BF16 ? PAGED_BF16 : PAGED_F32;
    view->k = kv->k; view->v = kv->v; view->k_scales = kv->k_scales; view->v_scales = kv->v_scales;
    view->starts = q->row_starts; view->lens = q->lens; view->table = q->page_table;
    view->n_seqs = q->n_seqs; view->n_rows = q->n_rows; view->width = q->table_width;
    view->ps_log = __builtin_ctz((unsigned)ps); view->n_pages = kv->n_pages; view->Hkv = kv->n_kv_heads;
    return PD_OK;
}

static pd_status check_q_heads(const char *who, const PagedView &p, int n_q_heads)
{
    if (n_q_heads < 1 || n_q_heads > 1024 || n_q_heads % p.Hkv != 0 || (int64_t)p.n_rows * n_q_heads >= (1ll << 31)) {
        set_error("%s: n_q_heads %d is not a multiple of n_kv_heads up to 1024, or n_rows * n_q_heads reaches 2^31", who, n_q_heads);
        return PD_ERR_SHAPE;
    }
    return PD_OK;
}

// a tensor of rows: pointer, stride
static pd_status check_rows(const char *who, const char *what, const void *ptr, int64_t stride, int heads, int hd, int dtype)
{
    if (!ptr || !aligned16(ptr)) {
        set_error("%s: %s is NULL or not 16-byte aligned", who, what);
        return PD_ERR_INVALID_ARG;
    }
    if (stride < (int64_t)heads * hd || stride > (1ll << 31) || stride % (dtype == PD_F32 ? 4 : 8) != 0) {
        set_error("%s: row stride of %s (%lld) is smaller than a row, above 2^31 or not a multiple of 16 bytes", who, what, (long long)stride);
        return PD_ERR_SHAPE;
    }
    return PD_OK;
}

#define CHECK(expr)                       \
    do {                                  \
        const pd_status st_ = (expr);     \
        if (st_ != PD_OK) return st_;     \
    } while (0)

static pd_status launched(const char *who, hipError_t e)
{
    if (e == hipSuccess) return PD_OK;
    set_error("%s: %s", who, hipGetErrorString(e));
    return PD_ERR_DEVICE;
}

extern "C" pd_status pd_paged_append(const pd_paged_kv *kv, const pd_paged_seqs *seqs, const pd_paged_rows *r, void *stream)
{
    static const char who[] = "pd_paged_append";
    PagedAppendArgs a;
    int kind;
    if (!r) {
        set_error("%s: NULL argument", who);
        return PD_ERR_INVALID_ARG;
    }
    CHECK(check_call(who, kv, seqs, &a.p, &kind));
    if (seqs->n_seqs == 0 || seqs->n_rows == 0) return PD_OK;    // tensors of nothing may be NULL
    const int hd = kv->head_dim;
    CHECK(check_rows(who, "k", r->k, r->k_stride, kv->n_kv_heads, hd, kv->dtype));
    CHECK(check_rows(who, "v", r->v, r->v_stride, kv->n_kv_heads, hd, kv->dtype));
    if (r->q) {
        CHECK(check_q_heads(who, a.p, r->n_q_heads));
        CHECK(check_rows(who, "q", r->q, r->q_stride, r->n_q_heads, hd, kv->dtype));
        CHECK(check_rows(who, "q_out", r->q_out, r->q_out_stride, r->n_q_heads, hd, kv->dtype));
    }
    if (!(r->rope_base >= 0.f) || !isfinite(r->rope_base)) {
        set_error("%s: rope_base must be 0 or positive and finite", who);
        return PD_ERR_INVALID_ARG;
    }
    a.q = r->q; a.k = r->k; a.v = r->v; a.q_out = r->q_out;
    a.q_stride = r->q_stride; a.k_stride = r->k_stride; a.v_stride = r->v_stride; a.q_out_stride = r->q_out_stride;
    a.Hq = r->n_q_heads;
    a.rope = r->rope_base > 0.f;
    for (int c = 0; c < 64; ++c)
        a.turns[c] = a.rope && c < hd / 2 ? pow((double)r->rope_base, -2.0 * c / hd) / 6.283185307179586 : 0.0;
    return launched(who, launch_paged_append(kind, hd, a, (hipStream_t)stream));
}

extern "C" pd_status pd_paged_attention_workspace(const pd_paged_kv *kv, const pd_paged_seqs *seqs, int32_t n_q_heads, int64_t *bytes)
{
    static const char who[] = "pd_paged_attention_workspace";
    PagedView p;
    int kind;
    if (!bytes) {
        set_error("%s: NULL argument", who);
        return PD_ERR_INVALID_ARG;
    }
    CHECK(check_call(who, kv, seqs, &p, &kind));
    CHECK(check_q_heads(who, p, n_q_heads));
    *bytes = seqs->n_seqs == 0 || seqs->n_rows == 0 ? 0 : (int64_t)paged_attn_plan(kind, kv->head_dim, p, n_q_heads).bytes;
    return PD_OK;
}

extern "C" pd_status pd_paged_attention(const pd_paged_kv *kv, const pd_paged_seqs *seqs, const void *q, int64_t q_stride, int32_t n_q_heads,
                                        float scale, void *out, void *workspace, int64_t workspace_bytes, void *stream)
{
    static const char who[] = "pd_paged_attention";
    PagedAttnArgs a;
    int kind;
    memset(&a, 0, sizeof(a));
    CHECK(check_call(who, kv, seqs, &a.p, &kind));
    CHECK(check_q_heads(who, a.p, n_q_heads));
    if (seqs->n_seqs == 0 || seqs->n_rows == 0) return PD_OK;
    const int hd = kv->head_dim;
    CHECK(check_rows(who, "q", q, q_stride, n_q_heads, hd, kv->dtype));
    if (!out || !aligned16(out) || !(scale > 0.f) || !isfinite(scale)) {
        set_error("%s: out is NULL or not 16-byte aligned, or scale is not positive and finite", who);
        return PD_ERR_INVALID_ARG;
    }
    const PagedAttnPlan plan = paged_attn_plan(kind, hd, a.p, n_q_heads);
    if (plan.bytes > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < (int64_t)plan.bytes)) {
        set_error("%s: needs a 16-byte aligned workspace of %zu bytes", who, plan.bytes);
        return PD_ERR_INVALID_ARG;
    }
    a.q = q; a.q_stride = q_stride; a.out = out; a.Hq = n_q_heads; a.G = n_q_heads / a.p.Hkv; a.scale = scale;
    return launched(who, launch_paged_attention(kind, hd, a, plan, (char *)workspace, (hipStream_t)stream));
}
