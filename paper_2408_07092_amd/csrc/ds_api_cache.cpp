// C-ABI layer of prompt attention and of the paged cache: argument validation only; every device
// step is enqueued through the launchers declared in ds_cache.h.
#include <algorithm>
#include <cstdint>

#include <hip/hip_runtime.h>

#include "ds_cache.h"

using namespace ds;

static bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

#define DS_TRY(expr)                                  \
    do {                                              \
        if ((expr) != hipSuccess) return DS_ERR_HIP;  \
    } while (0)

static bool heads_ok(int Hq, int Hkv, int d, int dtype)
{
    return Hq >= 1 && Hkv >= 1 && Hkv <= 65535 && Hq <= 65535 && Hq % Hkv == 0 && d == kD && (dtype == DS_F16 || dtype == DS_BF16);
}

// *m = *prm with the dense strides in the place of zeros
static bool prompt_ok(const ds_prompt_t *prm, ds_prompt_t *m)
{
    *m = *prm;
    if (m->n_seqs < 1 || m->total_q < 0 || m->max_kv < 0 || !heads_ok(m->Hq, m->Hkv, m->d, m->dtype)) return false;
    const int64_t row = (int64_t)m->Hq * kD, most = 1ll << 30;
    if (m->q_stride == 0) m->q_stride = row;
    if (m->out_stride == 0) m->out_stride = row;
    if (m->kv_stride == 0) m->kv_stride = (int64_t)m->Hkv * kD;
    if (m->kv_head_stride == 0) m->kv_head_stride = kD;
    for (int64_t s : {m->q_stride, m->out_stride, m->kv_stride, m->kv_head_stride})
        if (s % 8 != 0) return false;
    if (m->q_stride < row || m->out_stride < row || m->kv_stride < kD || m->kv_head_stride < kD || m->kv_elems < 0) return false;
    if (m->q_stride > most || m->out_stride > most || m->kv_stride > 1ll << 24 || m->kv_head_stride > 1ll << 40) return false;
    // (a launch holds less than 2^32 threads, and rows are numbered in 32 bits)
    return ((int64_t)m->total_q / kPromptRows + m->n_seqs) * m->Hq < 1ll << 24;
}

static bool pages_ok(const ds_pages_t *p)
{
    if (p->page_tokens < 16 || p->page_tokens > 256 || (p->page_tokens & (p->page_tokens - 1))) return false;
    if (p->n_pages < 1 || p->n_pages > 1 << 20 || p->n_rows < 1 || p->n_rows > 65536 || p->max_pages < 1) return false;
    return (int64_t)p->max_pages * p->page_tokens <= kMostTokens && heads_ok(p->Hkv, p->Hkv, p->d, p->dtype);
}

static int log2_of(int x) { return __builtin_ctz((unsigned)x); }

extern "C" {

size_t ds_prompt_workspace_bytes(const ds_prompt_t *prm)
{
    ds_prompt_t m;
    PromptPlan p;
    if (!prm || !prompt_ok(prm, &m)) return 0;
    make_prompt_plan(m, &p);
    return p.total;
}

static PromptArgs prompt_args(const void *q, const void *K, const void *V, void *out, const int32_t *q_start,
                              const int32_t *kv_len, void *workspace, const ds_prompt_t &m, const PromptPlan &p)
{
    PromptArgs a{};
    a.part_ml = static_cast<float2 *>(workspace);
    a.part_acc = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.off_acc);
    a.q = q;
    a.K = K;
    a.V = V;
    a.out = out;
    a.q_start = q_start;
    a.kv_len = kv_len;
    a.q_stride = m.q_stride;
    a.out_stride = m.out_stride;
    a.kv_stride = m.kv_stride;
    a.kv_head_stride = m.kv_head_stride;
    a.kv_elems = m.kv_elems;
    a.n_seqs = m.n_seqs;
    a.Hq = m.Hq;
    a.Hkv = m.Hkv;
    a.G = p.G;
    a.total_q = m.total_q;
    a.n_tiles = p.n_tiles;
    a.n_split = p.n_split;
    return a;
}

ds_status_t ds_prompt_attention(const void *q, const void *K, const void *V, void *out, const int32_t *q_start,
                                const int32_t *kv_start, const int32_t *kv_len, void *workspace,
                                size_t workspace_bytes, const ds_prompt_t *prm, void *stream)
{
    if (!q_start || !kv_start || !kv_len || !workspace || !prm) return DS_ERR_NULL;
    // (arrays without an element may have no address)
    if (((!q || !out) && prm->total_q != 0) || ((!K || !V) && prm->kv_elems != 0)) return DS_ERR_NULL;
    ds_prompt_t m;
    PromptPlan p;
    if (!prompt_ok(prm, &m)) return DS_ERR_SHAPE;
    make_prompt_plan(m, &p, workspace_bytes);
    if (!aligned(q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(workspace, 16) ||
        !aligned(q_start, 4) || !aligned(kv_start, 4) || !aligned(kv_len, 4))
        return DS_ERR_ALIGN;
    if (workspace_bytes < p.total) return DS_ERR_WORKSPACE;
    if (m.total_q == 0) return DS_OK;
    PromptArgs a = prompt_args(q, K, V, out, q_start, kv_len, workspace, m, p);
    a.kv_start = kv_start;
    DS_TRY(launch_prompt(a, false, m.dtype, (hipStream_t)stream));
    return DS_OK;
}

ds_status_t ds_prompt_attention_paged(const void *q, const void *K_pages, const void *V_pages, void *out,
                                      const int32_t *q_start, const int32_t *rows, const int32_t *lens,
                                      const int32_t *table, void *workspace, size_t workspace_bytes,
                                      const ds_prompt_t *prm, const ds_pages_t *pages, void *stream)
{
    if (!K_pages || !V_pages || !q_start || !lens || !table || !workspace || !prm || !pages) return DS_ERR_NULL;
    if ((!q || !out) && prm->total_q != 0) return DS_ERR_NULL;
    ds_prompt_t m;
    PromptPlan p;
    if (!prompt_ok(prm, &m) || !pages_ok(pages)) return DS_ERR_SHAPE;
    if (pages->Hkv != m.Hkv || pages->dtype != m.dtype || (!rows && m.n_seqs > pages->n_rows)) return DS_ERR_SHAPE;
    make_prompt_plan(m, &p, workspace_bytes);
    if (!aligned(q, 16) || !aligned(K_pages, 256) || !aligned(V_pages, 256) || !aligned(out, 16) ||
        !aligned(workspace, 16) || !aligned(q_start, 4) || !aligned(rows, 4) || !aligned(lens, 4) || !aligned(table, 4))
        return DS_ERR_ALIGN;
    if (workspace_bytes < p.total) return DS_ERR_WORKSPACE;
    if (m.total_q == 0) return DS_OK;
    PromptArgs a = prompt_args(q, K_pages, V_pages, out, q_start, lens, workspace, m, p);
    a.rows = rows;
    a.table = table;
    a.n_pages = pages->n_pages;
    a.page_log2 = log2_of(pages->page_tokens);
    a.max_pages = pages->max_pages;
    a.n_table = pages->n_rows;
    DS_TRY(launch_prompt(a, true, m.dtype, (hipStream_t)stream));
    return DS_OK;
}

static bool paged_ok(const ds_pages_t *g, int32_t n_seqs, int32_t Hq, int32_t max_len)
{
    if (!pages_ok(g) || n_seqs < 1 || max_len < 0 || !heads_ok(Hq, g->Hkv, g->d, g->dtype)) return false;
    const int64_t units = (int64_t)n_seqs * g->Hkv * ((Hq / g->Hkv + 15) / 16);
    return units <= (1ll << 31) / (((int64_t)g->max_pages * g->page_tokens + kPiece - 1) / kPiece + kLead);
}

size_t ds_paged_workspace_bytes(const ds_pages_t *pages, int32_t n_seqs, int32_t Hq, int32_t max_len)
{
    if (!pages || !paged_ok(pages, n_seqs, Hq, max_len)) return 0;
    PagedPlan p;
    make_paged_plan(*pages, n_seqs, Hq, max_len, &p);
    return p.total;
}

ds_status_t ds_paged_decode(const void *q, const void *K_pages, const void *V_pages, float *out,
                            const int32_t *rows, const int32_t *lens, const int32_t *table, void *workspace,
                            size_t workspace_bytes, const ds_pages_t *pages, int32_t n_seqs, int32_t Hq,
                            int32_t max_len, void *stream)
{
    if (!q || !K_pages || !V_pages || !out || !lens || !table || !workspace || !pages) return DS_ERR_NULL;
    if (!paged_ok(pages, n_seqs, Hq, max_len) || (!rows && n_seqs > pages->n_rows)) return DS_ERR_SHAPE;
    if (!aligned(q, 16) || !aligned(K_pages, 256) || !aligned(V_pages, 256) || !aligned(out, 16) ||
        !aligned(workspace, 16) || !aligned(rows, 4) || !aligned(lens, 4) || !aligned(table, 4))
        return DS_ERR_ALIGN;
    PagedPlan p;
    make_paged_plan(*pages, n_seqs, Hq, max_len, &p);
    if (workspace_bytes < p.total) return DS_ERR_WORKSPACE;
    PagedArgs a{};
    a.q = q;
    a.K = K_pages;
    a.V = V_pages;
    a.out = out;
    a.part = static_cast<float *>(workspace);
    a.arrived = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + p.off_arrived);
    a.rows = rows;
    a.lens = lens;
    a.table = table;
    a.n = n_seqs;
    a.Hkv = pages->Hkv;
    a.G = p.G;
    a.passes = p.passes;
    a.join_here = p.join_here;
    a.n_pages = pages->n_pages;
    a.page_log2 = log2_of(pages->page_tokens);
    a.max_pages = pages->max_pages;
    a.n_table = pages->n_rows;
    DS_TRY(launch_paged(a, p, pages->dtype, (hipStream_t)stream));
    return DS_OK;
}

ds_status_t ds_append_paged(const void *k_new, const void *v_new, void *K_pages, void *V_pages,
                            const int32_t *new_start, const int32_t *rows, const int32_t *start,
                            const int32_t *table, const ds_pages_t *pages, int32_t n_seqs, int32_t total_new,
                            int64_t new_stride, void *stream)
{
    if (!K_pages || !V_pages || !new_start || !start || !table || !pages || ((!k_new || !v_new) && total_new != 0)) return DS_ERR_NULL;
    if (!pages_ok(pages) || n_seqs < 1 || total_new < 0 || (!rows && n_seqs > pages->n_rows)) return DS_ERR_SHAPE;
    const int64_t row = (int64_t)pages->Hkv * kD;
    if (new_stride == 0) new_stride = row;
    if (new_stride < row || new_stride % 8 != 0 || new_stride > 1ll << 30) return DS_ERR_SHAPE;
    // (four wavefronts to a workgroup, and a launch holds less than 2^32 threads)
    if ((int64_t)total_new * ((pages->Hkv + 7) / 8) > (1ll << 26) - 4) return DS_ERR_SHAPE;
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(K_pages, 256) || !aligned(V_pages, 256) ||
        !aligned(new_start, 4) || !aligned(rows, 4) || !aligned(start, 4) || !aligned(table, 4))
        return DS_ERR_ALIGN;
    if (total_new == 0) return DS_OK;
    AppendPagedArgs a{};
    a.k_new = static_cast<const u32x4 *>(k_new);
    a.v_new = static_cast<const u32x4 *>(v_new);
    a.K = static_cast<u32x4 *>(K_pages);
    a.V = static_cast<u32x4 *>(V_pages);
    a.new_start = new_start;
    a.rows = rows;
    a.start = start;
    a.table = table;
    a.new_stride = new_stride / 8;
    a.n = n_seqs;
    a.total_new = total_new;
    a.Hkv = pages->Hkv;
    a.n_pages = pages->n_pages;
    a.page_log2 = log2_of(pages->page_tokens);
    a.max_pages = pages->max_pages;
    a.n_table = pages->n_rows;
    DS_TRY(launch_append_paged(a, (hipStream_t)stream));
    return DS_OK;
}

// The books' arguments, checked; DS_OK and *a filled in.
static ds_status_t books(int32_t *refs, int32_t *table, const int32_t *lens, const int32_t *rows, int32_t *status,
                         const ds_pages_t *pages, int32_t n, PagesArgs *a)
{
    if (!refs || !table || !lens || !rows || !status || !pages) return DS_ERR_NULL;
    if (!pages_ok(pages) || n < 1 || n > kPagesListed) return DS_ERR_SHAPE;
    if (!aligned(refs, 16) || !aligned(table, 4) || !aligned(lens, 4) || !aligned(rows, 4) || !aligned(status, 4))
        return DS_ERR_ALIGN;
    *a = PagesArgs{};
    a->refs = refs;
    a->table = table;
    a->lens = const_cast<int32_t *>(lens);
    a->rows = rows;
    a->status = status;
    a->n = n;
    a->n_pages = pages->n_pages;
    a->page_log2 = log2_of(pages->page_tokens);
    a->max_pages = pages->max_pages;
    a->n_rows = pages->n_rows;
    return DS_OK;
}

ds_status_t ds_pages_extend(int32_t *refs, int32_t *table, int32_t *lens, const int32_t *rows, const int32_t *n_new,
                            int32_t *start, int32_t *status, const ds_pages_t *pages, int32_t n, void *stream)
{
    if (!n_new || !start) return DS_ERR_NULL;
    PagesArgs a;
    const ds_status_t rc = books(refs, table, lens, rows, status, pages, n, &a);
    if (rc != DS_OK) return rc;
    if (!aligned(n_new, 4) || !aligned(start, 4)) return DS_ERR_ALIGN;
    a.n_new = n_new;
    a.start = start;
    DS_TRY(launch_pages_extend(a, (hipStream_t)stream));
    return DS_OK;
}

ds_status_t ds_pages_fork(int32_t *refs, int32_t *table, int32_t *lens, const int32_t *src, const int32_t *dst,
                          int32_t *copies, int32_t *n_copies, int32_t *status, const ds_pages_t *pages, int32_t n,
                          void *stream)
{
    if (!dst || !copies || !n_copies) return DS_ERR_NULL;
    PagesArgs a;
    const ds_status_t rc = books(refs, table, lens, src, status, pages, n, &a);
    if (rc != DS_OK) return rc;
    if (!aligned(dst, 4) || !aligned(copies, 16) || !aligned(n_copies, 4)) return DS_ERR_ALIGN;
    a.dst = dst;
    a.copies = reinterpret_cast<int4 *>(copies);
    a.n_copies = n_copies;
    DS_TRY(launch_pages_fork(a, (hipStream_t)stream));
    return DS_OK;
}

ds_status_t ds_pages_free(int32_t *refs, int32_t *table, int32_t *lens, const int32_t *rows, int32_t *status,
                          const ds_pages_t *pages, int32_t n, void *stream)
{
    PagesArgs a;
    const ds_status_t rc = books(refs, table, lens, rows, status, pages, n, &a);
    if (rc != DS_OK) return rc;
    DS_TRY(launch_pages_free(a, (hipStream_t)stream));
    return DS_OK;
}

size_t ds_pages_workspace_bytes(const ds_pages_t *pages) { return pages && pages_ok(pages) ? pages_workspace(pages->n_pages) : 0; }

ds_status_t ds_pages_compact(int32_t *refs, int32_t *table, const int32_t *lens, int32_t *copies, int32_t *n_copies,
                             int32_t *status, void *workspace, size_t workspace_bytes, const ds_pages_t *pages,
                             void *stream)
{
    if (!copies || !n_copies || !workspace) return DS_ERR_NULL;
    PagesArgs a;
    const ds_status_t rc = books(refs, table, lens, lens, status, pages, 1, &a);  // (there is no list of rows)
    if (rc != DS_OK) return rc;
    if (!aligned(copies, 16) || !aligned(n_copies, 4) || !aligned(workspace, 16)) return DS_ERR_ALIGN;
    if (workspace_bytes < pages_workspace(pages->n_pages)) return DS_ERR_WORKSPACE;
    a.copies = reinterpret_cast<int4 *>(copies);
    a.n_copies = n_copies;
    DS_TRY(launch_pages_compact(a, workspace, (hipStream_t)stream));
    return DS_OK;
}

ds_status_t ds_pages_copy(void *K_pages, void *V_pages, const int32_t *copies, const int32_t *n_copies,
                          const ds_pages_t *pages, int32_t max_copies, void *stream)
{
    if (!K_pages || !V_pages || !copies || !n_copies || !pages) return DS_ERR_NULL;
    if (!pages_ok(pages) || max_copies < 0) return DS_ERR_SHAPE;
    if ((int64_t)max_copies * pages->Hkv * pages->page_tokens > 1ll << 32) return DS_ERR_SHAPE;
    if (!aligned(K_pages, 256) || !aligned(V_pages, 256) || !aligned(copies, 16) || !aligned(n_copies, 4)) return DS_ERR_ALIGN;
    if (max_copies == 0) return DS_OK;
    CopyPagesArgs a{};
    a.K = static_cast<u32x4 *>(K_pages);
    a.V = static_cast<u32x4 *>(V_pages);
    a.copies = reinterpret_cast<const int4 *>(copies);
    a.n_copies = n_copies;
    a.max_copies = max_copies;
    a.Hkv = pages->Hkv;
    a.n_pages = pages->n_pages;
    a.page_log2 = log2_of(pages->page_tokens);
    DS_TRY(launch_pages_copy(a, (hipStream_t)stream));
    return DS_OK;
}

}  // extern "C"
