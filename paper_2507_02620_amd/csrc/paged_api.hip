// Host side of the C ABI for contexts in 8-bit pages and for attention over whole prompts: validation, then one or two launches.
#include <math.h>

#include <algorithm>
#include <climits>
#include <new>

#include "paged_api.hpp"

extern thread_local int g_last_hip;

#define HIP_TRY(expr)                 \
    do {                              \
        hipError_t e__ = (expr);      \
        if (e__ != hipSuccess) {      \
            g_last_hip = (int)e__;    \
            return FS_EHIP;           \
        }                             \
    } while (0)

static_assert(FS_PAGE_TOKENS == PAGE_TOK && FS_MAX_BATCH == PAGED_MAX_REQ && FS_MAX_SEQ_LIST == SEQ_LIST, "header and kernels agree");

int pool_dev(const fs_page_pool* p, PoolDev* d) {
    if (!p || !p->codes || !p->scales || !p->ref || !p->table || !p->length || !p->work) return FS_EINVAL;
    if (((uintptr_t)p->codes & 15) || (((uintptr_t)p->scales | (uintptr_t)p->ref | (uintptr_t)p->table | (uintptr_t)p->length | (uintptr_t)p->work) & 3))
        return FS_EINVAL;
    if (p->n_pages < 1 || p->n_pages > (1 << 24) || p->n_layers < 1 || p->n_kv_heads < 1 || p->n_seqs < 1 || p->max_pages < 1) return FS_EINVAL;
    if (p->head_dim != 64 && p->head_dim != 128) return FS_EINVAL;
    if (p->max_pages > (1 << 24) || (long long)p->n_layers * p->n_kv_heads > (1 << 20)) return FS_EINVAL;
    *d = PoolDev{(unsigned char*)p->codes, p->scales, p->ref,        p->table,    p->length,  p->work,
                 p->n_pages,               p->n_layers, p->n_kv_heads, p->head_dim, p->n_seqs, p->max_pages};
    return FS_OK;
}

int valid_rows(int dtype, int hd, const fs_kv_cache& kv) {
    const int epf = dtype == FS_F32 ? 4 : 8;
    if (!kv.base || ((uintptr_t)kv.base & 15)) return FS_EINVAL;
    if (kv.stride_tok < hd || kv.stride_tok % epf || kv.stride_head % epf || kv.stride_kv % epf || kv.stride_layer % epf) return FS_EINVAL;
    if (kv.stride_head < 0 || kv.stride_kv < 0 || kv.stride_layer < 0) return FS_EINVAL;
    return FS_OK;
}

int valid_paged_item(const PoolDev& p, const fs_paged_item& it) {
    if (it.l_s < 0 || it.seg_off < 0 || it.l_glo < 0 || it.n_paged < 0) return FS_EINVAL;
    if (it.seq < 0 || it.seq >= p.n_seqs || it.n_paged > it.l_glo) return FS_EINVAL;
    if (it.n_paged > (long long)p.max_pages * PAGE_TOK) return FS_ECAP;
    if ((long long)it.seg_off + it.l_s > FS_MAX_TREE) return FS_ECAP;
    const long long L = (long long)it.l_glo + it.seg_off + it.l_s;
    if (L - it.n_paged > it.kv_capacity || L > (1LL << 30)) return FS_ECAP;
    return FS_OK;
}

namespace {

// Sequence numbers in range; no destination twice, none among the sources.
int fill_lists(const PoolDev& p, SeqLists& l, const int32_t* a, const int32_t* b, int n, bool b_is_seq) {
    if (n < 0 || (n > 0 && (!a || (b_is_seq && !b)))) return FS_EINVAL;
    if (n > SEQ_LIST) return FS_ECAP;
    l.n = n;
    for (int i = 0; i < n; ++i) {
        l.a[i] = a[i];
        l.b[i] = b ? b[i] : 0;
        if (a[i] < 0 || a[i] >= p.n_seqs) return FS_EINVAL;
        if (b_is_seq && (b[i] < 0 || b[i] >= p.n_seqs)) return FS_EINVAL;
    }
    const int32_t* dst = b_is_seq ? b : a;
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j)
            if ((i != j && dst[i] == dst[j]) || (b_is_seq && dst[i] == a[j])) return FS_EINVAL;
    return FS_OK;
}

size_t partial_bytes(int Hq, int Hkv, int hd, int rows, int splits) {
    const size_t Rpad = ((size_t)(Hq / Hkv) * rows + 15) / 16 * 16;
    return (size_t)splits * Hkv * Rpad * (hd + 2) * sizeof(float);
}

// Scratch of calls of up to `rows` rows.  Fewer rows are split further, into as many splits as `most` allows a KV head's stacked rows, and the products of
// blocks of 64 and whole splits go up and down: the largest one counts.
size_t scratch_bytes(int Hq, int Hkv, int hd, int rows, int (*most)(int, long long)) {
    const long long R = (long long)(Hq / Hkv) * rows;
    const int last = most(Hkv, R);
    size_t bytes = partial_bytes(Hq, Hkv, hd, rows, last);
    for (long long r = 64; r < R && most(Hkv, r) > last; r += 64) bytes = std::max(bytes, partial_bytes(Hkv, Hkv, hd, (int)r, most(Hkv, r)));
    return bytes;
}

// Operands of an attention over pages, and their checks.
int fill_base(const PoolDev& p, int layer, int dtype, int n_q_heads, const fs_kv_cache& kv, const uint64_t* anc, const void* q, long long ldq, void* out,
              long long ldo, float scale, long long rows, PagedBase* to) {
    PagedBase& a = *to;
    const int epf = dtype == FS_F32 ? 4 : 8;
    const long long width = (long long)n_q_heads * p.hd;
    if (!q || !out || q == out || (((uintptr_t)q | (uintptr_t)out) & 15) || ((uintptr_t)anc & 7)) return FS_EINVAL;
    if (ldq < width || ldo < width || ldq % epf || ldo % epf) return FS_EINVAL;
    a.q = q; a.o = out; a.ldq = ldq; a.ldo = ldo;
    a.codes = p.codes; a.scales = p.scales; a.table = p.table; a.anc = anc;
    a.page_tiles = (long long)p.n_layers * 2 * p.Hkv; a.n_pages = p.n_pages; a.max_pages = p.max_pages; a.tile0 = layer * 2 * p.Hkv;
    a.Hq = n_q_heads; a.Hkv = p.Hkv; a.hd = p.hd; a.G = n_q_heads / p.Hkv;
    a.layer_off = layer * kv.stride_layer; a.stride_kv = kv.stride_kv; a.stride_head = kv.stride_head; a.stride_tok = kv.stride_tok;
    a.scale_log2 = (scale > 0.f ? scale : 1.f / sqrtf((float)p.hd)) * 1.4426950408889634f;
    a.rows = (int)rows;
    if ((long long)a.G * rows > (1 << 24) || p.Hkv > 65535) return FS_ECAP;
    return FS_OK;
}

}  // namespace

int fill_shared(const PoolDev& p, const fs_paged_item* items, int n_items, const fs_prefix_group* groups, int n_groups, SharedPlan* plan) {
    if (n_groups < 1 || n_groups > n_items || !groups) return FS_EINVAL;
    SharedArgs& a = plan->a;
    SharedReq own[PAGED_MAX_REQ];
    a.n_req = a.n_prefix = 0;
    int at = 0, row = 0;
    for (int g = 0; g < n_groups; ++g) {
        const int n = groups[g].n_items, shared = groups[g].n_shared;
        if (n < 1 || n > n_items - at || shared < 0 || shared % PAGE_TOK) return FS_EINVAL;
        const int row0 = row, req0 = a.n_req, lead = at;
        int last = at;
        for (; at < lead + n; ++at) {
            const fs_paged_item& it = items[at];
            if (it.l_s == 0) continue;
            if (shared > it.n_paged) return FS_EINVAL;
            SharedReq r{};
            (PagedReq&)r = PagedReq{it.kv.base, it.seq, it.n_paged, row, it.l_s, it.l_glo, it.seg_off};
            r.group = -1;
            own[a.n_req++] = r;
            row += it.l_s;
            last = at;
        }
        const int live = a.n_req - req0;
        if (shared == 0 || live == 0 || (live == 1 && last == lead)) continue;  // (one request reads its own pages in one pass)
        for (int i = req0; i < a.n_req; ++i) {
            own[i].first = shared / PAGE_TOK;
            own[i].group = a.n_prefix;
        }
        SharedReq r{};
        (PagedReq&)r = PagedReq{nullptr, items[lead].seq, shared, row0, row - row0, shared, 0};
        a.req[a.n_prefix++] = r;
    }
    std::copy(own, own + a.n_req, a.req + a.n_prefix);
    return at == n_items ? FS_OK : FS_EINVAL;
}

extern "C" {

int fs_paged_store(const fs_page_pool* pool, int dtype, const fs_store_item* items, int n_items, int32_t* written, void* stream) {
    StoreArgs a{};
    int rc = pool_dev(pool, &a.p);
    if (rc) return rc;
    if (dtype != FS_F32 && dtype != FS_BF16) return FS_EDTYPE;
    if (!items || n_items < 1) return FS_EINVAL;
    if (n_items > FS_MAX_BATCH) return FS_ECAP;
    const int elem = dtype == FS_F32 ? 4 : 2;
    long long pages = 0;
    for (int i = 0; i < n_items; ++i) {
        const fs_store_item& it = items[i];
        if (it.n_tokens < 0 || it.first_page < 0 || it.slot0 < 0 || it.seq < 0 || it.seq >= pool->n_seqs) return FS_EINVAL;
        if (it.n_tokens == 0) continue;
        rc = valid_rows(dtype, pool->head_dim, it.kv);
        if (rc) return rc;
        const long long n = ((long long)it.n_tokens + PAGE_TOK - 1) / PAGE_TOK;
        if (it.first_page + n > pool->max_pages) return FS_ECAP;
        for (int j = 0; j < a.n; ++j) {  // the same page twice
            const StoreItem& o = a.it[j];
            if (o.seq == it.seq && it.first_page < o.first_page + (o.n_tokens + PAGE_TOK - 1) / PAGE_TOK && o.first_page < it.first_page + n) return FS_EINVAL;
        }
        a.it[a.n++] = StoreItem{(const char*)it.kv.base + it.slot0 * it.kv.stride_tok * elem, it.kv.stride_layer, it.kv.stride_kv, it.kv.stride_head,
                                it.kv.stride_tok, it.seq, it.first_page, it.n_tokens, (int)pages};
        pages += n;
    }
    if (pages == 0) return FS_OK;
    if (pages > 65535) return FS_ECAP;
    a.written = written;
    HIP_TRY(launch_paged_store(dtype, a, (int)pages, (hipStream_t)stream));
    return FS_OK;
}

int fs_page_grow(const fs_page_pool* pool, const int32_t* seqs, const int32_t* n_tokens, int n, int32_t* status, void* stream) {
    PoolDev p;
    SeqLists l{};
    int rc = pool_dev(pool, &p);
    if (!rc) rc = fill_lists(p, l, seqs, n_tokens, n, false);
    if (rc) return rc;
    if (!status || (n > 0 && !n_tokens)) return FS_EINVAL;
    for (int i = 0; i < n; ++i) {
        if (n_tokens[i] < 0) return FS_EINVAL;
        if (n_tokens[i] > (long long)p.max_pages * PAGE_TOK) return FS_ECAP;
    }
    if (n == 0) return FS_OK;
    HIP_TRY(launch_page_grow(p, l, status, (hipStream_t)stream));
    return FS_OK;
}

int fs_page_fork(const fs_page_pool* pool, const int32_t* src, const int32_t* dst, int n, int32_t* status, void* stream) {
    PoolDev p;
    SeqLists l{};
    int rc = pool_dev(pool, &p);
    if (!rc) rc = fill_lists(p, l, src, dst, n, true);
    if (rc) return rc;
    if (!status) return FS_EINVAL;
    if (n == 0) return FS_OK;
    HIP_TRY(launch_page_fork(p, l, status, (hipStream_t)stream));
    return FS_OK;
}

int fs_page_free(const fs_page_pool* pool, const int32_t* seqs, int n, void* stream) {
    PoolDev p;
    SeqLists l{};
    int rc = pool_dev(pool, &p);
    if (!rc) rc = fill_lists(p, l, seqs, nullptr, n, false);
    if (rc) return rc;
    if (n == 0) return FS_OK;
    HIP_TRY(launch_page_free(p, l, (hipStream_t)stream));
    return FS_OK;
}

int fs_page_compact(const fs_page_pool* pool, int32_t* status, void* stream) {
    PoolDev p;
    int rc = pool_dev(pool, &p);
    if (rc) return rc;
    if (!status) return FS_EINVAL;
    HIP_TRY(launch_page_compact(p, status, (hipStream_t)stream));
    return FS_OK;
}

int fs_page_copy(const fs_page_pool* dst, const fs_page_pool* src, const int32_t* src_pages, const int32_t* dst_pages, int n, void* stream) {
    PoolDev d, s;
    SeqLists l{};
    int rc = pool_dev(dst, &d);
    if (!rc) rc = pool_dev(src, &s);
    if (rc) return rc;
    if (d.n_layers != s.n_layers || d.Hkv != s.Hkv || d.hd != s.hd) return FS_EINVAL;
    if (n < 0 || (n > 0 && (!src_pages || !dst_pages))) return FS_EINVAL;
    if (n > SEQ_LIST) return FS_ECAP;
    const bool same = d.codes == s.codes;
    for (int i = 0; i < n; ++i) {
        if (src_pages[i] < 0 || src_pages[i] >= s.n_pages || dst_pages[i] < 0 || dst_pages[i] >= d.n_pages) return FS_EINVAL;
        for (int j = 0; j < n; ++j)
            if ((i != j && dst_pages[i] == dst_pages[j]) || (same && dst_pages[i] == src_pages[j])) return FS_EINVAL;
        l.a[i] = src_pages[i];
        l.b[i] = dst_pages[i];
    }
    l.n = n;
    if (n == 0) return FS_OK;
    HIP_TRY(launch_page_copy(d, s, l, (hipStream_t)stream));
    return FS_OK;
}

size_t fs_paged_attention_workspace_bytes(int n_q_heads, int n_kv_heads, int head_dim, int rows) {
    if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || (head_dim != 64 && head_dim != 128) || rows < 1) return 0;
    return scratch_bytes(n_q_heads, n_kv_heads, head_dim, rows, paged_max_splits);
}

int fs_paged_attention(const fs_page_pool* pool, int layer, int dtype, int n_q_heads, const fs_paged_item* items, int n_items, const uint64_t* anc,
                       const void* q, long long ldq, void* out, long long ldo, float scale, void* workspace, size_t workspace_bytes, void* stream) {
    PoolDev p;
    int rc = pool_dev(pool, &p);
    if (rc) return rc;
    if (dtype != FS_F32 && dtype != FS_BF16) return FS_EDTYPE;
    if (layer < 0 || layer >= p.n_layers || n_q_heads < 1 || n_q_heads % p.Hkv || !items || n_items < 1) return FS_EINVAL;
    if (n_items > FS_MAX_BATCH) return FS_ECAP;
    if (!(scale >= 0.f) || !(scale < INFINITY)) return FS_EINVAL;
    PagedArgs a{};
    const fs_kv_cache* kv0 = nullptr;
    long long rows = 0;
    for (int i = 0; i < n_items; ++i) {
        const fs_paged_item& it = items[i];
        rc = valid_paged_item(p, it);
        if (rc) return rc;
        if (it.l_s == 0) continue;
        rc = valid_rows(dtype, p.hd, it.kv);
        if (rc) return rc;
        if (!kv0) kv0 = &it.kv;
        if (it.kv.stride_layer != kv0->stride_layer || it.kv.stride_kv != kv0->stride_kv || it.kv.stride_head != kv0->stride_head ||
            it.kv.stride_tok != kv0->stride_tok)
            return FS_EINVAL;
        a.req[a.n_req++] = PagedReq{it.kv.base, it.seq, it.n_paged, (int)rows, it.l_s, it.l_glo, it.seg_off};
        rows += it.l_s;
    }
    if (rows == 0) return FS_OK;
    rc = fill_base(p, layer, dtype, n_q_heads, *kv0, anc, q, ldq, out, ldo, scale, rows, &a);
    if (rc) return rc;
    const int mtw = paged_plan(dtype, a);
    if ((long long)a.n_req * a.row_blocks > 65535) return FS_ECAP;
    if (a.n_splits > 1) {
        const size_t need = partial_bytes(n_q_heads, p.Hkv, p.hd, a.rows, a.n_splits);
        if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return FS_EWS;
        a.part_o = (float*)workspace;
        a.part_ml = a.part_o + (size_t)a.n_splits * a.Hkv * a.Rpad * a.hd;
    }
    HIP_TRY(launch_paged_attention(dtype, a, mtw, (hipStream_t)stream));
    return FS_OK;
}

size_t fs_shared_attention_workspace_bytes(int n_q_heads, int n_kv_heads, int head_dim, int rows) {
    if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || (head_dim != 64 && head_dim != 128) || rows < 1) return 0;
    return scratch_bytes(n_q_heads, n_kv_heads, head_dim, rows, shared_max_places);
}

int fs_shared_attention(const fs_page_pool* pool, int layer, int dtype, int n_q_heads, const fs_paged_item* items, int n_items,
                        const fs_prefix_group* groups, int n_groups, const uint64_t* anc, const void* q, long long ldq, void* out, long long ldo, float scale,
                        void* workspace, size_t workspace_bytes, void* stream) {
    PoolDev p;
    int rc = pool_dev(pool, &p);
    if (rc) return rc;
    if (dtype != FS_F32 && dtype != FS_BF16) return FS_EDTYPE;
    if (layer < 0 || layer >= p.n_layers || n_q_heads < 1 || n_q_heads % p.Hkv || !items || n_items < 1) return FS_EINVAL;
    if (n_items > FS_MAX_BATCH) return FS_ECAP;
    if (!(scale >= 0.f) || !(scale < INFINITY)) return FS_EINVAL;
    const fs_kv_cache* kv0 = nullptr;
    long long rows = 0;
    for (int i = 0; i < n_items; ++i) {
        const fs_paged_item& it = items[i];
        rc = valid_paged_item(p, it);
        if (rc) return rc;
        if (it.l_s == 0) continue;
        rc = valid_rows(dtype, p.hd, it.kv);
        if (rc) return rc;
        if (!kv0) kv0 = &it.kv;
        if (it.kv.stride_layer != kv0->stride_layer || it.kv.stride_kv != kv0->stride_kv || it.kv.stride_head != kv0->stride_head ||
            it.kv.stride_tok != kv0->stride_tok)
            return FS_EINVAL;
        rows += it.l_s;
    }
    SharedPlan sp;
    rc = fill_shared(p, items, n_items, groups, n_groups, &sp);
    if (rc) return rc;
    if (rows == 0) return FS_OK;
    if (sp.a.n_prefix == 0)
        return fs_paged_attention(pool, layer, dtype, n_q_heads, items, n_items, anc, q, ldq, out, ldo, scale, workspace, workspace_bytes, stream);
    rc = fill_base(p, layer, dtype, n_q_heads, *kv0, anc, q, ldq, out, ldo, scale, rows, &sp.a);
    if (rc) return rc;
    shared_plan(dtype, sp);
    if (sp.wgs > INT_MAX / 512) return FS_ECAP;
    const size_t need = partial_bytes(n_q_heads, p.Hkv, p.hd, (int)rows, sp.places);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return FS_EWS;
    sp.place(workspace);
    HIP_TRY(launch_shared_attention(dtype, sp, (hipStream_t)stream));
    return FS_OK;
}

int fs_prompt_attention(int dtype, int n_q_heads, int n_kv_heads, int head_dim, const int32_t* cu_seqlens, int n_seqs, const fs_rows* q, const fs_rows* k,
                        const fs_rows* v, const fs_rows* out, float scale, void* stream) {
    if (dtype != FS_F32 && dtype != FS_BF16) return FS_EDTYPE;
    if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || (head_dim != 64 && head_dim != 128)) return FS_EINVAL;
    if (!cu_seqlens || n_seqs < 0 || !q || !k || !v || !out) return FS_EINVAL;
    if (!(scale >= 0.f) || !(scale < INFINITY) || n_q_heads > 65535) return FS_EINVAL;
    if (cu_seqlens[0] < 0) return FS_EINVAL;
    for (int i = 0; i < n_seqs; ++i)
        if (cu_seqlens[i + 1] < cu_seqlens[i]) return FS_EINVAL;
    if (n_seqs == 0 || cu_seqlens[n_seqs] == cu_seqlens[0]) return FS_OK;
    const int epf = dtype == FS_F32 ? 4 : 8;
    for (const fs_rows* r : {q, k, v, out}) {
        if (!r->base || ((uintptr_t)r->base & 15)) return FS_EINVAL;
        if (r->stride_tok < 0 || r->stride_head < 0 || r->stride_tok % epf || r->stride_head % epf) return FS_EINVAL;
        // 64 rows of a head are addressed with 32-bit byte offsets
        if (r->stride_tok > (1 << 24)) return FS_EINVAL;
    }
    // rows of the result do not overlap one another (heads within tokens or tokens within heads), nor begin where an operand does
    const long long tokens = cu_seqlens[n_seqs];
    if (out->stride_tok < head_dim || (n_q_heads > 1 && out->stride_head < head_dim)) return FS_EINVAL;
    if (n_q_heads > 1 && out->stride_tok < (n_q_heads - 1) * out->stride_head + head_dim && out->stride_head < (tokens - 1) * out->stride_tok + head_dim)
        return FS_EINVAL;
    if ((tokens / 16 + n_seqs) * n_q_heads > (1LL << 23)) return FS_ECAP;  // workgroups of one launch
    if (out->base == q->base || out->base == k->base || out->base == v->base) return FS_EINVAL;
    PromptArgs a{};
    a.q = q->base; a.k = k->base; a.v = v->base; a.o = out->base;
    a.q_tok = q->stride_tok; a.q_head = q->stride_head; a.k_tok = k->stride_tok; a.k_head = k->stride_head;
    a.v_tok = v->stride_tok; a.v_head = v->stride_head; a.o_tok = out->stride_tok; a.o_head = out->stride_head;
    a.scale_log2 = (scale > 0.f ? scale : 1.f / sqrtf((float)head_dim)) * 1.4426950408889634f;
    a.Hq = n_q_heads; a.Hkv = n_kv_heads; a.G = n_q_heads / n_kv_heads; a.hd = head_dim;
    try {  // (the order of the sequences is worked out in host memory)
        HIP_TRY(launch_prompt_attention(dtype, a, cu_seqlens, n_seqs, (hipStream_t)stream));
    } catch (const std::bad_alloc&) {
        return FS_EINVAL;
    }
    return FS_OK;
}

}  // extern "C"
