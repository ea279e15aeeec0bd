// C ABI of the cache operators (include/elsaa_cache.h): argument validation,
// workspace layout, launch sequences.
#include <math.h>

#include "cache.h"

using namespace elsaa;

namespace {

size_t align256(size_t x) { return (x + 255) / 256 * 256; }
bool misaligned(const void *p, size_t a) { return (uintptr_t)p % a != 0; }

template <typename F>
cudaError_t timed(const char *name, cudaStream_t st, F fn) {
    return timed_launch(
        name, st, [](void *f) { return (*(F *)f)(); }, &fn);
}

#define ELSAA_CACHE_LAUNCH(name, st, expr)                                  \
    do {                                                                    \
        const cudaError_t e_ = timed(name, st, [&] { return expr; });       \
        if (e_ != cudaSuccess)                                              \
            return set_last_error(ELSAA_ERR_CUDA, "%s: %s", name,           \
                                  cudaGetErrorString(e_));                  \
    } while (0)

// The view of a valid cache; T = 0: no new tokens in the call.
int make_view(const elsaa_cache *p, int T, CacheView *v) {
    auto bad = [](const char *m) {
        return set_last_error(ELSAA_ERR_INVALID_ARG, "%s", m);
    };
    auto no = [](const char *m) {
        return set_last_error(ELSAA_ERR_UNSUPPORTED, "%s", m);
    };
    if (!p) return bad("cache is NULL");
    if (p->B <= 0 || p->H <= 0 || p->H_kv <= 0 || p->num_pages <= 0 ||
        p->max_pages <= 0)
        return bad("B, H, H_kv, num_pages and max_pages must be positive");
    if (p->H % p->H_kv != 0) return bad("H must be a multiple of H_kv");
    if (p->dtype != ELSAA_BF16 && p->dtype != ELSAA_FP32)
        return bad("dtype must be ELSAA_BF16 or ELSAA_FP32");
    if (p->impl != ELSAA_IMPL_AUTO && p->impl != ELSAA_IMPL_SIMT)
        return bad("impl must be AUTO or SIMT");
    if (!(p->scale >= 0.f) || !isfinite(p->scale))
        return bad("scale must be finite and >= 0");
    if (p->d_h != 32 && p->d_h != 64 && p->d_h != 128)
        return no("d_h must be 32, 64 or 128");
    if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 &&
        p->page_size != 128)
        return no("page_size must be 16, 32, 64 or 128");
    if (p->B > kCacheMaxB) return no("B must be at most 4096");
    if (p->H > 65535) return no("H must be at most 65535");
    if ((long)p->max_pages * p->page_size > kCacheMaxSlots)
        return no("max_pages * page_size must be at most 2^31 - 2^16");
    if ((long)p->num_pages * p->H_kv > 0x7fffffffL / p->page_size)
        return no("num_pages * H_kv * page_size must fit in int32");
    if (!p->k || !p->v || !p->k_scale || !p->v_scale || !p->bounds ||
        !p->page_table || !p->lengths)
        return bad("k, v, k_scale, v_scale, bounds, page_table and lengths "
                   "must be non-NULL");
    if (misaligned(p->k, 16) || misaligned(p->v, 16) ||
        misaligned(p->bounds, 16) || misaligned(p->status, 16))
        return bad("k, v, bounds and status must be 16-byte aligned");
    CacheView &c = *v;
    c = CacheView{};
    c.B = p->B;
    c.H = p->H;
    c.Hkv = p->H_kv;
    c.G = p->H / p->H_kv;
    c.d = p->d_h;
    c.ps = p->page_size;
    c.num_pages = p->num_pages;
    c.max_pages = p->max_pages;
    c.T = T;
    c.dtype = p->dtype;
    c.scale = p->scale > 0.f ? p->scale : 1.0f / sqrtf((float)p->d_h);
    c.k = (uint8_t *)p->k;
    c.v = (uint8_t *)p->v;
    c.ks = p->k_scale;
    c.vs = p->v_scale;
    c.bounds = p->bounds;
    c.table = p->page_table;
    c.lengths = p->lengths;
    c.status = (DeviceStatus *)p->status;
    return ELSAA_OK;
}

int check_queries(const CacheView &c) {
    if (c.T <= 0)
        return set_last_error(ELSAA_ERR_INVALID_ARG, "T must be positive");
    if (c.T > 64 || c.G * c.T > 128)
        return set_last_error(ELSAA_ERR_UNSUPPORTED,
                              "T must be at most 64 and T * H / H_kv at most "
                              "128");
    if ((long)c.B * c.H * c.T > 1L << 30)
        return set_last_error(ELSAA_ERR_UNSUPPORTED,
                              "B * H * T must be at most 2^30");
    // the tiles of all columns, with a few more for every item
    const long tiles =
        ((long)c.max_pages * c.ps + kCacheTile - 1) / kCacheTile + 7;
    if (tiles * c.B > (1L << 31) / ((long)c.H * c.T))
        return set_last_error(ELSAA_ERR_UNSUPPORTED,
                              "B * H * T * max_pages * page_size must be at "
                              "most about 2^38");
    return ELSAA_OK;
}

int check_keep(int keep) {
    if (keep > kCacheMaxSlots)
        return set_last_error(ELSAA_ERR_UNSUPPORTED,
                              "keep must be at most 2^31 - 2^16");
    return ELSAA_OK;
}

// Workspace of one call: split items | lse2 | pieces | scores (attention), or
// page keys (select), or counts | pool rows (evict).
struct Layout {
    size_t split, lse2, part, scores, total;
    int cols, groups, ctas;
};
Layout attention_layout(const CacheView &c, bool tc, bool weights) {
    Layout l;
    const int gt = c.G * c.T;
    const long heads = (long)c.B * c.Hkv;
    const long held = heads * c.max_pages * c.ps * 2 * c.d;
    l.cols = tc ? cache_tc_cols(gt, held) : cache_simt_cols(gt);
    l.groups = (gt + l.cols - 1) / l.cols;
    // no more than the table has tiles for, or than may share the items
    const long tiles =
        ((long)c.max_pages * c.ps + kCacheTile - 1) / kCacheTile;
    const long share = tiles < kCacheMaxPieces ? tiles : kCacheMaxPieces;
    const long full = tc ? kCacheTcCtas : kCacheSimtCtas;
    const long most = heads * share;  // in one group
    l.ctas = (int)(most * l.groups < full ? most * l.groups : full);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += align256(bytes);
        return was;
    };
    l.split = take(sizeof(CacheSplit) * l.ctas);
    l.lse2 = take(sizeof(float) * (size_t)c.B * c.H * c.T);
    // a workspace for T tokens serves fewer, which may be one wider group
    long rows = (long)l.ctas * l.cols;
    if (tc && gt > 16 && rows < 16 * (most < full ? most : full))
        rows = 16 * (most < full ? most : full);
    l.part = take(sizeof(float) * 2 * rows * (c.d + 2));
    l.scores = at;
    if (weights)
        take(sizeof(float) * (size_t)c.B * c.H * c.T * c.max_pages * c.ps);
    l.total = at;
    return l;
}
bool on_tensor_cores(const elsaa_cache *cache, const CacheView &c) {
    return cache->impl == ELSAA_IMPL_AUTO && cache_attn_tc_supported(c);
}
size_t select_bytes(const CacheView &c) {
    return align256(sizeof(uint32_t) * (size_t)c.B * c.Hkv * c.max_pages);
}
size_t evict_bytes(const CacheView &c, int keep) {
    return align256(sizeof(int) * (size_t)c.B) +
           align256(sizeof(int32_t) * (size_t)c.B * c.Hkv * keep);
}

int check_workspace(const void *ws, size_t bytes, size_t need) {
    if (!ws) return set_last_error(ELSAA_ERR_WORKSPACE, "workspace is NULL");
    if (misaligned(ws, 256))
        return set_last_error(ELSAA_ERR_WORKSPACE,
                              "workspace must be 256-byte aligned");
    if (bytes < need)
        return set_last_error(ELSAA_ERR_WORKSPACE,
                              "workspace too small: %zu bytes given, %zu "
                              "needed",
                              bytes, need);
    return ELSAA_OK;
}

}  // namespace

extern "C" int elsaa_cache_workspace_size(const elsaa_cache *cache, int T,
                                          int weights, int keep,
                                          size_t *bytes) {
    clear_last_error();
    if (!bytes)
        return set_last_error(ELSAA_ERR_INVALID_ARG, "bytes is NULL");
    CacheView c;
    int rc = make_view(cache, T, &c);
    if (rc == ELSAA_OK) rc = check_queries(c);
    if (rc != ELSAA_OK) return rc;
    if (keep < 0)
        return set_last_error(ELSAA_ERR_INVALID_ARG, "keep must be >= 0");
    rc = check_keep(keep);
    if (rc != ELSAA_OK) return rc;
    // fewer tokens never need more
    size_t n =
        attention_layout(c, on_tensor_cores(cache, c), weights != 0).total;
    if (select_bytes(c) > n) n = select_bytes(c);
    if (evict_bytes(c, keep) > n) n = evict_bytes(c, keep);
    *bytes = n;
    return ELSAA_OK;
}

extern "C" int elsaa_cache_append(const elsaa_cache *cache, int T,
                                  const void *k, const void *v,
                                  const int32_t *new_len, void *stream) {
    clear_last_error();
    CacheView c;
    const int rc = make_view(cache, T, &c);
    if (rc != ELSAA_OK) return rc;
    if (T <= 0)
        return set_last_error(ELSAA_ERR_INVALID_ARG, "T must be positive");
    // a sequence with few of the T rows may be at the end of its table already:
    // the pages that all T would take from there on are numbered too
    if (T > kCacheMaxSlots - (long)c.max_pages * c.ps)
        return set_last_error(ELSAA_ERR_UNSUPPORTED,
                              "T + max_pages * page_size must be at most "
                              "2^31 - 2^16");
    if (!k || !v)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "k and v must be non-NULL");
    if (misaligned(k, 16) || misaligned(v, 16))
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "k and v must be 16-byte aligned");
    c.new_len = new_len;
    cudaStream_t st = (cudaStream_t)stream;
    ELSAA_CACHE_LAUNCH("cache_append", st, launch_cache_append(c, k, v, st));
    return ELSAA_OK;
}

extern "C" int elsaa_cache_select(const elsaa_cache *cache, int T,
                                  const void *q, const int32_t *new_len,
                                  int n_sel, int first, int last,
                                  int32_t *pages, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    clear_last_error();
    CacheView c;
    int rc = make_view(cache, T, &c);
    if (rc == ELSAA_OK) rc = check_queries(c);
    if (rc != ELSAA_OK) return rc;
    if (!q || !pages)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "q and pages must be non-NULL");
    if (misaligned(q, 16))
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "q must be 16-byte aligned");
    if (n_sel <= 0 || first < 0 || last < 0 || first > n_sel ||
        last > n_sel - first)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "n_sel must be positive, first and last >= 0 "
                              "and first + last at most n_sel");
    if (n_sel > kCacheMaxSlots / c.ps)
        return set_last_error(ELSAA_ERR_UNSUPPORTED,
                              "n_sel * page_size must be at most 2^31 - 2^16");
    rc = check_workspace(workspace, workspace_bytes, select_bytes(c));
    if (rc != ELSAA_OK) return rc;
    c.new_len = new_len;
    cudaStream_t st = (cudaStream_t)stream;
    ELSAA_CACHE_LAUNCH("cache_select", st,
                       launch_cache_select(c, q, n_sel, first, last, pages,
                                           (float *)workspace, st));
    return ELSAA_OK;
}

extern "C" int elsaa_cache_attention(const elsaa_cache *cache, int T,
                                     const void *q, const int32_t *new_len,
                                     const int32_t *pages, int n_sel,
                                     const float *weight_in,
                                     float *weight_out, void *o, float *lse,
                                     void *workspace, size_t workspace_bytes,
                                     void *stream) {
    clear_last_error();
    CacheAttn A = {};
    int rc = make_view(cache, T, &A.c);
    if (rc == ELSAA_OK) rc = check_queries(A.c);
    if (rc != ELSAA_OK) return rc;
    const CacheView &c = A.c;
    if (!q || !o)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "q and o must be non-NULL");
    if (misaligned(q, 16) || misaligned(o, 16))
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "q and o must be 16-byte aligned");
    if (misaligned(weight_in, 16) || misaligned(weight_out, 16))
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "weight_in and weight_out must be 16-byte "
                              "aligned");
    if (weight_in && !weight_out)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "weight_in needs weight_out");
    if (pages && (n_sel <= 0 || (long)n_sel * c.ps > 0x7fffffffL))
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "n_sel must be positive and n_sel * page_size "
                              "fit in int32");
    const bool tc = on_tensor_cores(cache, c);
    const Layout l = attention_layout(c, tc, weight_out != nullptr);
    rc = check_workspace(workspace, workspace_bytes, l.total);
    if (rc != ELSAA_OK) return rc;
    char *ws = (char *)workspace;
    A.c.new_len = new_len;
    A.q = q;
    A.o = o;
    A.lse = lse;
    A.pages = pages;
    A.n_sel = pages ? n_sel : 0;
    A.weight_in = weight_in;
    A.weight_out = weight_out;
    A.cols = l.cols;
    A.groups = l.groups;
    A.ctas = l.ctas;
    const long items = (long)c.B * c.Hkv * l.groups;
    const long table = (long)c.max_pages * c.ps;
    const long listed = pages ? (long)n_sel * c.ps : table;
    const long tiles =
        ((listed < table ? listed : table) + kCacheTile - 1) / kCacheTile;
    A.whole = tc && c.B <= kCacheWholeSeqs && items <= kCacheTcCtas &&
              tiles <= kCacheWhole &&
              tiles - items * tiles / kCacheTcCtas <= kCacheMore;
    A.per_t = (65535u + T) / T;
    if (A.whole) A.ctas = (int)items;
    A.split = (CacheSplit *)(ws + l.split);
    A.part = (float *)(ws + l.part);
    if (weight_out) {
        A.lse2 = (float *)(ws + l.lse2);
        A.scores = (float *)(ws + l.scores);
        A.slots = (long)c.max_pages * c.ps;
    }
    cudaStream_t st = (cudaStream_t)stream;
    if (tc)
        ELSAA_CACHE_LAUNCH("cache_attn_tc", st, launch_cache_attn_tc(A, st));
    else
        ELSAA_CACHE_LAUNCH("cache_attn_simt", st,
                           launch_cache_attn_simt(A, st));
    if (!A.whole)
        ELSAA_CACHE_LAUNCH("cache_merge", st, launch_cache_merge(A, tc, st));
    if (weight_out)
        ELSAA_CACHE_LAUNCH("cache_weights", st, launch_cache_weights(A, st));
    return ELSAA_OK;
}

extern "C" int elsaa_cache_evict(const elsaa_cache *cache,
                                 const float *weight, int keep, int recent,
                                 const int32_t *dst_table, int dst_pages,
                                 float *weight_out, int32_t *lengths_out,
                                 int32_t *kept, void *workspace,
                                 size_t workspace_bytes, void *stream) {
    clear_last_error();
    CacheView c;
    int rc = make_view(cache, 0, &c);
    if (rc != ELSAA_OK) return rc;
    if (!weight || !dst_table || !weight_out || !lengths_out)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "weight, dst_table, weight_out and lengths_out "
                              "must be non-NULL");
    if (weight == weight_out)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "weight_out must not be weight");
    if (keep <= 0 || recent < 0 || recent > keep)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "keep must be positive and recent in [0, keep]");
    rc = check_keep(keep);
    if (rc != ELSAA_OK) return rc;
    if (dst_pages <= 0 || (long)dst_pages * c.ps < keep)
        return set_last_error(ELSAA_ERR_INVALID_ARG,
                              "dst_pages * page_size must be at least keep");
    rc = check_workspace(workspace, workspace_bytes, evict_bytes(c, keep));
    if (rc != ELSAA_OK) return rc;
    CacheKept out;
    out.count = (int *)workspace;
    out.rows = (int32_t *)((char *)workspace +
                           align256(sizeof(int) * (size_t)c.B));
    out.kept = kept;
    out.weight_out = weight_out;
    out.dst_pages = dst_pages;
    cudaStream_t st = (cudaStream_t)stream;
    ELSAA_CACHE_LAUNCH("cache_keep", st,
                       launch_cache_keep(c, weight, keep, recent, out, st));
    ELSAA_CACHE_LAUNCH("cache_compact", st,
                       launch_cache_compact(c, keep, out.rows, out.count,
                                            dst_table, dst_pages, lengths_out,
                                            st));
    return ELSAA_OK;
}
