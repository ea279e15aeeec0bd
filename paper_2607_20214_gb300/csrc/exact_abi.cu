// C ABI of exact attention (include/elsaa_exact.h): argument validation,
// workspace layout, launches.
#include <math.h>

#include "exact.h"

using namespace elsaa;

namespace {

size_t align256(size_t x) { return (x + 255) / 256 * 256; }
bool misaligned(const void *p) { return (uintptr_t)p % 16 != 0; }
int bad(const char *m) {
    return set_last_error(ELSAA_ERR_INVALID_ARG, "%s", m);
}
int no(const char *m) {
    return set_last_error(ELSAA_ERR_UNSUPPORTED, "%s", m);
}

template <typename F>
cudaError_t timed(const char *name, cudaStream_t st, F fn) {
    return timed_launch(
        name, st, [](void *f) { return (*(F *)f)(); }, &fn);
}

#define ELSAA_EXACT_LAUNCH(name, st, expr)                                  \
    do {                                                                    \
        const cudaError_t e_ = timed(name, st, [&] { return expr; });       \
        if (e_ != cudaSuccess)                                              \
            return set_last_error(ELSAA_ERR_CUDA, "%s: %s", name,           \
                                  cudaGetErrorString(e_));                  \
    } while (0)

int make_view(const elsaa_exact *p, ExactView *a) {
    if (!p) return bad("exact is NULL");
    if (p->B <= 0 || p->H <= 0 || p->H_kv <= 0 || p->N_q <= 0 || p->N_k <= 0)
        return bad("B, H, H_kv, N_q and N_k must be positive");
    if (p->H % p->H_kv != 0) return bad("H must be a multiple of H_kv");
    if (p->dtype != ELSAA_BF16 && p->dtype != ELSAA_FP32)
        return bad("dtype must be ELSAA_BF16 or ELSAA_FP32");
    if (p->causal != 0 && p->causal != 1)
        return bad("causal must be 0 or 1");
    if (p->impl != ELSAA_IMPL_AUTO && p->impl != ELSAA_IMPL_SIMT)
        return bad("impl must be AUTO or SIMT");
    // (times log2 e it must still be finite)
    if (!(p->scale >= 0.f && p->scale <= 1e38f))
        return bad("scale must be at least 0 and at most 1e38");
    if (p->d_h != 32 && p->d_h != 64 && p->d_h != 128)
        return no("d_h must be 32, 64 or 128");
    if (p->H > 65535) return no("H must be at most 65535");
    const long most = 1L << 30;
    if (p->N_q > most / p->B / p->H || p->N_k > most / p->B / p->H_kv)
        return no("B * H * N_q and B * H_kv * N_k must be at most 2^30");
    *a = ExactView{};
    a->B = p->B;
    a->H = p->H;
    a->Hkv = p->H_kv;
    a->G = p->H / p->H_kv;
    a->Nq = p->N_q;
    a->Nk = p->N_k;
    a->d = p->d_h;
    a->dtype = p->dtype;
    a->causal = p->causal;
    a->scale = p->scale > 0.f ? p->scale : 1.0f / sqrtf((float)p->d_h);
    return ELSAA_OK;
}

bool on_tensor_cores(const elsaa_exact *p) {
    return p->dtype == ELSAA_BF16 && p->impl == ELSAA_IMPL_AUTO;
}

// status, two work counters and a flag | D_i, or what CTAs leave of divided rows | the
// same of the backward pass
struct Layout {
    size_t next_item, scratch, part, total;
};
Layout layout(const ExactView &a, bool tensor, bool backward) {
    Layout l;
    l.next_item = sizeof(DeviceStatus);
    l.scratch = align256(l.next_item + 3 * sizeof(int));
    size_t most = tensor ? exact_share_bytes(a) : exact_chunk_bytes(a);
    const size_t delta = sizeof(float) * (size_t)a.B * a.H * a.Nq;
    if (backward && delta > most) most = delta;
    l.part = l.total = l.scratch + align256(most);
    if (backward)
        l.total +=
            align256(tensor ? exact_part_bytes(a) : exact_add_bytes(a));
    return l;
}

int check_workspace(const void *ws, size_t bytes, size_t need) {
    if (!ws) return set_last_error(ELSAA_ERR_WORKSPACE, "workspace is NULL");
    if ((uintptr_t)ws % 256 != 0)
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

extern "C" int elsaa_exact_workspace_size(const elsaa_exact *exact,
                                          int backward, size_t *bytes) {
    clear_last_error();
    if (!bytes) return bad("bytes is NULL");
    ExactView a;
    const int rc = make_view(exact, &a);
    if (rc != ELSAA_OK) return rc;
    *bytes = layout(a, on_tensor_cores(exact), backward != 0).total;
    return ELSAA_OK;
}

extern "C" int elsaa_exact_forward(const elsaa_exact *exact, const void *q,
                                   const void *k, const void *v,
                                   const int32_t *q_len,
                                   const int32_t *k_len, void *o, float *lse,
                                   void *workspace, size_t workspace_bytes,
                                   void *stream) {
    clear_last_error();
    ExactView a;
    int rc = make_view(exact, &a);
    if (rc != ELSAA_OK) return rc;
    if (!q || !k || !v || !o) return bad("q, k, v and o must be non-NULL");
    for (const void *p : {q, k, v, (const void *)o, (const void *)lse})
        if (misaligned(p)) return bad("tensors must be 16-byte aligned");
    const bool tensor = on_tensor_cores(exact);
    const Layout l = layout(a, tensor, false);
    rc = check_workspace(workspace, workspace_bytes, l.total);
    if (rc != ELSAA_OK) return rc;
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_len = q_len;
    a.k_len = k_len;
    a.out = o;
    a.lse = lse;
    a.status = (DeviceStatus *)workspace;
    cudaStream_t st = (cudaStream_t)stream;
    char *ws = (char *)workspace;
    if (tensor)
        ELSAA_EXACT_LAUNCH("exact_fwd_tc", st,
                           launch_exact_fwd_tc(a, (int *)(ws + l.next_item),
                                               (float *)(ws + l.scratch),
                                               st));
    else
        ELSAA_EXACT_LAUNCH("exact_fwd_simt", st,
                           launch_exact_fwd_simt(
                               a, (float *)(ws + l.scratch), st));
    return ELSAA_OK;
}

extern "C" int elsaa_exact_backward(
    const elsaa_exact *exact, const void *q, const void *k, const void *v,
    const void *o, const float *lse, const void *d_o, const int32_t *q_len,
    const int32_t *k_len, void *dq, void *dk, void *dv, void *workspace,
    size_t workspace_bytes, void *stream) {
    clear_last_error();
    ExactView a;
    int rc = make_view(exact, &a);
    if (rc != ELSAA_OK) return rc;
    if (!q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv)
        return bad("q, k, v, o, lse, d_o, dq, dk and dv must be non-NULL");
    for (const void *p : {q, k, v, o, (const void *)lse, d_o,
                          (const void *)dq, (const void *)dk,
                          (const void *)dv})
        if (misaligned(p)) return bad("tensors must be 16-byte aligned");
    const bool tensor = on_tensor_cores(exact);
    const Layout l = layout(a, tensor, true);
    rc = check_workspace(workspace, workspace_bytes, l.total);
    if (rc != ELSAA_OK) return rc;
    a.q = q;
    a.k = k;
    a.v = v;
    a.o = o;
    a.lse = const_cast<float *>(lse);
    a.d_o = d_o;
    a.q_len = q_len;
    a.k_len = k_len;
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    a.status = (DeviceStatus *)workspace;
    a.delta = (float *)((char *)workspace + l.scratch);
    cudaStream_t st = (cudaStream_t)stream;
    float *part = (float *)((char *)workspace + l.part);
    if (tensor) {
        int *next_item = (int *)((char *)workspace + l.next_item);
        int *far = next_item + 2;
        ELSAA_EXACT_LAUNCH("exact_delta", st,
                           launch_exact_delta(a, next_item, st));
        ELSAA_EXACT_LAUNCH("exact_dq_tc", st,
                           launch_exact_dq_tc(a, next_item, far, part, st));
        ELSAA_EXACT_LAUNCH("exact_dkv_tc", st,
                           launch_exact_dkv_tc(a, next_item + 1, far, part, st));
        ELSAA_EXACT_LAUNCH("exact_sum", st, launch_exact_sum(a, part, st));
        return ELSAA_OK;
    }
    ELSAA_EXACT_LAUNCH("exact_dq_simt", st,
                       launch_exact_bwd_simt(a, false, part, st));
    ELSAA_EXACT_LAUNCH("exact_dkv_simt", st,
                       launch_exact_bwd_simt(a, true, part, st));
    return ELSAA_OK;
}
