// C ABI of the paged key/value cache: host-side validation and dispatch only.
#include "../../include/attn_paged.h"
#include "attn_paged.hpp"

#include <algorithm>
#include <cmath>
#include <limits>

namespace {

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int check_paged(const attn_paged_params_t *p, bool e4m3)
{
    if (!p) return ATTN_ERR_NULL;
    const int64_t lim = std::numeric_limits<int32_t>::max();
    if (p->T < 0 || p->B < 0 || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv || p->pages < 1 || p->table_width < 1)
        return ATTN_ERR_SHAPE;
    if (p->D < 8 || p->D > 256 || p->D % (e4m3 ? 16 : 8)) return ATTN_ERR_SHAPE;
    if (p->page_size < 16 || p->page_size > 4096 || (p->page_size & (p->page_size - 1))) return ATTN_ERR_SHAPE;
    if (p->table_stride < p->table_width) return ATTN_ERR_STRIDE;
    if ((int64_t)p->table_width * p->page_size > (1 << 30) || (int64_t)p->T * p->Hq > lim ||
        p->Hq > 65535 ||
        // (work-groups of the appending kernel)
        ((int64_t)p->T / p->page_size + 2 * (int64_t)p->B) * p->Hkv * 2 + p->T > lim)
        return ATTN_ERR_SHAPE;
    for (int64_t s : {p->q_stride_t, p->q_stride_h, p->out_stride_t, p->out_stride_h})
        if (s < 0 || s % 8) return ATTN_ERR_STRIDE;
    // rows that are written lie apart (those that are read may be one)
    if ((p->T > 1 && p->out_stride_t < p->D) || (p->Hq > 1 && p->out_stride_h < p->D)) return ATTN_ERR_STRIDE;
    const int64_t size = e4m3 ? 1 : 2, unit = 16 / size;
    if (p->cache_stride_s < p->D || p->cache_stride_h < 1 || p->cache_stride_p < 1 || p->cache_stride_s % unit ||
        p->cache_stride_h % unit || p->cache_stride_p % unit || p->page_size * p->cache_stride_s * size > (1 << 30))
        return ATTN_ERR_STRIDE;
    return ATTN_OK;
}

attn::PagedBatch batch_of(const attn_paged_params_t *p, const int32_t *page_table, const int32_t *q_start,
                          const int32_t *kv_lens)
{
    attn::PagedBatch b;
    b.page_table = page_table; b.q_start = q_start; b.kv_lens = kv_lens;
    b.T = p->T; b.B = p->B; b.pages = p->pages; b.table_width = p->table_width;
    b.table_stride = p->table_stride;
    b.page_shift = __builtin_ctz((unsigned)p->page_size);
    return b;
}

template <typename E>
int append_impl(const void *K, const void *V, const void *Q, void *Q_rot, const float *cos_table,
                const float *sin_table, void *K_cache, void *V_cache, float *k_scale, float *v_scale,
                const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens,
                const attn_paged_params_t *p, void *hip_stream)
{
    if (!k_scale != !v_scale) return ATTN_ERR_NULL;
    const int rc = check_paged(p, k_scale != nullptr);
    if (rc != ATTN_OK) return rc;
    if (p->rot < 0 || p->rot > p->D || p->rot % 8) return ATTN_ERR_SHAPE;
    if (p->rot && p->table_rows < (int64_t)p->table_width * p->page_size) return ATTN_ERR_SHAPE;
    if (p->kv_stride_t < 0 || p->kv_stride_h < 0 || p->kv_stride_t % 8 || p->kv_stride_h % 8) return ATTN_ERR_STRIDE;
    if (p->T == 0 || p->B == 0) return ATTN_OK;
    if (!K || !V || !K_cache || !V_cache || !page_table || !q_start || !kv_lens || !Q != !Q_rot ||
        (p->rot && (!cos_table || !sin_table)))
        return ATTN_ERR_NULL;
    if (!aligned(K, 16) || !aligned(V, 16) || !aligned(Q, 16) || !aligned(Q_rot, 16) || !aligned(cos_table, 16) ||
        !aligned(sin_table, 16) || !aligned(K_cache, 16) || !aligned(V_cache, 16) || !aligned(k_scale, 4) ||
        !aligned(v_scale, 4) || !aligned(page_table, 4) || !aligned(q_start, 4) || !aligned(kv_lens, 4))
        return ATTN_ERR_ALIGN;
    attn::PagedAppendArgsT<E> a;
    a.b = batch_of(p, page_table, q_start, kv_lens);
    a.K = static_cast<const E *>(K); a.V = static_cast<const E *>(V);
    a.Q = static_cast<const E *>(Q); a.Q_rot = static_cast<E *>(Q_rot);
    a.cos_table = cos_table; a.sin_table = sin_table;
    a.K_cache = K_cache; a.V_cache = V_cache; a.k_scale = k_scale; a.v_scale = v_scale;
    a.Hq = p->Hq; a.Hkv = p->Hkv; a.D = p->D; a.rot = p->rot;
    a.q_stride_t = p->q_stride_t; a.q_stride_h = p->q_stride_h;
    a.out_stride_t = p->out_stride_t; a.out_stride_h = p->out_stride_h;
    a.kv_stride_t = p->kv_stride_t; a.kv_stride_h = p->kv_stride_h;
    a.cache_stride_p = p->cache_stride_p; a.cache_stride_h = p->cache_stride_h; a.cache_stride_s = p->cache_stride_s;
    return attn::launch_paged_append(a, static_cast<hipStream_t>(hip_stream)) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

template <typename E>
int fwd_impl(const void *Q, const void *K_cache, const void *V_cache, const float *k_scale, const float *v_scale,
             const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens, void *O, float *LSE,
             void *workspace, size_t workspace_bytes, const attn_paged_params_t *p, void *hip_stream)
{
    if (!k_scale != !v_scale) return ATTN_ERR_NULL;
    const int rc = check_paged(p, k_scale != nullptr);
    if (rc != ATTN_OK) return rc;
    if (p->max_q < 1 && p->T > 0) return ATTN_ERR_SHAPE;
    // (what all tiles of keys together count in the spans of the work-groups)
    const int64_t units = (int64_t)p->T * (p->Hq / p->Hkv) / 128 + p->B, keys = (int64_t)p->table_width * p->page_size;
    if (units > std::numeric_limits<int32_t>::max() ||
        units * (keys / 32 + 16) > std::numeric_limits<int32_t>::max() / p->Hkv)
        return ATTN_ERR_SHAPE;
    if (!std::isfinite(p->scale) || !(p->scale > 0.0f)) return ATTN_ERR_SCALE;
    if (p->T == 0 || p->B == 0) return ATTN_OK;
    if (!Q || !K_cache || !V_cache || !page_table || !q_start || !kv_lens || !O || !LSE) return ATTN_ERR_NULL;
    if (!aligned(Q, 16) || !aligned(K_cache, 16) || !aligned(V_cache, 16) || !aligned(k_scale, 4) ||
        !aligned(v_scale, 4) || !aligned(page_table, 4) || !aligned(q_start, 4) || !aligned(kv_lens, 4) ||
        !aligned(O, 16) || !aligned(LSE, 4))
        return ATTN_ERR_ALIGN;
    if (workspace && (!aligned(workspace, 256) || workspace_bytes < attn_fwd_paged_workspace_bytes(p)))
        return ATTN_ERR_WORKSPACE;
    attn::PagedFwdArgsT<E> a;
    a.b = batch_of(p, page_table, q_start, kv_lens);
    a.Q = static_cast<const E *>(Q); a.O = static_cast<E *>(O); a.LSE = LSE;
    a.K_cache = K_cache; a.V_cache = V_cache; a.k_scale = k_scale; a.v_scale = v_scale;
    a.Hq = p->Hq; a.Hkv = p->Hkv; a.Dr = p->D; a.causal = p->causal != 0; a.max_q = p->max_q;
    a.scale_log2e = p->scale * 1.4426950408889634f;
    a.q_stride_t = p->q_stride_t; a.q_stride_h = p->q_stride_h;
    a.out_stride_t = p->out_stride_t; a.out_stride_h = p->out_stride_h;
    a.cache_stride_p = p->cache_stride_p; a.cache_stride_h = p->cache_stride_h; a.cache_stride_s = p->cache_stride_s;
    a.workspace = workspace;
    return attn::launch_paged_fwd(a, static_cast<hipStream_t>(hip_stream)) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

}  // namespace

extern "C" {

void attn_paged_params_contiguous(attn_paged_params_t *p, int32_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D,
                                  int32_t pages, int32_t page_size, int32_t table_width, float scale, int32_t causal)
{
    if (!p) return;
    p->T = T; p->B = B; p->Hq = Hq; p->Hkv = Hkv; p->D = D;
    p->pages = pages; p->page_size = page_size; p->table_width = table_width;
    p->table_stride = table_width;
    p->max_q = T; p->causal = causal; p->rot = 0; p->table_rows = 0; p->scale = scale;
    p->q_stride_h = p->out_stride_h = D; p->q_stride_t = p->out_stride_t = (int64_t)Hq * D;
    p->kv_stride_h = D; p->kv_stride_t = (int64_t)Hkv * D;
    p->cache_stride_s = D; p->cache_stride_h = (int64_t)page_size * D;
    p->cache_stride_p = (int64_t)Hkv * page_size * D;
}

int attn_paged_append(const void *K, const void *V, const void *Q, void *Q_rot, const float *cos_table,
                      const float *sin_table, void *K_cache, void *V_cache, float *k_scale, float *v_scale,
                      const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens,
                      const attn_paged_params_t *p, void *hip_stream)
{
    return append_impl<__bf16>(K, V, Q, Q_rot, cos_table, sin_table, K_cache, V_cache, k_scale, v_scale, page_table,
                               q_start, kv_lens, p, hip_stream);
}

int attn_paged_append_f16(const void *K, const void *V, const void *Q, void *Q_rot, const float *cos_table,
                          const float *sin_table, void *K_cache, void *V_cache, float *k_scale, float *v_scale,
                          const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens,
                          const attn_paged_params_t *p, void *hip_stream)
{
    return append_impl<_Float16>(K, V, Q, Q_rot, cos_table, sin_table, K_cache, V_cache, k_scale, v_scale, page_table,
                                 q_start, kv_lens, p, hip_stream);
}

size_t attn_fwd_paged_workspace_bytes(const attn_paged_params_t *p)
{
    if (check_paged(p, false) != ATTN_OK || p->max_q < 1 || p->T == 0 || p->B == 0) return 0;
    // (which cache it is going to be is not known here)
    const int64_t keys = (int64_t)p->table_width * p->page_size;
    return std::max(attn::paged_plan(p->T, p->B, p->Hq, p->Hkv, p->D, p->max_q, keys, false).bytes,
                    attn::paged_plan(p->T, p->B, p->Hq, p->Hkv, p->D, p->max_q, keys, true).bytes);
}

int attn_fwd_paged(const void *Q, const void *K_cache, const void *V_cache, const float *k_scale, const float *v_scale,
                   const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens, void *O, float *LSE,
                   void *workspace, size_t workspace_bytes, const attn_paged_params_t *p, void *hip_stream)
{
    return fwd_impl<__bf16>(Q, K_cache, V_cache, k_scale, v_scale, page_table, q_start, kv_lens, O, LSE, workspace,
                            workspace_bytes, p, hip_stream);
}

int attn_fwd_paged_f16(const void *Q, const void *K_cache, const void *V_cache, const float *k_scale,
                       const float *v_scale, const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens,
                       void *O, float *LSE, void *workspace, size_t workspace_bytes, const attn_paged_params_t *p,
                       void *hip_stream)
{
    return fwd_impl<_Float16>(Q, K_cache, V_cache, k_scale, v_scale, page_table, q_start, kv_lens, O, LSE, workspace,
                              workspace_bytes, p, hip_stream);
}

}  // extern "C"
