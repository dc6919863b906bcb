// Attention over the paged key/value cache (include/attn_paged.h).
#include "attn_paged.hpp"

namespace attn {

// One wave for each row and query head: 64 keys at a time, first a score a lane, then four columns a lane.
__global__ void __launch_bounds__(64) attn_paged_fwd_kernel(const PagedFwdArgs a, const int longer)
{
    __shared__ float probs[64];
    __shared__ int64_t at[64];
    const int t = blockIdx.x, hq = blockIdx.y, h = hq / (a.Hq / a.Hkv), l = threadIdx.x, D = a.Dr;
    const int b = paged_seq_of(a.b, t);
    if (b == a.b.B) return;
    const PagedSeq s = paged_seq(a.b, b);
    if (t < s.first || (int64_t)s.n * (a.Hq / a.Hkv) <= longer || s.n > a.max_q) return;
    const int seen = a.causal ? min(s.len, s.len - s.n + t - s.first + 1) : s.len;
    const elem *q = a.Q + t * a.q_stride_t + hq * a.q_stride_h;
    auto value = [&](const void *cache, int64_t i, float scale) {
        return a.k_scale ? __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)cache)[i], 0) * scale
                         : (float)((const elem *)cache)[i];
    };
    float m = -INFINITY, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < seen; k0 += 64) {
        const int k = k0 + l;
        float x = -INFINITY;
        int page = -1;
        if (k < seen) page = a.b.page_of(b, k);
        if (a.b.is_page(page)) {
            const int64_t i = page * a.cache_stride_p + h * a.cache_stride_h +
                              (k & (a.b.page_size() - 1)) * a.cache_stride_s;
            const float scale = a.k_scale ? a.k_scale[(int64_t)page * a.Hkv + h] : 1.f;
            x = 0.f;
            for (int c = 0; c < D; ++c) x += (float)q[c] * value(a.K_cache, i + c, scale);
            x *= a.scale_log2e;
            at[l] = i;
        }
        float top = x;
        for (int d = 32; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
        const float m_new = fmaxf(m, top);
        if (m_new == -INFINITY) continue;
        float p = fast_exp2(x - m_new), all = p;
        for (int d = 32; d; d /= 2) all += __shfl_xor(all, d);
        const float keep = fast_exp2(m - m_new);
        sum = sum * keep + all;
        m = m_new;
        // (a key that is not seen has probability 0 and no place)
        probs[l] = a.v_scale && p > 0.f ? p * a.v_scale[(int64_t)page * a.Hkv + h] : p;
        __syncthreads();
        for (int i = 0; i < 4; ++i) o[i] *= keep;
        for (int j = 0; j < 64; ++j)
            if (probs[j] > 0.f)
                for (int i = 0; i < 4; ++i)
                    if (l + 64 * i < D) o[i] += probs[j] * value(a.V_cache, at[j] + l + 64 * i, 1.f);
        __syncthreads();
    }
    elem *out = a.O + t * a.out_stride_t + hq * a.out_stride_h;
    for (int i = 0; i < 4; ++i)
        if (l + 64 * i < D) out[l + 64 * i] = (elem)(sum > 0.f ? o[i] / sum : 0.f);
    if (l == 0) a.LSE[(int64_t)t * a.Hq + hq] = sum > 0.f ? (m + fast_log2(sum)) * kLn2 : -INFINITY;
}

int launch_paged_fwd(const PagedFwdArgs &a, hipStream_t st)
{
    const PagedPlan p = paged_plan(a.b.B, a.Hq, a.Hkv, a.Dr, a.max_q, (int64_t)a.b.table_width << a.b.page_shift,
                                   a.k_scale != nullptr);
    if (p.decode_rows && launch_paged_decode(a, p.kernel_d, p.decode_rows, a.workspace ? p.decode_workers : 0, st) != 0) return -1;
    if (p.chunks)
        hipLaunchKernelGGL(attn_paged_fwd_kernel, dim3(a.b.T, a.Hq), dim3(64), 0, st, a, p.decode_rows);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace attn
