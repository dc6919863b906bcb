// Appending rows to the paged key/value cache (include/attn_paged.h): K rotated on the way, Q beside it.
#include "attn_paged.hpp"

namespace attn {

constexpr int kAppendThreads = 256;
constexpr float kE4m3Max = 448.0f;

// Column c of a row at position p, rotated: the same two fused multiply-adds as the rotary kernel's.
__device__ __forceinline__ float rotated(const PagedAppendArgs &a, const elem *row, int c, int64_t p)
{
    const int half = a.rot / 2;
    const float x = (float)row[c];
    if (c >= a.rot) return x;
    const int j = c < half ? c : c - half;
    const float cs = a.cos_table[p * half + j], sn = a.sin_table[p * half + j];
    return c < half ? __builtin_fmaf(x, cs, -((float)row[c + half] * sn)) : __builtin_fmaf(x, cs, (float)row[j] * sn);
}

// One work-group for each token: its Q row, and with a 16-bit cache its K and V rows.
__global__ void __launch_bounds__(kAppendThreads) attn_paged_append_kernel(const PagedAppendArgs a)
{
    const int t = blockIdx.x, b = paged_seq_of(a.b, t);
    if (b == a.b.B) return;
    const PagedSeq s = paged_seq(a.b, b);
    const int p = s.len - s.n + t - s.first;
    if (t < s.first || p < 0) return;
    const int D = a.D;
    if (a.Q_rot) {
        for (int i = threadIdx.x; i < a.Hq * D / 2; i += kAppendThreads) {
            // (both columns of a pair by one thread: Q_rot may be Q)
            const int h = i / (D / 2), j = i - h * (D / 2), half = a.rot / 2;
            const int c0 = j < half ? j : j + half, c1 = j < half ? j + half : j + D / 2;
            const int lo = j < half ? c0 : 2 * j, hi = j < half ? c1 : 2 * j + 1;
            const elem *row = a.Q + t * a.q_stride_t + h * a.q_stride_h;
            const float y0 = rotated(a, row, lo, p), y1 = rotated(a, row, hi, p);
            elem *out = a.Q_rot + t * a.out_stride_t + h * a.out_stride_h;
            out[lo] = (elem)y0;
            out[hi] = (elem)y1;
        }
    }
    const int page = a.b.page_of(b, p);
    if (a.k_scale || !a.b.is_page(page)) return;
    for (int i = threadIdx.x; i < a.Hkv * D; i += kAppendThreads) {
        const int h = i / D, c = i - h * D;
        const int64_t from = t * a.kv_stride_t + h * a.kv_stride_h;
        const int64_t to = page * a.cache_stride_p + h * a.cache_stride_h +
                           (p & (a.b.page_size() - 1)) * a.cache_stride_s + c;
        ((elem *)a.K_cache)[to] = (elem)rotated(a, a.K + from, c, p);
        ((elem *)a.V_cache)[to] = a.V[from + c];
    }
}

// The least power of two, 2^-100 at least, by which values of up to amax (> 0) fit e4m3: 448 = 1.75 * 2^8.
__device__ __forceinline__ float e4m3_scale(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    return __uint_as_float((uint32_t)(min(max(e, -100), 120) + 127) << 23);
}
__device__ __forceinline__ uint8_t to_e4m3(float x)
{
    x = fminf(fmaxf(x, -kE4m3Max), kE4m3Max);
    return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false);
}

// e4m3 cache: one work-group for each page that gets rows (slot), head and tensor.  Sequence b has the slots from
// q_start[b] / P + 2 b on: n rows touch at most n / P + 2 pages, so they do not reach into the next one's.
__global__ void __launch_bounds__(kAppendThreads) attn_paged_append8_kernel(const PagedAppendArgs a)
{
    __shared__ float most[kAppendThreads];
    const int P = a.b.page_size(), sh = a.b.page_shift, u = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, D = a.D;
    int b = 0;
    while (b < a.b.B && (min(max(a.b.q_start[b + 1], 0), a.b.T) >> sh) + 2 * (b + 1) <= u) ++b;
    if (b == a.b.B) return;
    const PagedSeq s = paged_seq(a.b, b);
    const int older = max(s.len - s.n, 0), slot = u - (s.first >> sh) - 2 * b;
    if (slot < 0) return;
    const int in_seq = (older >> sh) + slot;  // which of the sequence's pages
    if (s.n == 0 || ((int64_t)in_seq << sh) >= s.len) return;
    const int page = a.b.page_of(b, in_seq << sh);
    if (!a.b.is_page(page)) return;
    const int p0 = in_seq << sh, lo = max(older, p0), hi = min(s.len, p0 + P);
    const elem *from = (blockIdx.z ? a.V : a.K) + h * a.kv_stride_h;
    uint8_t *to = (uint8_t *)(blockIdx.z ? a.V_cache : a.K_cache) + page * a.cache_stride_p + h * a.cache_stride_h;
    float *scale = (blockIdx.z ? a.v_scale : a.k_scale) + (int64_t)page * a.Hkv + h;
    const int t0 = s.first + s.n - s.len;  // packed row of position 0
    auto value = [&](int i) {
        const int p = lo + i / D, c = i % D;
        const elem *row = from + (t0 + p) * a.kv_stride_t;
        return blockIdx.z ? (float)row[c] : rotated(a, row, c, p);
    };
    float amax = 0.f;
    for (int i = tid; i < (hi - lo) * D; i += kAppendThreads) amax = fmaxf(amax, fabsf(value(i)));
    most[tid] = amax;
    __syncthreads();
    for (int n = kAppendThreads / 2; n; n /= 2) {
        if (tid < n) most[tid] = fmaxf(most[tid], most[tid + n]);
        __syncthreads();
    }
    const float before = lo > p0 ? *scale : 0.f;
    const float by = fmaxf(e4m3_scale(most[0]), before);
    if (by > before)
        for (int i = tid; i < (lo - p0) * D; i += kAppendThreads) {
            uint8_t *x = to + i / D * a.cache_stride_s + i % D;
            *x = to_e4m3(__builtin_amdgcn_cvt_f32_fp8(*x, 0) * (before / by));
        }
    for (int i = tid; i < (hi - lo) * D; i += kAppendThreads)
        to[(lo - p0 + i / D) * a.cache_stride_s + i % D] = to_e4m3(value(i) / by);
    __syncthreads();
    if (tid == 0) *scale = by;
}

int launch_paged_append(const PagedAppendArgs &a, hipStream_t st)
{
    if (a.Q_rot || !a.k_scale)
        hipLaunchKernelGGL(attn_paged_append_kernel, dim3(a.b.T), dim3(kAppendThreads), 0, st, a);
    if (a.k_scale)
        hipLaunchKernelGGL(attn_paged_append8_kernel, dim3((a.b.T >> a.b.page_shift) + 2 * a.b.B, a.Hkv, 2),
                           dim3(kAppendThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace attn
