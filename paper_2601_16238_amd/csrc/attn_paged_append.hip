// Appending rows to the paged key/value cache (include/attn_paged.h): K rotated on the way, Q beside it.
//
// Nothing is computed that would count: the kernels move bytes.  A row is worked on in units of twice W columns: columns
// j .. j+W-1 and their partners j + rot/2 .., which are rotated together, or 2 W consecutive ones behind the rotated.
// W = 8 (16-byte accesses) where such units cover a row, that is rot and D are multiples of 16, otherwise 4: prompts of 13K
// tokens (272 MB, fp16 or bf16) in 51.5 us, 5.3 TB/s, which is what a copy reaches; 61.9 with W = 4.
#include "attn_paged.hpp"

#include <algorithm>

namespace attn {

constexpr float kE4m3Max = 448.0f;
constexpr int kAppendKeep = 4;  // units that a thread keeps in registers

template <int W>
struct Unit {
    float a[W], b[W];  // columns A .. and B ..
};
template <int W>
struct Columns {
    int A, B;
    bool turned;
    __device__ Columns(int u, int rot)
    {
        const int pairs = rot / (2 * W);
        turned = u < pairs;
        A = turned ? u * W : rot + (u - pairs) * 2 * W;
        B = turned ? A + rot / 2 : A + W;
    }
};
template <int W>
__device__ __forceinline__ void load_columns(const elem *p, float (&x)[W])
{
    typedef elem vec __attribute__((ext_vector_type(W)));
    const vec v = *(const vec *)p;
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = (float)v[i];
}
template <int W>
__device__ __forceinline__ void store_columns(elem *p, const float (&x)[W])
{
    typedef elem vec __attribute__((ext_vector_type(W)));
    typedef float vecf __attribute__((ext_vector_type(W)));
    vecf v;
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = x[i];
    *(vec *)p = __builtin_convertvector(v, vec);
}
// Rotated by row p of the tables: the two fused multiply-adds of the rotary kernel, so that both give the same bits.
template <int W>
__device__ __forceinline__ void turn(const PagedAppendArgs &a, int64_t p, int j, Unit<W> &x)
{
    const float *cs = a.cos_table + p * (a.rot / 2) + j, *sn = a.sin_table + p * (a.rot / 2) + j;
#pragma unroll
    for (int q = 0; q < W; q += 4) {
        const f32x4 c = *(const f32x4 *)(cs + q), s = *(const f32x4 *)(sn + q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = x.a[q + i], hi = x.b[q + i];
            x.a[q + i] = __builtin_fmaf(lo, c[i], -(hi * s[i]));
            x.b[q + i] = __builtin_fmaf(hi, c[i], lo * s[i]);
        }
    }
}

// i divided by the units of a row.
__device__ __forceinline__ int row_of(const PagedAppendArgs &a, int i) { return a.nu_magic ? __umulhi(i, a.nu_magic) : i; }

// A work-group for each token, so that its sequence, position and page are found once for all heads.
// The rows of token t by one work-group: of Q, and (KV) of K and V, with a 16-bit cache.
template <int W, bool KV>
__device__ __forceinline__ void append_token(const PagedAppendArgs &a, int t)
{
    const int b = paged_seq_of(a.b, t);
    if (b == a.b.B) return;
    const PagedSeq s = paged_seq_scalar(a.b, __builtin_amdgcn_readfirstlane(b));
    const int p = s.len - s.n + t - s.first;
    if (t < s.first || p < 0) return;
    const int nu = a.D / (2 * W), Hq = a.Q_rot ? a.Hq : 0;
    int page = -1;
    if (KV) page = scalar_load(a.b.page_table + (int64_t)b * a.b.table_stride + (p >> a.b.page_shift));
    const int rows = Hq + (KV && a.b.is_page(page) ? 2 * a.Hkv : 0);
    const int64_t to = page * a.cache_stride_p + (p & (a.b.page_size() - 1)) * a.cache_stride_s;
    for (int i = threadIdx.x; i < rows * nu; i += blockDim.x) {
        const int row = row_of(a, i), u = i - row * nu;
        const bool is_q = row < Hq, is_k = row < Hq + a.Hkv;
        const int h = is_q ? row : is_k ? row - Hq : row - Hq - a.Hkv;
        const Columns<W> c(u, is_k ? a.rot : 0);
        const elem *from = is_q ? a.Q + t * a.q_stride_t + h * a.q_stride_h
                                : (is_k ? a.K : a.V) + t * a.kv_stride_t + h * a.kv_stride_h;
        elem *out = is_q ? a.Q_rot + t * a.out_stride_t + h * a.out_stride_h
                         : (elem *)(is_k ? a.K_cache : a.V_cache) + to + h * a.cache_stride_h;
        Unit<W> x;
        load_columns<W>(from + c.A, x.a);
        load_columns<W>(from + c.B, x.b);
        if (c.turned) turn<W>(a, p, c.A, x);
        store_columns<W>(out + c.A, x.a);
        store_columns<W>(out + c.B, x.b);
    }
}

template <int W>
__global__ void __launch_bounds__(512) attn_paged_append_kernel(const PagedAppendArgs a)
{
    append_token<W, true>(a, blockIdx.x);
}

// The least power of two, 2^-100 at least, by which values of up to amax fit e4m3: 448 = 1.75 * 2^8.
__device__ __forceinline__ float e4m3_scale(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    return __uint_as_float((uint32_t)(min(max(e, -100), 120) + 127) << 23);
}
__device__ __forceinline__ uint32_t to_e4m3(float x0, float x1, float x2, float x3)
{
    auto in = [](float x) { return fminf(fmaxf(x, -kE4m3Max), kE4m3Max); };
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(in(x0), in(x1), 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(in(x2), in(x3), lo, true);
}
template <int W>
__device__ __forceinline__ void store_codes(uint8_t *p, const float (&x)[W], float by)
{
#pragma unroll
    for (int i = 0; i < W; i += 4)
        *(uint32_t *)(p + i) = to_e4m3(x[i] * by, x[i + 1] * by, x[i + 2] * by, x[i + 3] * by);
}

// e4m3 cache: one work-group for each page that gets rows (slot), head and tensor; behind them one for each token's Q.
// Sequence b has the slots from q_start[b] / P + 2 b on: n rows touch at most n / P + 2 pages, so they do not reach into
// the next one's.  A page's new values are read once, where a thread can keep its units of them (kAppendKeep), and a second
// time for pages of more than kAppendKeep THREADS units.
// Bound by the rows' way through memory: prompts of 19K tokens (229 MB) in 51 us, 4.4 TB/s of the 5.1 that a copy reaches;
// one token each of 64 sequences in 5 us, that is by latency: q_start, lengths, page, then values and scale.
// A wave for each page, head and tensor where it can keep the new rows of a page (of a sequence of average length), otherwise
// four, us with 64 / 256 threads, D = 128 and 8 K/V heads: 64 sequences of 1 row 5.1 / 7.0, 32 rows 10.7 / 13.5;
// 32 sequences of 100 rows, pages of 16 rows 15.4 / 21.4, of 64 18.2 / 16.6, of 256 24.3 / 15.7; 4000 rows in one page of 4096
// 764 / 206.  (Twice as many values kept: 58 instead of 50 us for the prompts, fewer waves are resident.)
template <int W, int THREADS>
__global__ void __launch_bounds__(THREADS) attn_paged_append8_kernel(const PagedAppendArgs a, const int slots)
{
    constexpr int kKeep = kAppendKeep, kWaves = THREADS / 64;
    __shared__ float most[kWaves];
    const int tid = threadIdx.x, l = tid & 63;
    if ((int)blockIdx.x >= slots * a.Hkv * 2) {
        append_token<W, false>(a, blockIdx.x - slots * a.Hkv * 2);
        return;
    }
    const int z = blockIdx.x & 1, h = (blockIdx.x >> 1) % a.Hkv, slot = (blockIdx.x >> 1) / a.Hkv;
    const int P = a.b.page_size(), sh = a.b.page_shift, D = a.D;
    int b = -1;
    for (int b0 = 0; b0 < a.b.B && b < 0; b0 += 64) {
        const int i = b0 + l;
        const int end = (min(max(a.b.q_start[min(i, a.b.B - 1) + 1], 0), a.b.T) >> sh) + 2 * (i + 1);
        const uint64_t behind = __builtin_amdgcn_ballot_w64(i < a.b.B && end > slot);
        if (behind) b = b0 + __builtin_ctzll(behind);
    }
    if (b < 0) return;
    const PagedSeq s = paged_seq_scalar(a.b, __builtin_amdgcn_readfirstlane(b));
    const int older = max(s.len - s.n, 0), nth = slot - (s.first >> sh) - 2 * b;
    if (nth < 0) return;
    const int in_seq = (older >> sh) + nth;  // which of the sequence's pages
    if (s.n == 0 || ((int64_t)in_seq << sh) >= s.len) return;
    const int page = scalar_load(a.b.page_table + (int64_t)b * a.b.table_stride + in_seq);
    if (!a.b.is_page(page)) return;
    const int p0 = in_seq << sh, lo = max(older, p0), hi = min(s.len, p0 + P);
    const int rot = z ? 0 : a.rot, nu = D / (2 * W), units = (hi - lo) * nu;
    const elem *from = (z ? a.V : a.K) + h * a.kv_stride_h;
    uint8_t *to = (uint8_t *)(z ? a.V_cache : a.K_cache) + page * a.cache_stride_p + h * a.cache_stride_h;
    float *scale = (z ? a.v_scale : a.k_scale) + (int64_t)page * a.Hkv + h;
    const int t0 = s.first + s.n - s.len;  // packed row of position 0
    // which unit: row and columns
    auto unit = [&](int i, Unit<W> &x) __attribute__((always_inline)) {
        const int row = row_of(a, i), p = lo + row;
        const Columns<W> c(i - row * nu, rot);
        const elem *src = from + (t0 + p) * a.kv_stride_t;
        load_columns<W>(src + c.A, x.a);
        load_columns<W>(src + c.B, x.b);
        if (c.turned) turn<W>(a, p, c.A, x);
    };
    auto largest = [&](const Unit<W> &x, float most_) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < W; ++i) most_ = fmaxf(most_, fmaxf(fabsf(x.a[i]), fabsf(x.b[i])));
        return most_;
    };
    auto store = [&](int i, const Unit<W> &x, float by) __attribute__((always_inline)) {
        const int row = row_of(a, i);
        const Columns<W> c(i - row * nu, rot);
        uint8_t *out = to + (lo - p0 + row) * a.cache_stride_s;
        store_codes<W>(out + c.A, x.a, by);
        store_codes<W>(out + c.B, x.b, by);
    };
    Unit<W> kept[kKeep];
    float amax = 0.f;
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
        const int i = tid + k * THREADS;
        if (i < units) {
            unit(i, kept[k]);
            amax = largest(kept[k], amax);
        }
    }
    for (int i = tid + kKeep * THREADS; i < units; i += THREADS) {
        Unit<W> x;
        unit(i, x);
        amax = largest(x, amax);
    }
#pragma unroll
    for (int d = 32; d; d /= 2) amax = fmaxf(amax, __shfl_xor(amax, d));
    if constexpr (kWaves > 1) {
        if (l == 0) most[tid >> 6] = amax;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWaves; ++i) amax = fmaxf(amax, most[i]);
    }
    const float before = lo > p0 ? *scale : 0.f;
    const float now = fmaxf(e4m3_scale(amax), before), by = 1.0f / now;
    // the older keys take the larger scale
    if (now > before && lo > p0) {
        const float ratio = before / now;
        for (int i = tid; i < (lo - p0) * (D / 16); i += THREADS) {
            const int row = i / (D / 16);
            u32x4 *at = (u32x4 *)(to + row * a.cache_stride_s + (i - row * (D / 16)) * 16), v = *at;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8(v[k], false),
                            y = __builtin_amdgcn_cvt_pk_f32_fp8(v[k], true);
                v[k] = to_e4m3(x[0] * ratio, x[1] * ratio, y[0] * ratio, y[1] * ratio);
            }
            *at = v;
        }
    }
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
        const int i = tid + k * THREADS;
        if (i < units) store(i, kept[k], by);
    }
    for (int i = tid + kKeep * THREADS; i < units; i += THREADS) {
        Unit<W> x;
        unit(i, x);
        store(i, x, by);
    }
    // (every wave has read the old one)
    if constexpr (kWaves > 1) __syncthreads();
    if (tid == 0) *scale = now;
}

template <int W>
static int launch_append_w(PagedAppendArgs a, hipStream_t st)
{
    const int nu = a.D / (2 * W);
    a.nu_magic = (uint32_t)((((uint64_t)1 << 32) + nu - 1) / nu);
    if (!a.k_scale) {
        const int units = ((a.Q_rot ? a.Hq : 0) + 2 * a.Hkv) * nu;
        const int threads = units >= 512 ? 512 : (units + 63) / 64 * 64;
        hipLaunchKernelGGL(attn_paged_append_kernel<W>, dim3(a.b.T), dim3(threads), 0, st, a);
    } else {
        const int slots = (a.b.T >> a.b.page_shift) + 2 * a.b.B;
        const dim3 grid((unsigned)(slots * a.Hkv * 2 + (a.Q_rot ? a.b.T : 0)));
        const int64_t rows = std::min<int64_t>(a.b.page_size(), (a.b.T + a.b.B - 1) / a.b.B);
        if (rows * nu <= kAppendKeep * 64)
            hipLaunchKernelGGL((attn_paged_append8_kernel<W, 64>), grid, dim3(64), 0, st, a, slots);
        else
            hipLaunchKernelGGL((attn_paged_append8_kernel<W, 256>), grid, dim3(256), 0, st, a, slots);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_paged_append(const PagedAppendArgs &a, hipStream_t st)
{
    return a.rot % 16 == 0 && a.D % 16 == 0 ? launch_append_w<8>(a, st) : launch_append_w<4>(a, st);
}

}  // namespace attn
