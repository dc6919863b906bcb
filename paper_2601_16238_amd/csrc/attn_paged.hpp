// Argument blocks, launch entry points and device helpers of the paged key/value cache (include/attn_paged.h).
#pragma once
#include "attn_device.hpp"

namespace attn {

// What the batch looks like in device memory.
struct PagedBatch {
    const int32_t *page_table, *q_start, *kv_lens;
    int T, B, pages, page_shift, table_width, table_stride;
    __host__ __device__ int page_size() const { return 1 << page_shift; }
    // the page that holds position p of sequence b
    __device__ int page_of(int b, int p) const { return page_table[(int64_t)b * table_stride + (p >> page_shift)]; }
    __device__ bool is_page(int id) const { return (unsigned)id < (unsigned)pages; }
};

template <typename E>
struct PagedAppendArgsT {
    PagedBatch b;
    const E *K, *V, *Q;
    E *Q_rot;
    const float *cos_table, *sin_table;
    void *K_cache, *V_cache;
    float *k_scale, *v_scale;  // NULL: 16-bit cache
    int Hq, Hkv, D, rot;
    uint32_t nu_magic;  // ceil(2^32 / units of a row); one unit: 0
    int64_t q_stride_t, q_stride_h, out_stride_t, out_stride_h, kv_stride_t, kv_stride_h;
    int64_t cache_stride_p, cache_stride_h, cache_stride_s;
};

template <typename E>
struct PagedFwdArgsT {
    PagedBatch b;
    const E *Q;
    const void *K_cache, *V_cache;
    const float *k_scale, *v_scale;  // NULL: 16-bit cache
    E *O;
    float *LSE;
    int Hq, Hkv, Dr, causal, max_q;
    float scale_log2e;
    int64_t q_stride_t, q_stride_h, out_stride_t, out_stride_h;
    int64_t cache_stride_p, cache_stride_h, cache_stride_s;
    void *workspace;
};
typedef PagedAppendArgsT<elem> PagedAppendArgs;
typedef PagedFwdArgsT<elem> PagedFwdArgs;

int launch_paged_append(const PagedAppendArgsT<__bf16> &a, hipStream_t st);
int launch_paged_append(const PagedAppendArgsT<_Float16> &a, hipStream_t st);
int launch_paged_fwd(const PagedFwdArgsT<__bf16> &a, hipStream_t st);
int launch_paged_fwd(const PagedFwdArgsT<_Float16> &a, hipStream_t st);
int launch_paged_decode(const PagedFwdArgsT<__bf16> &a, int D, int max_rows, int workers, hipStream_t st);
int launch_paged_decode(const PagedFwdArgsT<_Float16> &a, int D, int max_rows, int workers, hipStream_t st);

int launch_paged_chunk(const PagedFwdArgsT<__bf16> &a, int D, int workers, hipStream_t st);
int launch_paged_chunk(const PagedFwdArgsT<_Float16> &a, int D, int workers, hipStream_t st);

// Work in spans: a work-group takes the same number of tiles of keys as every other, from wherever its span begins to
// wherever it ends.  Of a unit of rows that several have worked on, each leaves a partial result in the workspace: in slot
// 2 w, or 2 w + 1 if it holds the unit's first tile, rows x D fp32 of O relative to a maximum m, in the kernel's own order,
// then m and the sums l, [2 workers][rows] each; and the one that holds the first tile says what is to be joined.
struct PagedJoin {
    int first, head, row0, rows;  // packed row and K/V head of the unit; its rows are row0 .. row0+rows-1 of their grid
    int pieces;                   // workers w, w+1, ..; 0: nothing
};
__host__ __device__ constexpr int64_t paged_slots_bytes(int64_t workers, int rows, int D)
{
    return 2 * workers * rows * (D + 2) * 4;
}
__host__ __device__ constexpr int64_t paged_span_bytes(int64_t workers, int rows, int D)
{
    return (paged_slots_bytes(workers, rows, D) + workers * (int64_t)sizeof(PagedJoin) + 255) / 256 * 256;
}
constexpr float kJoinMinusHuge = -1.0e30f;  // what a maximum starts from
template <typename E>
struct PagedSlots {
    float *part, *m, *l;
    PagedJoin *join;
    __host__ __device__ PagedSlots(void *workspace, int64_t workers, int rows, int D)
        : part((float *)workspace), m(part + 2 * workers * rows * D), l(m + 2 * workers * rows),
          join((PagedJoin *)(l + 2 * workers * rows)) {}
};

// Which kernel a call takes, by what the host knows of the batch.
struct PagedPlan {
    int kernel_d;     // 64, 128 or 256
    int decode_rows;  // the decoding kernel, for sequences of up to so many rows (new tokens times the query heads of a
                      // K/V head); 0: the kernel of many rows
    int workers;      // 0: one work-group for each unit of rows
    size_t bytes;     // workspace
};
// Tiles of a span, at least (every piece that the join counts has to have one).  us with 1 / 2 / 4, few rows: 10.9 / 12.3 /
// 15.1 (one sequence of 1000 keys), 12.5 / 13.7 / 16.0 (4000); many rows: 16.1 / 19.1 / 25.6 (two sequences of up to 11 rows
// and 807 keys, D = 192), 26.6 / 25.6 / 27.7 (5 of up to 206 and 780), 28.1 / 25.7 / 24.6 (one of 104 and 2089); batches drawn
// over the whole range 1 % faster with 2 than with 1 and 4 % than with 4.
constexpr int kDecodeSpan = 1, kChunkSpan = 2;
// A table of up to so many tiles is not cut, and nothing joined.  us uncut / cut, few rows, 600 keys: 8.2 / 10.4 (one sequence),
// 29.7 / 32.1 (64); 1000 keys: 11.1 / 11.0 (one; e4m3 11.9 / 10.3), 44.7 / 47.9 (64).  Many rows, 310 keys: 25.8 / 36.0 (5
// sequences of up to 273 rows, D = 192), 9.8 / 18.5 (7 of up to 212); 494 keys: 11.2 / 10.4 (one of 19); beyond, 676 keys:
// 26.8 / 19.1 (22 of up to 150).
constexpr int kWholeTiles = 8;
constexpr int chunk_rows(int D) { return D == 128 ? 256 : 128; }  // of a unit, in the kernel of many rows
PagedPlan paged_plan(int64_t T, int64_t B, int Hq, int Hkv, int D, int max_q, int64_t keys, bool e4m3);

// Rows and keys of a sequence, inside the buffers whatever device memory holds.
struct PagedSeq {
    int first, n, len;  // first packed row, rows, keys
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedBatch &a, int b)
{
    PagedSeq s;
    s.first = min(max(a.q_start[b], 0), a.T);
    s.n = max(min(a.q_start[b + 1], a.T) - s.first, 0);
    s.len = min(max(a.kv_lens[b], 0), a.table_width << a.page_shift);
    return s;
}

// The sequence that packed row t belongs to, or B: the first whose end lies behind t.  By a whole wave, t the same in
// all lanes.
__device__ __forceinline__ int paged_seq_of(const PagedBatch &a, int t)
{
    const int l = threadIdx.x & 63;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int b = b0 + l;
        const uint64_t behind = __builtin_amdgcn_ballot_w64(b < a.B && a.q_start[min(b, a.B - 1) + 1] > t);
        if (behind) return b0 + __builtin_ctzll(behind);
    }
    return a.B;
}

// Sum of two numbers that are not negative, at most lim.
__device__ __forceinline__ int add_up_to(int a, int b, int lim) { return (int)min((unsigned)a + (unsigned)b, (unsigned)lim); }

// Sum over a work-group's threads up to this one, over those before it, and over all of them, each at most lim.
template <int NW>
__device__ __forceinline__ int block_scan(int v, int lim, int *lds, int &before, int &all)
{
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(v, d);
        if (l >= d) v = add_up_to(v, x, lim);
    }
    before = __shfl_up(v, 1);
    if (l == 0) before = 0;
    __syncthreads();
    if (l == 63) lds[w] = v;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        if (i < w) {
            v = add_up_to(v, lds[i], lim);
            before = add_up_to(before, lds[i], lim);
        }
        all = add_up_to(all, lds[i], lim);
    }
    return v;
}

// A value of device memory that no kernel writes while this one runs, by a scalar load.
template <typename T>
__device__ __forceinline__ T scalar_load(const T *p)
{
    return *(const __attribute__((address_space(4))) T *)(uintptr_t)p;
}
__device__ __forceinline__ PagedSeq paged_seq_scalar(const PagedBatch &a, int b)
{
    PagedSeq s;
    s.first = min(max(scalar_load(a.q_start + b), 0), a.T);
    s.n = max(min(scalar_load(a.q_start + b + 1), a.T) - s.first, 0);
    s.len = min(max(scalar_load(a.kv_lens + b), 0), a.table_width << a.page_shift);
    return s;
}

// The span of worker w of `workers`: `tiles(seq)` are those of a sequence with one head, of which there are `heads`.
// Where the span begins: sequence b, and how many tiles lie in front of that sequence (all heads).
// The sums end at what an int32 holds.  Row ranges that lie apart never get there (the host has checked), others, which
// are an error of the caller's, do not lead outside the buffers that way: a sequence that is found has its tiles.
struct PagedSpan {
    int64_t begin, front, size;
    int left, b;  // tiles of the span (0: none)
    PagedSeq seq;
    int tiles;    // of sequence b
};
__device__ __forceinline__ int64_t div_up(int64_t x, int y)
{
    // (a division of 64 bits takes four times as long)
    return x < (1 << 30) ? (int64_t)(((unsigned)x + y - 1) / (unsigned)y) : (x + y - 1) / y;
}
template <int NW, typename Tiles>
__device__ __forceinline__ PagedSpan paged_span(const PagedBatch &a, int heads, int w, int workers, int least, int *lds,
                                                Tiles tiles)
{
    const int tid = threadIdx.x, l = tid & 63, B = a.B;
    PagedSpan s = {};
    const int lim = 0x7fffffff / heads;
    auto cut = [&](int64_t total) __attribute__((always_inline)) {
        s.size = max((int64_t)least, div_up(total, workers));
        s.begin = w * s.size;
        s.left = __builtin_amdgcn_readfirstlane((int)max(min(s.size, total - s.begin), (int64_t)0));
    };
    if (B <= 64) {
        // every wave by itself: without barriers, and with what it has loaded
        const PagedSeq q = paged_seq(a, min(l, B - 1));
        const int mine = l < B ? tiles(q) : 0;
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(sum, d);
            if (l >= d) sum = add_up_to(sum, x, lim);
        }
        cut((int64_t)__builtin_amdgcn_readlane(sum, 63) * heads);
        if (s.left == 0) return s;
        s.b = __builtin_ctzll(__builtin_amdgcn_ballot_w64((int64_t)sum * heads > s.begin));
        s.front = s.b ? (int64_t)__builtin_amdgcn_readlane(sum, s.b - 1) * heads : 0;
        s.seq.first = __builtin_amdgcn_readlane(q.first, s.b);
        s.seq.n = __builtin_amdgcn_readlane(q.n, s.b);
        s.seq.len = __builtin_amdgcn_readlane(q.len, s.b);
        s.tiles = __builtin_amdgcn_readlane(mine, s.b);
        return s;
    }
    int total = 0, front = 0, sum = 0, before = 0, all = 0;
    auto sums = [&](int b0) __attribute__((always_inline)) {
        sum = block_scan<NW>(b0 + tid < B ? tiles(paged_seq(a, b0 + tid)) : 0, lim, lds, before, all);
    };
    for (int b0 = 0; b0 < B; b0 += NW * 64) {
        sums(b0);
        total = add_up_to(total, all, lim);
    }
    cut((int64_t)total * heads);
    if (s.left == 0) return s;
    // (one round: its sums are still there)
    for (int b0 = 0; b0 < B; b0 += NW * 64) {
        if (B > NW * 64) sums(b0);
        const int behind = add_up_to(front, all, lim);
        if ((int64_t)behind * heads > s.begin) {
            __syncthreads();
            const int from = add_up_to(front, before, lim);
            if ((int64_t)add_up_to(front, sum, lim) * heads > s.begin && (int64_t)from * heads <= s.begin) {
                lds[0] = b0 + tid;
                lds[1] = from;
            }
            __syncthreads();
            s.b = __builtin_amdgcn_readfirstlane(lds[0]);
            s.front = (int64_t)__builtin_amdgcn_readfirstlane(lds[1]) * heads;
            s.seq = paged_seq_scalar(a, s.b);
            s.tiles = __builtin_amdgcn_readfirstlane(tiles(s.seq));
            return s;
        }
        front = behind;
    }
    return s;
}

// Global -> LDS transfer as dma16 (attn_device.hpp), of 16 bytes from an address of each lane's.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16_from(const void *p, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 ::"s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(p) : "m0");
}
#pragma clang diagnostic pop

// Four e4m3 codes times the power of two of `scale`.
__device__ __forceinline__ elem4 from_e4m3(uint32_t codes, float scale)
{
#ifdef ATTN_F16
    const elem2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, false),
                hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, true);
#else
    const elem2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false),
                hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
#endif
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
}
__device__ __forceinline__ elem8 from_e4m3(uint32_t lo, uint32_t hi, float scale_lo, float scale_hi)
{
    return __builtin_shufflevector(from_e4m3(lo, scale_lo), from_e4m3(hi, scale_hi), 0, 1, 2, 3, 4, 5, 6, 7);
}
// What the conversion leaves of a scale, in 1 .. 2; 0 of 0.
__device__ __forceinline__ float scale_rest(float scale)
{
    const uint32_t u = __float_as_uint(scale);
    return u ? __uint_as_float((u & 0x7fffffu) | 0x3f800000u) : 0.f;
}

}  // namespace attn
