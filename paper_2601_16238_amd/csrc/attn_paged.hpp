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

// Which kernels a call takes, by what the host knows of the batch: the decoding kernel for the sequences of up to
// decode_rows rows (new tokens times the query heads of a K/V head; 0: it is not launched), the other for longer ones.
struct PagedPlan {
    int kernel_d;     // 64, 128 or 256
    int decode_rows, decode_workers;  // workers 0: one work-group for each sequence and K/V head
    bool chunks;
    size_t bytes;     // workspace
};
PagedPlan paged_plan(int64_t B, int Hq, int Hkv, int D, int max_q, int64_t keys, bool e4m3);

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

}  // namespace attn
