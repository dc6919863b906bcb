// Attention over the paged key/value cache (include/attn_paged.h): which kernel a call takes.
#include "attn_paged.hpp"

#include <algorithm>

namespace attn {

#ifndef ATTN_F16
PagedPlan paged_plan(int64_t T, int64_t B, int Hq, int Hkv, int D, int max_q, int64_t keys, bool e4m3)
{
    PagedPlan p = {};
    p.kernel_d = D <= 64 ? 64 : D <= 128 ? 128 : 256;
    // Up to 32 rows a work-group's waves share nothing; beyond (D above 128: 16), the accumulators of all rows in each
    // wave leave room for one work-group a compute unit.  us of this / the other kernel, 8 sequences, 8 K/V heads: 32 rows, 8000
    // keys, D = 128 59 / 60, e4m3 42 / 66, D = 64 35 / 38, 500 keys 19 / 21; 64 rows (four blocks a wave, no longer built)
    // 77 / 66, e4m3 85 / 65, D = 64 65 / 42; 32 rows with D = 256 137 / 115.
    const int G = Hq / Hkv, most = p.kernel_d == 256 ? 16 : 32;
    const int64_t rows = (int64_t)max_q * G;
    if (rows <= most) {
        p.decode_rows = (int)rows;
        const int tile = p.kernel_d == 256 && !e4m3 ? 64 : 128;
        const int64_t tiles = (keys + tile - 1) / tile;
        if (tiles <= kWholeTiles) return p;
        const int lds = p.kernel_d * (e4m3 ? 1 : 2) * 64 * 2 * (tile / 32), per_cu = 160 * 1024 / (lds + 4096);
        p.workers = (int)std::min<int64_t>(256 * std::min(per_cu, 2), B * Hkv * ((tiles + kDecodeSpan - 1) / kDecodeSpan));
        p.bytes = paged_span_bytes(p.workers, rows <= 16 ? 16 : 32, p.kernel_d);
        return p;
    }
    // A batch that may hold long sequences: all of it by the kernel of many rows, also the sequences of one token next
    // to a chunk, which are bound by their keys' way from memory there as well, while the chunk's products run (one launch for
    // each kind took 148 us where this took 141, 15 sequences beside a chunk of 512 tokens, e4m3).
    // (units, at most: of every sequence one that is not full)
    const int unit = chunk_rows(p.kernel_d);
    // (D = 64: two work-groups a compute unit, prompts 445 us; with one 554)
    const int64_t units = (T * G / unit + std::min(B, T)) * Hkv, tiles = (keys + 63) / 64;
    if (tiles <= kWholeTiles) return p;
    p.workers = (int)std::min<int64_t>(p.kernel_d == 64 ? 512 : 256, units * ((tiles + kChunkSpan - 1) / kChunkSpan));
    p.bytes = paged_span_bytes(p.workers, unit, p.kernel_d);
    return p;
}
#endif

int launch_paged_fwd(const PagedFwdArgs &a, hipStream_t st)
{
    const PagedPlan p = paged_plan(a.b.T, a.b.B, a.Hq, a.Hkv, a.Dr, a.max_q, (int64_t)a.b.table_width << a.b.page_shift,
                                   a.k_scale != nullptr);
    const int workers = a.workspace ? p.workers : 0;
    return p.decode_rows ? launch_paged_decode(a, p.kernel_d, p.decode_rows, workers, st)
                         : launch_paged_chunk(a, p.kernel_d, workers, st);
}

}  // namespace attn
