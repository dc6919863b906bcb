// Attention over the paged cache for sequences of many rows (prompts and chunks of them).
//
// The rows of a unit of work are kBR = 32 NW consecutive ones of a sequence and K/V head, new token by new token and
// within it query head by query head, so that a tile of 64 keys is read once for all heads that share it; a wave has
// 32 of them.  S^T = K Q^T and O^T += V^T P^T by 32x32x16 MFMA with the scores of a query in one lane; K and V tiles
// reach LDS row-major, two buffers each.  16-bit tiles come by direct transfers, 16 rows (of one page) to a buffer
// resource; slots behind the last key, pages that are none and columns that do not exist read as zero.  e4m3 tiles
// pass through registers, where they are converted once for all waves: K exactly, V with its power of two; what is
// left of V's scale is added to the exponent of the probabilities and taken out of their sums.
//
// Work is cut into equal spans of tiles, as for few rows (attn_paged_decode.hip).
#include "attn_paged.hpp"

namespace attn {

template <int D, bool E8>
struct ChunkCfg {
    static constexpr int kNW = 4;
    static constexpr int kThreads = kNW * 64;
    static constexpr int kBR = kNW * 32;
    static constexpr int kBC = 64;
    using L = Pieces<D>;
    static constexpr int kPieces = kBC / L::kRows;            // transfers of a 16-bit tile
    static constexpr int kPerWave = kPieces / kNW;
    static constexpr int kTile = L::base(kPieces);            // bytes
    static constexpr int kHalf = kTile / 2;                   // 32 rows further
    static constexpr int kOffV = 2 * kTile;
    static constexpr int kLds = 4 * kTile;
    static constexpr int kChunks = D / 16;                    // 16-byte pieces of an e4m3 row
    static constexpr int kPerThread = kBC * kChunks / kThreads;
    static constexpr int kWaves = D > 128 ? 1 : 2;            // a SIMD
    static_assert(kPieces % kNW == 0 && kBC * kChunks % kThreads == 0, "staging divides evenly");
    static_assert(kWaves * kLds <= 160 * 1024, "LDS of a compute unit");
};

// Units of rows of a sequence: rt has the rows rt BR .. of the sequence's n G.
__device__ __forceinline__ int chunk_row_tiles(const PagedSeq &s, int G, int max_q, int BR)
{
    return s.n > max_q ? 0 : (int)(((unsigned)(s.n * G) + BR - 1) / BR);
}
// Tiles of keys that the rows up to the end of new token `token` see (none: one, in which nothing is seen).
__device__ __forceinline__ int chunk_tiles(const PagedSeq &s, bool causal, int token)
{
    const int keys = causal ? min(s.len - s.n + min(token, s.n - 1) + 1, s.len) : s.len;
    return max((keys + 63) >> 6, 1);
}
// Walks over a sequence's units: their last tokens, without a division each.
struct ChunkWalk {
    int quot, rem, G, token, left;
    __device__ ChunkWalk(int G_, int BR) : quot(BR / G_), rem(BR % G_), G(G_), token(-1), left(0) {}
    // the last token that the next unit has a row of
    __device__ int next()
    {
        // rows so far: (rt + 1) BR = tokens G + left
        token += quot;
        left += rem;
        if (left >= G) { left -= G; ++token; }
        return left ? token + 1 : token;
    }
};
__device__ __forceinline__ int chunk_cost(const PagedSeq &s, int G, int max_q, int BR, bool causal)
{
    const int row_tiles = chunk_row_tiles(s, G, max_q, BR);
    ChunkWalk walk(G, BR);
    int sum = 0;
    for (int rt = 0; rt < row_tiles; ++rt) sum += chunk_tiles(s, causal, walk.next());
    return sum;
}

constexpr float kChunkOverflow = 1024.0f;  // a lane's sum of a score block above this moves the reference maximum
constexpr float kChunkMinusHuge = -1.0e30f;

template <int D, bool E8, bool SPLIT>
__global__ void __launch_bounds__((ChunkCfg<D, E8>::kThreads))
    __attribute__((amdgpu_waves_per_eu(ChunkCfg<D, E8>::kWaves, ChunkCfg<D, E8>::kWaves)))
attn_paged_chunk_kernel(const PagedFwdArgs a, const PagedSlots<elem> slots)
{
    using C = ChunkCfg<D, E8>;
    using L = typename C::L;
    constexpr int KS = D / 16, DB = D / 32, NW = C::kNW, BR = C::kBR, BC = C::kBC;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ int scan[NW];

    const int tid = threadIdx.x, l = tid & 63, r = l & 31, h = l >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.Hq / a.Hkv, Hkv = a.Hkv, Dr = a.Dr, B = a.b.B;
    const bool causal = a.causal;

    // ---- the span: consecutive units of one XCD, which share K/V heads
    struct Unit { int b, h, rt, t, tiles, token; };
    PagedSeq s;
    int row_tiles, todo;
    Unit u;
    ChunkWalk walk(G, BR);
    PagedSpan span = {};
    const int me = SPLIT ? xcd_contiguous_order(blockIdx.x, gridDim.x) : blockIdx.x;
    auto set_seq = [&](const PagedSeq &q) __attribute__((always_inline)) {
        s = q;
        row_tiles = chunk_row_tiles(q, G, a.max_q, BR);
    };
    if constexpr (SPLIT) {
        span = paged_span<NW>(a.b, Hkv, me, gridDim.x, kChunkSpan, scan,
                              [&](const PagedSeq &q) { return chunk_cost(q, G, a.max_q, BR, causal); });
        todo = span.left;
        if (tid == 0) slots.join[me].pieces = 0;
        if (todo == 0) return;
        u.b = span.b;
        set_seq(span.seq);
        // which head, which unit of it and which of its tiles
        int cost = 0;
        for (int rt = 0; rt < row_tiles; ++rt) cost += chunk_tiles(s, causal, walk.next());
        int in = (int)(span.begin - span.front);
        u.h = in / cost;
        in -= u.h * cost;
        walk = ChunkWalk(G, BR);
        u.rt = 0;
        while (true) {
            u.token = walk.next();
            u.tiles = chunk_tiles(s, causal, u.token);
            if (in < u.tiles) break;
            in -= u.tiles;
            ++u.rt;
        }
        u.t = in;
    } else {
        // one work-group for each unit: row tiles of a sequence from floor(first G / BR) + b on
        const int64_t slot = blockIdx.x / Hkv;
        u.h = blockIdx.x % Hkv;
        int b = -1;
        for (int b0 = 0; b0 < B && b < 0; b0 += 64) {
            const int bl = min(b0 + l, B - 1);
            const PagedSeq q = paged_seq(a.b, bl);
            const int64_t from = (int64_t)q.first * G / BR + bl;
            const uint64_t is = __builtin_amdgcn_ballot_w64(b0 + l < B && slot >= from &&
                                                            slot < from + chunk_row_tiles(q, G, a.max_q, BR));
            if (is) b = __builtin_amdgcn_readfirstlane(b0 + __builtin_ctzll(is));
        }
        if (b < 0) return;
        set_seq(paged_seq_scalar(a.b, b));
        u.rt = __builtin_amdgcn_readfirstlane((int)(slot - ((int64_t)s.first * G / BR + b)));
        u.b = b;
        for (int rt = 0; rt <= u.rt; ++rt) u.token = walk.next();
        u.tiles = chunk_tiles(s, causal, u.token);
        u.t = 0;
        todo = u.tiles;
    }

    // ---- staging
    const uint32_t row_bytes = (uint32_t)a.cache_stride_s * (E8 ? 1 : 2);
    constexpr uint32_t kPast = 1u << 31;
    const uint32_t lds0 = lds_address(smem);
    const uint32_t voff = L::lane_offset(l, row_bytes, Dr, kPast);
    struct Tile { int id[4]; float k[4], v[4]; };  // pages of its 16-key groups, and their scales
    auto ids_of = [&](int kt, Tile &t) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int key = kt * BC + 16 * g;
            int id = key < s.len ? scalar_load(a.b.page_table + (int64_t)u.b * a.b.table_stride +
                                               (key >> a.b.page_shift)) : -1;
            if (!a.b.is_page(id)) id = -1;
            t.id[g] = id;
            if constexpr (E8) {
                t.k[g] = id < 0 ? 1.f : scalar_load(a.k_scale + (int64_t)id * Hkv + u.h);
                t.v[g] = id < 0 ? 1.f : scalar_load(a.v_scale + (int64_t)id * Hkv + u.h);
            }
        }
    };
    // group g of tile kt: offset of its first row in the cache, and the bytes that exist of it
    auto place = [&](int kt, int id, int g, uint32_t &bytes) __attribute__((always_inline)) {
        const int key = kt * BC + 16 * g, rows = id < 0 ? 0 : min(s.len - key, 16);
        bytes = rows > 0 ? (uint32_t)(rows - 1) * row_bytes + Dr * (E8 ? 1 : 2) : 0;
        return ((int64_t)(id < 0 ? 0 : id) * a.cache_stride_p + u.h * a.cache_stride_h +
                (key & (a.b.page_size() - 1)) * a.cache_stride_s) * (E8 ? 1 : 2);
    };
    auto transfer = [&](int kt, const Tile &t, int buf) __attribute__((always_inline)) {
        if constexpr (!E8) {
#pragma unroll
            for (int n = 0; n < C::kPerWave; ++n) {
                const int ii = w + n * NW, row0 = ii * L::kRows, g = n * NW * L::kRows / 16 + (w * L::kRows) / 16;
                uint32_t bytes;
                // (which group: known when compiled but for D = 64, where a wave's is its own)
                const int id = D == 64 ? (g == 0 ? t.id[0] : g == 1 ? t.id[1] : g == 2 ? t.id[2] : t.id[3])
                                       : t.id[n * NW * L::kRows / 16];
                const int64_t off = place(kt, id, g, bytes);
                const uint32_t soff = (row0 & 15) * row_bytes, lds = lds0 + buf * C::kTile + L::base(ii);
                dma16_between(make_desc((const char *)a.K_cache + off, bytes), lds, voff, soff);
                dma16_between(make_desc((const char *)a.V_cache + off, bytes), lds + C::kOffV, voff, soff);
            }
        }
    };
    // e4m3: 16 codes a thread and step, of row (w + NW j) kBC / ..; a wave's rows lie in one group
    constexpr int RPW = 64 / C::kChunks;  // rows of a wave's step
    u32x4 ck[E8 ? C::kPerThread : 1], cv[E8 ? C::kPerThread : 1];
    auto fetch = [&](int kt, const Tile &t) __attribute__((always_inline)) {
        if constexpr (E8) {
#pragma unroll
            for (int j = 0; j < C::kPerThread; ++j) {
                const int row0 = (w + NW * j) * RPW, g = row0 / 16;
                uint32_t bytes;
                const int id = g == 0 ? t.id[0] : g == 1 ? t.id[1] : g == 2 ? t.id[2] : t.id[3];
                const int64_t off = place(kt, id, g, bytes);
                const int c = l % C::kChunks;
                const uint32_t at = c * 16 < Dr ? (row0 % 16 + l / C::kChunks) * row_bytes + c * 16 : kPast;
                ck[j] = buf_load16(make_rsrc((const char *)a.K_cache + off, bytes), at, 0);
                cv[j] = buf_load16(make_rsrc((const char *)a.V_cache + off, bytes), at, 0);
            }
        }
    };
    auto convert = [&](const Tile &t, int buf) __attribute__((always_inline)) {
        if constexpr (E8) {
#pragma unroll
            for (int j = 0; j < C::kPerThread; ++j) {
                const int row0 = (w + NW * j) * RPW, g = row0 / 16, row = row0 + l / C::kChunks, c = l % C::kChunks;
                const float sv = g == 0 ? t.v[0] : g == 1 ? t.v[1] : g == 2 ? t.v[2] : t.v[3];
                char *const k = smem + buf * C::kTile;
                *(elem8 *)(k + L::at(row, 2 * c)) = from_e4m3(ck[j].x, ck[j].y, 1.f, 1.f);
                *(elem8 *)(k + L::at(row, 2 * c + 1)) = from_e4m3(ck[j].z, ck[j].w, 1.f, 1.f);
                *(elem8 *)(k + C::kOffV + L::at(row, 2 * c)) = from_e4m3(cv[j].x, cv[j].y, sv, sv);
                *(elem8 *)(k + C::kOffV + L::at(row, 2 * c + 1)) = from_e4m3(cv[j].z, cv[j].w, sv, sv);
            }
        }
    };

    const int k_lane = L::at(r, h);
    int v_lane[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
        v_lane[j] = C::kOffV + L::at(8 * j + 4 * h + ((l & 15) >> 2), 2 * ((l >> 4) & 1) + ((l >> 1) & 1)) + (l & 1) * 8;

    // ---- units
    while (true) {
        const int rows = min(s.n * G - u.rt * BR, BR), t0 = u.t, t1 = min(u.tiles, u.t + todo);
        const int row = u.rt * BR + w * 32 + r;             // the lane's row of the sequence and head
        const int tok = row / G, head = u.h * G + row - tok * G;
        // the last key that it sees
        const int seen = causal ? min(s.len - s.n + tok, s.len - 1) : s.len - 1;
        // ... and the wave's first row (all see that many)
        const int all_see = causal ? __builtin_amdgcn_readfirstlane(min(s.len - s.n + (u.rt * BR + w * 32) / G, s.len - 1))
                                   : s.len - 1;
        Tile cur, next;
        ids_of(t0, cur);
        transfer(t0, cur, 0);
        fetch(t0, cur);
        // the unit's rows of Q to the second buffers, in the layout of the tiles: 64 in K's, 64 in V's
        {
            constexpr int CPR = D / 8;
#pragma unroll
            for (int i = 0; i < BR * CPR / C::kThreads; ++i) {
                const int id = tid + i * C::kThreads, qr = id / CPR, c = id % CPR;
                const int q = u.rt * BR + qr, t = q / G;
                u32x4 x = {0u, 0u, 0u, 0u};
                if (qr < rows && c * 8 < Dr)
                    x = *(const u32x4 *)(a.Q + (s.first + t) * a.q_stride_t + (u.h * G + q - t * G) * a.q_stride_h + c * 8);
                *(u32x4 *)(smem + C::kTile + (qr >> 6) * C::kOffV + L::at(qr & 63, c)) = x;
            }
        }
        convert(cur, 0);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        elem8 qf[KS];
        {
            const char *Qs = smem + C::kTile + (w >> 1) * C::kOffV + (w & 1) * C::kHalf + k_lane;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const elem8 *)(Qs + L::step(ks));
        }
        float m = kChunkMinusHuge, lsum = 0.f;
        f32x16 o[DB];
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] = 0.f;

        if (t0 + 1 < t1) ids_of(t0 + 1, next);
        for (int kt = t0; kt < t1; ++kt) {
            const int buf = (kt - t0) & 1;
            // (the other buffers' last reads, of Q or tile kt - 1, are done)
            __syncthreads();
            if (kt + 1 < t1) {
                transfer(kt + 1, next, buf ^ 1);
                fetch(kt + 1, next);
            }
            const char *Kt = smem + buf * C::kTile;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x16 x;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    x = mfma32(*(const elem8 *)(Kt + half * C::kHalf + L::step(ks) + k_lane), qf[ks], x);
                float c[2] = {a.scale_log2e, a.scale_log2e}, rest[2] = {0.f, 0.f}, inv[2] = {1.f, 1.f};
                if constexpr (E8)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        // (not 0, which a masked score would turn into NaN)
                        c[g] = fmaxf(c[g] * cur.k[2 * half + g], 1e-38f);
                        const float left = scale_rest(cur.v[2 * half + g]);
                        rest[g] = left > 0.f ? fast_log2(left) : 0.f;
                        inv[g] = left > 0.f ? 1.f / left : 1.f;
                    }
                const int kb = kt * BC + 32 * half;
                if (kb + 31 > all_see || cur.id[2 * half] < 0 || cur.id[2 * half + 1] < 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = acc_row(i, h);
                        if (key > seen - kb || cur.id[2 * half + (i >= 8)] < 0) x[i] = -INFINITY;
                    }
                }
                float e[16], part[2];
                auto probs = [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        part[g] = 0.f;
#pragma unroll
                        for (int i = 8 * g; i < 8 * g + 8; ++i) {
                            e[i] = fast_exp2(__builtin_fmaf(x[i], c[g], rest[g] - m));
                            part[g] += e[i];
                        }
                    }
                };
                probs();
                if (__builtin_amdgcn_ballot_w64(part[0] + part[1] > kChunkOverflow)) {
                    float t[2];
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        t[g] = x[8 * g];
#pragma unroll
                        for (int i = 1; i < 8; ++i) t[g] = fmaxf(t[g], x[8 * g + i]);
                        t[g] *= c[g];
                    }
                    const float to = fmaxf(m, xhalf_max(fmaxf(t[0], t[1]))), alpha = fast_exp2(m - to);
                    m = to;
                    lsum *= alpha;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
                    probs();
                }
                lsum += E8 ? part[0] * inv[0] + part[1] * inv[1] : part[0] + part[1];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const elem8 p = pack8(e[8 * g], e[8 * g + 1], e[8 * g + 2], e[8 * g + 3], e[8 * g + 4], e[8 * g + 5],
                                          e[8 * g + 6], e[8 * g + 7]);
                    const char *Vt = Kt + (2 * half + g) * L::kRows16;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
                        o[db] = mfma32(join8(lds_read_tr((const elem *)(Vt + db * L::kBlock + v_lane[0])),
                                             lds_read_tr((const elem *)(Vt + db * L::kBlock + v_lane[1]))), p, o[db]);
                }
            }
            if (kt + 1 < t1) {
                convert(next, buf ^ 1);
                cur = next;
                if (kt + 2 < t1) ids_of(kt + 2, next);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        __syncthreads();  // all tiles are read: the buffers take the rows of O

        const float lt = xhalf_sum(lsum);
        const bool from_start = t0 == 0, to_end = t1 == u.tiles;
        const bool there = w * 32 + r < rows;
        if (!SPLIT || (from_start && to_end)) {
            const float by = lt > 0.f ? 1.f / lt : 0.f;
            char *const stg = smem + w * C::kHalf;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(elem4 *)(stg + L::at(r, 4 * db + g) + 8 * h) =
                        pack4(o[db][4 * g] * by, o[db][4 * g + 1] * by, o[db][4 * g + 2] * by, o[db][4 * g + 3] * by);
            asm volatile("" ::: "memory");  // a wave's LDS accesses execute in order
            constexpr int CPR = D / 8, RPI = 64 / CPR;
            const int lr = l / CPR, lc = l % CPR;
#pragma unroll
            for (int j = 0; j < 32 / RPI; ++j) {
                const u32x4 v = *(const u32x4 *)(stg + L::at(RPI * j + lr, lc));
                const int in = w * 32 + RPI * j + lr, q = u.rt * BR + in, t = q / G;
                if (in < rows && lc * 8 < Dr)
                    *(u32x4 *)(a.O + (s.first + t) * a.out_stride_t + (u.h * G + q - t * G) * a.out_stride_h + lc * 8) = v;
            }
            if (there && h == 0)
                a.LSE[(int64_t)(s.first + tok) * a.Hq + head] = lt > 0.f ? (m + fast_log2(lt)) * kLn2 : -INFINITY;
        } else {
            const int64_t slot = 2 * (int64_t)me + (from_start ? 1 : 0);
            if (there) {
                float *const part = slots.part + (slot * BR + w * 32 + r) * D;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        *(f32x4 *)(part + 32 * db + 8 * g + 4 * h) =
                            f32x4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
                if (h == 0) {
                    slots.m[slot * BR + w * 32 + r] = m;
                    slots.l[slot * BR + w * 32 + r] = lt;
                }
            }
            if (from_start && tid == 0) {
                const int64_t last = span.begin + span.left - 1 + (u.tiles - t1);
                slots.join[me] = PagedJoin{s.first, u.h, u.rt * BR, rows, (int)(last / span.size) - me + 1};
            }
        }
        todo -= t1 - t0;
        if (!SPLIT || todo == 0) return;
        __syncthreads();  // the rows of O are read: the buffers take the next unit's tiles
        u.t = 0;
        if (++u.rt == row_tiles) {
            u.rt = 0;
            walk = ChunkWalk(G, BR);
            if (++u.h == Hkv) {
                u.h = 0;
                do set_seq(paged_seq_scalar(a.b, ++u.b)); while (row_tiles == 0);
            }
        }
        u.token = walk.next();
        u.tiles = chunk_tiles(s, causal, u.token);
    }
}

template <int D, bool E8>
static int launch_chunk_t(const PagedFwdArgs &a, int workers, hipStream_t st)
{
    using C = ChunkCfg<D, E8>;
    const void *kernel = workers ? (const void *)attn_paged_chunk_kernel<D, E8, true>
                                 : (const void *)attn_paged_chunk_kernel<D, E8, false>;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, C::kLds) != hipSuccess) return -1;
    const PagedSlots<elem> slots(a.workspace, workers, C::kBR, D);
    if (!workers) {
        const int64_t units = (int64_t)a.b.T * (a.Hq / a.Hkv) / C::kBR + a.b.B;
        hipLaunchKernelGGL((attn_paged_chunk_kernel<D, E8, false>), dim3((unsigned)(units * a.Hkv)), dim3(C::kThreads),
                           C::kLds, st, a, slots);
    } else {
        hipLaunchKernelGGL((attn_paged_chunk_kernel<D, E8, true>), dim3(workers), dim3(C::kThreads), C::kLds, st, a, slots);
        hipLaunchKernelGGL((attn_paged_join_kernel<D, 1>), dim3(workers, C::kBR * D / 1024), dim3(256), 0, st, a, slots,
                           C::kBR);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_paged_chunk(const PagedFwdArgs &a, int D, int workers, hipStream_t st)
{
    if (a.k_scale)
        return D == 64 ? launch_chunk_t<64, true>(a, workers, st)
             : D == 128 ? launch_chunk_t<128, true>(a, workers, st)
                        : launch_chunk_t<256, true>(a, workers, st);
    return D == 64 ? launch_chunk_t<64, false>(a, workers, st)
         : D == 128 ? launch_chunk_t<128, false>(a, workers, st)
                    : launch_chunk_t<256, false>(a, workers, st);
}

}  // namespace attn
