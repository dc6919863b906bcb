// Attention over the paged cache for sequences of many rows (prompts and chunks of them).
//
// The rows of a unit of work are kBR = 32 NW consecutive ones of a sequence and K/V head, new token by new token and
// within it query head by query head, so that a tile of 64 keys is read once for all heads that share it; a wave has
// 32 of them.  S^T = K Q^T and O^T += V^T P^T by 32x32x16 MFMA with the scores of a query in one lane.  A
// step forms the scores of 32 keys, the probabilities of the 32 before them and the products with V of the 32 before
// those: three independent pieces of work in one block of code, so that the matrix pipe and the vector ALU overlap inside
// a wave.  K and V tiles reach LDS row-major, two or three buffers each: two steps share a pair of tiles of 64 keys, K's 32 keys
// ahead of the probabilities and V's 32 behind.  16-bit tiles come by direct transfers, 16 rows (of one page) to a buffer
// resource; slots behind the last key, pages that are none and columns that do not exist read as zero.  e4m3 tiles
// pass through registers, where they are converted once for all waves: K exactly, V with its power of two; what is
// left of V's scale is added to the exponent of the probabilities and taken out of their sums.
//
// Work is cut into equal spans of tiles, as for few rows (attn_paged_decode.hip).
//
// Bound by the products and the exponentials beside them: a unit's tile of 256 rows and 64 keys takes 2.1 us of a compute unit
// (2.2 with e4m3), 1.0 PFLOP/s of the 1.2 that a large product reaches.  Prompts of 16.6K tokens (567 GFLOP) in 600 us and 15
// for the join, 512 tokens after 3584 keys (32 GFLOP) in 45 + 9, half of it beginnings and ends: a span's place, the first
// tiles' way and the partial results, 128 KB each.
// Eight waves of 32 rows a work-group with D = 128, so that a tile's way from L2 serves 256 rows: prompts 619 us, 798 with
// four; 16-bit tiles in three buffers: 15 sequences of one token beside a chunk 86 us, 95 with two, prompts the same.
#include "attn_paged.hpp"

#include <type_traits>

namespace attn {

template <int D, bool E8>
struct ChunkCfg {
    static constexpr int kNW = D == 128 ? 8 : 4;
    static constexpr int kThreads = kNW * 64;
    static constexpr int kBR = kNW * 32;
    static_assert(kBR == chunk_rows(D), "as planned");
    static constexpr int kBC = 64;
    using L = Pieces<D>;
    static constexpr int kPieces = kBC / L::kRows;            // transfers of a 16-bit tile
    static constexpr int kPerWave = kPieces / kNW;
    static constexpr int kTile = L::base(kPieces);            // bytes
    static constexpr int kHalf = kTile / 2;                   // 32 rows further
    static constexpr int kBufs = D == 128 && !E8 ? 3 : 2;     // of K, and of V
    static constexpr int kOffV = kBufs * kTile;
    static constexpr int kAreas = kNW / 2;                    // 64 rows of Q each
    // (and behind everything the rows of O on their way out, 64 bytes of each at a time)
    static constexpr int kOut = (2 * kBufs + kAreas - 2) * kTile, kOutWave = 32 * 64 + 4 * 16;
    static constexpr int kLds = kOut + kNW * kOutWave;
    static constexpr int kWaveRows = kBC / kNW;               // of a tile, fetched by a wave
    // place of rows 64 i .. of Q: the last buffers, and behind them
    __device__ static int area(int i)
    {
        return i == 0 ? (kBufs - 1) * kTile : i == 1 ? kOffV + (kBufs - 1) * kTile : (2 * kBufs + i - 2) * kTile;
    }
    static constexpr int kChunks = D / 16;                    // 16-byte pieces of an e4m3 row
    static constexpr int kPerThread = kBC * kChunks / kThreads;
    static constexpr int kWaves = D > 128 ? 1 : 2;            // a SIMD
    static constexpr int kPerUnit = kWaves * 4 / kNW;         // work-groups of a compute unit
    static_assert(kPieces % kNW == 0 && kBC * kChunks % kThreads == 0 && 16 % kWaveRows == 0, "staging divides evenly");
    static_assert(kPerUnit * kLds <= 160 * 1024, "LDS of a compute unit");
};

// sum of floor((a i + b) / m) over i = 0 .. n-1, by the steps of Euclid's algorithm on (a, m).
__device__ __forceinline__ int64_t floor_sum(unsigned n, unsigned m, unsigned a, unsigned b)
{
    int64_t sum = 0;
    while (n) {
        if (a >= m) {
            sum += (int64_t)n * (n - 1) / 2 * (a / m);
            a %= m;
        }
        if (b >= m) {
            sum += (int64_t)n * (b / m);
            b %= m;
        }
        const unsigned most = a * n + b;
        if (most < m) break;
        n = most / m;
        b = most % m;
        const unsigned t = a;
        a = m;
        m = t;
    }
    return sum;
}
// What spans count: a tile as 2, or, 16-bit, as 1 where one or two waves have rows (sequences of few rows next to long ones),
// and the beginning and end of a unit, where its rows come and go, as 6.  15 sequences of one token beside a chunk: 86 us with
// such tiles as 1, 94 as 2; e4m3, whose tiles wait for the codes' way to the registers whatever the rows are, 111 as 1
// and 98 as 2.  The ends as 0 / 4 / 6 / 8: prompts 837 / 755 / 725 / 711 us when they took longest, 665 / - / 657 / 655
// since their rows are requested together; as 10: mixed batches 98 -> 101.
constexpr int kTileCost = 2, kLightCost = 1, kLightRows = 64, kChunkEnd = 6;
// The units of a sequence and K/V head, unit rt with the rows rt BR .. of the sequence's n G, and their tiles of 64 keys:
// those that its last row sees (none: one, in which nothing is seen).  Under a causal mask these are
//     ceil((len - n + ceil((rt + 1) BR / G)) / 64) = floor((len - n) / 64) + floor(((rt + 1) BR + r G + 64 G - 1) / (64 G)),
// r = (len - n) mod 64, but for the last unit, which ends with the sequence, and the first `ones`, which see 64 at most.
struct ChunkUnits {
    int units, last, q0, ones, len, cost;  // cost: of a tile
    unsigned m, b, BR;
    bool causal;
    __device__ ChunkUnits() {}
    __device__ ChunkUnits(const PagedSeq &s, int G, int max_q, int BR_, bool causal_, int light)
        : len(s.len), BR(BR_), causal(causal_)
    {
        units = s.n > max_q ? 0 : (int)(((unsigned)(s.n * G) + BR - 1) / BR);
        last = max((s.len + 63) >> 6, 1);
        cost = s.n * G <= kLightRows ? light : kTileCost;
        const int before = s.len - s.n;
        q0 = before >> 6;
        m = 64u * G;
        b = BR + (unsigned)(before & 63) * G + m - 1;
        ones = before >= 64 ? 0 : min((int)((unsigned)(64 - before) * G / BR), units);
    }
    __device__ int tiles(int rt) const
    {
        if (!causal || rt == units - 1) return last;
        return rt < ones ? 1 : q0 + (int)((BR * rt + b) / m);
    }
    // cost of the units in front of unit k
    __device__ int64_t front(int k) const { return (int64_t)k * kChunkEnd + cost * tiles_in_front(k); }
    __device__ int64_t tiles_in_front(int k) const
    {
        if (!causal) return (int64_t)k * last;
        int64_t sum = 0;
        const int body = min(k, max(units - 1, 0)), ramp = body - min(body, ones);
        sum += min(body, ones) + (int64_t)ramp * q0 + floor_sum(ramp, m, BR, b + BR * ones);
        return k == units && units ? sum + last : sum;
    }
    // the unit that position `at` lies in, and what lies in front of it; by a whole wave, 64 candidates at a time
    __device__ int find(int at, int &in_front_of_it) const
    {
        int lo = 0, n = units;  // in lo .. lo + n - 1
        in_front_of_it = 0;
        while (n > 1) {
            const int step = (n + 63) >> 6, k = min(lo + (int)(threadIdx.x & 63) * step, lo + n - 1);
            const int f = (int)front(k);
            const int c = __popcll(__builtin_amdgcn_ballot_w64(f <= at && (int)(threadIdx.x & 63) * step < n)) - 1;
            in_front_of_it = __builtin_amdgcn_readlane(f, c);
            n = min(step, lo + n - (lo + c * step));
            lo += c * step;
        }
        return __builtin_amdgcn_readfirstlane(lo);
    }
};

// A lane's sum of the probabilities of its 16 keys above this moves the reference maximum: until then they stay inside the exponents
// of either type (fp16: up to 2^15), so that rounding them to it costs the same; sums and products are fp32.
constexpr float kChunkOverflow = 1024.0f;
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
    struct Unit { int b, h, rt, t, tiles, cost, at; };  // cost of a tile; at: where in the unit's cost the span goes on
    PagedSeq s;
    int todo;
    Unit u;
    int64_t begin_at = 0, size = 0;  // of the span
    int left = 0;
    const int me = SPLIT ? xcd_contiguous_order(blockIdx.x, gridDim.x) : blockIdx.x;
    auto units_of = [&](const PagedSeq &q) { return ChunkUnits(q, G, a.max_q, BR, causal, E8 ? kTileCost : kLightCost); };
    auto next_unit = [&]() __attribute__((always_inline)) {
        // (what the sequence's units are is found again rather than kept: the scalar registers are few)
        ChunkUnits units = units_of(s);
        u.t = u.at = 0;
        if (++u.rt == units.units) {
            u.rt = 0;
            if (++u.h == Hkv) {
                u.h = 0;
                do units = units_of(s = paged_seq_scalar(a.b, ++u.b)); while (units.units == 0);
            }
        }
        u.tiles = units.tiles(u.rt);
        u.cost = units.cost;
    };
    if constexpr (SPLIT) {
        const PagedSpan span = paged_span<NW>(a.b, Hkv, me, gridDim.x, kTileCost * kChunkSpan, scan, [&](const PagedSeq &q) {
            const ChunkUnits c = units_of(q);
            return (int)c.front(c.units);
        });
        begin_at = span.begin;
        size = span.size;
        todo = left = span.left;
        if (tid == 0) slots.join[me].pieces = 0;
        if (todo == 0) return;
        u.b = span.b;
        s = span.seq;
        const ChunkUnits units = units_of(s);
        // which head, which unit of it and which of its tiles
        const int cost = span.tiles;
        int in = __builtin_amdgcn_readfirstlane((int)(span.begin - span.front));
        u.h = in / cost;
        in -= u.h * cost;
        int front;
        u.rt = units.find(in, front);
        u.tiles = units.tiles(u.rt);
        u.cost = units.cost;
        // (a tile is the span's in which its cost begins)
        in -= front;
        u.at = in;
        u.t = (in + units.cost - 1) >> (units.cost - 1);  // (the cost is 1 or 2)
        if (u.t < u.tiles && u.t * units.cost >= in + todo) return;
        if (u.t >= u.tiles) {  // the span begins with the end of a unit
            todo -= u.tiles * units.cost + kChunkEnd - in;
            if (todo <= 0) return;
            next_unit();
        }
    } else {
        // one work-group for each unit: those of a sequence from floor(first G / BR) + b on
        const int64_t slot = blockIdx.x / Hkv;
        u.h = blockIdx.x % Hkv;
        int b = -1;
        for (int b0 = 0; b0 < B && b < 0; b0 += 64) {
            const int bl = min(b0 + l, B - 1);
            const PagedSeq q = paged_seq(a.b, bl);
            const int64_t from = (int64_t)q.first * G / BR + bl;
            const uint64_t is = __builtin_amdgcn_ballot_w64(b0 + l < B && slot >= from && slot < from + units_of(q).units);
            if (is) b = __builtin_amdgcn_readfirstlane(b0 + __builtin_ctzll(is));
        }
        if (b < 0) return;
        s = paged_seq_scalar(a.b, b);
        const ChunkUnits units = units_of(s);
        u.b = b;
        u.rt = __builtin_amdgcn_readfirstlane((int)(slot - ((int64_t)s.first * G / BR + b)));
        u.tiles = units.tiles(u.rt);
        u.cost = units.cost;
        u.t = u.at = 0;
        todo = u.tiles * units.cost;
    }

    // ---- staging
    const uint32_t row_bytes = (uint32_t)a.cache_stride_s * (E8 ? 1 : 2);
    constexpr uint32_t kPast = 1u << 31;
    const uint32_t lds0 = lds_address(smem);
    const uint32_t voff = L::lane_offset(l, row_bytes, Dr, kPast);
    // Set j: the groups 4 j + 2 .. 4 j + 5 of 16 keys each, counted from the unit's first key that the span has; they are
    // K's tile j and V's tile j + 1.  A wave fetches rows of one group, `own`, and tells the others what its
    // scores are multiplied with, what is added to the exponents of its probabilities (minus infinity: no page, or behind
    // the last key) and what their sum is multiplied with.
    const int own = w * C::kWaveRows / 16, own_row = w * C::kWaveRows % 16;
    struct Const { float c, rest, inv, unused; };
    constexpr int kSets = 4;
    __shared__ Const consts[kSets][4];
    int key0 = 0, key1 = 0;  // the keys of the unit that the span has
    auto key_of = [&](int j, int g) { return key0 + 64 * j + 32 + 16 * g; };
    auto id_of = [&](int j) __attribute__((always_inline)) {
        const int key = key_of(j, own);
        if constexpr (!E8)
            return key >= key0 && key < key1 ? scalar_load(a.b.page_table + (int64_t)u.b * a.b.table_stride +
                                                           (key >> a.b.page_shift)) : -1;
        // (loads without branches, here and of the scales, of what is there in any case)
        const int at = max(min(key, s.len - 1), 0) >> a.b.page_shift;
        const int id = scalar_load(a.b.page_table + (int64_t)u.b * a.b.table_stride + at);
        return key >= key0 && key < key1 ? id : -1;
    };
    // the wave's group: offset of its first row in the cache, bytes that exist of it, and its scales
    struct Group { int64_t off; uint32_t bytes; float k, v; };
    auto group_of = [&](int j, int id) __attribute__((always_inline)) {
        const bool is = a.b.is_page(id);
        const int key = key_of(j, own), page = is ? id : 0;
        Group t;
        t.bytes = is ? (uint32_t)(min(s.len - key, 16) - 1) * row_bytes + Dr * (E8 ? 1 : 2) : 0;
        t.off = (page * a.cache_stride_p + u.h * a.cache_stride_h + (key & (a.b.page_size() - 1)) * a.cache_stride_s) *
                (E8 ? 1 : 2);
        if constexpr (E8) {
            const float k = scalar_load(a.k_scale + (int64_t)page * Hkv + u.h),
                        v = scalar_load(a.v_scale + (int64_t)page * Hkv + u.h);
            t.k = is ? k : 1.f;
            t.v = is ? v : 1.f;
        }
        return t;
    };
    auto tell = [&](int j, const Group &t) __attribute__((always_inline)) {
        Const x = {a.scale_log2e, t.bytes ? 0.f : -INFINITY, 1.f, 0.f};
        if constexpr (E8) {
            // (not 0, which a masked score would turn into NaN)
            x.c = fmaxf(a.scale_log2e * t.k, 1e-38f);
            const float left = scale_rest(t.v);
            if (t.bytes && left > 0.f) {
                x.rest = fast_log2(left);
                x.inv = 1.f / left;
            }
        }
        if (l == 0 && own_row == 0) consts[(j + 1) % kSets][own] = x;
    };
    // piece n of the wave's rows of a 16-bit tile of K (tensor 0) or V
    auto transfer = [&](int tensor, desc_t d, int buf, int n) __attribute__((always_inline)) {
        if constexpr (!E8)
            dma16_between(d, lds0 + (tensor ? C::kOffV : 0) + buf * C::kTile + L::base(w * C::kPerWave + n), voff,
                          (own_row + n * L::kRows) * row_bytes);
    };
    auto desc_of = [&](int tensor, const Group &t) __attribute__((always_inline)) {
        return make_desc((const char *)(tensor ? a.V_cache : a.K_cache) + t.off, t.bytes);
    };
    // e4m3: 16 codes a thread and step
    constexpr int RPW = 64 / C::kChunks;  // rows of a wave's step
    u32x4 ck[E8 ? C::kPerThread : 1], cv[E8 ? C::kPerThread : 1];
    const uint32_t at8 = l % C::kChunks * 16 < Dr ? l / C::kChunks * row_bytes + l % C::kChunks * 16 : kPast;
    auto fetch = [&](int tensor, const Group &t, auto &codes) __attribute__((always_inline)) {
        if constexpr (E8) {
            const rsrc_t d = make_rsrc((const char *)(tensor ? a.V_cache : a.K_cache) + t.off, t.bytes);
#pragma unroll
            for (int n = 0; n < C::kPerThread; ++n) codes[n] = buf_load16(d, at8, (own_row + n * RPW) * row_bytes);
        }
    };
    auto convert = [&](int tensor, float by, int buf, const auto &codes, int shift = 0) __attribute__((always_inline)) {
        if constexpr (E8) {
#pragma unroll
            for (int n = 0; n < C::kPerThread; ++n) {
                const int row = C::kWaveRows * w + n * RPW + l / C::kChunks + shift, c = l % C::kChunks;
                char *const to = smem + (tensor ? C::kOffV : 0) + buf * C::kTile;
                *(elem8 *)(to + L::at(row, 2 * c)) = from_e4m3(codes[n].x, codes[n].y, by, by);
                *(elem8 *)(to + L::at(row, 2 * c + 1)) = from_e4m3(codes[n].z, codes[n].w, by, by);
            }
        }
    };

    const int k_lane = L::at(r, h);
    int v_lane[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
        v_lane[j] = C::kOffV + L::at(8 * j + 4 * h + ((l & 15) >> 2), 2 * ((l >> 4) & 1) + ((l >> 1) & 1)) + (l & 1) * 8;

    // x / G for 0 <= x < 2^17: the product is off by less than x / G 2^-22, and x + 1/2 is 1/2 away from any multiple of G
    const float inv_group = 1.0f / (float)G;
    auto over_group = [&](int x) { return (int)(((float)x + 0.5f) * inv_group); };

    // ---- the beginning of a unit.  Everything that its first tiles need is requested at once, while the unit before it
    // leaves: the 32 keys of sub-tile 0 of K to the first half of V's tile 0 (which nobody has), that tile's second half, the
    // tiles 0 (and 1) of K and V, and the wave's rows of Q to the buffers that are free.
    constexpr int A = C::kBufs - 1;  // 16-bit tiles are requested so many ahead of their use
    int rows = 0, t0 = 0, t1 = 0;       // rows, tiles
    int base_tok = 0, base_head = 0;    // the first row: new token, and which query head of the K/V head's
    Group sets[3] = {};  // of sets j, j + 1, .. j + A
    constexpr int F = E8 ? 2 : A;  // sets in use ahead of tile j's; e4m3: one more, in registers
    Group following = {};          // e4m3: set j + F
    int ahead = -1;                // the page of the set behind them
    auto begin = [&]() __attribute__((always_inline)) {
        rows = min(s.n * G - u.rt * BR, BR);
        t0 = u.t;
        t1 = min(u.tiles, (u.at + todo + u.cost - 1) >> (u.cost - 1));
        base_tok = u.rt * BR / G;
        base_head = u.rt * BR - base_tok * G;
        key0 = t0 * BC;
        key1 = min(t1 * BC, s.len);
        const int id0 = id_of(-1), id1 = id_of(0), id2 = id_of(1), id3 = F > 1 ? id_of(2) : id2;
        ahead = E8 ? id_of(F + 1) : id3;
        sets[0] = group_of(-1, id0);
        sets[1] = group_of(0, id1);
        if constexpr (F > 1) sets[2] = group_of(1, id2);
        if constexpr (E8) following = group_of(F, id3);
        tell(-1, sets[0]);
        tell(0, sets[1]);
        if constexpr (F > 1) tell(1, sets[2]);
        auto transfer_all = [&](int tensor, const Group &t, int buf) __attribute__((always_inline)) {
            const desc_t d = desc_of(tensor, t);
#pragma unroll
            for (int n = 0; n < C::kPerWave; ++n) transfer(tensor, d, buf, n);
        };
        if constexpr (!E8) {
            if (own >= 2) {
                const desc_t d = desc_of(0, sets[0]);
#pragma unroll
                for (int n = 0; n < C::kPerWave; ++n)
                    dma16_between(d, lds0 + C::kOffV + L::base(w * C::kPerWave + n - C::kPieces / 2), voff,
                                  (own_row + n * L::kRows) * row_bytes);
                transfer_all(1, sets[0], 0);
            }
            transfer_all(0, sets[1], 0);
            if constexpr (A > 1) {
                transfer_all(1, sets[1], 1);
                transfer_all(0, sets[2], 1);
            }
        }
        // (rows behind the unit's last are the last again, columns that do not exist column 0, which K's zeros take out)
#pragma unroll
        for (int n = 0; n < 32 / L::kRows; ++n) {
            const int row = min(w * 32 + n * L::kRows + L::lane_row(l), rows - 1), t = over_group(base_head + row);
            const int c = L::lane_chunk(l) * 8;
            dma16_from(a.Q + (s.first + base_tok + t) * a.q_stride_t + (u.h * G + base_head + row - t * G) * a.q_stride_h +
                           (c < Dr ? c : 0),
                       lds0 + C::area(w >> 1) + L::base((w & 1) * (32 / L::kRows) + n));
        }
    };
    // ... e4m3: what passes through registers
    auto begin_registers = [&]() __attribute__((always_inline)) {
        if constexpr (E8) {
            fetch(0, sets[0], ck);
            fetch(1, sets[0], cv);
        }
    };

    // ---- units
    begin();
    begin_registers();
    while (true) {
        const int in_tok = over_group(base_head + w * 32 + r);  // of the lane's row
        // the last key that it sees
        const int seen = causal ? min(s.len - s.n + base_tok + in_tok, s.len - 1) : s.len - 1;
        // ... and the wave's first row (all see that many)
        const int first_sees = s.len - s.n + base_tok + over_group(base_head + w * 32);
        const int all_see = causal ? __builtin_amdgcn_readfirstlane(min(first_sees, s.len - 1)) : s.len - 1;
        const int T = t1 - t0;
        const bool active = w * 32 < rows;  // (a wave without rows only fetches)
        if constexpr (E8) {
            if (own >= 2) {
                convert(1, 1.f, 0, ck, -32);
                convert(1, sets[0].v, 0, cv);
            }
            fetch(0, sets[1], ck);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        elem8 qf[KS];
        {
            const char *Qs = smem + C::area(w >> 1) + (w & 1) * C::kHalf + k_lane;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const elem8 *)(Qs + L::step(ks));
        }
        float m = kChunkMinusHuge, lsum = 0.f;
        f32x16 o[DB], sa, sb;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sa[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sa = mfma32(*(const elem8 *)(smem + C::kOffV + L::step(ks) + k_lane), qf[ks], sa);
        if constexpr (E8) {
            convert(0, 1.f, 0, ck);
            // (the codes of the tiles behind, on their way for a whole tile)
            fetch(1, sets[1], cv);
            fetch(0, sets[2], ck);
        }
        elem8 pp[2];  // probabilities of the sub-tile before
#pragma unroll
        for (int i = 0; i < 8; ++i) pp[0][i] = pp[1][i] = (elem)0.f;

        constexpr int NS = KS / 4, NP = 2 * NS;  // phases of four products: with K, with V
        elem8 f[2][4];
        // (per-lane LDS addresses of the current tiles, opaque to the compiler, so that step and block are folded into the
        // immediate offsets of the LDS instructions)
        int k_base = 0, v_base0 = 0, v_base1 = 0;
        auto set_bases = [&](int buf) __attribute__((always_inline)) {
            k_base = k_lane + buf * C::kTile;
            v_base0 = v_lane[0] + buf * C::kTile;
            v_base1 = v_lane[1] + buf * C::kTile;
            asm volatile("" : "+v"(k_base), "+v"(v_base0), "+v"(v_base1));
        };
        auto load = [&](int half, int p, elem8 (&to)[4]) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (p < NS) {
                    to[t] = *(const elem8 *)(smem + half * C::kHalf + L::step(4 * p + t) + k_base);
                } else {
                    const int i = 4 * (p - NS) + t;
                    const char *x = smem + (2 * half + i / DB) * L::kRows16 + i % DB * L::kBlock;
                    to[t] = join8(lds_read_tr((const elem *)(x + v_base0)), lds_read_tr((const elem *)(x + v_base1)));
                }
            }
        };
        // Step `half` of tile j: probabilities of sub-tile 2 j + half (scores in x), scores of the next into y, V times the
        // probabilities of the one before.  Between the products of the first step the next tiles are requested (in one
        // burst, the waves would all queue at the compute unit's vector-memory path while the matrix pipes idle).
        struct Pair { float c[2], rest[2], inv[2]; };  // of a sub-tile's two groups
        auto pair_of = [&](int j, int g) __attribute__((always_inline)) {
            Pair t;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const Const x = consts[(j + 1) % kSets][g + i];
                t.c[i] = E8 ? pin_scalar(x.c) : a.scale_log2e;
                t.rest[i] = pin_scalar(x.rest);
                t.inv[i] = E8 ? pin_scalar(x.inv) : 1.f;
            }
            return t;
        };
        desc_t Kd, Vd;
        auto step = [&](bool masked, int half, int kb, int fill, const Pair &t, f32x16 &x, f32x16 &y)
                        __attribute__((always_inline)) {
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (acc_row(i, h) > seen - kb) x[i] = -INFINITY;
            }
            float e[16], part[2] = {0.f, 0.f}, off[2] = {t.rest[0] - m, t.rest[1] - m};
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = 0.f;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                if (p + 1 < NP) load(half, p + 1, f[(p + 1) & 1]);
                else if (half == 0) load(1, 0, f[0]);
                if (half == 0 && p % (NP / C::kPerWave) == 0) {
                    static_assert(NP % C::kPerWave == 0, "pieces divide evenly");
                    transfer(0, Kd, fill, p / (NP / C::kPerWave));
                    transfer(1, Vd, fill, p / (NP / C::kPerWave));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int n = 4 * (p - NS) + k;
                    if (p < NS) y = mfma32(f[p & 1][k], qf[4 * p + k], y);
                    else o[n % DB] = mfma32(f[p & 1][k], pp[n / DB], o[n % DB]);
                }
#pragma unroll
                for (int i = 16 * p / NP; i < 16 * (p + 1) / NP; ++i) {
                    e[i] = fast_exp2(__builtin_fmaf(x[i], t.c[i >= 8], off[i >= 8]));
                    part[i >= 8] += e[i];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(part[0] + part[1] > kChunkOverflow) != 0, 0)) {
                // a probability has outgrown the reference maximum (always the first ones): it moves to the running maximum
                float top[2];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    top[g] = x[8 * g];
#pragma unroll
                    for (int i = 1; i < 8; ++i) top[g] = fmaxf(top[g], x[8 * g + i]);
                    top[g] = top[g] * t.c[g] + t.rest[g];
                }
                const float to = fmaxf(m, xhalf_max(fmaxf(top[0], top[1]))), alpha = fast_exp2(m - to);
                m = to;
                lsum *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
                part[0] = part[1] = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    e[i] = fast_exp2(__builtin_fmaf(x[i], t.c[i >= 8], t.rest[i >= 8] - m));
                    part[i >= 8] += e[i];
                }
            }
            lsum += E8 ? part[0] * t.inv[0] + part[1] * t.inv[1] : part[0] + part[1];
#pragma unroll
            for (int g = 0; g < 2; ++g)
                pp[g] = pack8(e[8 * g], e[8 * g + 1], e[8 * g + 2], e[8 * g + 3], e[8 * g + 4], e[8 * g + 5], e[8 * g + 6],
                              e[8 * g + 7]);
        };
        Pair behind = pair_of(-1, 2);
        int buf = 0;
        for (int j = 0; j < T; ++j) {
            // tiles j are there (and those behind them on their way), and tiles j - 1 are read
            wait_vm_and_barrier<E8 ? 63 : (A - 1) * 2 * C::kPerWave>();
            const int fill = buf + A >= C::kBufs ? buf + A - C::kBufs : buf + A;
            set_bases(buf);
            load(0, 0, f[0]);
            const Pair first = pair_of(j, 0), second = pair_of(j, 2);
            const int kb = key0 + 64 * j;
            // the tiles A further: set j + A as K's, set j + A - 1 as V's; e4m3: one more, into registers
            const Group newest = E8 ? following : group_of(j + F, ahead);
            if constexpr (!E8) ahead = id_of(j + F + 1);
            tell(j + F, newest);
            if constexpr (!E8) {
                Kd = desc_of(0, newest);
                Vd = desc_of(1, sets[F]);
            }
            if (active) {
                step(kb + 31 > all_see, 0, kb, fill, behind, sa, sb);
            } else if constexpr (!E8) {
#pragma unroll
                for (int n = 0; n < C::kPerWave; ++n) {
                    transfer(0, Kd, fill, n);
                    transfer(1, Vd, fill, n);
                }
            }
            convert(1, sets[1].v, fill, cv);
            fetch(1, sets[2], cv);
            if (active) step(kb + 63 > all_see, 1, kb + 32, fill, first, sb, sa);
            convert(0, 1.f, fill, ck);
            fetch(0, newest, ck);
            // (scalar loads just before the barrier, which waits for them: inside a step, every wait for LDS would)
            if constexpr (E8) {
                following = group_of(j + F + 1, ahead);
                ahead = id_of(j + F + 2);
            }
            behind = second;
            if constexpr (F > 1) {
                sets[1] = sets[2];
                sets[2] = newest;
            } else {
                sets[1] = newest;
            }
            buf = buf + 1 == C::kBufs ? 0 : buf + 1;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        // the last probabilities' products
        set_bases(buf);
#pragma unroll
        for (int p = 0; p < NS; ++p) {
            load(0, NS + p, f[0]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                o[(4 * p + t) % DB] = mfma32(f[0][t], pp[(4 * p + t) / DB], o[(4 * p + t) % DB]);
        }
        __syncthreads();  // all tiles are read

        // The next unit's first tiles and rows come while this one's leave.
        struct { int rows, base_tok, base_head, h, first, row0, begins, last; bool from_start, to_end; } e =
            {rows, base_tok, base_head, u.h, s.first, u.rt * BR, left - todo, (u.tiles - 1) * u.cost, t0 == 0,
             t1 == u.tiles};
        todo -= e.to_end ? u.tiles * u.cost - u.at + kChunkEnd : todo;
        const bool more = SPLIT && todo > 0;
        if (more) {
            next_unit();
            begin();
        }
        const float lt = xhalf_sum(lsum);
        const bool there = w * 32 + r < e.rows;
        if (!SPLIT || (e.from_start && e.to_end)) {
            const float by = lt > 0.f ? 1.f / lt : 0.f;
            // 32 columns of the wave's rows at a time, through LDS: 16 bytes a lane, 64 of a row
            char *const stg = smem + C::kOut + w * C::kOutWave;
            auto at = [](int row, int chunk) { return row * 64 + row / 8 * 16 + chunk * 16; };
            elem *out[2];
            bool store[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int in = w * 32 + 16 * j + l / 4, t = over_group(e.base_head + in);
                store[j] = in < e.rows;
                out[j] = a.O + (e.first + e.base_tok + t) * a.out_stride_t +
                         (e.h * G + e.base_head + in - t * G) * a.out_stride_h + l % 4 * 8;
            }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(elem4 *)(stg + at(r, g) + 8 * h) =
                        pack4(o[db][4 * g] * by, o[db][4 * g + 1] * by, o[db][4 * g + 2] * by, o[db][4 * g + 3] * by);
                asm volatile("" ::: "memory");  // a wave's LDS accesses execute in order
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4 v = *(const u32x4 *)(stg + at(16 * j + l / 4, l % 4));
                    if (store[j] && db * 32 + l % 4 * 8 < Dr) *(u32x4 *)(out[j] + db * 32) = v;
                }
                asm volatile("" ::: "memory");
            }
            if (there && h == 0)
                a.LSE[(int64_t)(e.first + e.base_tok + in_tok) * a.Hq + e.h * G + e.base_head + w * 32 + r - in_tok * G] =
                    lt > 0.f ? (m + fast_log2(lt)) * kLn2 : -INFINITY;
        } else {
            const int64_t slot = 2 * (int64_t)me + (e.from_start ? 1 : 0);
            if (w * 32 < e.rows) {
                // as the accumulators lie: every store of a wave is 1 KB
                float *const part = slots.part + slot * BR * D + w * 32 * D + l * 4;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        *(f32x4 *)(part + (4 * db + g) * 256) =
                            f32x4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
                if (h == 0) {
                    slots.m[slot * BR + w * 32 + r] = m;
                    slots.l[slot * BR + w * 32 + r] = lt;
                }
            }
            if (e.from_start && tid == 0) {
                const int64_t last = begin_at + e.begins + e.last;  // where the unit's last tile begins
                slots.join[me] = PagedJoin{e.first, e.h, e.row0, e.rows, min((int)(last / size), (int)gridDim.x - 1) - me + 1};
            }
        }
        if (!more) return;
        begin_registers();
    }
}

// The partial results of the units that worker blockIdx.y has the first tile of, joined: a work-group has 32 rows and 32
// columns (grid x), a thread four columns of a row in all pieces, two, four or eight of them at a time and with no load that
// waits for another but the record's.
// Bound by those two latencies and by the partial results' bytes: 320 of 128 KB in 9.3 us (512 new tokens after 3584 keys), 500
// in 15 (prompts; 22 when eight are always read).  The parts of a unit are neighbours in the grid, on all eight XCDs: with the
// workers as the first index, every fourth of which has a unit's beginning, 11.6 us.
template <int D>
__global__ void __launch_bounds__(256) attn_paged_join_rows_kernel(const PagedFwdArgs a, const PagedSlots<elem> s)
{
    constexpr int DB = D / 32, R = chunk_rows(D);
    __shared__ __attribute__((aligned(16))) elem out[32][40];
    const int me = blockIdx.y, part = blockIdx.x;
    const PagedJoin j = s.join[me];
    const int tid = threadIdx.x, r = tid & 31, g = tid >> 6, h = tid >> 5 & 1, w = part / DB, db = part % DB;
    if (j.pieces == 0 || w * 32 >= j.rows) return;
    const int row = w * 32 + r;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    float top = kJoinMinusHuge, all = 0.f;
    auto add = [&](auto count, int i0) __attribute__((always_inline)) {
        constexpr int kPieces = decltype(count)::value;
        float m[kPieces], l[kPieces];
        f32x4 y[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            // (behind the last piece: the last again)
            const int i = min(i0 + k, j.pieces - 1);
            const int64_t slot = 2 * (int64_t)(me + i) + (i == 0);
            m[k] = s.m[slot * R + row];
            l[k] = s.l[slot * R + row];
            y[k] = *(const f32x4 *)(s.part + slot * R * D + w * 32 * D + (4 * db + g) * 256 + (tid & 63) * 4);
        }
        float to = top;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) to = fmaxf(to, m[k]);
        const float keep = fast_exp2(top - to);
        x *= keep;
        all *= keep;
        top = to;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const float by = i0 + k < j.pieces ? fast_exp2(m[k] - to) : 0.f;
            x += y[k] * by;
            all += l[k] * by;
        }
    };
    int i0 = 0;
    for (; j.pieces - i0 > 4; i0 += 8) add(std::integral_constant<int, 8>{}, i0);
    if (j.pieces - i0 > 2) add(std::integral_constant<int, 4>{}, i0);
    else if (j.pieces > i0) add(std::integral_constant<int, 2>{}, i0);
    const float inv = all > 0.f ? 1.f / all : 0.f;
    *(elem4 *)&out[r][8 * g + 4 * h] = pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    const int G = a.Hq / a.Hkv;
    if (db == 0 && tid < 32 && row < j.rows) {
        const int q = j.row0 + row, t = q / G;
        a.LSE[(int64_t)(j.first + t) * a.Hq + j.head * G + q - t * G] = all > 0.f ? (top + fast_log2(all)) * kLn2 : -INFINITY;
    }
    __syncthreads();
    // 16 bytes a lane, 64 of a row
    const int in = w * 32 + tid / 4, col = 32 * db + tid % 4 * 8;
    if (tid >= 128 || in >= j.rows || col >= a.Dr) return;
    const int q = j.row0 + in, t = q / G;
    *(u32x4 *)(a.O + (j.first + t) * a.out_stride_t + (j.head * G + q - t * G) * a.out_stride_h + col) =
        *(const u32x4 *)&out[tid / 4][tid % 4 * 8];
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
        hipLaunchKernelGGL(attn_paged_join_rows_kernel<D>, dim3(C::kBR / 32 * (D / 32), workers), dim3(256), 0, st, a, slots);
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
