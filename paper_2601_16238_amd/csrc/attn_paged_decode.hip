// Attention over the paged cache for sequences of few rows (decoding, speculative decoding): the query heads of a K/V
// head times the new tokens are at most 16 RB rows, so that K and V are read once and nothing else counts.
//
//   S^T = K Q^T (16x16x32 MFMA: keys by rows), p = exp2(c s - m), O^T += V^T P^T.
//
// Work: the tiles of TK keys of all sequences and K/V heads, one after the other, are cut into as many equal spans as
// there are work-groups, whatever the lengths are: the lengths are known on the device only (a captured graph is
// replayed with others), so each work-group adds them up itself.  A span that begins or ends inside a sequence
// writes a partial result (m, l, O); attn_paged_join_kernel joins those.
//
// A work-group is NW waves, and each wave works through 32 keys of a tile on its own (nothing is shared but the end of
// a sequence, where the waves' results are added): K and V reach the wave's own LDS by direct transfers, those of the
// next tile while this one is computed on, also across the end of a sequence, with no barrier in between.  The 16 keys
// of a half block lie in one page, whose rows up to the sequence's last key are one buffer resource: slots behind it,
// pages that are none and columns that do not exist read as zero and fetch nothing.
//
// LDS: 16-byte chunk c of row R lies in 64-byte pieces of rows one after the other (four neighbouring lanes of a
// transfer fetch 64 contiguous bytes), exchanged within 64 bytes by f(R), so that the 16 rows of a K read and the
// 8 (16) rows of two V transpose reads lie in different banks.
//
// Bound by memory: 8 sequences of 8K keys, 268 MB, in 44 us and 4.6 for the join, 5.5 TB/s (a plain read reaches 6.2, 7.0 with
// the non-temporal hint, without which this takes 52); the transfers alone, with nothing computed, take 44 as well.  131K
// keys of e4m3 in 48 + 7 us, 64 ragged sequences of e4m3 (342 MB) in 62 + 5; the transfers alone 46 and 59.
//
// e4m3: the codes are converted to the tensors' type exactly; K's scale multiplies the scores of its 16 keys, V's power
// of two is applied by the conversion and the rest of it to the probabilities before their one rounding.
#include "attn_paged.hpp"

namespace attn {

typedef elem8 frag;
__device__ __forceinline__ f32x4 mfma16(frag a, frag b, f32x4 c)
{
#ifdef ATTN_F16
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
#else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#endif
}
template <int D, bool E8>
struct DecodeCfg {
    static constexpr int kSize = E8 ? 1 : 2;
    // (at D = 256 four waves' buffers of 16-bit keys do not fit)
    static constexpr int kNW = D == 256 && !E8 ? 2 : 4;
    static constexpr int kThreads = kNW * 64;
    static constexpr int kTK = kNW * 32;                    // keys of a tile
    static constexpr int kRows = 1024 / (D * kSize);        // rows of a transfer
    static constexpr int kPieces = 32 / kRows;              // transfers of a wave's K (V) of a tile
    static constexpr int kBlock = kRows * 64;               // the next 64 bytes of the rows of a piece
    static constexpr int kHalf = 16 / kRows * 1024;         // 16 rows further
    static constexpr int kStage = 2 * kPieces * 1024;       // a wave's K and V of a tile
    static constexpr int kLds = kNW * 2 * kStage;
    static constexpr bool kFlip = D == 256 && !E8;          // two rows a piece
    static constexpr int kSteps = D / 32, kDB = D / 16;
    static_assert(kStage >= 16 * D * 4, "the waves' results are added in a stage");
    static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
    // exchange of the chunks of row R, linear in the bits of R
    __host__ __device__ static constexpr int f(int R)
    {
        const int x = R >> 2;
        return (E8 ? (x & 1) | ((((x >> 1) ^ (x >> 2)) & 1) << 1) : ((x & 1) << 1) | ((x >> 1) & 1)) |
               (kFlip ? ((R >> 1) & 1) << 2 : 0);
    }
    // byte offset of chunk c of row R
    __host__ __device__ static constexpr int at(int R, int c)
    {
        const int x = c ^ f(R);
        return R / kRows * 1024 + x / 4 * kBlock + R % kRows * 64 + x % 4 * 16;
    }
};

// The tiles of a sequence that the kernel takes: one of 1 .. max_rows rows.  (No key: one tile, which has none.)
__device__ __forceinline__ int decode_tiles(const PagedSeq &s, int G, int max_rows, int TK)
{
    return s.n < 1 || (int64_t)s.n * G > max_rows ? 0 : max(1, (s.len + TK - 1) / TK);
}

// What the end of a unit counts as, in tiles: the waves wait for each other there.  (Without it the spans of short
// sequences, which end many, were the last to be done: 64 ragged ones in 77 us; 64.4 counted as 1, 62.7 as 2, 63.9 as 3.)
constexpr int kUnitEnd = 2;

// SPLIT: work-groups with spans, partial results in the workspace.  Otherwise one work-group for each sequence and K/V head.
// (Two work-groups a compute unit: without the bound, 32 rows and e4m3 take 260 registers and 63 us instead of 42.)
template <int D, int RB, bool E8, bool SPLIT>
__global__ void __launch_bounds__((DecodeCfg<D, E8>::kThreads), (D <= 128 ? 2 : 1))
attn_paged_decode_kernel(const PagedFwdArgs a, const int max_rows)
{
    using C = DecodeCfg<D, E8>;
    constexpr int NW = C::kNW, TK = C::kTK, R = 16 * RB, KP = C::kPieces;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ int scan[NW];
    __shared__ float sm[NW][R], sl[NW][R];

    const int tid = threadIdx.x, l = tid & 63, m16 = l & 15, g = l >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.Hq / a.Hkv, Hkv = a.Hkv, Dr = a.Dr, B = a.b.B;
    const PagedSlots<elem> slots(a.workspace, gridDim.x, R, D);

    // ---- where the span begins
    struct Unit { int b, h, t, tiles, first, n, len; };  // sequence, K/V head, tile
    auto set_seq = [&](Unit &u, const PagedSeq &s) __attribute__((always_inline)) {
        u.first = s.first;
        u.n = s.n;
        u.len = s.len;
        u.tiles = decode_tiles(s, G, max_rows, TK);
    };
    Unit nx;
    int left;  // of the span, from the tile nx on
    auto next_unit = [&](Unit &u) __attribute__((always_inline)) {
        u.t = 0;
        if (++u.h < Hkv) return;
        u.h = 0;
        do {
            ++u.b;
            if (u.b < B) set_seq(u, paged_seq_scalar(a.b, u.b));
        } while (u.b < B && u.tiles == 0);
    };
    PagedSpan span = {};
    if constexpr (SPLIT) {
        span = paged_span<NW>(a.b, Hkv, blockIdx.x, gridDim.x, kDecodeSpan, scan,
                              [&](const PagedSeq &s) {
            const int tiles = decode_tiles(s, G, max_rows, TK);
            return tiles ? tiles + kUnitEnd : 0;
        });
        if (tid == 0) slots.join[blockIdx.x].pieces = 0;
        if (span.left == 0) return;
        nx.b = span.b;
        set_seq(nx, span.seq);
        const int in = __builtin_amdgcn_readfirstlane((int)(span.begin - span.front));
        nx.h = in / (nx.tiles + kUnitEnd);
        nx.t = in - nx.h * (nx.tiles + kUnitEnd);
        left = span.left;
        if (nx.t >= nx.tiles) {  // it begins with the end of a unit
            left -= nx.tiles + kUnitEnd - nx.t;
            if (left <= 0) return;
            next_unit(nx);
        }
    } else {
        nx.b = blockIdx.x / Hkv;
        nx.h = blockIdx.x % Hkv;
        nx.t = 0;
        set_seq(nx, paged_seq_scalar(a.b, nx.b));
        left = nx.tiles;
        if (left == 0) return;
    }

    // ---- lanes
    const uint32_t row_bytes = (uint32_t)a.cache_stride_s * C::kSize;
    constexpr uint32_t kPast = 1u << 31;  // an offset behind every resource
    // what a lane fetches of a piece: its row, and (exchanged by the piece's f) its chunk
    const int fetch_row = l / 4 % C::kRows, fetch_chunk = (l / (4 * C::kRows) * 4 + l % 4) ^ C::f(fetch_row);
    const uint32_t fetch_off = fetch_row * row_bytes;
    const uint32_t stage0 = lds_address(smem) + w * 2 * C::kStage;
    const char *const mine = smem + w * 2 * C::kStage;
    // row reads of K: row m16 of a half, chunk 4 s + g; in the second half f may differ
    const int k_at[2][2] = {{C::at(m16, g), C::at(m16, 4 + g)}, {C::at(16 + m16, g), C::at(16 + m16, 4 + g)}};
    // transpose reads of V: column block db of 16, rows 4 g + e (16-bit; the second read is 16 rows further; e4m3: both)
    int v_at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (E8) {
            const int e = m16 >> 1, row = e < 4 ? 4 * g + e : 12 + 4 * g + e;
            v_at[j] = C::kPieces * 1024 + C::at(row, j) + (l & 1) * 8;
        } else {
            v_at[j] = C::kPieces * 1024 + C::at(4 * g + (m16 >> 2), 2 * j + ((l >> 1) & 1)) + (l & 1) * 8;
        }
    }
    // ---- transfers
    struct Pages { int id[2]; };           // of the wave's two half blocks of a tile
    struct Scales { float k[2], v[2]; };
    auto pages_of = [&](const Unit &u) __attribute__((always_inline)) {
        Pages p;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int key = u.t * TK + w * 32 + 16 * hf;
            // (without a branch: there is an entry in any case)
            const int at = max(min(key, u.len - 1), 0) >> a.b.page_shift;
            const int id = scalar_load(a.b.page_table + (int64_t)u.b * a.b.table_stride + at);
            p.id[hf] = key < u.len ? id : -1;
        }
        return p;
    };
    auto issue = [&](const Unit &u, const Pages &p, int buf, Scales &sc) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the buffer's last reads are done
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int key = u.t * TK + w * 32 + 16 * hf;
            const bool is = a.b.is_page(p.id[hf]);
            const int rows = is ? min(u.len - key, 16) : 0;
            const int id = is ? p.id[hf] : 0;
            const uint32_t bytes = rows > 0 ? (uint32_t)(rows - 1) * row_bytes + Dr * C::kSize : 0;
            const int64_t off = (id * a.cache_stride_p + u.h * a.cache_stride_h +
                                 (key & (a.b.page_size() - 1)) * a.cache_stride_s) * C::kSize;
            const desc_t Kd = make_desc((const char *)a.K_cache + off, bytes),
                         Vd = make_desc((const char *)a.V_cache + off, bytes);
            if constexpr (E8) {
                const float k = scalar_load(a.k_scale + (int64_t)id * Hkv + u.h),
                            v = scalar_load(a.v_scale + (int64_t)id * Hkv + u.h);
                sc.k[hf] = is ? k : 1.f;
                sc.v[hf] = is ? v : 1.f;
            }
#pragma unroll
            for (int n = 0; n < KP / 2; ++n) {
                const int pc = hf * (KP / 2) + n, chunk = fetch_chunk ^ C::f(pc * C::kRows);
                const uint32_t voff = chunk * 16 < Dr * C::kSize ? fetch_off + chunk * 16 : kPast;
                const uint32_t soff = n * C::kRows * row_bytes, lds = stage0 + buf * C::kStage + pc * 1024;
                dma16_between_nt(Kd, lds, voff, soff);
                dma16_between_nt(Vd, lds + KP * 1024, voff, soff);
            }
        }
    };

    Pages nx_pages = pages_of(nx);
    Scales sc = {};
    issue(nx, nx_pages, 0, sc);

    // the lane's rows (as columns of S^T): query head and new token
    int row_q[RB], row_h[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        row_q[rb] = (16 * rb + m16) / G;
        row_h[rb] = 16 * rb + m16 - row_q[rb] * G;
    }

    // ---- a sequence's and head's state
    frag q[RB][C::kSteps];
    // (the next unit's, requested with its first keys: where there are registers for them)
    constexpr bool kAhead = RB == 1;
    frag next_q[kAhead ? RB : 1][C::kSteps];
    f32x4 o[RB][C::kDB];
    float m[RB], lsum[RB];
    constexpr float kMinusHuge = -1.0e30f;
    // Probabilities up to 2^8 before the reference maximum moves: inside the exponents of either type (fp16: up to 2^15), so
    // that rounding them to it costs the same; sums and products are fp32.
    constexpr float kSlack = 8.f;
    auto load_q = [&](const Unit &u, auto &to) __attribute__((always_inline)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const bool is = row_q[rb] < u.n;
            const elem *row = a.Q + (u.first + (is ? row_q[rb] : 0)) * a.q_stride_t +
                              (u.h * G + (is ? row_h[rb] : 0)) * a.q_stride_h;
#pragma unroll
            for (int s = 0; s < C::kSteps; ++s) {
                // (e4m3: a lane's 16 bytes of K are 16 columns, which make two steps)
                const int col = E8 ? s / 2 * 64 + g * 16 + s % 2 * 8 : s * 32 + g * 8;
                to[rb][s] = as_elem8(ld_row16(row, col, Dr));
            }
        }
    };
    auto begin_unit = [&](const Unit &u) __attribute__((always_inline)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            m[rb] = kMinusHuge;
            lsum[rb] = 0.f;
#pragma unroll
            for (int db = 0; db < C::kDB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if constexpr (kAhead) {
#pragma unroll
            for (int s = 0; s < C::kSteps; ++s) q[0][s] = next_q[0][s];
        } else {
            load_q(u, q);
        }
    };
    auto compute = [&](const Unit &u, const Pages &p, int buf, const Scales &sc) __attribute__((always_inline)) {
        const int kb = u.t * TK + w * 32;
        if (kb >= u.len) return;
        const char *at = mine + buf * C::kStage;
        f32x4 s[2][RB];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) s[hf][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < C::kSteps; ++st) {
                if constexpr (E8) {
                    if (st % 2) continue;
                    const u32x4 c = *(const u32x4 *)(at + k_at[hf][0] + st / 2 * C::kBlock);
                    const frag k0 = from_e4m3(c.x, c.y, 1.f, 1.f), k1 = from_e4m3(c.z, c.w, 1.f, 1.f);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        s[hf][rb] = mfma16(k0, q[rb][st], s[hf][rb]);
                        s[hf][rb] = mfma16(k1, q[rb][st + 1], s[hf][rb]);
                    }
                } else {
                    const frag k = C::kFlip ? *(const frag *)(at + k_at[hf][st % 2] + st / 2 * 2 * C::kBlock)
                                            : *(const frag *)(at + k_at[hf][0] + st * C::kBlock);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) s[hf][rb] = mfma16(k, q[rb][st], s[hf][rb]);
                }
            }
        }
        float c[2] = {a.scale_log2e, a.scale_log2e};
        if constexpr (E8) {  // (not 0, which a masked score would turn into NaN)
            c[0] = fmaxf(c[0] * sc.k[0], 1e-38f);
            c[1] = fmaxf(c[1] * sc.k[1], 1e-38f);
        }
        const bool pages = a.b.is_page(p.id[0]) && (kb + 16 >= u.len || a.b.is_page(p.id[1]));
        if (!pages || kb + 32 > u.len || (a.causal && kb + 32 > u.len - u.n + 1)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int seen = a.causal ? min(u.len, u.len - u.n + row_q[rb] + 1) : u.len;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const int lim = (a.b.is_page(p.id[hf]) ? seen : 0) - kb - 16 * hf - 4 * g;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i >= lim) s[hf][rb][i] = -INFINITY;
                }
            }
        }
        bool over = false;
        float top[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float t[2];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                t[hf] = fmaxf(fmaxf(s[hf][rb][0], s[hf][rb][1]), fmaxf(s[hf][rb][2], s[hf][rb][3])) * c[hf];
            top[rb] = fmaxf(t[0], t[1]);
            over |= top[rb] > m[rb] + kSlack;
        }
        if (__builtin_amdgcn_ballot_w64(over)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float t = xhalf_max(top[rb]);
                t = fmaxf(t, __shfl_xor(t, 16));
                const float to = fmaxf(m[rb], t), alpha = fast_exp2(m[rb] - to);
                m[rb] = to;
                lsum[rb] *= alpha;
#pragma unroll
                for (int db = 0; db < C::kDB; ++db) o[rb][db] *= alpha;
            }
        }
        frag pr[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float e[2][4];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[hf][i] = fast_exp2(__builtin_fmaf(s[hf][rb][i], c[hf], -m[rb]));
                    lsum[rb] += e[hf][i];
                }
            if constexpr (E8) {
                // what the conversion leaves of V's scale: in 1 .. 2 (0: 0)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const float rest = scale_rest(sc.v[hf]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[hf][i] *= rest;
                }
            }
            pr[rb] = pack8(e[0][0], e[0][1], e[0][2], e[0][3], e[1][0], e[1][1], e[1][2], e[1][3]);
        }
#pragma unroll
        for (int db = 0; db < C::kDB; ++db) {
            frag v;
            if constexpr (E8) {
                typedef int i32x2 __attribute__((ext_vector_type(2)));
                const i32x2 c8 = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (i32x2 __attribute__((address_space(3))) *)(at + v_at[db % 4] + db / 4 * C::kBlock));
                v = from_e4m3(c8.x, c8.y, sc.v[0], sc.v[1]);
            } else {
                const char *x = C::kFlip ? at + v_at[db % 4] + db / 4 * 2 * C::kBlock
                                         : at + v_at[db % 2] + db / 2 * C::kBlock;
                v = join8(lds_read_tr((const elem *)x), lds_read_tr((const elem *)(x + C::kHalf)));
            }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) o[rb][db] = mfma16(v, pr[rb], o[rb][db]);
        }
    };
    // The waves' results together, in the stage that has just been worked through.
    auto end_unit = [&](const Unit &u, bool from_start, bool to_end, int buf) __attribute__((always_inline)) {
        float ls[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            ls[rb] = xhalf_sum(lsum[rb]);
            ls[rb] += __shfl_xor(ls[rb], 16);
            if (g == 0) {
                sm[w][16 * rb + m16] = m[rb];
                sl[w][16 * rb + m16] = ls[rb];
            }
        }
        __syncthreads();
        const int rows = u.n * G;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (from_start ? 1 : 0);
        if (SPLIT && from_start && !to_end && tid == 0) {
            // the unit's last tile lies u.tiles - u.t - 1 behind this one, the span's last
            const int64_t last = span.begin + span.left - 1 + (u.tiles - 1 - u.t);
            slots.join[blockIdx.x] = PagedJoin{u.first, u.h, 0, rows,
                                                   min((int)(last / span.size), (int)gridDim.x - 1) - (int)blockIdx.x + 1};
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            if (16 * rb >= rows) break;
            const int r = 16 * rb + m16;
            float top = sm[0][r], all = 0.f;
#pragma unroll
            for (int i = 1; i < NW; ++i) top = fmaxf(top, sm[i][r]);
#pragma unroll
            for (int i = 0; i < NW; ++i) all += sl[i][r] * fast_exp2(sm[i][r] - top);
            const float mul = fast_exp2(m[rb] - top);
            // [16 rows][D] fp32, 16-byte chunks exchanged by the row
            char *const out = smem + (w * 2 + buf) * C::kStage;
#pragma unroll
            for (int db = 0; db < C::kDB; ++db)
                *(f32x4 *)(out + m16 * (D * 4) + ((4 * db + g) ^ m16) * 16) = o[rb][db] * mul;
            if (w == 0 && g == 0 && r < rows) {
                if (from_start && to_end)
                    a.LSE[(int64_t)(u.first + row_q[rb]) * a.Hq + u.h * G + row_h[rb]] =
                        all > 0.f ? (top + fast_log2(all)) * kLn2 : -INFINITY;
                else {
                    slots.m[slot * R + r] = top;
                    slots.l[slot * R + r] = all;
                }
            }
            // the sums of the rows, for the threads that store them
            __shared__ float inv[16];
            if (w == 0 && g == 0) inv[m16] = all > 0.f ? 1.f / all : 0.f;
            __syncthreads();
            for (int i = tid; i < 16 * (D / 4); i += C::kThreads) {
                const int row = i / (D / 4), c4 = i % (D / 4), rr = 16 * rb + row;
                if (rr >= rows || 4 * c4 >= Dr) continue;
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < NW; ++k)
                    x += *(const f32x4 *)(smem + (k * 2 + buf) * C::kStage + row * (D * 4) + (c4 ^ row) * 16);
                if (from_start && to_end) {
                    const int t = rr / G, h = rr - t * G;
                    const float by = inv[row];
                    *(elem4 *)(a.O + (u.first + t) * a.out_stride_t + (u.h * G + h) * a.out_stride_h + 4 * c4) =
                        pack4(x[0] * by, x[1] * by, x[2] * by, x[3] * by);
                } else {
                    *(f32x4 *)(slots.part + (slot * R + rr) * D + 4 * c4) = x;
                }
            }
            __syncthreads();
        }
    };

    // ---- the span: tile cur, whose transfers are on their way; nx behind it, which the span may not hold any more
    Unit cur = nx;
    Pages cur_pages = nx_pages;
    if constexpr (kAhead) load_q(cur, next_q);
    begin_unit(cur);
    bool from_start = cur.t == 0;
    int buf = 0;
    // u and what is left of the span to the tile behind it
    auto advance = [&](Unit &u) __attribute__((always_inline)) {
        --left;
        if (++u.t < u.tiles) return;
        left -= SPLIT ? kUnitEnd : left;
        if (left > 0) next_unit(u);
    };
    advance(nx);
    bool more = left > 0;
    if (more) nx_pages = pages_of(nx);
    while (true) {
        Scales next_sc = {};
        if (more) {
            issue(nx, nx_pages, buf ^ 1, next_sc);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * KP) : "memory");
            if constexpr (kAhead) if (nx.t == 0) load_q(nx, next_q);
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        Unit nn = nx;
        Pages nn_pages = nx_pages;
        bool still = false;
        if (more) {
            advance(nn);
            still = left > 0;
            if (still) nn_pages = pages_of(nn);
        }
        compute(cur, cur_pages, buf, sc);
        const bool to_end = cur.t + 1 == cur.tiles;
        if (to_end || !more) {
            end_unit(cur, from_start, to_end, buf);
            if (!more) return;
            begin_unit(nx);
            from_start = true;
        }
        more = still;
        cur = nx;
        cur_pages = nx_pages;
        nx = nn;
        nx_pages = nn_pages;
        sc = next_sc;
        buf ^= 1;
    }
}

// The partial results of the units that worker blockIdx.y has the first tile of, joined.  A work-group has one row (grid x),
// PAR = 1024 / D groups of D / 4 threads that share the pieces, 64 at a time: a piece's maximum and sum in a lane.
// Bound by three accesses that wait for each other (record, maxima, rows) and the launch: 4.6 us for 64 units of 8 pieces, 7.2
// for 8 of 64.  The rows of a unit are neighbours in the grid, on all XCDs (workers first: 5.6 instead of 4.8 with 16 rows).
template <int D>
__global__ void __launch_bounds__(256) attn_paged_join_kernel(const PagedFwdArgs a, const PagedSlots<elem> s, const int R)
{
    constexpr int kCols = D / 4, PAR = 256 / kCols;
    __shared__ f32x4 sum[PAR][kCols];
    const PagedJoin j = s.join[blockIdx.y];
    const int tid = threadIdx.x, l = tid & 63, c = tid % kCols, p = tid / kCols, r = blockIdx.x;
    if (j.pieces == 0 || r >= j.rows) return;
    auto at = [&](int i) { return (2 * (int64_t)(blockIdx.y + i) + (i == 0)) * R + r; };
    const bool mine = 4 * c < a.Dr;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    float top = kJoinMinusHuge, all = 0.f;
    for (int i0 = 0; i0 < j.pieces; i0 += 64) {
        const int n = min(j.pieces - i0, 64);
        const bool is = l < n;
        const float m = is ? s.m[at(i0 + l)] : kJoinMinusHuge, sum_l = is ? s.l[at(i0 + l)] : 0.f;
        float to = fmaxf(top, m);
#pragma unroll
        for (int d = 32; d; d /= 2) to = fmaxf(to, __shfl_xor(to, d));
        const float weight = fast_exp2(m - to), keep = fast_exp2(top - to);
        float sums = sum_l * weight;
#pragma unroll
        for (int d = 32; d; d /= 2) sums += __shfl_xor(sums, d);
        x *= keep;
        all = all * keep + sums;
        top = to;
        // (the first piece lies in its worker's other slot)
        const float *const part = s.part + at(i0) * D + 4 * c;
        const int64_t step = 2 * (int64_t)R * D, back = i0 == 0 ? (int64_t)R * D : 0;
#pragma unroll 4
        for (int i = 0; i < n; i += PAR) {
            const int k = i + p;
            const float by = __shfl(weight, k & 63);
            if (k < n && mine) x += *(const f32x4 *)(part + k * step - (k ? back : 0)) * by;
        }
    }
    sum[p][c] = x;
    __syncthreads();
    if (p || !mine) return;
#pragma unroll
    for (int i = 1; i < PAR; ++i) x += sum[i][c];
    const float inv = all > 0.f ? 1.f / all : 0.f;
    const int G = a.Hq / a.Hkv, t = j.first + r / G, hq = j.head * G + r % G;
    *(elem4 *)(a.O + t * a.out_stride_t + hq * a.out_stride_h + 4 * c) = pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    if (c == 0) a.LSE[(int64_t)t * a.Hq + hq] = all > 0.f ? (top + fast_log2(all)) * kLn2 : -INFINITY;
}

template <int D, int RB, bool E8>
static int launch_decode_t(const PagedFwdArgs &a, int max_rows, int workers, hipStream_t st)
{
    using C = DecodeCfg<D, E8>;
    const void *kernel = workers ? (const void *)attn_paged_decode_kernel<D, RB, E8, true>
                                     : (const void *)attn_paged_decode_kernel<D, RB, E8, false>;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, C::kLds) != hipSuccess) return -1;
    if (!workers) {
        hipLaunchKernelGGL((attn_paged_decode_kernel<D, RB, E8, false>), dim3(a.b.B * a.Hkv), dim3(C::kThreads), C::kLds,
                           st, a, max_rows);
    } else {
        hipLaunchKernelGGL((attn_paged_decode_kernel<D, RB, E8, true>), dim3(workers), dim3(C::kThreads), C::kLds, st, a,
                           max_rows);
        hipLaunchKernelGGL(attn_paged_join_kernel<D>, dim3(max_rows, workers), dim3(256), 0, st, a,
                           PagedSlots<elem>(a.workspace, workers, 16 * RB, D), 16 * RB);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D, bool E8>
static int launch_decode_d(const PagedFwdArgs &a, int max_rows, int workers, hipStream_t st)
{
    if (max_rows <= 16) return launch_decode_t<D, 1, E8>(a, max_rows, workers, st);
    if constexpr (D <= 128) return launch_decode_t<D, 2, E8>(a, max_rows, workers, st);
    return -1;
}

int launch_paged_decode(const PagedFwdArgs &a, int D, int max_rows, int workers, hipStream_t st)
{
    if (a.k_scale)
        return D == 64 ? launch_decode_d<64, true>(a, max_rows, workers, st)
             : D == 128 ? launch_decode_d<128, true>(a, max_rows, workers, st)
                        : launch_decode_d<256, true>(a, max_rows, workers, st);
    return D == 64 ? launch_decode_d<64, false>(a, max_rows, workers, st)
         : D == 128 ? launch_decode_d<128, false>(a, max_rows, workers, st)
                    : launch_decode_d<256, false>(a, max_rows, workers, st);
}

}  // namespace attn
