// Attention over a paged cache of latent rows on gfx950 (the absorbed form).
//
// A token has one row c_j = [latent part, R values | rotary part, E values] for all query heads: it is their key, and its
// latent part their value.  Query row r = (token i, head h) of a sequence:
//
//     s_rj = scale <q_r, c_j>,   out_r = sum_j softmax_j(s_rj) c_j[0 .. R)     over the rows j up to token i's own.
//
// 2 (R + E) + 2 R flops a pair for 2 (R + E) bytes a row: M = W Hq query rows share every row that is read, so few heads
// are bound by the memory and 128 of them are about as much bound by the products (242 flops a byte).
//
// S^T = C Q^T and O^T = C^T P by 16x16x32 matrix instructions, 16 query rows a wave, one per lane % 16, so all soft-max state is lane
// local; one pass over the rows with a running maximum and sum.  A tile of 32 rows is contiguous in a page and goes from
// memory straight into LDS, once: the first product reads its rows, the second one the same rows transposed.  Queries and
// output stay in registers (72 and 128 of a lane's, for R = 512).
//
// A workgroup's waves are RG row groups x KG key groups: waves of one key group share tiles, the key groups take tiles in
// turn and are joined in LDS at the end.  Few sequences are shared by S workgroups, whose partials a second launch joins.
//
// What bounds it, R = 512, per row of every sequence (one long batch minus a shorter one, 256 sequences): 16 heads 6.2 TB/s, what
// reads alone reach; 64 heads 6.3 TB/s; 128 heads 940 TFLOP/s and 3.9 TB/s, where a large product of matrices reaches 1230.  There a
// wave's products wait for its own reads of LDS (256 bytes a clock: 30 % of it is used) and for the loads' issue, ~100 clocks each;
// the other wave of the SIMD covers a part, the matrix units are busy 40 % of the time.  Besides that, a call of 64 sequences x 16 heads x
// 1000 to 2000 rows (33 us; 18 for the bytes) has ~5 us until the first tile is there, lengths 1.3 times the mean in its longest
// workgroups, 3 us of partials and a joining launch of 4.7; one of 128 x 128 x 1894 to 3533 (135 us; 78 for the products) its lengths.
//
// P is rounded to bf16 for the second product (half a step: 2^-8 of an entry at most), since the rows are bf16 and the matrix instructions
// take operands of one type: in two parts it would be half as many products again, for an error that the output's own rounding (it is
// the operand of the product that brings the latent vectors to the heads' values) has too.  Sums and soft-max state are fp32.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ngc.h"
#include "ngc_device.h"
#include "ngc_latent.h"
#include "ngc_latent_shape.h"
#include "ngc_workspace.h"

namespace ngc {

constexpr int LT_LDS_KEYS = 128;            // rows in LDS: those of R = 512 fill a CU's

struct LatentArgs {
    const unsigned char *rows;              // bf16 [num_pages][page_rows][R + E]
    const int32_t *table;                   // [L][B][max_pages]
    const int32_t *len;                     // [L][B]
    const int32_t *n_new;                   // [B] or nullptr
    const unsigned char *q;                 // bf16 [launch layers][B][W][Hq][R + E]
    unsigned char *out;                     // bf16 [launch layers][B][W][Hq][R]
    float *lse_out;                         // fp32 [launch layers][B][W][Hq] or nullptr
    float *part_o;                          // [segments of the launch][S][M][R]
    float *part_ml;                         // [segments of the launch][S][M][2]
    int32_t *status;
    int seg0, nseg, blocks, S, M, W, Hq, B, cap;
    int max_pages, num_pages, page_shift;
    float scale, scale_log2e;
};

// A sequence's rows and its new tokens.
struct LatentSegment {
    int n, w;
    __device__ __forceinline__ LatentSegment(const LatentArgs &a, int seg, bool counts)
    {
        n = constant_word(a.len + a.seg0 + seg);
        w = a.n_new ? constant_word(a.n_new + seg % a.B) : a.W;
        const bool odd = n < 0 || n > a.cap, odd_new = w < 0 || w > a.W;
        if (counts) {
            if (odd) atomicAdd(&a.status[NGC_STATUS_LEN_CLAMPED], 1);
            if (odd_new) atomicAdd(&a.status[NGC_STATUS_LEN_CLAMPED], 1);
            if (n <= 0 && w != 0) atomicAdd(&a.status[NGC_STATUS_EMPTY_ATTN], 1);
        }
        n = n < 0 ? 0 : n > a.cap ? a.cap : n;
        w = w < 0 ? 0 : w > a.W ? a.W : w;
    }
    // How many rows query row r sees.
    __device__ __forceinline__ int limit(const LatentArgs &a, int r) const
    {
        const int sees = n - w + r / a.Hq + 1;
        return sees < 0 ? 0 : sees > n ? n : sees;
    }
};

// Where things are in a tile of KEYS rows in LDS: the latent parts, 16-byte piece p of row r at slot p ^ swizzle(r), then the rotary
// parts.
template <int R, int E, int KEYS>
struct LatentTile {
    static constexpr int ROW = (R + E) * 2, LAT = R * 2, ROT = E * 2;
    static constexpr int LAT_BYTES = KEYS * LAT, BYTES = KEYS * ROW;
    static constexpr int LAT_PIECES = LAT / 16, ROT_PIECES = ROT / 16;
    static constexpr int LAT_ROWS = 64 / LAT_PIECES, ROT_ROWS = 64 / ROT_PIECES;         // rows a wave-wide load brings
    static constexpr int LAT_LOADS = KEYS / LAT_ROWS, ROT_LOADS = KEYS / ROT_ROWS;
    static_assert(LAT_PIECES == 64 || LAT_PIECES == 32, "whole rows a load");
    static_assert(ROT_PIECES == 8 || ROT_PIECES == 4, "whole rows a load");
    __device__ static __forceinline__ int swizzle(int r) { return lds_swizzle<LAT_PIECES>(r); }
    __device__ static __forceinline__ int rot_swizzle(int r) { return lds_swizzle<ROT_PIECES>(r); }
    __device__ static __forceinline__ uint32_t piece(int r, int p)
    {
        if (p < LAT_PIECES) return (uint32_t)(r * LAT + (p ^ swizzle(r)) * 16);
        return (uint32_t)(LAT_BYTES + r * ROT + ((p - LAT_PIECES) ^ rot_swizzle(r)) * 16);
    }
};

__device__ __forceinline__ f32x4 product16(bf16x8 x, bf16x8 y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); }
// Over the 32 (16) rows of a tile: columns (rows read transposed) by weights.
__device__ __forceinline__ f32x4 add_rows(const u32x2 (&v)[2], const uint32_t (&w)[4], f32x4 c)
{
    return product16(__builtin_bit_cast(bf16x8, u32x4{v[0][0], v[0][1], v[1][0], v[1][1]}), __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]}), c);
}
__device__ __forceinline__ f32x4 add_rows(const u32x2 (&v)[1], const uint32_t (&w)[2], f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, v[0]), __builtin_bit_cast(s16x4, u32x2{w[0], w[1]}), c, 0, 0, 0);
}
// Row of a tile that score register e of a lane's quarter stands for: the scores of rows 0 .. 15, then (of 32) of 16 .. 31.
__device__ __forceinline__ int latent_key(int e, int quarter) { return 16 * (e / 4) + 4 * quarter + e % 4; }

// 2^8: the reference of the exponents moves only when a maximum has outgrown it by that.
constexpr float LT_LAZY = 8.0f;

// Waves per SIMD: what LDS leaves room for.
constexpr int latent_waves(int R, int NW) { return R == 512 ? NW / 4 : 2; }

// NW waves, RG row groups.
template <int R, int E, int NW, int RG>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(latent_waves(R, NW))))
void latent_attn_kernel(LatentArgs a)
{
    constexpr int KEYS = latent_keys(RG), HALVES = KEYS / 16, SLOTS = LT_LDS_KEYS / KEYS;
    using Tile = LatentTile<R, E, KEYS>;
    constexpr int KG = NW / RG;
    constexpr int NB = SLOTS / KG;                         // buffers of a key group
    static_assert(NB == 2, "a tile is on its way while one is worked on");
    constexpr int CHUNKS = (R + E) / 32, LAT_CHUNKS = R / 32, CT = R / 16;               // of the first product; column tiles of the second
    constexpr int LAT_LOADS = (Tile::LAT_LOADS + RG - 1) / RG, ROT_LOADS = (Tile::ROT_LOADS + RG - 1) / RG;      // of a wave, per tile
    // A wave is held up where it asks for a tile, about 100 clocks a load.  The two waves of a SIMD, of different key groups, do it at
    // different times: 343 us for 380 with 256 sequences of 4096 rows and 128 heads, R = 512.
    constexpr bool LATER = RG > 1;
    constexpr int PARTS = (NW * LT_ROWS * R * 4 + SLOTS * Tile::BYTES - 1) / (SLOTS * Tile::BYTES);       // the output goes through LDS in

    extern __shared__ __align__(256) unsigned char lds[];
    float *const red = reinterpret_cast<float *>(lds + SLOTS * Tile::BYTES);             // [2][waves][rows]
    uint32_t *const odd_waves = reinterpret_cast<uint32_t *>(red + 2 * NW * LT_ROWS);    // [waves]

    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    const int rg = wv % RG, kg = wv / RG;
    const int row = lane & 15, quarter = lane >> 4;
    // the row blocks of a share of a sequence follow one another on one XCD, whose L2 then has the rows for all but the first
    int share = (int)blockIdx.x, block = 0;
    if (a.blocks > 1) {
        const int first = (int)(blockIdx.x / (8u * (unsigned)a.blocks)) * 8, at = (int)blockIdx.x - first * a.blocks;
        const int here = a.nseg * a.S - first < 8 ? a.nseg * a.S - first : 8;
        block = at / here;
        share = first + at - block * here;
    }
    const int seg = share % a.nseg, split = share / a.nseg;
    const int stride = a.S * KG, first_tile = split * KG + kg;
    const int32_t *tab = a.table + (size_t)(a.seg0 + seg) * a.max_pages;
    auto tile_base = [&](int t) -> const unsigned char * {
        const int r0 = t * KEYS;
        int page = constant_word(tab + (r0 >> a.page_shift));
        page = (page < 0 || page >= a.num_pages) ? 0 : page;          // never leave the pool
        return a.rows + (((size_t)page << a.page_shift) + (r0 & ((1 << a.page_shift) - 1))) * Tile::ROW;
    };
    // ---- asked for before the lengths have arrived: queries (of rows that are none too) and the first tile (or the last there is room
    // for) ----
    const int block_row0 = block * RG * LT_ROWS;
    const int my_row = block_row0 + rg * LT_ROWS + row, q_row = my_row < a.M ? my_row : a.M - 1;
    const unsigned char *const first_base = tile_base(first_tile < a.cap / KEYS ? first_tile : a.cap / KEYS - 1);
    const LatentSegment s(a, seg, threadIdx.x == 0 && split == 0 && block == 0);

    unsigned char *const buffers = lds + kg * NB * Tile::BYTES;
    auto load_tile = [&](const unsigned char *base, unsigned char *to) {
        int lane_ = lane;
        __asm__ volatile("" : "+v"(lane_));                // (offsets are made where they are used, not kept over the loop)
        // the swizzle is linear in a row's bits: a lane's part of it, and the load's
        const int lrow = Tile::LAT_ROWS == 1 ? 0 : lane_ / Tile::LAT_PIECES, lp = lane_ % Tile::LAT_PIECES ^ Tile::swizzle(lrow);
#pragma unroll
        for (int i = 0; i < LAT_LOADS; ++i) {
            const int r0 = (i * RG + rg) * Tile::LAT_ROWS;
            start_load_to_lds16(base + r0 * Tile::ROW, (uint32_t)(lrow * Tile::ROW) + (uint32_t)(lp ^ Tile::swizzle(r0)) * 16, to + r0 * Tile::LAT);
        }
        const int rrow = lane_ / Tile::ROT_PIECES, rp = lane_ % Tile::ROT_PIECES ^ Tile::rot_swizzle(rrow);
#pragma unroll
        for (int i = 0; i < ROT_LOADS; ++i) {
            const int r0 = (i * RG + rg) % Tile::ROT_LOADS * Tile::ROT_ROWS;             // (what is left over loads a part again)
            start_load_to_lds16(base + r0 * Tile::ROW + Tile::LAT, (uint32_t)(rrow * Tile::ROW) + (uint32_t)(rp ^ Tile::rot_swizzle(r0)) * 16,
                                to + Tile::LAT_BYTES + r0 * Tile::ROT);
        }
    };
    load_tile(first_base, buffers);
    bf16x8 qop[CHUNKS];
    {
        const unsigned char *q = a.q + ((size_t)seg * a.M + q_row) * Tile::ROW + quarter * 16;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) qop[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(q + c * 64));
    }

    const int real_rows = s.w * a.Hq;                      // query rows of the sequence
    if (block_row0 >= real_rows) {
        wait_for_loads<0>();                               // nothing may be on its way to LDS that is not this workgroup's any more
        return;
    }
    const int limit = s.limit(a, q_row);
    // rows below `all` are seen by every query row of the workgroup, rows from `end` on by none
    const int all = s.limit(a, block_row0);
    const int last_row = block_row0 + RG * LT_ROWS - 1;
    const int end = s.limit(a, last_row < real_rows ? last_row : real_rows - 1);
    const int tiles = (end + KEYS - 1) / KEYS;
    f32x4 oacc[CT];                                        // registers e of column tile c: columns 16 c + 4 quarter + e
#pragma unroll
    for (int c = 0; c < CT; ++c) oacc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, m_ref = 0.f, l_run = 0.f;     // m_ref: m_run, or 0 as long as nothing has been seen

    // Where this lane's operands are in a tile.  Pieces 16 apart are 256 bytes apart whatever the swizzle, rows 16 apart have the same one,
    // and a tile begins at a multiple of 256: the other offsets differ from the first one's by bits.
    static_assert(Tile::BYTES % 256 == 0 && Tile::LAT % 256 == 0, "offsets differ by bits");
    const int read_row = 4 * quarter + row / 4, read_col = 4 * (row % 4);                // of the transposing reads
    const uint32_t lat0 = Tile::piece(row, quarter), rot0 = Tile::piece(row, Tile::LAT_PIECES + quarter);
    const uint32_t col0 = Tile::piece(read_row, read_col / 8) + (uint32_t)(read_col % 8) * 2;
    auto compute_tile = [&](int t, unsigned char *tile, auto between) {
        const uint32_t tile_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char *)tile;
        auto row_piece = [&](int c, int k) {               // chunk c of rows 16 k ..
            const uint32_t at = c < LAT_CHUNKS ? ((tile_at + lat0) ^ (uint32_t)(c % 4 * 64)) + (uint32_t)(c / 4 * 256 + k * 16 * Tile::LAT)
                                               : ((tile_at + rot0) ^ (uint32_t)((c - LAT_CHUNKS) * 64)) + (uint32_t)(k * 16 * Tile::ROT);
            return *(const u32x4 __attribute__((address_space(3))) *)(uintptr_t)at;
        };
        auto transposed = [&](int g, int c) {              // rows 16 g + 4 quarter .. + 3 of column tile c
            const uint32_t at = ((tile_at + col0) ^ (uint32_t)(c % 8 * 32)) + (uint32_t)(c / 8 * 256 + g * 16 * Tile::LAT);
            return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)at));
        };
        const int key0 = t * KEYS;
        constexpr int SCORES = 4 * HALVES;
        // GROUP chunks' rows (column tiles) are asked for DEPTH - 1 groups (a group) before their products run
        constexpr int GROUP = RG == 1 ? (CHUNKS % 6 == 0 ? 6 : 9) : R == 512 ? 1 : 3, VGROUP = RG == 1 ? 8 : 4, DEPTH = RG > 1 && R == 512 ? 4 : 2;
        static_assert(CHUNKS % GROUP == 0 && CT % VGROUP == 0, "whole groups");
        f32x4 sc[HALVES];
#pragma unroll
        for (int k = 0; k < HALVES; ++k) sc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 x[DEPTH][GROUP][HALVES];
        auto ask_rows = [&](int g) {
#pragma unroll
            for (int u = 0; u < GROUP; ++u)
#pragma unroll
                for (int k = 0; k < HALVES; ++k) x[g % DEPTH][u][k] = row_piece(g * GROUP + u, k);
        };
        u32x2 v[2][VGROUP][HALVES];
        auto ask_columns = [&](int g) {
#pragma unroll
            for (int u = 0; u < VGROUP; ++u)
#pragma unroll
                for (int h = 0; h < HALVES; ++h) v[g & 1][u][h] = transposed(h, g * VGROUP + u);
        };
#pragma unroll
        for (int g = 0; g < DEPTH - 1; ++g) ask_rows(g);
#pragma unroll
        for (int g = 0; g < CHUNKS / GROUP; ++g) {
            if (g + DEPTH - 1 < CHUNKS / GROUP) ask_rows(g + DEPTH - 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < GROUP; ++u)
#pragma unroll
                for (int k = 0; k < HALVES; ++k) sc[k] = product16(__builtin_bit_cast(bf16x8, x[g % DEPTH][u][k]), qop[g * GROUP + u], sc[k]);
            __builtin_amdgcn_sched_barrier(0);
        }
        const bool mixed = key0 + KEYS > all;              // not every query row of the workgroup sees all of the tile's rows
        between();
        // Values that are not finite, where some query row does not see their row: a weight of 0 would make NaN of them.  Every wave looks
        // at what it has loaded itself.  (In a round of several key groups some may have such a tile and some not.)
        if (RG == 1 ? mixed : (t - kg + KG) * KEYS > all) {
            unsigned char *const own = tile + (Tile::LAT_ROWS == 2 ? lane / 32 * Tile::LAT + lane % 32 * 16 : lane * 16);
            auto own_part = [&](auto &&f) {
#pragma unroll 1
                for (int k = 0; k < LAT_LOADS; ++k) {
                    u32x4 *const at = reinterpret_cast<u32x4 *>(own + (k * RG + rg) * Tile::LAT_ROWS * Tile::LAT);
                    f(at, *at);
                }
            };
            bool odd = false;
            if (mixed) own_part([&](u32x4 *, u32x4 x) { odd |= has_odd(u32x2{x[0], x[1]}) | has_odd(u32x2{x[2], x[3]}); });
            bool some = __ballot(odd) != 0;
            if constexpr (RG > 1) {
                if (lane == 0) odd_waves[wv] = some;
                lds_accesses_done();
                workgroup_barrier();
                uint32_t any = 0;
#pragma unroll
                for (int k = 0; k < NW; ++k) any |= odd_waves[k];
                some = __builtin_amdgcn_readfirstlane(any) != 0;
            }
            if (__builtin_expect(some, 0)) {
                // They become NaN in the columns of the query rows that see theirs: such a row's score is not finite, its weight NaN, or 0
                // for minus infinity, and NaN is what either makes of them.  How many of a column a query row sees is another product.
                // Then they become 0.
                if (mixed) {
                    uint32_t sees[SCORES / 2];
#pragma unroll
                    for (int e = 0; e < SCORES / 2; ++e)
                        sees[e] = (key0 + latent_key(2 * e, quarter) < limit ? 0x3F80u : 0u) | (key0 + latent_key(2 * e + 1, quarter) < limit ? 0x3F800000u : 0u);
#pragma unroll
                    for (int c = 0; c < CT; ++c) {
                        u32x2 y[HALVES];
#pragma unroll
                        for (int h = 0; h < HALVES; ++h) y[h] = odd_ones(transposed(h, c));
                        const f32x4 count = add_rows(y, sees, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int e = 0; e < 4; ++e) oacc[c][e] = count[e] > 0.f ? NAN : oacc[c][e];
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                if constexpr (RG > 1) {
                    lds_accesses_done();
                    workgroup_barrier();
                }
                if (mixed)
                    own_part([&](u32x4 *at, u32x4 x) {
                        u32x2 lo = {x[0], x[1]}, hi = {x[2], x[3]};
                        take_out_odd(lo);
                        take_out_odd(hi);
                        *at = u32x4{lo[0], lo[1], hi[0], hi[1]};
                    });
                lds_accesses_done();
                if constexpr (RG > 1) workgroup_barrier();
            }
        }
        ask_columns(0);                                    // (there when the weights are)
        __builtin_amdgcn_sched_barrier(0);
        float s_[SCORES];
#pragma unroll
        for (int e = 0; e < SCORES; ++e) s_[e] = sc[e / 4][e % 4];
        if (mixed) {
#pragma unroll
            for (int e = 0; e < SCORES; ++e) s_[e] = key0 + latent_key(e, quarter) < limit ? s_[e] : -INFINITY;
        }
        float tmx = s_[0];
#pragma unroll
        for (int e = 1; e < SCORES; ++e) tmx = max_no_nan(tmx, s_[e]);
        tmx = quad_rows_max(tmx);
        const bool outgrown = (tmx - m_run) * a.scale_log2e > LT_LAZY;     // of each row by itself: its results do not depend on its neighbours'
        if (__ballot(outgrown)) {
            const bool some = __ballot(m_run > -INFINITY) != 0;            // (nothing to scale on the first tile)
            const float m_new = outgrown ? tmx : m_run;
            const float alpha = m_new == m_run ? 1.0f : fast_exp2((m_run - m_new) * a.scale_log2e);
            l_run *= alpha;
            if (some) {
#pragma unroll
                for (int c = 0; c < CT; ++c) oacc[c] *= alpha;
            }
            m_run = m_new;
            m_ref = m_new == -INFINITY ? 0.f : m_new;
        }
        uint32_t p[SCORES / 2];
        float psum = 0.f;
#pragma unroll
        for (int e = 0; e < SCORES / 2; ++e) {
            // the difference first: scores of any size
            const f32x2 w = {fast_exp2((s_[2 * e] - m_ref) * a.scale_log2e), fast_exp2((s_[2 * e + 1] - m_ref) * a.scale_log2e)};
            psum += w[0] + w[1];
            p[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(w, bf16x2));
        }
        l_run += psum;
#pragma unroll
        for (int g = 0; g < CT / VGROUP; ++g) {
            if (g + 1 < CT / VGROUP) ask_columns(g + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < VGROUP; ++u) oacc[g * VGROUP + u] = add_rows(v[g & 1][u], p, oacc[g * VGROUP + u]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // ---- the tiles ----
    const int mine = first_tile < tiles ? (tiles - first_tile + stride - 1) / stride : 0;
    // how many rounds the workgroup takes (key group 0 has the most tiles)
    const int rounds = split * KG < tiles ? (tiles - split * KG + stride - 1) / stride : 0;
    own_rows_loaded();
    for (int i = 0; i < (RG == 1 ? mine : rounds); ++i) {
        const int t = first_tile + i * stride;
        wait_for_loads<0>();
        unsigned char *const tile = buffers + i % NB * Tile::BYTES;
        if constexpr (RG > 1) workgroup_barrier();         // (or a wave's tiles are its own)
        auto load_next = [&] {
            if (i + 1 < mine) load_tile(tile_base(t + stride), buffers + (i + 1) % NB * Tile::BYTES);
        };
        if (!LATER || kg % 2 == 0) load_next();
        // (a key group without a tile in the last round computes one that nobody sees)
        compute_tile(t, tile, [&] {
            if (LATER && kg % 2) load_next();
        });
    }
    wait_for_loads<0>();

    // ---- join the key groups, and out: through LDS, 16-byte piece p of query row r at slot p ^ r ----
    const float l = quad_rows_sum(l_run);
    if (quarter == 0) {
        red[wv * LT_ROWS + row] = m_run;
        red[(NW + wv) * LT_ROWS + row] = l;
    }
    __syncthreads();
    float m_all = -INFINITY, l_all = 0.f;
#pragma unroll
    for (int k = 0; k < KG; ++k) m_all = max_no_nan(m_all, red[(k * RG + rg) * LT_ROWS + row]);
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        // (a group has no weights where its sum is 0; one of NaN counts whatever its maximum, which leaves NaN out)
        const float mk = red[(k * RG + rg) * LT_ROWS + row], lk = red[(NW + k * RG + rg) * LT_ROWS + row];
        if (lk != 0.f) l_all += lk * fast_exp2((mk - m_all) * a.scale_log2e);
    }
    float part = l == 0.f ? 0.f : fast_exp2((m_run - m_all) * a.scale_log2e);
    if (a.S == 1) part = l_all == 0.f ? 0.f : part / l_all;
    if (kg == 0 && quarter == 0 && my_row < real_rows) {
        if (a.S == 1) {
            if (a.lse_out) a.lse_out[(size_t)seg * a.M + my_row] = l_all == 0.f ? -INFINITY : m_all * a.scale + logf(l_all);
        } else {
            st_device8(device_span(a.part_ml + ((size_t)seg * a.S + split) * a.M * 2, (uint32_t)a.M * 8u), (uint32_t)my_row * 8u,
                       f32x2{m_all, rounds == 0 ? -1.0f : l_all});                 // (-1: no partial)
        }
    }
    if (a.S > 1 && rounds == 0) return;                    // (nothing was seen: the join does not look at it)
    constexpr int COLS = R / PARTS, PIECES = COLS / 4;
    float *const mine_o = reinterpret_cast<float *>(lds) + wv * LT_ROWS * COLS;
    const float *const all_o = reinterpret_cast<const float *>(lds);
#pragma unroll
    for (int h = 0; h < PARTS; ++h) {
        if (h) __syncthreads();
#pragma unroll
        for (int c = h * CT / PARTS; c < (h + 1) * CT / PARTS; ++c) {
            const int piece = (16 * c - h * COLS) / 4 + quarter;
            *reinterpret_cast<f32x4 *>(mine_o + row * COLS + ((piece ^ row) & (PIECES - 1)) * 4) = oacc[c] * part;
        }
        __syncthreads();
        static_assert(RG * LT_ROWS * PIECES % (NW * 64) == 0, "whole rounds");
#pragma unroll
        for (int n = 0; n < RG * LT_ROWS * PIECES / (NW * 64); ++n) {
            const int i = n * NW * 64 + (int)threadIdx.x;
            const int piece = i % PIECES, rr = i / PIECES, g = rr / LT_ROWS, r = rr % LT_ROWS;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KG; ++k)
                o += *reinterpret_cast<const f32x4 *>(all_o + ((k * RG + g) * LT_ROWS + r) * COLS + ((piece ^ r) & (PIECES - 1)) * 4);
            const int to = block_row0 + rr, col = h * COLS + piece * 4;
            if (to >= real_rows) continue;
            if (a.S == 1) {
                const u32x2 b = {__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[0], o[1]}, bf16x2)),
                                 __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[2], o[3]}, bf16x2))};
                *reinterpret_cast<u32x2 *>(a.out + (((size_t)seg * a.M + to) * R + col) * 2) = b;
            } else {
                st_device16(device_span(a.part_o + ((size_t)seg * a.S + split) * a.M * R, (uint32_t)(a.M * R) * 4u), (uint32_t)(to * R + col) * 4u, o);
            }
        }
    }
}

// The partials are stored past the L2, which the end of a launch would have to write back before the next one begins (16 x 1000 rows, 32
// query rows 19.1 -> 16.1 us, 64 x 1500, 16: 29.5 -> 28.6).  A join in the same launch by the last of a segment's workgroups, which a
// ticket tells, took 2 to 6 us more than this one: a workgroup has to read alone what is read here by 16.
// Partials of a query row joined, a workgroup (two for R = 256 in one) a row: R / 4 threads.  The shares of all partials first, then the
// partials, JOIN_BATCH asked for at a time.
constexpr int JOIN_THREADS = 128, JOIN_BATCH = 8;
template <int R>
__global__ __launch_bounds__(JOIN_THREADS) void latent_join_kernel(LatentArgs a)
{
    constexpr int PER_ROW = R / 4, ROWS = JOIN_THREADS / PER_ROW;
    __shared__ float shares[ROWS][LT_MOST_SPLITS];
    const int sub = (int)threadIdx.x / PER_ROW, lane = lane_id();
    const int seg = (int)blockIdx.y, r = (int)blockIdx.x * ROWS + sub, col = (int)threadIdx.x % PER_ROW * 4;
    const int row = r < a.M ? r : a.M - 1;
    const float *ml = a.part_ml + ((size_t)seg * a.S * a.M + row) * 2;
    const float *po = a.part_o + ((size_t)seg * a.S * a.M + row) * R + col;
    f32x4 v[JOIN_BATCH];
    auto ask = [&](int i0) {                               // (what nobody has written is not looked at)
#pragma unroll
        for (int u = 0; u < JOIN_BATCH; ++u) v[u] = *reinterpret_cast<const f32x4 *>(po + (size_t)(i0 + u < a.S ? i0 + u : a.S - 1) * a.M * R);
    };
    ask(0);
    f32x2 x = {-INFINITY, -1.0f};                          // of partial `lane`; a sum of -1: there is none
    if (lane < a.S) x = *reinterpret_cast<const f32x2 *>(ml + (size_t)lane * a.M * 2);
    int tokens = a.n_new ? a.n_new[seg % a.B] : a.W;
    tokens = tokens < 0 ? 0 : tokens > a.W ? a.W : tokens;
    const bool real = r < tokens * a.Hq;
    const float m = wave_max_f(x[0]);
    const bool none = x[1] < 0.f, weighs = !none && x[1] != 0.f;       // (NaN weighs, whatever its maximum)
    const float wx = weighs ? fast_exp2((x[0] - m) * a.scale_log2e) : 0.f;
    const float l = wave_sum_f(weighs ? wx * x[1] : 0.f);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    if (col / 4 < 64) shares[sub][lane] = none ? -1.0f : wx * inv;     // a row's first wave
    __syncthreads();
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < a.S; i0 += JOIN_BATCH) {
        if (i0) ask(i0);
#pragma unroll
        for (int u = 0; u < JOIN_BATCH; ++u) {
            const float w = i0 + u < a.S ? shares[sub][i0 + u] : -1.0f;
            if (!(w < 0.f)) o += w * v[u];                 // (a share of 0 too: values that are not finite stay)
        }
    }
    if (!real) return;
    const u32x2 b = {__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[0], o[1]}, bf16x2)),
                     __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[2], o[3]}, bf16x2))};
    *reinterpret_cast<u32x2 *>(a.out + (((size_t)seg * a.M + r) * R + col) * 2) = b;
    if (col == 0 && a.lse_out) a.lse_out[(size_t)seg * a.M + r] = l == 0.f ? -INFINITY : m * a.scale + logf(l);
}

}  // namespace ngc

// ============================================================ host side ====

using namespace ngc;

extern "C" size_t ngc_latent_workspace_bytes(const ngc_paged_cache *pc, int32_t W)
{
    if (check_latent(pc) != NGC_OK || W < 1 || W > LATENT_MOST_TOKENS) return 0;
    const ngc_cache c = logical_geometry(pc);
    size_t most = 0;
    const int R = latent_width(pc->D);
    for (int w = 1; w <= W; ++w) {                         // (calls with fewer new tokens may be split more often)
        const int M = w * pc->Hq;
        for (int layers : {1, pc->L}) {
            for (int groups : {1, 4}) {                    // (which of them, and how many splits, is the hint's to say)
                const int nseg = layers * pc->B;
                const size_t bytes = latent_partial_bytes(nseg, latent_most_splits(latent_shape(groups, M), nseg, c.cap, R), M, R);
                most = bytes > most ? bytes : most;
            }
        }
    }
    return scratch_offset(&c) + most;
}

extern "C" int ngc_latent_attn(const ngc_paged_cache *pc, int32_t layer, const int32_t *n_new, int32_t W, const void *q, float scale,
                               int32_t max_len_hint, void *out, float *lse_out, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_latent(pc);
    if (rc) return rc;
    if (!q || !out || !ws || !aligned16(q) || !aligned16(out) || !aligned16(ws)) return NGC_EINVAL;
    if (W < 1 || !(scale > 0.f) || !(scale <= 2.35e38f) || max_len_hint < 0) return NGC_EINVAL;
    if (W > LATENT_MOST_TOKENS) return NGC_EUNSUPPORTED;
    int seg0, nseg;
    rc = paged_layer_range(pc, layer, &seg0, &nseg);
    if (rc) return rc;
    const ngc_cache c = logical_geometry(pc);
    if (ws_bytes < scratch_offset(&c)) return NGC_ENOSPC;
    const int R = latent_width(pc->D), M = W * pc->Hq;
    const int rows = max_len_hint > 0 && max_len_hint < c.cap ? max_len_hint : c.cap;
    int S = 1;
    const LatentShape shape = latent_shape(M, nseg, rows, R, &S);
    // (workgroups that share sequences are fewer than the chip holds, and so are the sequences that the join counts in its grid's y)
    if (!launchable((long long)nseg * shape.blocks, shape.waves * 64)) return NGC_EUNSUPPORTED;
    while (S > 1 && scratch_offset(&c) + latent_partial_bytes(nseg, S, M, R) > ws_bytes) S /= 2;

    LatentArgs a{};
    a.rows = reinterpret_cast<const unsigned char *>(pc->k_pool);
    a.table = pc->table; a.len = pc->len; a.n_new = n_new;
    a.q = reinterpret_cast<const unsigned char *>(q);
    a.out = reinterpret_cast<unsigned char *>(out);
    a.lse_out = lse_out;
    a.part_o = reinterpret_cast<float *>(reinterpret_cast<unsigned char *>(ws) + scratch_offset(&c));
    a.part_ml = a.part_o + (size_t)nseg * S * M * R;
    a.status = reinterpret_cast<int32_t *>(ws);
    a.seg0 = seg0; a.nseg = nseg; a.blocks = shape.blocks; a.S = S; a.M = M; a.W = W; a.Hq = pc->Hq; a.B = pc->B; a.cap = c.cap;
    a.max_pages = pc->max_pages; a.num_pages = pc->num_pages; a.page_shift = __builtin_ctz((unsigned)pc->page_rows);
    a.scale = scale;
    a.scale_log2e = scale * 1.4426950408889634f;
    hipStream_t st = (hipStream_t)stream;
    const void *fn;
    size_t lds;
#define NGC_PICK_LATENT(R_, E_) \
    lds = LT_LDS_KEYS * (R_ + E_) * 2 + (2 * 8 * LT_ROWS + 8) * sizeof(float); \
    fn = shape.groups == 1   ? reinterpret_cast<const void *>(&latent_attn_kernel<R_, E_, 4, 1>) \
                             : reinterpret_cast<const void *>(&latent_attn_kernel<R_, E_, 8, 4>)
    if (R == 512) { NGC_PICK_LATENT(512, 64); }
    else { NGC_PICK_LATENT(256, 32); }
#undef NGC_PICK_LATENT
    if (lds > 64 * 1024) NGC_HIP_CHECK(hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    rc = launch(fn, dim3((unsigned)(nseg * shape.blocks * S)), dim3(shape.waves * 64), lds, st, a);
    if (rc || S == 1) return rc;
    const int rows_a_group = JOIN_THREADS / (R / 4);
    fn = R == 512 ? reinterpret_cast<const void *>(&latent_join_kernel<512>) : reinterpret_cast<const void *>(&latent_join_kernel<256>);
    return launch(fn, dim3((unsigned)((M + rows_a_group - 1) / rows_a_group), (unsigned)nseg), dim3(JOIN_THREADS), 0, st, a);
}
