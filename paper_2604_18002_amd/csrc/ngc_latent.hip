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
// S^T = C Q^T and O^T = C^T P by matrix instructions, 32x32x16 for 32 query rows a wave and 16x16x32 for 16: one query row
// per lane % 32 (16), so all soft-max state is lane local; one pass over the rows with a running maximum and sum.  A tile of
// 32 rows is contiguous in a page and goes from memory straight into LDS, once: the first product reads its rows, the second
// one the same rows transposed.  Queries and output stay in registers (32 rows: 144 and 256 of the 512 of a lane).
//
// A workgroup's 4 waves are RG row groups x 4 / RG key groups: waves of one key group share tiles, the key groups take
// tiles in turn and are joined in LDS at the end.  Few sequences are shared by S workgroups, whose partials a second launch
// joins.
//
// P is rounded to bf16 for the second product (2^-9 of an entry at most), as the output is: it is the operand of the
// product that brings the latent vectors to the heads' values.  Sums and soft-max state are fp32.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ngc.h"
#include "ngc_device.h"
#include "ngc_latent.h"
#include "ngc_workspace.h"

namespace ngc {

constexpr int LT_WAVES = 4;
constexpr int LT_KEYS = 32;                 // rows of a tile

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

// Where things are in a tile of 32 rows in LDS: the latent parts, 16-byte piece p of row r at slot p ^ swizzle(r), then the rotary
// parts.
template <int R, int E>
struct LatentTile {
    static constexpr int ROW = (R + E) * 2, LAT = R * 2, ROT = E * 2;
    static constexpr int LAT_BYTES = LT_KEYS * LAT, BYTES = LT_KEYS * ROW;
    static constexpr int LAT_PIECES = LAT / 16, ROT_PIECES = ROT / 16;
    static constexpr int LAT_ROWS = 64 / LAT_PIECES, ROT_ROWS = 64 / ROT_PIECES;         // rows a wave-wide load brings
    static constexpr int LAT_LOADS = LT_KEYS / LAT_ROWS, ROT_LOADS = LT_KEYS / ROT_ROWS;
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

// A wave's matrix tiles, for 32 and for 16 query rows.  `row`: of the lane.  A score register e of a lane is the score of key
// key_of(e); eight consecutive ones are an operand of the second product.
template <int RT>
struct LatentMath;
template <>
struct LatentMath<32> {
    typedef f32x16 Acc;
    static constexpr int ROWS = 32, CHUNK = 16, KEYS = 32, COLS = 32, SCORES = 16, STEPS = 2;      // of 16 keys
    __device__ static __forceinline__ int row(int lane) { return lane & 31; }
    __device__ static __forceinline__ int part(int lane) { return lane >> 5; }
    __device__ static __forceinline__ int key_of(int e, int part) { return 8 * (e / 4) + 4 * part + e % 4; }
    __device__ static __forceinline__ Acc product(bf16x8 x, bf16x8 y, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0); }
    // first row and column of what a lane names in a transposing read: for keys 16 step + 8 g .. of columns 32 c ..
    __device__ static __forceinline__ int read_row(int lane) { return 4 * (lane >> 5) + (lane & 15) / 4; }
    __device__ static __forceinline__ int read_col(int lane) { return (lane & 16) + 4 * (lane & 3); }
    static constexpr int step_rows(int step, int g) { return 16 * step + 8 * g; }
    __device__ static __forceinline__ float top(float v) { return half_rows_max(v); }
    __device__ static __forceinline__ float sum(float v) { return half_rows_sum(v); }
    // registers 4 q .. 4 q + 3 of accumulator c hold columns col(c, q) .. + 3
    static constexpr int QUADS = 4;
    __device__ static __forceinline__ int col(int c, int q, int part) { return 32 * c + 8 * q + 4 * part; }
};
template <>
struct LatentMath<16> {
    typedef f32x4 Acc;
    static constexpr int ROWS = 16, CHUNK = 32, KEYS = 16, COLS = 16, SCORES = 8, STEPS = 1;       // of 32 keys
    __device__ static __forceinline__ int row(int lane) { return lane & 15; }
    __device__ static __forceinline__ int part(int lane) { return lane >> 4; }
    __device__ static __forceinline__ int key_of(int e, int part) { return 16 * (e / 4) + 4 * part + e % 4; }
    __device__ static __forceinline__ Acc product(bf16x8 x, bf16x8 y, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); }
    __device__ static __forceinline__ int read_row(int lane) { return 4 * (lane >> 4) + (lane & 15) / 4; }
    __device__ static __forceinline__ int read_col(int lane) { return 4 * (lane & 3); }
    static constexpr int step_rows(int, int g) { return 16 * g; }
    __device__ static __forceinline__ float top(float v) { return quad_rows_max(v); }
    __device__ static __forceinline__ float sum(float v) { return quad_rows_sum(v); }
    static constexpr int QUADS = 1;
    __device__ static __forceinline__ int col(int c, int, int part) { return 16 * c + 4 * part; }
};

// For s_waitcnt: at most `n` loads are still on their way, and no LDS operation.
constexpr int wait_loads(int n) { return 0x0070 | (n & 15) | (n >> 4 << 14); }

// 2^8: the reference of the exponents moves only when a maximum has outgrown it by that.
constexpr float LT_LAZY = 8.0f;

// Waves per SIMD (by registers: queries and output are (2 R + E) RT / 128 of a lane's), and tiles in LDS: four of R = 512 fill a CU's.
constexpr int latent_waves(int R, int RT) { return R == 256 && RT == 16 ? 2 : 1; }
constexpr int latent_slots(int R, int RT) { return R == 256 && RT == 32 ? 8 : 4; }

// The accumulators times alpha, where they are: left to itself the compiler keeps a second copy of them for the branch around this.
// (A matrix instruction's result may be read 18 cycles after its issue at the earliest.)
template <int CT, class Acc>
__device__ __forceinline__ void scale_all(Acc (&o)[CT], float alpha)
{
    if constexpr (CT * sizeof(Acc) <= 512) {
#pragma unroll
        for (int c = 0; c < CT; ++c) o[c] *= alpha;
    } else {
        __asm__ volatile("s_nop 15\n\ts_nop 7");
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < (int)(sizeof(Acc) / 4); ++e) {
                float x;
                __asm__ volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1"
                                 : "+a"(o[c][e]), "=&v"(x) : "v"(alpha));
            }
        __asm__ volatile("s_nop 3");
    }
}

// RT query rows a wave, RG row groups.
template <int R, int E, int RT, int RG>
__global__ __launch_bounds__(LT_WAVES * 64) __attribute__((amdgpu_waves_per_eu(latent_waves(R, RT))))
void latent_attn_kernel(LatentArgs a)
{
    using Tile = LatentTile<R, E>;
    using Math = LatentMath<RT>;
    constexpr int KG = LT_WAVES / RG;
    constexpr int SLOTS = latent_slots(R, RT);             // tiles in LDS
    constexpr int NB = SLOTS / KG;                         // buffers of a key group
    constexpr int CHUNKS = (R + E) / Math::CHUNK;          // of the first product
    constexpr int KTILES = LT_KEYS / Math::KEYS;           // score tiles per tile of rows
    constexpr int CT = R / Math::COLS;                     // column tiles of the second product
    constexpr int LAT_LOADS = (Tile::LAT_LOADS + RG - 1) / RG, ROT_LOADS = (Tile::ROT_LOADS + RG - 1) / RG;      // of a wave, per tile
    constexpr int LOADS = LAT_LOADS + ROT_LOADS;
    constexpr int HALVES = LT_WAVES * RT * R * 4 > SLOTS * Tile::BYTES ? 2 : 1;          // the output goes through LDS in so many parts
    static_assert(LT_WAVES * RT * R * 4 / HALVES <= SLOTS * Tile::BYTES, "a part of the output fits");

    extern __shared__ __align__(256) unsigned char lds[];
    float *const red = reinterpret_cast<float *>(lds + SLOTS * Tile::BYTES);             // [2][waves][RT]

    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    const int rg = wv % RG, kg = wv / RG;
    const int row = Math::row(lane), part = Math::part(lane);
    // the row blocks of a sequence follow one another on one XCD
    int seg = (int)blockIdx.x, block = 0;
    if (a.blocks > 1) {
        const int first = (int)(blockIdx.x / (8u * (unsigned)a.blocks)) * 8, at = (int)blockIdx.x - first * a.blocks;
        const int here = a.nseg - first < 8 ? a.nseg - first : 8;
        block = at / here;
        seg = first + at - block * here;
    }
    const int split = (int)blockIdx.y;
    const LatentSegment s(a, seg, threadIdx.x == 0 && split == 0 && block == 0);
    const int real_rows = s.w * a.Hq;                      // query rows of the sequence
    const int block_row0 = block * RG * RT;
    if (block_row0 >= real_rows) return;
    const int my_row = block_row0 + rg * RT + row;
    const int q_row = my_row < real_rows ? my_row : real_rows - 1;

    bf16x8 qop[CHUNKS];
    {
        const unsigned char *q = a.q + ((size_t)seg * a.M + q_row) * Tile::ROW + part * 16;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) qop[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(q + c * Math::CHUNK * 2));
    }
    const int limit = s.limit(a, q_row);
    // rows below `all` are seen by every query row of the workgroup, rows from `end` on by none
    const int all = s.limit(a, block_row0);
    const int last_row = block_row0 + RG * RT - 1;
    const int end = s.limit(a, last_row < real_rows ? last_row : real_rows - 1);
    const int tiles = (end + LT_KEYS - 1) / LT_KEYS;
    const int32_t *tab = a.table + (size_t)(a.seg0 + seg) * a.max_pages;
    const int stride = a.S * KG, first_tile = split * KG + kg;

    auto tile_base = [&](int t) -> const unsigned char * {
        const int r0 = t * LT_KEYS;
        int page = constant_word(tab + (r0 >> a.page_shift));
        page = (page < 0 || page >= a.num_pages) ? 0 : page;          // never leave the pool
        return a.rows + (((size_t)page << a.page_shift) + (r0 & ((1 << a.page_shift) - 1))) * Tile::ROW;
    };
    unsigned char *const buffers = lds + kg * NB * Tile::BYTES;
    auto load_tile = [&](int t, unsigned char *to) {
        const unsigned char *base = tile_base(t);
        int lane_ = lane;
        __asm__ volatile("" : "+v"(lane_));                // (offsets are made where they are used, not kept over the loop)
        // the swizzle is linear in a row's bits: a lane's part of it, and the load's
        const int lrow = Tile::LAT_ROWS == 1 ? 0 : lane_ / Tile::LAT_PIECES, lp = lane_ % Tile::LAT_PIECES ^ Tile::swizzle(lrow);
        const uint32_t lat = (uint32_t)(lrow * Tile::ROW);
#pragma unroll
        for (int i = 0; i < LAT_LOADS; ++i) {
            const int r0 = (i * RG + rg) * Tile::LAT_ROWS;
            load_to_lds16(base + r0 * Tile::ROW + (lat + (uint32_t)(lp ^ Tile::swizzle(r0)) * 16), to + r0 * Tile::LAT);
        }
        const int rrow = lane_ / Tile::ROT_PIECES, rp = lane_ % Tile::ROT_PIECES ^ Tile::rot_swizzle(rrow);
        const uint32_t rot = (uint32_t)(rrow * Tile::ROW);
#pragma unroll
        for (int i = 0; i < ROT_LOADS; ++i) {
            const int r0 = (i * RG + rg) % Tile::ROT_LOADS * Tile::ROT_ROWS;             // (what is left over loads a part again)
            load_to_lds16(base + r0 * Tile::ROW + Tile::LAT + (rot + (uint32_t)(rp ^ Tile::rot_swizzle(r0)) * 16), to + Tile::LAT_BYTES + r0 * Tile::ROT);
        }
    };

    typename Math::Acc oacc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int e = 0; e < Math::QUADS * 4; ++e) oacc[c][e] = 0.f;
    float m_run = -INFINITY, m_ref = 0.f, l_run = 0.f;     // m_ref: m_run, or 0 as long as nothing has been seen

    // Where this lane's operands are in a tile.  Pieces 16 apart are 256 bytes apart whatever the swizzle, rows 16 apart have the same one,
    // those of rows 8 apart differ by 3, and a tile begins at a multiple of 256: the other offsets differ from the first one's by bits.
    constexpr int PIECES_A_CHUNK = Math::CHUNK / 8, LAT_CHUNKS = R / Math::CHUNK, LAT_VARIANTS = 16 / PIECES_A_CHUNK;
    constexpr int COL_VARIANTS = 128 / Math::COLS;
    static_assert(Tile::BYTES % 256 == 0 && Tile::LAT % 256 == 0, "offsets differ by bits");
    const uint32_t lat0 = Tile::piece(row, part), rot0 = Tile::piece(row, Tile::LAT_PIECES + part);
    const uint32_t col0 = Tile::piece(Math::read_row(lane), Math::read_col(lane) / 8) + (uint32_t)(Math::read_col(lane) % 8) * 2;

    auto compute_tile = [&](int t, const unsigned char *tile) {
        uint32_t at_lat = lat0, at_rot = rot0, at_col = col0;
        __asm__ volatile("" : "+v"(at_lat), "+v"(at_rot), "+v"(at_col));
        const unsigned char __attribute__((address_space(3))) *const tile3 = (const unsigned char __attribute__((address_space(3))) *)tile;
        const uint32_t tile_at = (uint32_t)(uintptr_t)tile3;
        auto row_piece = [&](int c, int k) {               // chunk c of the rows of key tile k
            const uint32_t at = c < LAT_CHUNKS ? ((tile_at + at_lat) ^ (uint32_t)(c % LAT_VARIANTS * PIECES_A_CHUNK * 16)) + (uint32_t)(c / LAT_VARIANTS * 256 + k * Math::KEYS * Tile::LAT)
                                               : ((tile_at + at_rot) ^ (uint32_t)((c - LAT_CHUNKS) * PIECES_A_CHUNK * 16)) + (uint32_t)(k * Math::KEYS * Tile::ROT);
            return *(const u32x4 __attribute__((address_space(3))) *)(uintptr_t)at;
        };
        // keys 16 st + 8 g .. (of 32 query rows), 16 g .. (of 16), of column tile c
        auto transposed = [&](int st, int g, int c) {
            const uint32_t at = ((tile_at + at_col) ^ (uint32_t)(c % COL_VARIANTS * Math::COLS * 2 ^ (RT == 32 ? g * 48 : 0))) +
                                (uint32_t)(c / COL_VARIANTS * 256 + (RT == 32 ? st * 16 + g * 8 : g * 16) * Tile::LAT);
            return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)at));
        };
        const int key0 = t * LT_KEYS;
        const bool edge = key0 + LT_KEYS > all;            // not every query row of the workgroup sees all of the tile's rows
        typename Math::Acc sc[KTILES];
#pragma unroll
        for (int k = 0; k < KTILES; ++k)
#pragma unroll
            for (int e = 0; e < Math::QUADS * 4; ++e) sc[k][e] = 0.f;
        // GROUP chunks' rows are asked for while the products of those before run
        constexpr int GROUP = CHUNKS % 4 == 0 ? 4 : 3;
        static_assert(CHUNKS % GROUP == 0, "whole groups");
        u32x4 x[2][GROUP][KTILES];
        auto ask_rows = [&](int g0, u32x4 (&to)[GROUP][KTILES]) {
#pragma unroll
            for (int u = 0; u < GROUP; ++u)
#pragma unroll
                for (int k = 0; k < KTILES; ++k) to[u][k] = row_piece(g0 + u, k);
        };
        ask_rows(0, x[0]);
#pragma unroll
        for (int g = 0; g < CHUNKS / GROUP; ++g) {
            if (g + 1 < CHUNKS / GROUP) ask_rows((g + 1) * GROUP, x[(g + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < GROUP; ++u)
#pragma unroll
                for (int k = 0; k < KTILES; ++k) sc[k] = Math::product(__builtin_bit_cast(bf16x8, x[g & 1][u][k]), qop[g * GROUP + u], sc[k]);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the first columns, while the weights are made
        constexpr int VGROUP = RT == 32 ? 2 : 4;
        u32x2 v[2][VGROUP][Math::STEPS][2];
        auto ask_columns = [&](int c0, u32x2 (&to)[VGROUP][Math::STEPS][2]) {
#pragma unroll
            for (int u = 0; u < VGROUP; ++u)
#pragma unroll
                for (int st = 0; st < Math::STEPS; ++st)
#pragma unroll
                    for (int g = 0; g < 2; ++g) to[u][st][g] = transposed(st, g, c0 + u);
        };
        ask_columns(0, v[0]);
        __builtin_amdgcn_sched_barrier(0);
        float s_[Math::SCORES];
#pragma unroll
        for (int e = 0; e < Math::SCORES; ++e) s_[e] = KTILES == 1 ? sc[0][e % 16] : sc[e / 4 % KTILES][e % 4];
        if (edge) {
#pragma unroll
            for (int e = 0; e < Math::SCORES; ++e) s_[e] = key0 + Math::key_of(e, part) < limit ? s_[e] : -INFINITY;
        }
        float tmx = s_[0];
#pragma unroll
        for (int e = 1; e < Math::SCORES; ++e) tmx = max_no_nan(tmx, s_[e]);
        tmx = Math::top(tmx);
        const bool outgrown = (tmx - m_run) * a.scale_log2e > LT_LAZY;     // of each row by itself: its results do not depend on its neighbours'
        if (__ballot(outgrown)) {
            const bool some = __ballot(m_run > -INFINITY) != 0;       // (nothing to scale on the first tile)
            const float m_new = outgrown ? tmx : m_run;
            const float alpha = m_new == m_run ? 1.0f : fast_exp2((m_run - m_new) * a.scale_log2e);
            l_run *= alpha;
            if (some) scale_all(oacc, alpha);
            m_run = m_new;
            m_ref = m_new == -INFINITY ? 0.f : m_new;
        }
        uint32_t p[Math::SCORES / 2];
        float psum = 0.f;
#pragma unroll
        for (int e = 0; e < Math::SCORES / 2; ++e) {
            // the difference first: scores of any size
            const f32x2 w = {fast_exp2((s_[2 * e] - m_ref) * a.scale_log2e), fast_exp2((s_[2 * e + 1] - m_ref) * a.scale_log2e)};
            psum += w[0] + w[1];
            p[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(w, bf16x2));
        }
        l_run += psum;
        bool odd = false;
#pragma unroll
        for (int g = 0; g < CT / VGROUP; ++g) {
            if (g + 1 < CT / VGROUP) ask_columns((g + 1) * VGROUP, v[(g + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
            if (edge) {
#pragma unroll
                for (int u = 0; u < VGROUP; ++u)
#pragma unroll
                    for (int st = 0; st < Math::STEPS; ++st) odd |= take_out_odd(v[g & 1][u][st][0]) | take_out_odd(v[g & 1][u][st][1]);
            }
#pragma unroll
            for (int st = 0; st < Math::STEPS; ++st)
#pragma unroll
                for (int u = 0; u < VGROUP; ++u) {
                    const u32x2 lo = v[g & 1][u][st][0], hi = v[g & 1][u][st][1];
                    const bf16x8 vt = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
                    const bf16x8 w = __builtin_bit_cast(bf16x8, u32x4{p[4 * st], p[4 * st + 1], p[4 * st + 2], p[4 * st + 3]});
                    oacc[g * VGROUP + u] = Math::product(vt, w, oacc[g * VGROUP + u]);
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (__ballot(odd)) {
            // the query rows that see one of the rows with such values, and no others, become NaN
            for (int k = 0; k < LT_KEYS && key0 + k < end; ++k) {
                bool any = false;
#pragma unroll
                for (int i = 0; i < Tile::LAT; i += 512) any |= has_odd(*reinterpret_cast<const u32x2 *>(tile + k * Tile::LAT + i + lane * 8));
                if (__ballot(any) && key0 + k < limit) l_run = NAN;
            }
        }
    };

    // ---- the tiles ----
    constexpr int WAIT_LDS = 0xC07F;                       // lgkmcnt(0)
    const int mine = first_tile < tiles ? (tiles - first_tile + stride - 1) / stride : 0;
    // how many rounds the workgroup takes (key group 0 has the most tiles)
    const int rounds = split * KG < tiles ? (tiles - split * KG + stride - 1) / stride : 0;
    if constexpr (NB == 1) {
        static_assert(RG == 1, "no barrier");
        // a wave's tiles are its own
        for (int i = 0; i < mine; ++i) {
            load_tile(first_tile + i * stride, buffers);
            __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0)
            __asm__ volatile("" ::: "memory");
            compute_tile(first_tile + i * stride, buffers);
            __builtin_amdgcn_s_waitcnt(WAIT_LDS);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        int issued = 0;
        for (; issued < NB - 1 && issued < mine; ++issued) load_tile(first_tile + issued * stride, buffers + issued * Tile::BYTES);
        for (int i = 0; i < rounds; ++i) {
            const int ahead = issued - i - 1;              // tiles on their way behind this one
            // the tile has arrived, and what this wave has read
            if (ahead == NB - 2 && i < mine) __builtin_amdgcn_s_waitcnt(wait_loads((NB - 2) * LOADS));
            else __builtin_amdgcn_s_waitcnt(wait_loads(0));
            __asm__ volatile("" ::: "memory");
            if constexpr (RG > 1) __builtin_amdgcn_s_barrier();      // (or a wave's tiles are its own)
            __asm__ volatile("" ::: "memory");
            if (issued < mine) {
                load_tile(first_tile + issued * stride, buffers + issued % NB * Tile::BYTES);
                ++issued;
            }
            // (a key group without a tile in the last round computes one that nobody sees)
            compute_tile(first_tile + i * stride, buffers + i % NB * Tile::BYTES);
        }
    }

    // ---- join the key groups, and out: through LDS, 16-byte piece p of query row r at slot p ^ r ----
    const float l = Math::sum(l_run);
    if (part == 0) {
        red[wv * RT + row] = m_run;
        red[(LT_WAVES + wv) * RT + row] = l;
    }
    __syncthreads();
    float m_all = -INFINITY, l_all = 0.f;
#pragma unroll
    for (int k = 0; k < KG; ++k) m_all = max_no_nan(m_all, red[(k * RG + rg) * RT + row]);
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        const float mk = red[(k * RG + rg) * RT + row];
        if (mk > -INFINITY || mk != mk) l_all += red[(LT_WAVES + k * RG + rg) * RT + row] * fast_exp2((mk - m_all) * a.scale_log2e);
    }
    float share = m_run == -INFINITY ? 0.f : fast_exp2((m_run - m_all) * a.scale_log2e);
    if (a.S == 1) share = l_all == 0.f ? 0.f : share / l_all;
    if (kg == 0 && part == 0 && my_row < real_rows) {
        if (a.S == 1) {
            if (a.lse_out) a.lse_out[(size_t)seg * a.M + my_row] = l_all == 0.f ? -INFINITY : m_all * a.scale + logf(l_all);
        } else {
            float *ml = a.part_ml + (((size_t)seg * a.S + split) * a.M + my_row) * 2;
            ml[0] = m_all;
            ml[1] = l_all;
        }
    }
    if (a.S > 1 && rounds == 0) return;                    // (nothing was seen: the join does not look at it)
    constexpr int COLS = R / HALVES, PIECES = COLS / 4;
    float *const mine_o = reinterpret_cast<float *>(lds) + wv * RT * COLS;
    const float *const all_o = reinterpret_cast<const float *>(lds);
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        if (h) __syncthreads();
#pragma unroll
        for (int c = h * CT / HALVES; c < (h + 1) * CT / HALVES; ++c)
#pragma unroll
            for (int qd = 0; qd < Math::QUADS; ++qd) {
                const int piece = (Math::col(c, qd, part) - h * COLS) / 4;
                f32x4 o = {oacc[c][4 * qd], oacc[c][4 * qd + 1], oacc[c][4 * qd + 2], oacc[c][4 * qd + 3]};
                o = share == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * share;
                *reinterpret_cast<f32x4 *>(mine_o + row * COLS + ((piece ^ row) & (PIECES - 1)) * 4) = o;
            }
        __syncthreads();
        for (int i = threadIdx.x; i < RG * RT * PIECES; i += LT_WAVES * 64) {
            const int piece = i % PIECES, rr = i / PIECES, g = rr / RT, r = rr % RT;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KG; ++k)
                o += *reinterpret_cast<const f32x4 *>(all_o + ((k * RG + g) * RT + r) * COLS + ((piece ^ r) & (PIECES - 1)) * 4);
            const int to = block_row0 + rr, col = h * COLS + piece * 4;
            if (to >= real_rows) continue;
            if (a.S == 1) {
                const u32x2 b = {__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[0], o[1]}, bf16x2)),
                                 __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[2], o[3]}, bf16x2))};
                *reinterpret_cast<u32x2 *>(a.out + (((size_t)seg * a.M + to) * R + col) * 2) = b;
            } else {
                *reinterpret_cast<f32x4 *>(a.part_o + (((size_t)seg * a.S + split) * a.M + to) * R + col) = o;
            }
        }
    }
}

// Partials of a query row joined, a workgroup (two for R = 256 in one) a row: R / 4 threads.  The shares of all partials first, then the
// partials, JOIN_BATCH asked for at a time.
constexpr int JOIN_THREADS = 128, JOIN_BATCH = 8;
constexpr int LT_MOST_SPLITS = 128;
template <int R>
__global__ __launch_bounds__(JOIN_THREADS) void latent_join_kernel(LatentArgs a)
{
    constexpr int PER_ROW = R / 4, ROWS = JOIN_THREADS / PER_ROW;
    __shared__ float shares[ROWS][LT_MOST_SPLITS + JOIN_BATCH];
    const int sub = (int)threadIdx.x / PER_ROW, lane = lane_id();
    const int seg = (int)blockIdx.y, r = (int)blockIdx.x * ROWS + sub, col = (int)threadIdx.x % PER_ROW * 4;
    const LatentSegment s(a, seg, false);
    if ((int)blockIdx.x * ROWS >= s.w * a.Hq) return;
    const bool real = r < s.w * a.Hq;
    const int row = real ? r : 0;
    const float *ml = a.part_ml + ((size_t)seg * a.S * a.M + row) * 2;
    // of partials lane and 64 + lane
    f32x2 x = {-INFINITY, 0.f}, y = {-INFINITY, 0.f};
    if (lane < a.S) x = *reinterpret_cast<const f32x2 *>(ml + (size_t)lane * a.M * 2);
    if (lane + 64 < a.S) y = *reinterpret_cast<const f32x2 *>(ml + (size_t)(lane + 64) * a.M * 2);
    const float m = wave_max_f(fmaxf(x[0], y[0]));
    const float wx = x[0] == -INFINITY ? 0.f : fast_exp2((x[0] - m) * a.scale_log2e), wy = y[0] == -INFINITY ? 0.f : fast_exp2((y[0] - m) * a.scale_log2e);
    const float l = wave_sum_f((wx == 0.f ? 0.f : wx * x[1]) + (wy == 0.f ? 0.f : wy * y[1]));
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    if (col / 4 < 64) {                                    // a row's first wave
        shares[sub][lane] = wx * inv;
        shares[sub][lane + 64] = wy * inv;
        if (lane < JOIN_BATCH) shares[sub][LT_MOST_SPLITS + lane] = 0.f;
    }
    __syncthreads();
    const float *po = a.part_o + ((size_t)seg * a.S * a.M + row) * R + col;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < a.S; i0 += JOIN_BATCH) {
        f32x4 v[JOIN_BATCH];
#pragma unroll
        for (int u = 0; u < JOIN_BATCH; ++u) {             // (one without a share may not have been written)
            const int i = i0 + u < a.S ? i0 + u : a.S - 1;
            v[u] = *reinterpret_cast<const f32x4 *>(po + (size_t)i * a.M * R);
        }
#pragma unroll
        for (int u = 0; u < JOIN_BATCH; ++u) {
            const float w = i0 + u < a.S ? shares[sub][i0 + u] : 0.f;
            if (w != 0.f) o += w * v[u];
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

namespace {

// How M query rows are dealt to waves and workgroups.
struct LatentShape {
    int rows, groups, blocks, key_groups;
};
LatentShape latent_shape(int M)
{
    LatentShape s;
    s.rows = M <= 16 ? 16 : 32;
    s.groups = M <= 32 ? 1 : M <= 64 ? 2 : 4;
    s.blocks = (M + s.rows * s.groups - 1) / (s.rows * s.groups);
    s.key_groups = LT_WAVES / s.groups;
    return s;
}

// How many workgroups share a sequence's rows.
int latent_splits(const LatentShape &s, int nseg, int rows)
{
    const long long groups = (long long)nseg * s.blocks;
    const int rounds = (rows + LT_KEYS * s.key_groups - 1) / (LT_KEYS * s.key_groups);
    long long S = 256 / groups;
    if (S > rounds / 2) S = rounds / 2;
    if (S > LT_MOST_SPLITS) S = LT_MOST_SPLITS;
    return S < 1 ? 1 : (int)S;
}

size_t latent_partial_bytes(int nseg, int S, int M, int R) { return S == 1 ? 0 : (size_t)nseg * S * M * (R + 2) * sizeof(float); }

}  // namespace

extern "C" size_t ngc_latent_workspace_bytes(const ngc_paged_cache *pc, int32_t W)
{
    if (check_latent(pc) != NGC_OK || W < 1 || W > LATENT_MOST_TOKENS) return 0;
    const ngc_cache c = logical_geometry(pc);
    size_t most = 0;
    const int R = latent_width(pc->D);
    for (int w = 1; w <= W; ++w) {                         // (calls with fewer new tokens may be split more often)
        const int M = w * pc->Hq;
        for (int layers : {1, pc->L}) {
            const int nseg = layers * pc->B;
            const size_t bytes = latent_partial_bytes(nseg, latent_splits(latent_shape(M), nseg, c.cap), M, R);
            most = bytes > most ? bytes : most;
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
    const LatentShape shape = latent_shape(M);
    if ((long long)nseg * shape.blocks > 0x7FFFFFFFLL || nseg > 65535) return NGC_EUNSUPPORTED;
    const int rows = max_len_hint > 0 && max_len_hint < c.cap ? max_len_hint : c.cap;
    int S = latent_splits(shape, nseg, rows);
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
    lds = latent_slots(R_, shape.rows) * LatentTile<R_, E_>::BYTES + 2 * LT_WAVES * 32 * sizeof(float); \
    fn = shape.rows == 16   ? reinterpret_cast<const void *>(&latent_attn_kernel<R_, E_, 16, 1>) \
       : shape.groups == 1  ? reinterpret_cast<const void *>(&latent_attn_kernel<R_, E_, 32, 1>) \
       : shape.groups == 2  ? reinterpret_cast<const void *>(&latent_attn_kernel<R_, E_, 32, 2>) \
                            : reinterpret_cast<const void *>(&latent_attn_kernel<R_, E_, 32, 4>)
    if (R == 512) { NGC_PICK_LATENT(512, 64); }
    else { NGC_PICK_LATENT(256, 32); }
#undef NGC_PICK_LATENT
    if (lds > 64 * 1024) NGC_HIP_CHECK(hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    rc = launch(fn, dim3((unsigned)(nseg * shape.blocks), (unsigned)S), dim3(LT_WAVES * 64), lds, st, a);
    if (rc || S == 1) return rc;
    const int rows_a_group = JOIN_THREADS / (R / 4);
    fn = R == 512 ? reinterpret_cast<const void *>(&latent_join_kernel<512>) : reinterpret_cast<const void *>(&latent_join_kernel<256>);
    return launch(fn, dim3((unsigned)((M + rows_a_group - 1) / rows_a_group), (unsigned)nseg), dim3(JOIN_THREADS), 0, st, a);
}
