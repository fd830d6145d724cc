// Replay attention of latent layers, expanded form, forward and backward, on gfx950.
//
// All T positions of a trajectory at once.  Head h has keys k_j = [its own part, D values | rotary part, E = D / 2 values that
// all heads share] and values v_j of D; query i sees key j iff j <= i < death_j:
//
//     s_ij = scale <q_i, k_j>,  P_ij = exp(s_ij - lse_i),  o_i = sum_j P_ij v_j.
//
// With g_i the gradient that arrives at o_i and delta_i = <g_i, o_i>:
//
//     dv_j = sum_i P_ij g_i,   dS_ij = P_ij (<g_i, v_j> - delta_i),   dq_i = scale sum_j dS_ij k_j,   dk_j = scale sum_i dS_ij q_i,
//
// and the rotary part's gradient is the sum of the heads'.
//
// Kernels around the same units of 32 x 32 pairs by 32x32x16 matrix instructions, two workgroups a CU:
//   forward      four waves of 32 queries each walk tiles of two units of 32 keys: S^T = K Q^T, O^T += V^T P.
//   backward, q  the same walk, S^T and (V G^T) again, dQ^T += K^T dS; leaves delta and lse as the next one wants them.
//   backward, kv two waves for 32 keys (two such pairs in a workgroup) walk units of 32 queries: the first makes S = Q K^T, P and
//                dV^T += G^T P, the second, a unit behind, G V^T, dS of it and of P, and dK^T += Q^T dS: 20 products of 32 x 32 x 16 each
//                (D = 128), and the sums of 32 keys, 160 registers of a lane, in two waves.  P goes from one to the other in fp32.
// In each the pairs stand in registers as the first products leave them, which is the order the second products' operand
// needs if the rows of the other operand are read transposed in the same order: nothing crosses lanes but a row's maximum.
// The two backward kernels form S twice (7 products in place of 5), so that every sum has one owner: no atomics, the same
// bits again.
//
// 32 keys that are dead for all of a workgroup's queries are never loaded: pages are evicted whole.  Tiles of keys are made of two
// such units that live, wherever they are; keys are given to workgroups in the order of their ends, so that a workgroup's live about as
// long.  Pairs are masked one by one only on the diagonal, behind the sequence's end, or where keys die midway.
//
// What bounds it.  2 (2 D + E) flops a pair forward, 2 (3 (D + E) + 2 D) + 2 (2 D + E) backward (D = 128: 640 and 1664 with what is formed
// twice left out) on 16-bit inputs: the products, for more than some hundred positions.  Measured, 16 heads of 128: 8192 positions
// without evictions 920 TFLOP/s forward (371 us; two of them 945) and 670 to 690 backward, where a large product of matrices reaches 1230;
// 2 x 3000 to 3850 positions with evictions every 512, 126 us forward, 186 us the queries' and 292 us the keys' gradients.  A step of 32 x
// 32 pairs is 640 clocks of products and some 700 of vector work forward, and two waves overlap little of them: the matrix units are
// busy 45 % of the time without evictions.  With evictions a workgroup has few tiles and its first one, 2.5 us, and the look at the ends, 1.5, count.
//   Registers decide: two waves a SIMD have 256 each, and one more copy of the sums (a branch around a unit makes the compiler keep
// one) or offsets kept for every read (they differ in a bit: made where they are used) went to scratch, whose loads wait behind every
// tile on its way: the queries' gradient 245 us with 23 such registers, 190 without.
//   Not kept: one wave for 32 keys with all sums (one wave a SIMD, 380 us, nobody covers its waits: 320 with two waves); four pairs of
// waves a workgroup (317 us with evictions, keys that live for different times; 5 % faster without); units of keys one by one in
// a ring of four (forward 167 us for 137: a barrier and the offsets for every 32 keys); loads spread between the products.
//
// P and dS are rounded to bf16 (half a step: 2^-8 of an entry at most) for their second products, whose other operand is bf16 as it comes
// (in two parts, half as many products again), as outputs and gradients are; delta is of the output as it is stored, which is what a
// caller has kept.  Sums, maxima, lse and delta are fp32.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ngc.h"
#include "ngc_device.h"
#include "ngc_latent.h"
#include "ngc_workspace.h"

namespace ngc {

constexpr int LR_WAVES = 4;
constexpr int LR_OWN = 32;                   // queries (keys) of a wave
constexpr int LR_BLOCK = LR_WAVES * LR_OWN;  // of a workgroup
constexpr int LR_STEP = 32;                  // keys (queries) of a unit: a step of the math
constexpr int LR_MOST_POSITIONS = 64 * 64 * LR_STEP;       // a bit of a lane's words per LR_STEP keys
constexpr int KV_GROUPS = 2;                 // units of keys of a workgroup of the keys' gradients
constexpr int KV_BLOCK = KV_GROUPS * LR_OWN;
constexpr int kv_slots(int D) { return D == 128 ? 3 : 6; }     // units of queries in LDS, for two workgroups a CU
constexpr float LR_LAZY = 8.0f;              // the reference of the exponents moves when a maximum has outgrown it by 2^8
// Exponents are score * scale - reference in one operation, the reference rounded.  Its rounding is the same for all keys, and lse is of the
// rounded one; but it would reach 2^7, where weights overflow, at references of 2^31, and count where they move.  From this one on (there half a
// step is 2^-12, and what has been added up before such a move weighs 2^-8 at most) the scores' difference comes first.
constexpr float LR_FAR = 4096.0f;

struct LatentReplayArgs {
    const unsigned char *q;                  // bf16 [B][T][H][D + E]
    const unsigned char *kv;                 // bf16 [B][T][H][2 D]: keys, then values
    const unsigned char *rope;               // bf16, E values a position, rope_row bytes apart
    const int32_t *death;                    // [B][T] or nullptr
    const int32_t *n;                        // [B] or nullptr
    unsigned char *out;                      // bf16 [B][T][H][D]
    float *lse;                              // fp32 [B][H][T] (or nullptr, forward)
    // backward
    const unsigned char *dout;               // bf16 [B][T][H][D]
    unsigned char *dq, *dkv, *drope;         // bf16, as q and kv; [B][T][E]
    float *stats;                            // workspace, fp32 [B][H][2][T]: -lse in powers of 2, and delta
    float *part;                             // workspace, fp32 [B][H][T][E]: the heads' gradients of the rotary part
    size_t rope_row;
    int B, T, H;
    float scale, scale_log2e;
};

// Rows of BYTES in LDS behind one another: 16-byte piece p of row r at slot p ^ swizzle(r).
template <int BYTES>
struct LdsRows {
    static constexpr int PIECES = BYTES / 16, LOAD_ROWS = 64 / PIECES;
    static_assert(PIECES == 16 || PIECES == 8 || PIECES == 4, "whole rows a load");
    __device__ static __forceinline__ int swizzle(int r)
    {
        return lds_swizzle<PIECES>(r);
    }
    // LR_STEP rows from memory straight to LDS, rows `stride` bytes apart, by WAVES waves (this: wave wv of them); rows behind `last` are
    // that one again, and where there are more waves than loads, some load again what others do.  (The swizzle is linear in a row's bits:
    // a lane's part of it, and the load's.)
    template <int WAVES>
    static constexpr int LOADS = (LR_STEP / LOAD_ROWS + WAVES - 1) / WAVES;                // of a wave
    template <int WAVES>
    __device__ static __forceinline__ int row(int i, int wv) { return (i * WAVES + wv) * LOAD_ROWS % LR_STEP; }        // load i's first
    template <int WAVES>
    __device__ static __forceinline__ uint32_t offset(int i, uint32_t stride, int last, int wv, int lane)
    {
        const int lrow = lane / PIECES, piece = lane % PIECES ^ swizzle(lrow), r0 = row<WAVES>(i, wv), r = r0 + lrow;
        return (uint32_t)(r < last ? r : last) * stride + (uint32_t)(piece ^ swizzle(r0)) * 16u;
    }
    template <int WAVES>
    __device__ static __forceinline__ void load(const unsigned char *from, uint32_t stride, int last, unsigned char *to, int wv, int lane)
    {
#pragma unroll
        for (int i = 0; i < LOADS<WAVES>; ++i)
            start_load_to_lds16(from, offset<WAVES>(i, stride, last, wv, lane), to + row<WAVES>(i, wv) * BYTES);
    }
    // Offset of piece 2 c + half of row `li`: an operand of 16 values c of 32 rows.  (Rows 32 apart: 32 BYTES more.)
    __device__ static __forceinline__ uint32_t row_piece(int li, int half, int c)
    {
        return (uint32_t)(li * BYTES + (((2 * c + half) ^ swizzle(li)) & (PIECES - 1)) * 16);
    }
    // Where a lane points in a transposing read of rows 4 half + 8 g .. + 3 (16 more: 16 BYTES more), columns 32 c ..
    __device__ static __forceinline__ uint32_t column(int lane, int g, int c)
    {
        const int r = 4 * (lane >> 5) + (lane & 15) / 4 + 8 * g, col = 32 * c + (lane & 16) + 4 * (lane & 3);
        return (uint32_t)(r * BYTES + (((col / 8) ^ swizzle(r)) & (PIECES - 1)) * 16 + (col % 8) * 2);
    }
};

__device__ __forceinline__ bf16x8 operand(u32x4 x) { return __builtin_bit_cast(bf16x8, x); }
__device__ __forceinline__ f32x16 product(bf16x8 x, bf16x8 y, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ f32x16 zeros16()
{
    f32x16 x;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.f;
    return x;
}
// (A value of the loop's own: what is made of it is made where it is used, not kept in registers that the sums need.)
__device__ __forceinline__ uint32_t fresh(uint32_t x)
{
    __asm__ volatile("" : "+v"(x));
    return x;
}
// Row of a tile that register r of a lane's half stands for.
__device__ __forceinline__ int row_of(int r, int half) { return 8 * (r / 4) + 4 * half + r % 4; }

// acc += X^T w for 32 rows of X in LDS and 32 x 32 weights as the first products leave them, two of X's column tiles at a time, whose rows
// are asked for while the products of the two before run.
struct Columns {
    u32x2 v[2][2][2];                        // [column tile][16 rows][8 of them]
};
// Two column tiles of CT, rows of BYTES from x; `first`: where a lane points for column tile 0.  (Offsets of the others differ in a bit
// of their own: no register is kept for them.)
template <int BYTES, int CT>
__device__ __forceinline__ void ask_columns(const unsigned char *x, const uint32_t (&first)[2], int pair, Columns &to)
{
#pragma unroll
    for (int u = 0; u < 2 && 2 * pair + u < CT; ++u)
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int g = 0; g < 2; ++g) to.v[u][st][g] = read_transposed16(x + (first[g] ^ (2 * pair + u) * 64) + 16 * st * BYTES);
}
// `mixed`: some pairs are masked; values that are not finite are taken for 0 then.  Returns whether there were some.
template <int CT>
__device__ __forceinline__ bool add_columns(Columns &x, int pair, const uint32_t (&w)[8], bool mixed, f32x16 (&acc)[CT])
{
    bool odd = false;
    if (mixed) {
#pragma unroll
        for (int u = 0; u < 2 && 2 * pair + u < CT; ++u)
#pragma unroll
            for (int st = 0; st < 2; ++st) odd |= take_out_odd(x.v[u][st][0]) | take_out_odd(x.v[u][st][1]);
    }
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        const bf16x8 weights = operand(u32x4{w[4 * st], w[4 * st + 1], w[4 * st + 2], w[4 * st + 3]});
#pragma unroll
        for (int u = 0; u < 2 && 2 * pair + u < CT; ++u)
            acc[2 * pair + u] = product(operand(u32x4{x.v[u][st][0][0], x.v[u][st][0][1], x.v[u][st][1][0], x.v[u][st][1][1]}), weights, acc[2 * pair + u]);
    }
    return odd;
}

// Which of 32 rows in LDS have a value that is not finite, a bit each (the whole wave).
template <int BYTES>
__device__ __forceinline__ uint32_t odd_rows(const unsigned char *rows)
{
    uint32_t mask = 0;
    for (int r = 0; r < 32; ++r) {
        bool any = false;
        if (lane_id() * 8 < BYTES) any = has_odd(*reinterpret_cast<const u32x2 *>(rows + r * BYTES + lane_id() * 8));
        mask |= (uint32_t)(__ballot(any) != 0) << r;
    }
    return mask;
}

// What add_columns() has taken for 0 in a unit's rows, times weight(r), to who sees row r: sees(r).  (Both of a lane's column of the products.)
template <int BYTES, int CT, class Sees, class Weight>
__device__ __forceinline__ void add_odd_values(const unsigned char *x, Sees sees, Weight weight, f32x16 (&acc)[CT])
{
    const int half = lane_id() >> 5;
    for (uint32_t rows = odd_rows<BYTES>(x); rows; rows &= rows - 1) {
        const int r = __builtin_ctz(rows);
        const bool mine = sees(r);
        const float w = weight(r);
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const u32x2 v = *reinterpret_cast<const u32x2 *>(x + r * BYTES + (((4 * c + g) ^ LdsRows<BYTES>::swizzle(r)) & (LdsRows<BYTES>::PIECES - 1)) * 16 + half * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float f = __uint_as_float(e % 2 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
                    if (mine && !(__builtin_fabsf(f) < INFINITY)) acc[c][4 * g + e] += w * f;
                }
            }
    }
}
// NaN in the columns of who sees a value that is not finite: how many of them is another product.
template <int BYTES, int CT>
__device__ __forceinline__ void odd_becomes_nan(const unsigned char *x, const uint32_t (&first)[2], const uint32_t (&sees)[8], f32x16 (&acc)[CT])
{
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        f32x16 count = zeros16();
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            u32x2 y[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) y[g] = odd_ones(read_transposed16(x + (first[g] ^ c * 64) + 16 * st * BYTES));
            count = product(operand(u32x4{y[0][0], y[0][1], y[1][0], y[1][1]}), operand(u32x4{sees[4 * st], sees[4 * st + 1], sees[4 * st + 2], sees[4 * st + 3]}), count);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] = count[r] > 0.f ? NAN : acc[c][r];
        __builtin_amdgcn_sched_barrier(0);
    }
}
// Weight of row r (uniform) of a unit and this lane's column, of the 32 x 32 as packed for the second product.
__device__ __forceinline__ float weight_of(const uint32_t (&w)[8], int r)
{
    const int at = 4 * (r / 8) + r % 4;                    // register, in the half r / 4 % 2
    uint32_t x = w[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) x = at / 2 == e ? w[e] : x;
    x = __shfl(x, (lane_id() & 31) + (r / 4 % 2) * 32);
    return __uint_as_float(at % 2 ? x & 0xFFFF0000u : x << 16);
}

// Units of LR_STEP keys that some query of first .. last sees, and those that all of them see where causality lets them, as words of
// 64 units in the lanes.  The workgroup's waves look at a part of the keys each and share their words in `scratch` (LDS, 1 KB, free
// again behind the next barrier).
struct LiveUnits {
    uint32_t some_lo, some_hi, all_lo, all_hi;             // of units 64 lane .. + 31, and the 32 behind them
    int units;
    __device__ __forceinline__ LiveUnits(const int32_t *death, int units_, int n, int first, int last, int wv, uint32_t *scratch) : units(units_)
    {
        const int lane = lane_id();
        auto below = [&](int u0) { return units >= u0 + 32 ? 0xFFFFFFFFu : units <= u0 ? 0u : (1u << (units - u0)) - 1u; };
        some_lo = all_lo = below(64 * lane);
        some_hi = all_hi = below(64 * lane + 32);
        if (!death) return;
        constexpr int BATCH = 16;            // loads of 64 keys: a word of units
        const int words = (units + 2 * BATCH - 1) / (2 * BATCH);
        for (int at = wv; at < words; at += LR_WAVES) {
            const int u0 = at * 2 * BATCH;
            int d[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int j = (u0 + 2 * i) * LR_STEP + lane;
                d[i] = j < n ? death[j] : 0;
            }
            // bit 2 i of a word: of the lower half's unit
            uint32_t seen = 0, whole = 0;
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const bool inside = (u0 + 2 * i) * LR_STEP + lane < n;
                const uint64_t any = __ballot(inside && d[i] > first), not_all = __ballot(inside && d[i] <= last);
                seen |= ((uint32_t)any != 0 ? 1u : 0u) << (2 * i) | ((uint32_t)(any >> 32) != 0 ? 2u : 0u) << (2 * i);
                whole |= ((uint32_t)not_all == 0 ? 1u : 0u) << (2 * i) | ((uint32_t)(not_all >> 32) == 0 ? 2u : 0u) << (2 * i);
            }
            if (lane < 2) scratch[2 * at + lane] = lane ? whole : seen;
        }
        __syncthreads();
        auto mine = [&](int at, int which) { return at < words ? scratch[2 * at + which] : 0u; };
        some_lo = mine(2 * lane, 0);
        some_hi = mine(2 * lane + 1, 0);
        all_lo = mine(2 * lane, 1);
        all_hi = mine(2 * lane + 1, 1);
    }
    __device__ static __forceinline__ uint32_t word(uint32_t lo, uint32_t hi, int u)
    {
        const uint32_t a = (uint32_t)__builtin_amdgcn_readlane((int)lo, u / 64), b = (uint32_t)__builtin_amdgcn_readlane((int)hi, u / 64);
        return u / 32 % 2 ? b : a;
    }
    // The first live unit from u on, or `units`.  Uniform.
    __device__ __forceinline__ int next(int u) const
    {
        while (u < units) {
            const uint32_t w = word(some_lo, some_hi, u) >> (u % 32);
            if (w) return u + __builtin_ctz(w) < units ? u + __builtin_ctz(w) : units;
            u = (u / 32 + 1) * 32;
        }
        return units;
    }
    __device__ __forceinline__ bool whole(int u) const { return (word(all_lo, all_hi, u) >> (u % 32)) & 1u; }
};

// What a workgroup that owns queries (forward, backward q) or keys (backward kv) works on: `at_once` (trajectory, head)s at a time (0:
// all), the heaviest blocks of each first.  Where their number is a multiple of 8 each keeps to one XCD, whose L2 then has its rows.
// Few at a time read less (backward kv, 16 for all 32 of 2 x 3850 positions, 16 heads: half the misses, 437 us for 451 with
// backward q); the queries' owners read less in the first place and fare better with the heaviest of all first (16 x 1050 positions:
// 95 us for 100).
constexpr int KV_AT_ONCE = 16;
struct LatentReplayPlace {
    int block, b, h;
    __device__ __forceinline__ LatentReplayPlace(const LatentReplayArgs &a, int blocks, bool last_first, int at_once)
    {
        const int heads = a.B * a.H;
        if (at_once == 0) at_once = heads;
        const int chunk = (int)(blockIdx.x / (unsigned)(at_once * blocks)), r = (int)blockIdx.x - chunk * at_once * blocks;
        const int first = chunk * at_once, here = heads - first < at_once ? heads - first : at_once;
        const int i = r / here, bh = first + r % here;
        block = last_first ? blocks - 1 - i : i;
        b = bh / a.H;
        h = bh % a.H;
    }
    __device__ __forceinline__ int length(const LatentReplayArgs &a) const
    {
        const int n = a.n ? constant_word(a.n + b) : a.T;
        return n < 0 ? 0 : n > a.T ? a.T : n;
    }
};

// Live units of keys, two at a time, through two places in LDS, for the two kernels with queries of their own.  KEEP: a lane's offsets stay in
// registers; the forward pass has them left, the queries' gradient would send 8 others to scratch.
template <int D, bool KEEP>
struct KeyTiles {
    static constexpr int KB = D * 2, RB = D, ROT = LR_STEP * KB, V = ROT + LR_STEP * RB, UNIT = V + LR_STEP * KB, BYTES = 4 * UNIT;
    const LatentReplayArgs &a;
    const LiveUnits &live;
    unsigned char *here, *there;
    int b, h, wv, lane;
    int unit[2];                             // of the next tile, on its way (`units`: none)
    using Own = LdsRows<KB>;
    using Rot = LdsRows<RB>;
    static constexpr int OWN_LOADS = Own::template LOADS<LR_WAVES>, ROT_LOADS = Rot::template LOADS<LR_WAVES>;
    uint32_t own_at[OWN_LOADS], rot_at[ROT_LOADS];         // this lane's part of a unit that lies whole in memory
    __device__ __forceinline__ KeyTiles(const LatentReplayArgs &a_, const LiveUnits &live_, unsigned char *lds, int b_, int h_, int wv_, int lane_)
        : a(a_), live(live_), here(lds), there(lds + 2 * UNIT), b(b_), h(h_), wv(wv_), lane(lane_)
    {
#pragma unroll
        for (int i = 0; i < OWN_LOADS; ++i) own_at[i] = Own::template offset<LR_WAVES>(i, (uint32_t)a.H * (2 * KB), LR_STEP, wv, lane);
#pragma unroll
        for (int i = 0; i < ROT_LOADS; ++i) rot_at[i] = Rot::template offset<LR_WAVES>(i, (uint32_t)a.rope_row, LR_STEP, wv, lane);
        ask(0);
    }
    __device__ __forceinline__ bool more() const { return unit[0] < live.units; }
    __device__ __forceinline__ void ask(int from)
    {
        unit[0] = live.next(from);
        unit[1] = live.next(unit[0] + 1);
        if (!more()) return;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int first = unit[unit[i] < live.units ? i : 0] * LR_STEP;        // (none: the first again)
            const int last = a.T - 1 - first;              // of the memory; behind the sequence's end nothing is seen
            unsigned char *const to = there + i * UNIT;
            const unsigned char *const k = a.kv + (((size_t)b * a.T + first) * a.H + h) * (2 * KB);
            const unsigned char *const r = a.rope + ((size_t)b * a.T + first) * a.rope_row;
            if (KEEP && last >= LR_STEP - 1) {
#pragma unroll
                for (int j = 0; j < OWN_LOADS; ++j) start_load_to_lds16(k, own_at[j], to + Own::template row<LR_WAVES>(j, wv) * KB);
#pragma unroll
                for (int j = 0; j < ROT_LOADS; ++j) start_load_to_lds16(r, rot_at[j], to + ROT + Rot::template row<LR_WAVES>(j, wv) * RB);
#pragma unroll
                for (int j = 0; j < OWN_LOADS; ++j) start_load_to_lds16(k + KB, own_at[j], to + V + Own::template row<LR_WAVES>(j, wv) * KB);
            } else {
                const int lane_ = (int)fresh((uint32_t)lane);
                const uint32_t stride = (uint32_t)a.H * (2 * KB);
                Own::template load<LR_WAVES>(k, stride, last, to, wv, lane_);
                Rot::template load<LR_WAVES>(r, (uint32_t)a.rope_row, last, to + ROT, wv, lane_);
                Own::template load<LR_WAVES>(k + KB, stride, last, to + V, wv, lane_);
            }
        }
    }
    // The next tile, in LDS until the next call; u: its units.  By all waves.
    __device__ __forceinline__ const unsigned char *take(int (&u)[2])
    {
        u[0] = unit[0];
        u[1] = unit[1];
        unsigned char *const x = here;
        here = there;
        there = x;
        lds_loads_done();
        ask(u[1] + 1);
        __builtin_amdgcn_sched_barrier(0);
        return here;
    }
};

// The bits of 32 keys from key0 (uniform) that query i sees, of the 16 that stand in a lane's registers: register r, bit r.  (The keys'
// ends through the scalar unit: a vector load's result would be waited for behind all the tiles on their way.)
__device__ __forceinline__ uint32_t seen_keys(const int32_t *death, int key0, int n, int T, int i, int half)
{
    const int below = i < n - 1 ? i : n - 1;               // the last key that it may see
    uint32_t seen = 0;
    if (!death) {
#pragma unroll
        for (int r = 0; r < 16; ++r) seen |= (uint32_t)(key0 + row_of(r, half) <= below) << r;
    } else if (key0 + LR_STEP <= T) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int lower = constant_word(death + key0 + row_of(r, 0)), upper = constant_word(death + key0 + row_of(r, 1));
            seen |= (uint32_t)(key0 + row_of(r, half) <= below && i < (half ? upper : lower)) << r;
        }
    } else {
#pragma unroll 1
        for (int r = 0; r < 16; ++r) {
            const int j = key0 + row_of(r, half);
            seen |= (uint32_t)(j <= below && i < death[j < T ? j : T - 1]) << r;
        }
    }
    return seen;
}

// Whether this lane's query sees key r (uniform) of a unit, of the bits that its halves have.
__device__ __forceinline__ bool sees_key(uint32_t seen, int r)
{
    return (__shfl(seen, (lane_id() & 31) + (r / 4 % 2) * 32) >> (4 * (r / 8) + r % 4)) & 1u;
}

template <int D>
__global__ __launch_bounds__(LR_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2)))
void latent_replay_kernel(LatentReplayArgs a)
{
    using Tiles = KeyTiles<D, true>;
    constexpr int E = D / 2, KC = D / 16, RC = E / 16, DT = D / 32;
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    const int li = lane & 31, half = lane >> 5;
    const LatentReplayPlace at(a, (a.T + LR_BLOCK - 1) / LR_BLOCK, true, 0);
    const int n = at.length(a), i0 = at.block * LR_BLOCK;
    if (i0 >= n) return;
    const int wave0 = i0 + wv * LR_OWN, qpos = wave0 + li;
    const int wave_last = wave0 + LR_OWN - 1 < n ? wave0 + LR_OWN - 1 : n - 1, block_last = i0 + LR_BLOCK - 1 < n ? i0 + LR_BLOCK - 1 : n - 1;
    const int32_t *death = a.death ? a.death + (size_t)at.b * a.T : nullptr;
    bf16x8 q[KC + RC];
    {
        const unsigned char *row = a.q + (((size_t)at.b * a.T + (qpos < n ? qpos : n - 1)) * a.H + at.h) * ((D + E) * 2) + half * 16;
#pragma unroll
        for (int c = 0; c < KC + RC; ++c) q[c] = operand(*reinterpret_cast<const u32x4 *>(row + c * 32));
    }
    const LiveUnits live(death, block_last / LR_STEP + 1, n, i0, block_last, wv, reinterpret_cast<uint32_t *>(lds));
    Tiles tiles(a, live, lds, at.b, at.h, wv, lane);       // (its first tile goes behind the words)
    const uint32_t k_first = LdsRows<Tiles::KB>::row_piece(li, half, 0), r_first = LdsRows<Tiles::RB>::row_piece(li, half, 0);
    const uint32_t v_first[2] = {LdsRows<Tiles::KB>::column(lane, 0, 0), LdsRows<Tiles::KB>::column(lane, 1, 0)};
    f32x16 o[DT];
#pragma unroll
    for (int c = 0; c < DT; ++c) o[c] = zeros16();
    float m_run = -INFINITY, neg_m = 0.f, l_run = 0.f;     // m_run: a score; neg_m: -m_run scaled, or 0 as long as nothing has been seen

    auto step = [&](const unsigned char *unit, int key0, bool whole) {
        const bool mixed = !whole || key0 + LR_STEP - 1 > wave0 || key0 + LR_STEP > n;
        f32x16 sc = zeros16();
#pragma unroll
        for (int c = 0; c < KC; ++c) sc = product(operand(*reinterpret_cast<const u32x4 *>(unit + (k_first ^ c * 32))), q[c], sc);
#pragma unroll
        for (int c = 0; c < RC; ++c) sc = product(operand(*reinterpret_cast<const u32x4 *>(unit + Tiles::ROT + (r_first ^ c * 32))), q[KC + c], sc);
        const unsigned char *const values = unit + Tiles::V;
        Columns x[2];
        ask_columns<Tiles::KB, DT>(values, v_first, 0, x[0]);   // (there when the weights are)
        uint32_t seen = 0xFFFFu;
        if (mixed) {
            seen = seen_keys(death, key0, n, a.T, qpos, half);
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = (seen >> r) & 1u ? sc[r] : -INFINITY;
        }
        float top = sc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = max_no_nan(top, sc[r]);
        top = half_rows_max(top);
        const bool outgrown = (top - m_run) * a.scale_log2e > LR_LAZY;     // of each row by itself: its results do not depend on its neighbours'
        if (__ballot(outgrown)) {
            const float m_new = outgrown ? top : m_run;
            const float alpha = m_new == m_run ? 1.0f : fast_exp2((m_run - m_new) * a.scale_log2e);
            l_run *= alpha;
#pragma unroll
            for (int c = 0; c < DT; ++c) o[c] *= alpha;
            m_run = m_new;
            neg_m = m_new == -INFINITY ? 0.f : -(m_new * a.scale_log2e);
        }
        float ref = neg_m;
        const bool far = __builtin_fabsf(neg_m) > LR_FAR;
        if (__builtin_expect(__ballot(far) != 0, 0)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = far ? sc[r] - m_run : sc[r];
            ref = far ? 0.f : neg_m;
        }
        uint32_t w[8];
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p0 = fast_exp2(__builtin_fmaf(sc[2 * e], a.scale_log2e, ref)), p1 = fast_exp2(__builtin_fmaf(sc[2 * e + 1], a.scale_log2e, ref));
            sum += p0 + p1;
            w[e] = pack_bf16(p0, p1);
        }
        l_run += sum;
        bool odd = false;
#pragma unroll
        for (int pair = 0; pair < DT / 2; ++pair) {
            if (pair + 1 < DT / 2) ask_columns<Tiles::KB, DT>(values, v_first, pair + 1, x[(pair + 1) & 1]);
            odd |= add_columns(x[pair & 1], pair, w, mixed, o);
        }
        if (__builtin_expect(__ballot(odd) != 0, 0)) add_odd_values<Tiles::KB>(values, [&](int r) { return sees_key(seen, r); }, [&](int r) { return weight_of(w, r); }, o);
    };

    own_rows_loaded();
    // (the tiles that this wave sees first, in a loop without branches: with one in it the sums would be kept twice)
    int u[2];
    auto mine = [&](int unit) { return unit < live.units && wave0 < n && unit * LR_STEP <= wave_last; };
    while (mine(tiles.unit[1])) {
        const unsigned char *const here = tiles.take(u);
        step(here, u[0] * LR_STEP, live.whole(u[0]));
        step(here + Tiles::UNIT, u[1] * LR_STEP, live.whole(u[1]));
    }
    if (mine(tiles.unit[0])) {
        const unsigned char *const here = tiles.take(u);
        step(here, u[0] * LR_STEP, live.whole(u[0]));
    }
    while (tiles.more()) (void)tiles.take(u);

    // out, through LDS: rows leave as whole lines, past the keys and values in the L2 (16 x 1050 positions: 92 us for 96); 16-byte piece p of
    // row r at slot p ^ r
    const float l = half_rows_sum(l_run);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    if (a.lse && half == 0 && qpos < n) {
        const bool far = __builtin_fabsf(neg_m) > LR_FAR;
        const float log2_l = __builtin_amdgcn_logf(l), near = (log2_l - neg_m) * 0.6931471805599453f;
        a.lse[((size_t)at.b * a.H + at.h) * a.T + qpos] = l == 0.f ? -INFINITY : far ? __builtin_fmaf(m_run, a.scale, log2_l * 0.6931471805599453f) : near;
    }
    lds_loads_done();
    constexpr int OP = D / 8;
    unsigned char *const rows = lds + wv * LR_OWN * D * 2;
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = 32 * c + 8 * g + 4 * half;
            *reinterpret_cast<u32x2 *>(rows + li * (D * 2) + (((col / 8) ^ li) & (OP - 1)) * 16 + (col % 8) * 2) =
                u32x2{pack_bf16(o[c][4 * g] * inv, o[c][4 * g + 1] * inv), pack_bf16(o[c][4 * g + 2] * inv, o[c][4 * g + 3] * inv)};
        }
    __builtin_amdgcn_s_waitcnt(0xC07F);                    // lgkmcnt(0): a wave's rows are its own
    __asm__ volatile("" ::: "memory");
#pragma unroll
    for (int r0 = 0; r0 < LR_OWN; r0 += 64 / OP) {
        const int r = r0 + lane / OP, piece = lane % OP;
        const u32x4 x = *reinterpret_cast<const u32x4 *>(rows + r * (D * 2) + ((piece ^ r) & (OP - 1)) * 16);
        if (wave0 + r < n) __builtin_nontemporal_store(x, reinterpret_cast<u32x4 *>(a.out + ((((size_t)at.b * a.T + wave0 + r) * a.H + at.h) * D + piece * 8) * 2));
    }
}

// 32 rows of COLS gradients (a wave's own) from accumulators to bf16 rows in memory, through LDS as above.  `col0`: first column of
// the first accumulator in a row.
template <int CT>
__device__ __forceinline__ void store_rows(unsigned char *lds, const f32x16 (&acc)[CT], float scale, unsigned char *to, size_t stride, int rows)
{
    constexpr int PIECES = CT * 4;                         // 16-byte pieces of a row: 4, 8, 12 or 16
    const int lane = lane_id(), li = lane & 31, half = lane >> 5;
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __asm__ volatile("" ::: "memory");
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int piece = 4 * c + g;
            *reinterpret_cast<u32x2 *>(lds + li * (PIECES * 16) + (piece ^ (li & 3)) * 16 + half * 8) =
                u32x2{pack_bf16(acc[c][4 * g] * scale, acc[c][4 * g + 1] * scale), pack_bf16(acc[c][4 * g + 2] * scale, acc[c][4 * g + 3] * scale)};
        }
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __asm__ volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32 * PIECES / 64; ++i) {
        const int r = (i * 64 + lane) / PIECES, piece = (i * 64 + lane) % PIECES;
        const u32x4 x = *reinterpret_cast<const u32x4 *>(lds + r * (PIECES * 16) + (piece ^ (r & 3)) * 16);
        if (r < rows) __builtin_nontemporal_store(x, reinterpret_cast<u32x4 *>(to + r * stride + piece * 16));
    }
}

// Gradient of the queries, and delta.
template <int D>
__global__ __launch_bounds__(LR_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2)))
void latent_replay_dq_kernel(LatentReplayArgs a)
{
    using Tiles = KeyTiles<D, false>;
    constexpr int E = D / 2, KC = D / 16, RC = E / 16, DT = D / 32, ET = E / 32;
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    const int li = lane & 31, half = lane >> 5;
    const LatentReplayPlace at(a, (a.T + LR_BLOCK - 1) / LR_BLOCK, true, 0);
    const int n = at.length(a), i0 = at.block * LR_BLOCK;
    if (i0 >= n) return;
    const int wave0 = i0 + wv * LR_OWN, qpos = wave0 + li, q_row = qpos < n ? qpos : n - 1;
    const int wave_last = wave0 + LR_OWN - 1 < n ? wave0 + LR_OWN - 1 : n - 1, block_last = i0 + LR_BLOCK - 1 < n ? i0 + LR_BLOCK - 1 : n - 1;
    const int32_t *death = a.death ? a.death + (size_t)at.b * a.T : nullptr;
    bf16x8 q[KC + RC], g_[KC];
    float delta = 0.f;
    const size_t row = ((size_t)at.b * a.T + q_row) * a.H + at.h;
    {
        const unsigned char *qr = a.q + row * ((D + E) * 2) + half * 16, *gr = a.dout + row * (D * 2) + half * 16, *orow = a.out + row * (D * 2) + half * 16;
#pragma unroll
        for (int c = 0; c < KC + RC; ++c) q[c] = operand(*reinterpret_cast<const u32x4 *>(qr + c * 32));
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(gr + c * 32), y = *reinterpret_cast<const u32x4 *>(orow + c * 32);
            g_[c] = operand(x);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                delta += __uint_as_float(x[e] << 16) * __uint_as_float(y[e] << 16) + __uint_as_float(x[e] & 0xFFFF0000u) * __uint_as_float(y[e] & 0xFFFF0000u);
        }
        delta = half_rows_sum(delta);
    }
    const LiveUnits live(death, block_last / LR_STEP + 1, n, i0, block_last, wv, reinterpret_cast<uint32_t *>(lds));
    Tiles tiles(a, live, lds, at.b, at.h, wv, lane);       // (its first tile goes behind the words)
    const size_t stat = ((size_t)at.b * a.H + at.h) * a.T + q_row;
    const float neg_lse = -a.lse[stat] * 1.4426950408889634f;
    if (half == 0 && qpos < n) {
        float *const stats = a.stats + ((size_t)at.b * a.H + at.h) * 2 * a.T + qpos;
        stats[0] = neg_lse;
        stats[a.T] = delta;
    }
    const uint32_t k_first = LdsRows<Tiles::KB>::row_piece(li, half, 0), r_first = LdsRows<Tiles::RB>::row_piece(li, half, 0);
    const uint32_t kt_first[2] = {LdsRows<Tiles::KB>::column(lane, 0, 0), LdsRows<Tiles::KB>::column(lane, 1, 0)};
    const uint32_t rt_first[2] = {LdsRows<Tiles::RB>::column(lane, 0, 0), LdsRows<Tiles::RB>::column(lane, 1, 0)};
    f32x16 dk[DT], dr[ET];                                 // dQ^T: of the part that meets the heads' own keys, and of the rotary part
#pragma unroll
    for (int c = 0; c < DT; ++c) dk[c] = zeros16();
#pragma unroll
    for (int c = 0; c < ET; ++c) dr[c] = zeros16();

    auto step = [&](const unsigned char *unit, int key0, bool whole) {
        const bool mixed = !whole || key0 + LR_STEP - 1 > wave0 || key0 + LR_STEP > n;
        f32x16 sc = zeros16(), dp = zeros16();
        const uint32_t k_0 = fresh(k_first), r_0 = fresh(r_first);
#pragma unroll
        for (int c = 0; c < KC; ++c) sc = product(operand(*reinterpret_cast<const u32x4 *>(unit + (k_0 ^ c * 32))), q[c], sc);
#pragma unroll
        for (int c = 0; c < RC; ++c) sc = product(operand(*reinterpret_cast<const u32x4 *>(unit + Tiles::ROT + (r_0 ^ c * 32))), q[KC + c], sc);
#pragma unroll
        for (int c = 0; c < KC; ++c) dp = product(operand(*reinterpret_cast<const u32x4 *>(unit + Tiles::V + (k_0 ^ c * 32))), g_[c], dp);
        const uint32_t kt_0[2] = {fresh(kt_first[0]), fresh(kt_first[1])}, rt_0[2] = {fresh(rt_first[0]), fresh(rt_first[1])};
        Columns x[2];
        ask_columns<Tiles::KB, DT>(unit, kt_0, 0, x[0]);
        float ds[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = fast_exp2(__builtin_fmaf(sc[r], a.scale_log2e, neg_lse)) * (dp[r] - delta);
        if (mixed) {
            const uint32_t seen = seen_keys(death, key0, n, a.T, qpos, half);
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] = (seen >> r) & 1u ? ds[r] : 0.f;
        }
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = pack_bf16(ds[2 * e], ds[2 * e + 1]);
        bool odd = false;
#pragma unroll
        for (int pair = 0; pair < DT / 2; ++pair) {
            if (pair + 1 < DT / 2) ask_columns<Tiles::KB, DT>(unit, kt_0, pair + 1, x[(pair + 1) & 1]);
            else ask_columns<Tiles::RB, ET>(unit + Tiles::ROT, rt_0, 0, x[(pair + 1) & 1]);
            odd |= add_columns(x[pair & 1], pair, w, mixed, dk);
        }
        odd |= add_columns(x[DT / 2 & 1], 0, w, mixed, dr);
        if (__builtin_expect(__ballot(odd) != 0, 0)) {
            // a key that is seen and not finite has a dS of NaN, or of 0 where its score is minus infinity: NaN times such a value
            const uint32_t seen = seen_keys(death, key0, n, a.T, qpos, half);          // (again: it would be in the sums' way)
            uint32_t sees[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) sees[e] = ((seen >> 2 * e) & 1u ? 0x3F80u : 0u) | ((seen >> (2 * e + 1)) & 1u ? 0x3F800000u : 0u);
            odd_becomes_nan<Tiles::KB>(unit, kt_0, sees, dk);
            odd_becomes_nan<Tiles::RB>(unit + Tiles::ROT, rt_0, sees, dr);
        }
    };
    own_rows_loaded();
    // (the tiles that this wave sees first, in a loop without branches: with one in it the sums would be kept twice)
    int u[2];
    auto mine = [&](int unit) { return unit < live.units && wave0 < n && unit * LR_STEP <= wave_last; };
    while (mine(tiles.unit[1])) {
        const unsigned char *const here = tiles.take(u);
        step(here, u[0] * LR_STEP, live.whole(u[0]));
        step(here + Tiles::UNIT, u[1] * LR_STEP, live.whole(u[1]));
    }
    if (mine(tiles.unit[0])) {
        const unsigned char *const here = tiles.take(u);
        step(here, u[0] * LR_STEP, live.whole(u[0]));
    }
    while (tiles.more()) (void)tiles.take(u);
    lds_loads_done();
    unsigned char *const rows = lds + wv * LR_OWN * D * 2;
    unsigned char *const to = a.dq + (((size_t)at.b * a.T + wave0) * a.H + at.h) * ((D + E) * 2);
    const size_t stride = (size_t)a.H * ((D + E) * 2);
    store_rows(rows, dk, a.scale, to, stride, n - wave0);
    store_rows(rows, dr, a.scale, to + D * 2, stride, n - wave0);
}

// The unit of 32 keys that has place `rank` when they are ordered by the query that sees a key of theirs last, the latest first, and by
// position among those: the keys of a workgroup's waves then live about as long.  Whole workgroup; `scratch`: LDS of LR_ORDER_BYTES.
// (A counting sort: how many units end in each stretch of 32 queries, where each stretch begins, then the units in their order.)
constexpr int LR_MOST_UNITS = LR_MOST_POSITIONS / LR_STEP;
constexpr int LR_ORDER_BYTES = (LR_MOST_UNITS + LR_MOST_UNITS / 2 + 8 + 32) * 4;
template <int WAVES>
__device__ __forceinline__ int unit_by_end(const int32_t *death, int n, int rank, int *scratch)
{
    constexpr int THREADS = WAVES * 64;
    int *const count = scratch, *const tmp = scratch + LR_MOST_UNITS + 8;  // count[s]: of units that end in stretch s from the back
    uint16_t *const end_of = reinterpret_cast<uint16_t *>(scratch + LR_MOST_UNITS + 8 + 32);
    const int units = (n + LR_STEP - 1) / LR_STEP, lane = lane_id();
    for (int i = threadIdx.x; i <= units; i += THREADS) count[i] = 0;
    __syncthreads();
    constexpr int BATCH = 8;
    for (int u0 = 2 * wave_id(); u0 < units; u0 += 2 * WAVES * BATCH) {
        int d[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int j = (u0 + 2 * WAVES * i) * LR_STEP + lane;
            d[i] = j < n ? death[j] : 0;
            d[i] = d[i] < n ? d[i] : n;
            d[i] = d[i] > j ? d[i] : 0;                    // seen by nobody
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int u = u0 + 2 * WAVES * i + lane / 32;
            int last = d[i];
#pragma unroll
            for (int step = 1; step < 32; step *= 2) {
                const int other = __shfl_xor(last, step);
                last = last > other ? last : other;
            }
            if ((lane & 31) == 0 && u < units) {
                const int s = units - (last + LR_STEP - 1) / LR_STEP;      // 0: sees the last query's stretch; units: nobody's
                end_of[u] = (uint16_t)s;
                atomicAdd(&count[s], 1);
            }
        }
    }
    __syncthreads();
    // the stretch of this wave's unit, and its place there
    const int per = (units + THREADS) / THREADS;           // of units + 1 stretches
    const int lo = (int)threadIdx.x * per, hi = lo + per < units + 1 ? lo + per : units + 1;
    int mine = 0;
    for (int i = lo; i < hi; ++i) mine += count[i];
    int total;
    int before = block_excl_scan_i<THREADS>(mine, tmp, &total);
    for (int i = lo; i < hi; ++i) {
        const int c = count[i];
        count[i] = before;
        before += c;
    }
    __syncthreads();
    int s_lo = 0, s_hi = units;                            // the last stretch that begins at or before rank
    while (s_lo < s_hi) {
        const int mid = (s_lo + s_hi + 1) / 2;
        if (count[mid] <= rank) s_lo = mid;
        else s_hi = mid - 1;
    }
    int left = rank - count[s_lo], found = units;          // (beyond the last unit: none)
    for (int u0 = 0; u0 < units && found == units; u0 += 64) {
        const uint64_t here = __ballot(u0 + lane < units && end_of[u0 + lane < units ? u0 + lane : 0] == s_lo);
        const int some = __popcll(here);
        if (left < some) {
            uint64_t w = here;
            for (int i = 0; i < left; ++i) w &= w - 1;
            found = u0 + __builtin_ctzll(w);
        }
        left -= some;
    }
    __syncthreads();                                       // scratch is free again
    return __builtin_amdgcn_readfirstlane(found);
}

// Gradients of keys and values, and the head's of the rotary part.  Two waves for 32 keys: the first makes P of 32 queries, and with
// it dV; the second makes dS of it and of <g, v>, and with it dK and the rotary part's.
template <int D>
__global__ __launch_bounds__(2 * KV_GROUPS * 64) __attribute__((amdgpu_waves_per_eu(2)))
void latent_replay_dkv_kernel(LatentReplayArgs a)
{
    constexpr int E = D / 2, KC = D / 16, RC = E / 16, DT = D / 32, ET = E / 32, KB = D * 2, RB = E * 2, PAIRS = DT / 2;
    // 32 queries in LDS: their two parts, the gradients that arrive at them, and their statistics
    constexpr int ROT = LR_STEP * KB, G = ROT + LR_STEP * RB, STATS = G + LR_STEP * KB, BYTES = STATS + 2 * LR_STEP * 4;
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), wv = wave % KV_GROUPS, second = wave / KV_GROUPS;
    const int li = lane & 31, half = lane >> 5;
    const LatentReplayPlace at(a, (a.T + KV_BLOCK - 1) / KV_BLOCK, false, KV_AT_ONCE);
    const int n = at.length(a);
    if (at.block * KV_BLOCK >= n) return;
    const int32_t *death = a.death ? a.death + (size_t)at.b * a.T : nullptr;
    const int unit = death ? unit_by_end<2 * KV_GROUPS>(death, n, at.block * KV_GROUPS + wv, reinterpret_cast<int *>(lds)) : at.block * KV_GROUPS + wv;
    const int wave0 = unit * LR_OWN, key = wave0 + li, k_row = key < n ? key : n - 1;
    // queries key .. until - 1 see this lane's key
    int until = n;
    if (death) {
        const int d = death[k_row];
        until = d < n ? d : n;
    }
    if (key >= n) until = 0;
    auto larger = [](int x, int y) { return x > y ? x : y; };
    auto smaller = [](int x, int y) { return x < y ? x : y; };
    const int wave_end = __builtin_amdgcn_readfirstlane(wave_reduce(until, larger));
    // all of the wave's keys are seen by queries below this one, where causality lets them
    const int wave_all = __builtin_amdgcn_readfirstlane(wave_reduce(until, smaller));
    __shared__ int begins[KV_GROUPS], ends[KV_GROUPS];
    if (lane == 0) {
        begins[wv] = wave0;
        ends[wv] = wave_end;
    }
    __syncthreads();
    int begin = n, end = 0;
#pragma unroll
    for (int w = 0; w < KV_GROUPS; ++w) {
        begin = smaller(begin, begins[w]);
        end = larger(end, ends[w]);
    }
    const int first = __builtin_amdgcn_readfirstlane(begin) / LR_STEP, units = (__builtin_amdgcn_readfirstlane(end) + LR_STEP - 1) / LR_STEP;

    const bool some = first < units;                       // (no query sees any of the keys: no unit to read)
    const size_t stat = ((size_t)at.b * a.H + at.h) * a.T;
    const uint32_t q_stride = (uint32_t)a.H * ((D + E) * 2), g_stride = (uint32_t)a.H * KB;
    // A unit: the first waves bring the queries, the second ones the gradients and (each of them) the statistics.
    constexpr int Q_LOADS = LdsRows<KB>::template LOADS<KV_GROUPS> + LdsRows<RB>::template LOADS<KV_GROUPS>, G_LOADS = LdsRows<KB>::template LOADS<KV_GROUPS> + 1;
    constexpr int SLOTS = kv_slots(D);
    auto slot = [&](int u) { return lds + (u - first) % SLOTS * BYTES; };
    auto load_ahead = [&](int u_) {
        const int u = u_ < units ? u_ : units - 1;         // (the last one again into a free place)
        const int i = u * LR_STEP, last = a.T - 1 - i;
        unsigned char *const to = slot(u_);
        const size_t row = ((size_t)at.b * a.T + i) * a.H + at.h;
        int lane_ = lane;
        __asm__ volatile("" : "+v"(lane_));                // (offsets are made where they are used)
        if (!second) {
            const unsigned char *const q = a.q + row * ((D + E) * 2);
            LdsRows<KB>::template load<KV_GROUPS>(q, q_stride, last, to, wv, lane_);
            LdsRows<RB>::template load<KV_GROUPS>(q + KB, q_stride, last, to + ROT, wv, lane_);
        } else {
            LdsRows<KB>::template load<KV_GROUPS>(a.dout + row * KB, g_stride, last, to + G, wv, lane_);
            const int r = lane_ & 31;
            start_load_to_lds4(reinterpret_cast<const unsigned char *>(a.stats + stat * 2 + i), (uint32_t)((r < last ? r : last) + (lane_ >> 5) * a.T) * 4u, to + STATS);
        }
    };
    // P of a unit, from the first wave to the second: two places, fp32 as the products leave it.
    unsigned char *const exchange = lds + SLOTS * BYTES + wv * (2 * 4096) + lane * 16;
    auto place = [&](int u) { return exchange + (u & 1) * 4096; };
    // units mine_first .. mine_end - 1 have queries that see keys of this wave (a loop of their own: with a branch in it the sums would be
    // kept twice)
    const int mine_first = unit < units ? unit : units, mine_end = larger(mine_first, (wave_end + LR_STEP - 1) / LR_STEP);
    auto mixed_at = [&](int u) { return u * LR_STEP < wave0 + LR_OWN - 1 || (u + 1) * LR_STEP > wave_all; };
    // Weights of 0 for the pairs of a unit that are masked.
    auto mask = [&](int query0, uint32_t (&w)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = query0 + row_of(2 * e, half);
            w[e] &= (key <= i && i < until ? 0xFFFFu : 0u) | (key <= i + 1 && i + 1 < until ? 0xFFFF0000u : 0u);
        }
    };
    // acc += X y for a unit's rows: COUNT operands, at(c) in the unit and y(c), GROUP of them asked for while the products of those before run.
    auto rows_product = [&](auto count, const unsigned char *from, auto at_, auto y, f32x16 acc) {
        constexpr int COUNT = decltype(count)::value, GROUP = COUNT % 4 ? 3 : 4, GROUPS = COUNT / GROUP;
        static_assert(COUNT % GROUP == 0, "whole groups");
        u32x4 rows[2][GROUP];
        auto ask = [&](int g) {
#pragma unroll
            for (int u = 0; u < GROUP; ++u) rows[g & 1][u] = *reinterpret_cast<const u32x4 *>(from + at_(g * GROUP + u));
        };
        ask(0);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            if (g + 1 < GROUPS) ask(g + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < GROUP; ++u) acc = product(operand(rows[g & 1][u]), y(g * GROUP + u), acc);
            __builtin_amdgcn_sched_barrier(0);
        }
        return acc;
    };
    auto round_begins = [&](int u) {
        if (second) wait_for_loads<(SLOTS - 3) * G_LOADS>();   // unit u is there, P of the one before too
        else wait_for_loads<(SLOTS - 3) * Q_LOADS>();
        workgroup_barrier();                               // and everybody has left unit u - 2
        load_ahead(u + SLOTS - 2);
        __builtin_amdgcn_sched_barrier(0);
    };
    const unsigned char *const kr = a.kv + (((size_t)at.b * a.T + k_row) * a.H + at.h) * (2 * KB) + half * 16;
    unsigned char *const mine = lds + wave * LR_OWN * KB;
    const size_t stride = (size_t)a.H * (2 * KB);
    unsigned char *const to = a.dkv + (((size_t)at.b * a.T + wave0) * a.H + at.h) * (2 * KB);
    if (!second) {
        bf16x8 k[KC + RC];
        const unsigned char *const rr = a.rope + ((size_t)at.b * a.T + k_row) * a.rope_row + half * 16;
#pragma unroll
        for (int c = 0; c < KC; ++c) k[c] = operand(*reinterpret_cast<const u32x4 *>(kr + c * 32));
#pragma unroll
        for (int c = 0; c < RC; ++c) k[KC + c] = operand(*reinterpret_cast<const u32x4 *>(rr + c * 32));
        const uint32_t q_first = LdsRows<KB>::row_piece(li, half, 0), r_first = LdsRows<RB>::row_piece(li, half, 0);
        const uint32_t gt_first[2] = {LdsRows<KB>::column(lane, 0, 0), LdsRows<KB>::column(lane, 1, 0)};
        f32x16 dv[DT];
#pragma unroll
        for (int c = 0; c < DT; ++c) dv[c] = zeros16();
        own_rows_loaded();
        for (int u = first; some && u < first + SLOTS - 2; ++u) load_ahead(u);
        for (int u = first; u < mine_first; ++u) round_begins(u);
        for (int u = mine_first; u < mine_end; ++u) {
            round_begins(u);
            const unsigned char *const here = slot(u);
            const bool mixed = mixed_at(u);
            const uint32_t q_0 = fresh(q_first), r_0 = fresh(r_first);
            const f32x16 s = rows_product(std::integral_constant<int, KC + RC>{}, here, [&](int c) { return c < KC ? q_0 ^ c * 32 : ROT + (r_0 ^ (c - KC) * 32); },
                                          [&](int c) { return k[c]; }, zeros16());
            uint32_t w[8];
            Columns x[2];
            const uint32_t gt_0[2] = {fresh(gt_first[0]), fresh(gt_first[1])};
            ask_columns<KB, DT>(here + G, gt_0, 0, x[0]);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 neg_lse = *reinterpret_cast<const f32x4 *>(here + STATS + (8 * g + 4 * half) * 4);
                f32x4 p;
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = fast_exp2(__builtin_fmaf(s[4 * g + e], a.scale_log2e, neg_lse[e]));
                *reinterpret_cast<f32x4 *>(place(u) + g * 1024) = p;
                w[2 * g] = pack_bf16(p[0], p[1]);
                w[2 * g + 1] = pack_bf16(p[2], p[3]);
            }
            if (mixed) mask(u * LR_STEP, w);
            bool odd = false;
#pragma unroll
            for (int pair = 0; pair < PAIRS; ++pair) {
                if (pair + 1 < PAIRS) ask_columns<KB, DT>(here + G, gt_0, pair + 1, x[(pair + 1) & 1]);
                __builtin_amdgcn_sched_barrier(0);
                odd |= add_columns(x[pair & 1], pair, w, mixed, dv);
            }
            if (__builtin_expect(__ballot(odd) != 0, 0)) {
                const int i0 = u * LR_STEP;
                add_odd_values<KB>(here + G, [&](int r) { return key <= i0 + r && i0 + r < until; }, [&](int r) { return weight_of(w, r); }, dv);
            }
        }
        for (int u = mine_end; some && u <= units; ++u) round_begins(u);
        lds_loads_done();
        store_rows(mine, dv, 1.0f, to + KB, stride, n - wave0);
    } else {
        bf16x8 v[KC];
#pragma unroll
        for (int c = 0; c < KC; ++c) v[c] = operand(*reinterpret_cast<const u32x4 *>(kr + KB + c * 32));
        const uint32_t g_first = LdsRows<KB>::row_piece(li, half, 0);
        const uint32_t qt_first[2] = {LdsRows<KB>::column(lane, 0, 0), LdsRows<KB>::column(lane, 1, 0)};
        const uint32_t rt_first[2] = {LdsRows<RB>::column(lane, 0, 0), LdsRows<RB>::column(lane, 1, 0)};
        f32x16 dk[DT], dr[ET];
#pragma unroll
        for (int c = 0; c < DT; ++c) dk[c] = zeros16();
#pragma unroll
        for (int c = 0; c < ET; ++c) dr[c] = zeros16();
        own_rows_loaded();
        for (int u = first; some && u < first + SLOTS - 2; ++u) load_ahead(u);
        for (int u = first - 1; some && u < mine_first; ++u) round_begins(u + 1);
        for (int u = mine_first; u < mine_end; ++u) {
            round_begins(u + 1);
            const unsigned char *const here = slot(u);
            const bool mixed = mixed_at(u);
            const uint32_t g_0 = fresh(g_first);
            const f32x16 dp = rows_product(std::integral_constant<int, KC>{}, here, [&](int c) { return G + (g_0 ^ c * 32); }, [&](int c) { return v[c]; }, zeros16());
            uint32_t w[8];
            Columns x[2];
            const uint32_t qt_0[2] = {fresh(qt_first[0]), fresh(qt_first[1])};
            ask_columns<KB, DT>(here, qt_0, 0, x[0]);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 delta = *reinterpret_cast<const f32x4 *>(here + STATS + (LR_STEP + 8 * g + 4 * half) * 4);
                const f32x4 p = *reinterpret_cast<const f32x4 *>(place(u) + g * 1024);
                float ds[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) ds[e] = p[e] * (dp[4 * g + e] - delta[e]);
                w[2 * g] = pack_bf16(ds[0], ds[1]);
                w[2 * g + 1] = pack_bf16(ds[2], ds[3]);
            }
            if (mixed) mask(u * LR_STEP, w);
#pragma unroll
            for (int pair = 0; pair <= PAIRS; ++pair) {
                if (pair + 1 < PAIRS) ask_columns<KB, DT>(here, qt_0, pair + 1, x[(pair + 1) & 1]);
                else if (pair + 1 == PAIRS) ask_columns<RB, ET>(here + ROT, rt_first, 0, x[(pair + 1) & 1]);
                __builtin_amdgcn_sched_barrier(0);
                // (a query that sees the key and is not finite has made dS NaN)
                if (pair < PAIRS) (void)add_columns(x[pair & 1], pair, w, mixed, dk);
                else (void)add_columns(x[pair & 1], 0, w, mixed, dr);
            }
        }
        for (int u = mine_end; some && u < units; ++u) round_begins(u + 1);
        lds_loads_done();
        store_rows(mine, dk, a.scale, to, stride, n - wave0);
        if (key < n) {
            float *part = a.part + (stat + key) * E;
#pragma unroll
            for (int c = 0; c < ET; ++c)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f32x4 *>(part + 32 * c + 8 * g + 4 * half) =
                        f32x4{dr[c][4 * g] * a.scale, dr[c][4 * g + 1] * a.scale, dr[c][4 * g + 2] * a.scale, dr[c][4 * g + 3] * a.scale};
        }
    }
}

// The heads' gradients of the rotary part, added in their order: four values a thread.
template <int E>
__global__ __launch_bounds__(256) void latent_replay_rope_kernel(LatentReplayArgs a)
{
    constexpr int QUADS = E / 4;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long pos = i / QUADS;
    if (pos >= (long long)a.B * a.T) return;
    const int b = (int)(pos / a.T), t = (int)(pos % a.T), col = (int)(i % QUADS) * 4;
    int n = a.n ? a.n[b] : a.T;
    if (t >= n) return;
    const float *part = a.part + ((size_t)b * a.H * a.T + t) * E + col;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int h = 0; h < a.H; ++h) sum += *reinterpret_cast<const f32x4 *>(part + (size_t)h * a.T * E);
    *reinterpret_cast<u32x2 *>(a.drope + (pos * E + col) * 2) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
}

}  // namespace ngc

// ============================================================ host side ====

using namespace ngc;

namespace {

bool latent_replay_sizes(int32_t B, int32_t T, int32_t Hq, int32_t D) { return B > 0 && T > 0 && Hq > 0 && (D == 64 || D == 128); }

int check_latent_replay(const void *q, const void *kv, const void *rope, int64_t rope_stride, int32_t B, int32_t T, int32_t Hq, int32_t D,
                        float scale, const void *out)
{
    if (!q || !kv || !rope || !out || !aligned16(q) || !aligned16(kv) || !aligned16(rope) || !aligned16(out)) return NGC_EINVAL;
    if (!latent_replay_sizes(B, T, Hq, D) || rope_stride < D / 2 || rope_stride % 8 != 0) return NGC_EINVAL;
    if (!(scale > 0.f) || !(scale <= 2.35e38f)) return NGC_EINVAL;
    if (Hq > LATENT_MOST_HEADS || T > LR_MOST_POSITIONS || rope_stride > 1 << 20) return NGC_EUNSUPPORTED;
    if (!launchable((long long)((T + KV_BLOCK - 1) / KV_BLOCK) * B * Hq, 2 * KV_GROUPS * 64)) return NGC_EUNSUPPORTED;
    return NGC_OK;
}

LatentReplayArgs latent_replay_args(const void *q, const void *kv, const void *rope, int64_t rope_stride, const int32_t *death, const int32_t *n,
                                    int32_t B, int32_t T, int32_t Hq, float scale)
{
    LatentReplayArgs a{};
    a.q = reinterpret_cast<const unsigned char *>(q);
    a.kv = reinterpret_cast<const unsigned char *>(kv);
    a.rope = reinterpret_cast<const unsigned char *>(rope);
    a.death = death; a.n = n;
    a.rope_row = (size_t)rope_stride * 2;
    a.B = B; a.T = T; a.H = Hq;
    a.scale = scale;
    a.scale_log2e = scale * 1.4426950408889634f;
    return a;
}

size_t latent_replay_stats_bytes(int32_t B, int32_t T, int32_t Hq) { return align256((size_t)B * Hq * T * 2 * sizeof(float)); }

int launch_blocks(const void *fn, const LatentReplayArgs &args, int block, int threads, size_t lds, hipStream_t st)
{
    LatentReplayArgs a = args;
    if (lds > 64 * 1024) NGC_HIP_CHECK(hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    return launch(fn, dim3((unsigned)((a.T + block - 1) / block * a.B * a.H)), dim3(threads), lds, st, a);
}

}  // namespace

extern "C" size_t ngc_latent_replay_workspace_bytes(int32_t B, int32_t T, int32_t Hq, int32_t D)
{
    if (!latent_replay_sizes(B, T, Hq, D)) return 0;
    return latent_replay_stats_bytes(B, T, Hq) + (size_t)B * Hq * T * (D / 2) * sizeof(float);
}

extern "C" int ngc_latent_replay_attn(const void *q, const void *kv, const void *rope, int64_t rope_stride, const int32_t *death,
                                      const int32_t *n, int32_t B, int32_t T, int32_t Hq, int32_t D, float scale, void *out,
                                      float *lse_out, void *stream)
{
    const int rc = check_latent_replay(q, kv, rope, rope_stride, B, T, Hq, D, scale, out);
    if (rc) return rc;
    LatentReplayArgs a = latent_replay_args(q, kv, rope, rope_stride, death, n, B, T, Hq, scale);
    a.out = reinterpret_cast<unsigned char *>(out);
    a.lse = lse_out;
    const void *fn = D == 128 ? reinterpret_cast<const void *>(&latent_replay_kernel<128>)
                              : reinterpret_cast<const void *>(&latent_replay_kernel<64>);
    return launch_blocks(fn, a, LR_BLOCK, LR_WAVES * 64, D == 128 ? KeyTiles<128, true>::BYTES : KeyTiles<64, true>::BYTES, (hipStream_t)stream);
}

extern "C" int ngc_latent_replay_attn_backward(const void *q, const void *kv, const void *rope, int64_t rope_stride, const int32_t *death,
                                               const int32_t *n, const void *out, const float *lse, const void *dout, int32_t B,
                                               int32_t T, int32_t Hq, int32_t D, float scale, void *dq, void *dkv, void *drope, void *ws,
                                               size_t ws_bytes, void *stream)
{
    int rc = check_latent_replay(q, kv, rope, rope_stride, B, T, Hq, D, scale, out);
    if (rc) return rc;
    if (!lse || !dout || !dq || !dkv || !drope || !ws) return NGC_EINVAL;
    if (!aligned16(dout) || !aligned16(dq) || !aligned16(dkv) || !aligned16(drope) || !aligned16(ws)) return NGC_EINVAL;
    if (ws_bytes < ngc_latent_replay_workspace_bytes(B, T, Hq, D)) return NGC_ENOSPC;
    LatentReplayArgs a = latent_replay_args(q, kv, rope, rope_stride, death, n, B, T, Hq, scale);
    a.out = reinterpret_cast<unsigned char *>(const_cast<void *>(out));    // (only read)
    a.lse = const_cast<float *>(lse);
    a.dout = reinterpret_cast<const unsigned char *>(dout);
    a.dq = reinterpret_cast<unsigned char *>(dq);
    a.dkv = reinterpret_cast<unsigned char *>(dkv);
    a.drope = reinterpret_cast<unsigned char *>(drope);
    a.stats = reinterpret_cast<float *>(ws);
    a.part = reinterpret_cast<float *>(reinterpret_cast<unsigned char *>(ws) + latent_replay_stats_bytes(B, T, Hq));
    hipStream_t st = (hipStream_t)stream;
    const size_t lds = D == 128 ? KeyTiles<128, true>::BYTES : KeyTiles<64, true>::BYTES;
    const void *fn = D == 128 ? reinterpret_cast<const void *>(&latent_replay_dq_kernel<128>)
                              : reinterpret_cast<const void *>(&latent_replay_dq_kernel<64>);
    rc = launch_blocks(fn, a, LR_BLOCK, LR_WAVES * 64, lds, st);
    if (rc) return rc;
    fn = D == 128 ? reinterpret_cast<const void *>(&latent_replay_dkv_kernel<128>) : reinterpret_cast<const void *>(&latent_replay_dkv_kernel<64>);
    rc = launch_blocks(fn, a, KV_BLOCK, 2 * KV_GROUPS * 64, kv_slots(D) * (lds / 4 + 2 * LR_STEP * sizeof(float)) + KV_GROUPS * 2 * 4096, st);
    if (rc) return rc;
    const long long threads = (long long)B * T * (D / 2 / 4);
    fn = D == 128 ? reinterpret_cast<const void *>(&latent_replay_rope_kernel<64>) : reinterpret_cast<const void *>(&latent_replay_rope_kernel<32>);
    return launch(fn, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a);
}
