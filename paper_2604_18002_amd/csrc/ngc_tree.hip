// Attention for a tree of drafted tokens over the surviving cache rows on gfx950.
//
// A sequence has W drafted tokens (nodes) behind its cache; node i attends to all n cached rows and to those drafted
// nodes that lie on its way from the root, itself included:
//
//     out_i = softmax_j( scale <q_i, k_j> ) v_j   over   j in cache  and  j in anc(i) = {i, parent(i), ..}.
//
// The drafted rows live in buffers of their own, as a projection writes them ([B][W][Hkv][D]): nothing that may be
// rejected enters the cache.  A KV head serves R = W G query rows (G query heads per node), so a segment's K and V are
// read once for all of them: 4 D R flops for 4 D bytes, memory bound below ~64 rows, bound by the products beyond.
//
// S^T = K Q^T and O^T = V^T P by 32x32x16 matrix instructions: one query row per lane % 32, so all soft-max state is lane
// local and crosses lanes once, between the two halves; one pass over the keys with a running maximum and sum.  K and V go
// from memory straight into LDS, V is read transposed from there.  Two kernels:
//   tree_narrow_kernel  a workgroup has 32 query rows; every wave has all of them and walks key tiles of its own, without a
//                       barrier;
//   tree_attn_kernel    4 waves share tiles of 64 keys, wave (wq, wk) has row block wq of WQ = 2 or 4 and part wk of the keys;
//                       more than 128 rows are several workgroups.
// The first reads a segment's keys once for every 32 rows, from L2 while all of them are at work at the same time, and is the
// faster one where little else goes on (tree_shape() has the rule and its figures).
// The drafted rows are one more tile behind those of the cache, masked by a word of ancestor bits per lane.
//
// P enters the second product as three bf16 parts (24 bits): with two (2^-17 of an entry lost at most) the output would be
// 2.2e-6 (of its norm) from the 64-bit result, where products in 32 bits are 3e-7 to 1.2e-6 away; with three it is 1.2e-7 to
// 7.2e-7.  That is 4 products per 32x32x32 block in place of 3.
//
// Few segments are shared by S workgroups that take tiles in turn; each leaves an unnormalised partial (max, sum, O) and
// a second launch joins them (tree_splits() has the rule and its figures).
//
// What it measures (one layer, HIP graph): 128 x 28/4 heads x 2713 rows, chains of 4 (R = 28) 113.5 us, the rows at 6.4 TB/s;
// with lengths of 1894-3533 121 us (the last workgroups have the chip to themselves); trees of 9 (R = 63) 127 us; 32 x 28/4 x
// 4096, trees of 64 (R = 448) 239 us, 507 TFLOP/s by the formula, 1020 as issued; the large matrix product of this card reaches 1241.
// What bounds the products: a 32x32x16 product occupies the matrix unit for 32 cycles and keeps the vector unit from issuing
// for about 16 of them (a loop of 1 product and 16 multiply-adds takes 38 ns on one wave, 8 of them 22.6, 4 of them 15.1), so
// the 32 products and ~200 vector instructions of a step of 32 keys take ~1600 cycles wherever they stand.
// Measured and not kept: the exponentials of 16 keys between the products of the 16 before (no change, see above); the
// remainders of P by a bf16 dot product (3 instead of 5 instructions a pair: 4 % slower); 64 rows in a wave of tree_narrow_kernel
// (one wave per SIMD: 128 segments x 1493 rows 30 -> 32-40 us); 8 waves and 128 keys per workgroup (R 33-64: 0.90-1.04 of the time,
// R 65-128: 0.96-1.12); joining the partials in the same launch by tickets (as fast or slower, and state to keep); 8 waves with 32 rows (one workgroup on a CU
// gets its rows at ~50 KB a microsecond however many waves ask: 0.82-1.12, 0.98 at the best choice of each geometry).
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/ngc.h"
#include "ngc_device.h"
#include "ngc_workspace.h"

namespace ngc {

constexpr int TREE_WAVES = 4;
constexpr int TREE_QW = 32;                 // query rows per wave
constexpr int TREE_MT = 32;                 // keys per step of the math
constexpr int TREE_PARTS = 3;               // bf16 parts of P
// Start of the running max: the smallest finite number, so that 2^(x - m) is 0 for x = -inf without a special case and every finite
// score is above it or equal to it.
constexpr float TREE_M_INIT = -FLT_MAX;
// The reference of the exponents moves only when a maximum has outgrown it by 2^8.
constexpr float TREE_LAZY = 8.0f;
// Rows whose maximum lies beyond this are computed again, key by key (see odd_row()): half a step of the maximum, rounded to 32 bits,
// is a common factor in all weights, 2 at 2^24, but more than 2^x can hold from 2^31 on.
constexpr float TREE_FAR = 16777216.0f;

struct TreeArgs {
    const unsigned char *k, *v;         // the cache's rows, or the pools
    const int32_t *len;
    const unsigned char *k_draft, *v_draft;   // bf16 [launch layers][B][W][Hkv][D]
    const int32_t *parent;              // [B][W]
    const int32_t *n_draft;             // [B] or nullptr
    const unsigned char *q;             // bf16 [launch layers][B][W][Hq][D]
    float *out;                         // fp32, as q
    float *lse_out;                     // fp32 [launch layers][B][W][Hq] or nullptr
    float *part_o;                      // [segments of the launch][S][R][D]
    float *part_ml;                     // [segments of the launch][S][R][2]
    int32_t *status;
    int seg0, nseg, blocks, S, W, G, B, Hkv, cap;
    float scale_log2e;
    const int32_t *table;               // paged layout only
    int max_pages, num_pages, page_shift;
};

// How a segment's keys are dealt out: tiles of `keys`, the drafted rows in tiles of their own, `waves` tiles to a workgroup at a time.
struct TreeTiles {
    int keys, waves;
    __host__ __device__ int groups(int n, int nd) const
    {
        return ((n + keys - 1) / keys + (nd + keys - 1) / keys + waves - 1) / waves;
    }
};

// A word that nobody writes during the launch, at a wave-uniform address: through the scalar unit.  (Behind a load to LDS the
// compiler takes any memory for changed, loads the word into a vector register and waits for everything in front of it.)
__device__ __forceinline__ int32_t constant_word(const int32_t *p)
{
    return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>((uintptr_t)p);
}

// What a workgroup has to know about its segment.
struct TreeSegment {
    int seg_local, h;
    size_t seq;                         // launch layer * B + sequence
    int b;
    int n, nd;                          // rows in the cache, drafted nodes; as they are in memory until clamp()

    __device__ __forceinline__ TreeSegment(const TreeArgs &a, int seg_local)
        : seg_local(seg_local), h(seg_local % a.Hkv), seq((size_t)(seg_local / a.Hkv)),
          b((int)(seq % a.B)), n(constant_word(a.len + a.seg0 + seg_local)),
          nd(a.n_draft ? constant_word(a.n_draft + b) : a.W)
    {
    }
    __device__ __forceinline__ void clamp(const TreeArgs &a, bool counts)
    {
        if (n < 0 || n > a.cap) {
            if (counts) atomicAdd(&a.status[NGC_STATUS_LEN_CLAMPED], 1);
            n = n < 0 ? 0 : a.cap;
        }
        if (nd < 0 || nd > a.W) {
            if (counts && h == 0) atomicAdd(&a.status[NGC_STATUS_BAD_TREE], 1);
            nd = nd < 0 ? 0 : a.W;
        }
    }
};

// A workgroup's segment and row block.  Workgroups go round-robin to the 8 XCDs: the row blocks of a segment follow one another on
// one of them, so that its rows come from memory once, while they are at work together (with the row block as the slowest
// coordinate instead, 100 segments x 3000 rows in 6 blocks of 32 take 119 us in place of 87; 128 x 4096 in 4 of 128 248, not 245).
struct TreePlace {
    int seg, block;
    __device__ __forceinline__ TreePlace(const TreeArgs &a) : seg((int)blockIdx.x), block(0)
    {
        if (a.blocks == 1) return;
        const int first = (int)(blockIdx.x / (8u * (unsigned)a.blocks)) * 8, at = (int)blockIdx.x - first * a.blocks;
        const int here = a.nseg - first < 8 ? a.nseg - first : 8;
        block = at / here;
        seg = first + at - block * here;
    }
};

// The bits of a node's ancestors, itself included, in lane = node; steps of 1, 2, 4, .. up the tree.  A parent that does
// not come before its child is taken for none.
__device__ __forceinline__ uint64_t tree_ancestors(const TreeArgs &a, int up, int nd, bool counts)      // up: of node = lane
{
    const int lane = lane_id();
    up = lane < nd ? up : -1;
    const bool bad = up < -1 || up >= lane;
    const uint64_t bad_nodes = __ballot(bad && lane < nd);
    if (counts && lane == 0 && bad_nodes) atomicAdd(&a.status[NGC_STATUS_BAD_TREE], __popcll(bad_nodes));
    up = bad ? -1 : up;
    uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
#pragma unroll
    for (int step = 0; step < 6; ++step) {
        const int from = up < 0 ? lane : up;
        lo |= (uint32_t)__shfl((int)lo, from);
        hi |= (uint32_t)__shfl((int)hi, from);
        const int next = __shfl(up, from);
        up = up < 0 ? -1 : next;
    }
    return (uint64_t)hi << 32 | lo;
}

// The sums are rescaled only when a maximum has outgrown the reference: any reference gives the same quotients, and
// probabilities up to 2^TREE_LAZY lose nothing in fp32 or in their bf16 parts.  `top`: of the row, in the scaled domain.
template <int DT>
__device__ __forceinline__ void raise_reference(float top, float &m_run, float &l_run, f32x16 (&oacc)[DT])
{
    if (__ballot(top > m_run + TREE_LAZY)) {
        const float m_new = max_no_nan(m_run, top);
        const float alpha = (m_new == m_run) ? 1.0f : fast_exp2(m_run - m_new);
        l_run *= alpha;
#pragma unroll
        for (int c = 0; c < DT; ++c) oacc[c] *= alpha;
        m_run = m_new;
    }
}

// P of 32 keys from their raw scores with this lane's row, in bf16 parts; returns its sum.  The (positive) scale is applied inside the
// exponent's multiply-add.
__device__ __forceinline__ float tree_weights(const f32x16 &sc, float scale_log2e, float m_run, uint32_t (&part)[TREE_PARTS][8])
{
    const float neg_m = -m_run;
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f32x2 p = {fast_exp2(__builtin_fmaf(sc[2 * e], scale_log2e, neg_m)),       // -inf gives 0
                   fast_exp2(__builtin_fmaf(sc[2 * e + 1], scale_log2e, neg_m))};
        psum += p[0] + p[1];
#pragma unroll
        for (int i = 0; i < TREE_PARTS; ++i) {        // rounded to bf16; the remainder is exact
            const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
            part[i][e] = w;
            if (i + 1 < TREE_PARTS) p = f32x2{p[0] - __uint_as_float(w << 16), p[1] - __uint_as_float(w & 0xFFFF0000u)};
        }
    }
    return psum;
}

// O += P V for 32 keys.  vop: [16-key chunk][d tile][keys 4 half .. +3, 8 + 4 half .. +3].
template <int DT>
__device__ __forceinline__ void add_products(const u32x2 (&vop)[2][DT][2], const uint32_t (&part)[TREE_PARTS][8], f32x16 (&oacc)[DT])
{
#pragma unroll
    for (int kc = 0; kc < 2; ++kc) {
        bf16x8 v[DT];
#pragma unroll
        for (int c = 0; c < DT; ++c)
            v[c] = __builtin_bit_cast(bf16x8, u32x4{vop[kc][c][0][0], vop[kc][c][0][1], vop[kc][c][1][0], vop[kc][c][1][1]});
#pragma unroll
        for (int i = 0; i < TREE_PARTS; ++i) {
            const bf16x8 p = __builtin_bit_cast(bf16x8, u32x4{part[i][4 * kc], part[i][4 * kc + 1], part[i][4 * kc + 2],
                                                              part[i][4 * kc + 3]});
#pragma unroll
            for (int c = 0; c < DT; ++c) oacc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[c], p, oacc[c], 0, 0, 0);
        }
    }
}

// Values of drafted V rows that are not finite would reach rows that do not see them, through a product with P = 0.  They become 0 in
// LDS, in every slot of the tile that is multiplied (behind the last drafted row stand copies of it), and are added, by themselves, to
// the rows that see them.
__device__ __forceinline__ bool take_out_odd_values(unsigned char *piece)      // of 16 bytes; whether it had any
{
    u32x4 x = *reinterpret_cast<const u32x4 *>(piece);
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if ((x[e] & 0x7F80u) == 0x7F80u) { odd = true; x[e] &= 0xFFFF0000u; }
        if ((x[e] & 0x7F800000u) == 0x7F800000u) { odd = true; x[e] &= 0xFFFFu; }
    }
    if (odd) *reinterpret_cast<u32x4 *>(piece) = x;
    return odd;
}
// Those of up to 32 drafted rows, `stride` bytes apart in memory, that `sees` has a bit for.
template <int DT>
__device__ __forceinline__ void add_odd_values(const unsigned char *rows, uint32_t stride, int count, uint32_t sees, f32x16 (&oacc)[DT])
{
    const int half = lane_id() >> 5;
    for (int j = 0; j < count; ++j) {
        const bool seen = ((sees >> j) & 1u) != 0;
        // of lane half: d = 32 c + 8 g + 4 half + i.  (The address is made opaque: nothing of it is kept over the loop.)
        const unsigned char *row = rows + (size_t)j * stride + half * 8;
        __asm__ volatile("" : "+v"(row));
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const u32x2 x = *reinterpret_cast<const u32x2 *>(row + (32 * c + 8 * g) * 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t bits = i & 1 ? x[i / 2] & 0xFFFF0000u : x[i / 2] << 16;
                    if (seen && (bits & 0x7F800000u) == 0x7F800000u) oacc[c][4 * g + i] += __uint_as_float(bits);
                }
            }
    }
}

// Whether a row has to be looked at again: four of its values are not all finite (0 x is NaN for those; a sum that is not finite though they
// are is looked at in vain), or its scores are far.
__device__ __forceinline__ bool is_odd(f32x4 o, float m)
{
    return 0.f * ((o[0] + o[1]) + (o[2] + o[3])) != 0.f || fabsf(m) > TREE_FAR;
}

// Four values (of D, by D / 4 consecutive lanes that call this together) of an output row that is odd, with its maximum m and sum of weights.
//   Infinities  By the formula, whose weights are positive, an infinity in a V row that is seen makes the output that infinity; the
//               products gave NaN, because parts of P are 0 or below 0 and weights may be 0 in 32 bits.  So what is not finite in
//               the rows that the output sees is added up by itself.
//   Far scores  A weight's exponent is the difference of two scaled scores that are rounded alike.
// Rare, and slow, key after key by a quarter of D lanes (32 x 28/4 heads x 4096 rows, trees of 64: an infinity in every segment 12 ms, all
// scores far 29; 1 x 32/8 x 16000, chains of 8: 3.2 and 8.0).
template <int D>
__device__ __forceinline__ f32x4 odd_row(int seg_local, int row, int piece, f32x4 o, float &m, float &sum)
{
#pragma clang fp contract(off)
    const bool far = fabsf(m) > TREE_FAR;
    if (!far && !(sum > 0.f && sum < INFINITY)) return o;   // scores that are not finite: NaN
    // Arguments and segment once more from where they come: nothing of this is kept in registers over the kernel's loop.
    auto args = __builtin_amdgcn_kernarg_segment_ptr();
    __asm__ volatile("" : "+s"(args));
    const TreeArgs &a = *reinterpret_cast<const TreeArgs *>((uintptr_t)args);
    TreeSegment s(a, seg_local);
    s.clamp(a, false);
    constexpr int ROW_BYTES = D * 2;
    auto value = [](u32x2 x, int e) { return __uint_as_float(e & 1 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16); };
    const u32x2 q = *reinterpret_cast<const u32x2 *>(a.q + ((s.seq * a.W + row / a.G) * (a.G * a.Hkv) + s.h * a.G + row % a.G) * ROW_BYTES + piece * 8);
    f32x4 infinities = {0.f, 0.f, 0.f, 0.f}, acc = {0.f, 0.f, 0.f, 0.f};
    float top = TREE_M_INIT, l = 0.f;
    auto add = [&](u32x2 k, u32x2 v) {
        float p = 0.f;
        if (far) {
            float score = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) score += value(q, e) * value(k, e);
#pragma unroll
            for (int step = 1; step < D / 4; step *= 2) score += __shfl_xor(score, step);
            score *= a.scale_log2e;
            if (score > top) {
                const float alpha = fast_exp2(top - score);
                l *= alpha;
                acc *= alpha;
                top = score;
            }
            p = fast_exp2(score - top);
            l += p;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float f = value(v, e);
            const bool finite = fabsf(f) < INFINITY;
            infinities[e] += finite ? 0.f : f;
            acc[e] += finite ? p * f : 0.f;
        }
    };
    auto piece_of = [&](const unsigned char *rows, size_t at) { return *reinterpret_cast<const u32x2 *>(rows + at * ROW_BYTES + piece * 8); };
    const size_t seg = (size_t)(a.seg0 + seg_local);
    constexpr int BATCH = 4;                                // asked for together
    for (int j0 = 0; j0 < s.n; j0 += BATCH) {
        u32x2 k[BATCH] = {}, v[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int j = j0 + u < s.n ? j0 + u : s.n - 1;
            size_t at = seg * a.cap + j;
            if (a.table) {
                int page = a.table[seg * a.max_pages + (j >> a.page_shift)];
                page = (page < 0 || page >= a.num_pages) ? 0 : page;
                at = ((size_t)page << a.page_shift) + (j & ((1 << a.page_shift) - 1));
            }
            v[u] = piece_of(a.v, at);
            if (far) k[u] = piece_of(a.k, at);
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u)
            if (j0 + u < s.n) add(k[u], v[u]);
        const f32x4 x = infinities;
        if (!far && x[0] != x[0] && x[1] != x[1] && x[2] != x[2] && x[3] != x[3]) return x;     // NaN: nothing more to find
    }
    for (int j = row / a.G; j >= 0;) {
        const size_t at = (s.seq * a.W + j) * a.Hkv + s.h;
        add(piece_of(a.k_draft, at), piece_of(a.v_draft, at));
        const int up = a.parent[(size_t)s.b * a.W + j];
        j = up < j ? up : -1;
    }
    if (far) {
        o = acc / l;
        m = top;
        sum = l;
    }
    if (!far || l == l)                                     // (NaN among the scores: NaN)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = infinities[e] != 0.f ? infinities[e] : o[e];
    return o;
}
// The lanes of a row decide together.
template <int D>
__device__ __forceinline__ bool row_is_odd(bool mine)
{
    const uint64_t lanes = (((uint64_t)1 << (D / 4)) - 1) << (lane_id() / (D / 4) * (D / 4));
    return (__ballot(mine) & lanes) != 0;
}

template <int D, int WQ, bool ONCE, bool PAGED>
__global__ __launch_bounds__(TREE_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2)))
void tree_attn_kernel(TreeArgs a)
{
    constexpr int WK = TREE_WAVES / WQ;
    constexpr int KT = 64;                                 // keys per LDS tile
    constexpr int STEPS = KT / (TREE_MT * WK);             // steps of a wave per tile
    constexpr int ROW_BYTES = D * 2;
    constexpr int DT = D / 32;                             // 32-wide d tiles of the second product
    constexpr int KCH = D / 16;                            // 16-wide d chunks of the first product
    constexpr int TILE_LDS = KT * ROW_BYTES;
    constexpr int PIECES = ROW_BYTES / 16;                 // 16-byte pieces per row
    constexpr int LOAD_ROWS = 64 / PIECES;                 // rows one wave-wide load brings
    constexpr int WAVE_ROWS = KT / TREE_WAVES;             // rows of a tile that a wave loads: inside one page
    constexpr int LOADS = WAVE_ROWS / LOAD_ROWS;
    constexpr int RB = TREE_QW * WQ;                       // query rows of the workgroup
    static_assert(TREE_MT * PIECES % (TREE_WAVES * 64) == 0, "a step's rows are cleaned by whole workgroups");

    __shared__ __align__(16) unsigned char lds_k0[TILE_LDS], lds_k1[TILE_LDS], lds_v0[TILE_LDS], lds_v1[TILE_LDS];
    __shared__ float red_m[TREE_WAVES][TREE_QW], red_l[TREE_WAVES][TREE_QW];

    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    const int wq = wv % WQ, wk = wv / WQ;
    const int li = lane & 31, half = lane >> 5;
    const TreePlace place(a);
    const int split = (int)blockIdx.y, block = place.block;
    TreeSegment s(a, place.seg);
    const int G = a.G, Hq = a.G * a.Hkv;
    const int row_base = block * RB, wave_row0 = row_base + wq * TREE_QW;

    // ---- asked for before the lengths have arrived: parents, queries (32 rows per wave, lane % 32 = row) and the first tile ----
    const int up = a.parent[(size_t)s.b * a.W + (lane < a.W ? lane : a.W - 1)];      // (of lanes that are no node it is not looked at)
    const int my_row = wave_row0 + li < a.W * G ? wave_row0 + li : a.W * G - 1;
    const int node = my_row / G;
    bf16x8 qop[KCH];
    {
        const unsigned char *qrow = a.q + ((s.seq * a.W + node) * Hq + s.h * G + my_row % G) * ROW_BYTES;
#pragma unroll
        for (int c = 0; c < KCH; ++c)
            qop[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qrow + c * 32 + half * 16));
    }
    const unsigned char *kseg = PAGED ? a.k : a.k + (size_t)(a.seg0 + s.seg_local) * a.cap * ROW_BYTES;
    const unsigned char *vseg = PAGED ? a.v : a.v + (size_t)(a.seg0 + s.seg_local) * a.cap * ROW_BYTES;
    const int32_t *tab = PAGED ? a.table + (size_t)(a.seg0 + s.seg_local) * a.max_pages : nullptr;
    auto row_base_of = [&](int r0) -> size_t {             // of a cached row, in bytes
        if constexpr (!PAGED) return (size_t)r0 * ROW_BYTES;
        int page = constant_word(tab + (r0 >> a.page_shift));
        page = (page < 0 || page >= a.num_pages) ? 0 : page;          // never leave the pool
        return (((size_t)page << a.page_shift) + (r0 & ((1 << a.page_shift) - 1))) * ROW_BYTES;
    };
    // Rows of a tile go straight from memory to LDS: a wave-wide load brings LOAD_ROWS whole rows, lane after lane.  The K
    // pieces of row r are stored at slot (piece ^ (r & SWZ)), so that reading one piece of 32 consecutive rows meets every
    // bank; the V pieces at (piece ^ v_swizzle(r)), so that reading 32 bytes of 4 consecutive rows does.
    constexpr int SWZ = PIECES - 1;
    auto v_swizzle = [](int r) { return (2 * r) & (PIECES < 16 ? SWZ : 7); };
    auto k_swizzle = [](int r) { return r & SWZ; };
    const int lrow = lane / PIECES, lslot = lane % PIECES;
    auto load_row = [&](const unsigned char *row, int slot_row, unsigned char *to, auto swizzle) {
        const unsigned char *at = row + (uint32_t)(lslot ^ swizzle(slot_row + lrow)) * 16u;
        if constexpr (ONCE) load_once_to_lds16(at, to + slot_row * ROW_BYTES);
        else load_to_lds16(at, to + slot_row * ROW_BYTES);
    };
    int t = split;
    const int S = a.S;
    {   // the first tile as if it were full (rows behind the capacity are the last one again): where it is not, it is asked for again
        int r0 = t * KT + wv * WAVE_ROWS;
        r0 = r0 < a.cap ? r0 : a.cap - 1;
        const size_t base0 = row_base_of(r0);
        const int most = a.cap - 1 - r0;
#pragma unroll
        for (int r = 0; r < LOADS; ++r) {
            const int row = r * LOAD_ROWS + lrow < most ? r * LOAD_ROWS + lrow : most;
            load_row(kseg + base0 + (uint32_t)row * ROW_BYTES, wv * WAVE_ROWS + r * LOAD_ROWS, lds_k0, k_swizzle);
        }
        __builtin_amdgcn_sched_barrier(0);                 // in this order: it is waited for in this order
#pragma unroll
        for (int r = 0; r < LOADS; ++r) {
            const int row = r * LOAD_ROWS + lrow < most ? r * LOAD_ROWS + lrow : most;
            load_row(vseg + base0 + (uint32_t)row * ROW_BYTES, wv * WAVE_ROWS + r * LOAD_ROWS, lds_v0, v_swizzle);
        }
        __asm__ volatile("" ::: "memory");
    }
    s.clamp(a, threadIdx.x == 0 && split == 0 && block == 0);
    const int R = s.nd * G;                                // query rows that there are
    const int n = s.n, nd = s.nd;
    const int cache_tiles = (n + KT - 1) / KT;
    const int tiles = cache_tiles + 1;                     // the last one: the drafted rows
    if (row_base >= R || split >= tiles) {                 // (uniform; the merge counts tiles too)
        __builtin_amdgcn_s_waitcnt(0x0F70);                // nothing may be on its way to LDS that is not this workgroup's any more
        return;
    }
    const bool active = wave_row0 < R;                     // (a last block may have waves without query rows)
    const size_t draft_at = ((s.seq * a.W) * a.Hkv + s.h) * ROW_BYTES;
    const uint32_t draft_row = (uint32_t)a.Hkv * ROW_BYTES;
    // First of the wave's rows in cache tile t, the segment's last row where there are none; paged: its place in the pools.
    auto first_row = [&](int t) {
        const int r0 = t * KT + wv * WAVE_ROWS;
        return r0 < n ? r0 : n - 1;
    };
    auto tile_base = [&](int t) -> size_t {                // of the wave's first row, in bytes
        return t >= cache_tiles ? draft_at : row_base_of(first_row(t));
    };
    auto load = [&](int t, size_t base, const unsigned char *cached, const unsigned char *drafts, unsigned char *to, auto swizzle) {
        const bool drafted = t >= cache_tiles;
        const unsigned char *src = drafted ? drafts + base : cached + base;
        const uint32_t stride = drafted ? draft_row : (uint32_t)ROW_BYTES;
        const int first = drafted ? 0 : first_row(t);                  // what `base` names
        const int last = drafted ? nd - 1 : n - 1;
        const int start = drafted ? wv * WAVE_ROWS : first;
#pragma unroll
        for (int r = 0; r < LOADS; ++r) {
            int row = start + r * LOAD_ROWS + lrow;
            row = row < last ? row : last;
            load_row(src + (uint32_t)(row - first) * stride, wv * WAVE_ROWS + r * LOAD_ROWS, to, swizzle);
        }
    };
    auto load_k = [&](int t, size_t base, unsigned char *to) { load(t, base, kseg, a.k_draft, to, k_swizzle); };
    auto load_v = [&](int t, size_t base, unsigned char *to) { load(t, base, vseg, a.v_draft, to, v_swizzle); };

    // Asked for in this order, here and in the loop: K of a tile, its V, K of the next tile, its V, ..
    if ((t + 1) * KT > n) {
        const size_t base0 = tile_base(t);
        __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): not before what was asked for in vain has arrived
        __asm__ volatile("" ::: "memory");
        load_k(t, base0, lds_k0);
        load_v(t, base0, lds_v0);
    }
    size_t base1 = tile_base(t + S), base2 = tile_base(t + 2 * S);     // of the next tile and the one after it

    uint32_t sees_lo, sees_hi;             // drafted nodes that this lane's row sees
    {
        const uint64_t anc = tree_ancestors(a, up, nd, wv == 0 && split == 0 && block == 0 && s.h == 0);
        sees_lo = (uint32_t)__shfl((int)(uint32_t)anc, node);
        sees_hi = (uint32_t)__shfl((int)(uint32_t)(anc >> 32), node);
    }

    f32x16 oacc[DT];
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[c][r] = 0.f;
    float m_run = TREE_M_INIT, l_run = 0.f;

    // LDS offsets of this lane's operands.  K: piece 2c + half of row li.  V: a transposing read gives lane x of 16 the
    // column d0 + x of 4 rows if lane x points at the 4 values from d0 + 4 (x % 4) of row x / 4; the rows are the keys
    // its half contracts over in a 16-key chunk (4 half .. +3 and 8 + 4 half .. +3: the order the scores come in).
    uint32_t koff[KCH];
#pragma unroll
    for (int c = 0; c < KCH; ++c) koff[c] = (uint32_t)(li * ROW_BYTES + (((2 * c + half) ^ (li & SWZ)) * 16));
    uint32_t vrd[DT];
    {
        const int row = 4 * half + (lane & 15) / 4;       // + 16 kc + 8 g: the same row modulo 8 for every g, kc
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            const int d0 = 32 * c + (lane & 16) + 4 * (lane & 3);
            vrd[c] = (uint32_t)(row * ROW_BYTES + (((d0 / 8) ^ v_swizzle(row)) * 16) + (d0 % 8) * 2);
        }
    }

    // Raw scores of 32 keys with this lane's row: register r holds key 8 (r / 4) + 4 half + r % 4 of them.
    auto scores = [&](const unsigned char *lk) {
        f32x16 sc;
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = 0.f;
        u32x4 kop[KCH];
#pragma unroll
        for (int c = 0; c < KCH; ++c) kop[c] = *reinterpret_cast<const u32x4 *>(lk + koff[c]);
#pragma unroll
        for (int c = 0; c < KCH; ++c)
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kop[c]), qop[c], sc, 0, 0, 0);
        return sc;
    };
    // O += P V for 32 keys and their raw scores.
    auto add_values = [&](const unsigned char *lv, const f32x16 &sc) {
        u32x2 vop[2][DT][2];
#pragma unroll
        for (int kc = 0; kc < 2; ++kc)
#pragma unroll
            for (int c = 0; c < DT; ++c)
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    vop[kc][c][g] = read_transposed16(lv + vrd[c] + (16 * kc + 8 * g) * ROW_BYTES);
        __builtin_amdgcn_sched_barrier(0);     // the V rows arrive while the exponentials are made
        uint32_t part[TREE_PARTS][8];
        l_run += tree_weights(sc, a.scale_log2e, m_run, part);
        add_products(vop, part, oacc);
    };

    // One tile, in two parts with a barrier in front of each.  In front of the first: everybody's K rows are there, and the V
    // buffer of the tile before is read out, so the next tile's V is asked for.  In front of the second: everybody's V rows
    // are there, and the K buffer is read out, so K of the tile after the next is asked for.  Each wait is for all but the
    // newest two halves of a tile (48 KB of a workgroup's 64 are on their way or waited for at any time), except in a
    // workgroup's last two tiles, where less follows.
    constexpr int WAIT_OLDER = 0x0070 | (2 * LOADS);       // vmcnt(2 LOADS); lgkmcnt(0): what this wave has read has arrived
    constexpr int WAIT_ALL = 0x0070;                       // vmcnt(0) lgkmcnt(0)
    auto tile_step = [&](auto main, unsigned char *lk, unsigned char *lv, unsigned char *next_v) {
        constexpr bool MAIN = decltype(main)::value;       // two more tiles follow: this one is a full tile of the cache
        __builtin_amdgcn_s_waitcnt(MAIN ? WAIT_OLDER : WAIT_ALL);
        __asm__ volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" ::: "memory");
        if (MAIN || t + S < tiles) load_v(t + S, base1, next_v);
        __builtin_amdgcn_sched_barrier(0);
        const bool drafted = !MAIN && t >= cache_tiles;
        f32x16 sc[STEPS];
        int steps = STEPS;                                 // of this wave that have keys
        if (active) {
            if (!MAIN) {
                const int keys = (drafted ? nd : n - t * KT) - wk * STEPS * TREE_MT;
                steps = keys <= 0 ? 0 : keys <= TREE_MT ? 1 : STEPS;
            }
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                if (!MAIN && st >= steps) break;
                sc[st] = scores(lk + (wk * STEPS + st) * TREE_MT * ROW_BYTES);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        bool odd = false;
        __builtin_amdgcn_s_waitcnt(MAIN ? WAIT_OLDER : WAIT_ALL);
        __asm__ volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" ::: "memory");
        if (MAIN || t + 2 * S < tiles) load_k(t + 2 * S, base2, lk);
        base1 = base2;
        base2 = tile_base(t + 3 * S);
        if (drafted) {
            bool any = false;
            for (int first = 0; first < nd; first += TREE_MT)
#pragma unroll
                for (int i = 0; i < TREE_MT * PIECES; i += TREE_WAVES * 64)
                    any |= take_out_odd_values(lv + (first * PIECES + i + (int)threadIdx.x) * 16);
            odd = __syncthreads_or(any) != 0;
        }
        if (!active || steps == 0) return;
        __builtin_amdgcn_sched_barrier(0);
        float top = -INFINITY;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            if (!MAIN && st >= steps) break;
            if constexpr (!MAIN) {
                const int at = (wk * STEPS + st) * TREE_MT, left = n - (t * KT + at);
                const uint32_t sees = drafted ? (at == 0 ? sees_lo : sees_hi) : left >= TREE_MT ? 0xFFFFFFFFu : (1u << left) - 1u;
                const uint32_t w = sees >> (4 * half);
#pragma unroll
                for (int r = 0; r < 16; ++r) sc[st][r] = (w >> (8 * (r / 4) + r % 4)) & 1u ? sc[st][r] : -INFINITY;
            }
#pragma unroll
            for (int r = 0; r < 16; r += 2) top = max_or_nan(max_or_nan(top, sc[st][r]), sc[st][r + 1]);
        }
        raise_reference(half_rows_max(top) * a.scale_log2e, m_run, l_run, oacc);
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            if (!MAIN && st >= steps) break;
            add_values(lv + (wk * STEPS + st) * TREE_MT * ROW_BYTES, sc[st]);
        }
        if (odd && wk == 0) {
#pragma unroll 1
            for (int j = 0; j < nd; j += 32)
                add_odd_values(a.v_draft + draft_at + (size_t)j * draft_row, draft_row, nd - j < 32 ? nd - j : 32, j == 0 ? sees_lo : sees_hi, oacc);
        }
    };
    // (The compiler keeps account of what is on its way and makes a read of a buffer wait for it: it must find the same order on
    // every way into the loop, or it has everything waited for.  The waits above are its builtin for the same reason.)
    if (t + 3 * S < tiles) {
        load_k(t + S, base1, lds_k1);
        do {
            tile_step(std::true_type{}, lds_k0, lds_v0, lds_v1);
            t += S;
            tile_step(std::true_type{}, lds_k1, lds_v1, lds_v0);
            t += S;
        } while (t + 3 * S < tiles);
    } else if (t + S < tiles) {
        load_k(t + S, base1, lds_k1);
    }
    for (bool even = true; t < tiles; t += S, even = !even)
        tile_step(std::false_type{}, even ? lds_k0 : lds_k1, even ? lds_v0 : lds_v1, even ? lds_v1 : lds_v0);

    // ---- join the waves of a row block, normalise, write --------------------------
    // O goes through LDS, so that a row's D values leave as whole cache lines: a wave's own 32 rows in its part of the tile
    // buffers, 16-byte piece p of row r at slot p ^ r.
    constexpr int OP = D / 4;                              // 16-byte pieces per output row
    constexpr int O_LDS = TREE_QW * D * 4;
    static_assert(O_LDS <= TILE_LDS, "a wave's output rows fit a tile buffer");
    __syncthreads();                                       // every wave is done with the tiles
    auto rows_of = [&](int w) { return w == 0 ? lds_k0 : w == 1 ? lds_k1 : w == 2 ? lds_v0 : lds_v1; };
    {
        const float l = half_rows_sum(l_run);
        if (half == 0) { red_m[wv][li] = active ? m_run : TREE_M_INIT; red_l[wv][li] = active ? l : 0.f; }
        unsigned char *mine = rows_of(wv);
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {   // register (c, 4g + i) holds d = 32 c + 8 g + 4 half + i
                const int piece = 8 * c + 2 * g + half;
                *reinterpret_cast<f32x4 *>(mine + li * (D * 4) + ((piece ^ li) & (OP - 1)) * 16) =
                    f32x4{oacc[c][4 * g], oacc[c][4 * g + 1], oacc[c][4 * g + 2], oacc[c][4 * g + 3]};
            }
    }
    __syncthreads();
    constexpr int ROWS = TREE_WAVES * 64 / OP;             // rows per workgroup-wide store
    const int piece = threadIdx.x % OP;
    auto joined = [&](int r0, float &m_all, float &l_all) {
        const int q = r0 / TREE_QW, i = r0 % TREE_QW;
        float f[WK];
        m_all = TREE_M_INIT, l_all = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) m_all = fmaxf(m_all, red_m[w * WQ + q][i]);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WK; ++w) {
            f[w] = WK == 1 ? 1.f : fast_exp2(red_m[w * WQ + q][i] - m_all);
            l_all += red_l[w * WQ + q][i] * f[w];
            o += *reinterpret_cast<const f32x4 *>(rows_of(w * WQ + q) + i * (D * 4) + ((piece ^ i) & (OP - 1)) * 16) * f[w];
        }
        return o;
    };
    float m_all, l_all;
    auto write = [&](int row, f32x4 o, auto store) {
        const size_t at = (s.seq * a.W + row / G) * Hq + s.h * G + row % G;
        store(o, reinterpret_cast<f32x4 *>(a.out + at * D) + piece);
        if (a.lse_out && piece == 0) a.lse_out[at] = (m_all + __log2f(l_all)) * 0.6931471805599453f;
    };
    bool odd = false;
    for (int r0 = threadIdx.x / OP; r0 < RB; r0 += ROWS) {
        const int row = row_base + r0;
        if (row >= R) break;
        f32x4 o = joined(r0, m_all, l_all);
        if (a.S == 1 || tiles == 1) {
            o *= 1.0f / l_all;          // (with four quotients, a rounding less, 256 x 12/2 heads x 100 rows, chains of 6, take 16.3 us, not 15.95)
            odd |= is_odd(o, m_all);
            write(row, o, [](f32x4 x, f32x4 *at) { __builtin_nontemporal_store(x, at); });
        } else {
            const size_t at = ((size_t)s.seg_local * a.S + split) * (size_t)(a.W * G) + row;
            *(reinterpret_cast<f32x4 *>(a.part_o + at * D) + piece) = o;
            if (piece == 0) *reinterpret_cast<f32x2 *>(a.part_ml + at * 2) = f32x2{m_all, l_all};
        }
    }
    if (__ballot(odd) == 0) return;
    for (int r0 = threadIdx.x / OP; r0 < RB && row_base + r0 < R; r0 += ROWS) {
        const f32x4 o = joined(r0, m_all, l_all) * (1.0f / l_all);
        if (row_is_odd<D>(is_odd(o, m_all)))
            write(row_base + r0, odd_row<D>(s.seg_local, row_base + r0, piece, o, m_all, l_all), [](f32x4 x, f32x4 *at) { *at = x; });
    }
}

// 32 query rows.  Every wave walks key tiles of its own, 32 keys each (tile t belongs to wave t % 4 of workgroup
// (t / 4) % S), through its own part of LDS: no barrier until the end.  A tile's K and V have one buffer each; the next
// tile's K is requested as soon as this one's has been read into registers, its V likewise, so that 8 to 16 KB of every
// wave are on their way, two workgroups a CU.  The drafted rows are the last one or two tiles.
template <int D, bool ONCE, bool PAGED>
__global__ __launch_bounds__(TREE_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2)))
void tree_narrow_kernel(TreeArgs a)
{
    constexpr int ROW_BYTES = D * 2;
    constexpr int DT = D / 32, KCH = D / 16;
    constexpr int TILE_LDS = TREE_MT * ROW_BYTES;
    constexpr int PIECES = ROW_BYTES / 16;
    constexpr int LOAD_ROWS = 64 / PIECES;
    constexpr int LOADS = TREE_MT / LOAD_ROWS;
    constexpr int OP = D / 4;                              // 16-byte pieces per output row

    __shared__ __align__(16) unsigned char lds_k[TREE_WAVES * TILE_LDS], lds_v[TREE_WAVES * TILE_LDS];
    __shared__ float red_m[TREE_WAVES][TREE_QW], red_l[TREE_WAVES][TREE_QW];

    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    const int li = lane & 31, half = lane >> 5;
    const TreePlace place(a);
    const int split = (int)blockIdx.y, block = place.block, row_base = block * TREE_QW;
    const int G = a.G, Hq = a.G * a.Hkv;
    TreeSegment s(a, place.seg);

    // ---- asked for before the lengths have arrived: parents, queries and the wave's first tile ----
    const int up = a.parent[(size_t)s.b * a.W + (lane < a.W ? lane : a.W - 1)];      // (of lanes that are no node it is not looked at)
    const int my_row = row_base + li < a.W * G ? row_base + li : a.W * G - 1;
    const int node = my_row / G;
    bf16x8 qop[KCH];
    {
        const unsigned char *qrow = a.q + ((s.seq * a.W + node) * Hq + s.h * G + my_row % G) * ROW_BYTES;
#pragma unroll
        for (int c = 0; c < KCH; ++c)
            qop[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qrow + c * 32 + half * 16));
    }
    const unsigned char *kseg = PAGED ? a.k : a.k + (size_t)(a.seg0 + s.seg_local) * a.cap * ROW_BYTES;
    const unsigned char *vseg = PAGED ? a.v : a.v + (size_t)(a.seg0 + s.seg_local) * a.cap * ROW_BYTES;
    const int32_t *tab = PAGED ? a.table + (size_t)(a.seg0 + s.seg_local) * a.max_pages : nullptr;
    auto row_base_of = [&](int r0) -> size_t {             // of a cached row, in bytes
        if constexpr (!PAGED) return (size_t)r0 * ROW_BYTES;
        int page = constant_word(tab + (r0 >> a.page_shift));
        page = (page < 0 || page >= a.num_pages) ? 0 : page;          // never leave the pool
        return (((size_t)page << a.page_shift) + (r0 & ((1 << a.page_shift) - 1))) * ROW_BYTES;
    };
    constexpr int SWZ = PIECES - 1;
    auto v_swizzle = [](int r) { return (2 * r) & (PIECES < 16 ? SWZ : 7); };
    auto k_swizzle = [](int r) { return r & SWZ; };
    auto load_piece = [](const unsigned char *from, unsigned char *to) {
        if constexpr (ONCE) load_once_to_lds16(from, to);
        else load_to_lds16(from, to);
    };
    const int lrow = lane / PIECES, lslot = lane % PIECES;
    unsigned char *const wk = lds_k + wv * TILE_LDS, *const wvl = lds_v + wv * TILE_LDS;
    const int step = a.S * TREE_WAVES;
    int t = split * TREE_WAVES + wv;
    {   // the tile as if it were full (rows behind the capacity are the last one again): where it is not, it is asked for again
        int r0 = t * TREE_MT;
        r0 = r0 < a.cap ? r0 : a.cap - 1;
        const size_t base0 = row_base_of(r0);
        const int most = a.cap - 1 - r0;
        auto whole = [&](const unsigned char *rows, unsigned char *to, auto swizzle) {
#pragma unroll
            for (int r = 0; r < LOADS; ++r) {
                const int slot_row = r * LOAD_ROWS + lrow, row = slot_row < most ? slot_row : most;
                load_piece(rows + base0 + (uint32_t)row * ROW_BYTES + (uint32_t)(lslot ^ swizzle(slot_row)) * 16u, to + r * LOAD_ROWS * ROW_BYTES);
            }
        };
        whole(kseg, wk, k_swizzle);
        __builtin_amdgcn_sched_barrier(0);                 // K first: it is waited for first
        whole(vseg, wvl, v_swizzle);
        __asm__ volatile("" ::: "memory");
    }
    s.clamp(a, threadIdx.x == 0 && split == 0 && block == 0);
    const int n = s.n, nd = s.nd;
    const int rows_left = nd * G - row_base, R = rows_left < TREE_QW ? rows_left : TREE_QW;      // query rows of the block
    const int cache_tiles = (n + TREE_MT - 1) / TREE_MT;
    const int tiles = cache_tiles + (nd + TREE_MT - 1) / TREE_MT;
    const int parts = (tiles + TREE_WAVES - 1) / TREE_WAVES < a.S ? (tiles + TREE_WAVES - 1) / TREE_WAVES : a.S;   // with tiles
    if (R <= 0 || split >= parts) {
        __builtin_amdgcn_s_waitcnt(0x0F70);                // nothing may be on its way to LDS that is not this workgroup's any more
        return;
    }
    const size_t draft_at = ((s.seq * a.W) * a.Hkv + s.h) * ROW_BYTES;
    const uint32_t draft_row = (uint32_t)a.Hkv * ROW_BYTES;
    auto tile_base = [&](int t) -> size_t {                // of a cache tile, in bytes; a tile lies inside one page
        t = t < cache_tiles ? t : cache_tiles - 1;
        return t < 0 ? 0 : row_base_of(t * TREE_MT);
    };
    // K (or V) rows of a tile, straight to LDS; rows behind the last are the last one again
    auto load = [&](int t, size_t base, const unsigned char *cached, const unsigned char *drafts, unsigned char *to, auto swizzle) {
        const bool drafted = t >= cache_tiles;
        const int first = (drafted ? t - cache_tiles : t) * TREE_MT;
        const int last = (drafted ? nd : n) - 1 - first;
        const uint32_t stride = drafted ? draft_row : (uint32_t)ROW_BYTES;
        const unsigned char *src = drafted ? drafts + draft_at + (size_t)first * draft_row : cached + base;
#pragma unroll
        for (int r = 0; r < LOADS; ++r) {
            const int slot_row = r * LOAD_ROWS + lrow;
            const int row = slot_row < last ? slot_row : last;
            load_piece(src + ((uint32_t)row * stride + (uint32_t)(lslot ^ swizzle(slot_row)) * 16u), to + r * LOAD_ROWS * ROW_BYTES);
        }
    };
    auto load_k = [&](int t, size_t base) { load(t, base, kseg, a.k_draft, wk, k_swizzle); };
    auto load_v = [&](int t, size_t base) { load(t, base, vseg, a.v_draft, wvl, v_swizzle); };

    size_t base1 = 0;
    if (t < tiles) {
        if ((t + 1) * TREE_MT > n) {
            const size_t base0 = tile_base(t);
            __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0): not before what was asked for in vain has arrived
            __asm__ volatile("" ::: "memory");
            load_k(t, base0);
            __builtin_amdgcn_sched_barrier(0);
            load_v(t, base0);
        }
        base1 = tile_base(t + step);
    } else {
        __builtin_amdgcn_s_waitcnt(0x0F70);                // (its part of LDS takes the wave's output)
        __asm__ volatile("" ::: "memory");
    }
    uint32_t sees_lo, sees_hi;             // drafted nodes that this lane's row sees
    {
        const uint64_t anc = tree_ancestors(a, up, nd, wv == 0 && split == 0 && block == 0 && s.h == 0);
        sees_lo = (uint32_t)__shfl((int)(uint32_t)anc, node);
        sees_hi = (uint32_t)__shfl((int)(uint32_t)(anc >> 32), node);
    }

    f32x16 oacc[DT];
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[c][r] = 0.f;
    float m_run = TREE_M_INIT, l_run = 0.f;
    uint32_t koff[KCH];
#pragma unroll
    for (int c = 0; c < KCH; ++c) koff[c] = (uint32_t)(li * ROW_BYTES + (((2 * c + half) ^ (li & SWZ)) * 16));
    uint32_t vrd[DT];
    {
        const int row = 4 * half + (lane & 15) / 4;
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            const int d0 = 32 * c + (lane & 16) + 4 * (lane & 3);
            vrd[c] = (uint32_t)(row * ROW_BYTES + (((d0 / 8) ^ v_swizzle(row)) * 16) + (d0 % 8) * 2);
        }
    }

    constexpr int WAIT_LDS = 0xC07F;                       // lgkmcnt(0)
    constexpr int WAIT_OLDER = 0x0F70 | LOADS;             // vmcnt(LOADS): all but the newest tile half is there
    auto tile_step = [&](int t, auto next) {
        // (a tile that is not full, or drafted, is a wave's last: what comes after it is less than a step of the deal)
        constexpr bool NEXT = decltype(next)::value;
        const bool drafted = !NEXT && t >= cache_tiles;
        const int chunk = t - cache_tiles;
        const int left = n - t * TREE_MT;
        const bool full = NEXT || (!drafted && left >= TREE_MT);
        const uint32_t sees = drafted ? (chunk == 0 ? sees_lo : sees_hi) : full ? 0xFFFFFFFFu : (1u << left) - 1u;
        __builtin_amdgcn_s_waitcnt(WAIT_OLDER);            // K; V is still on its way
        __asm__ volatile("" ::: "memory");
        u32x4 kop[KCH];
#pragma unroll
        for (int c = 0; c < KCH; ++c) kop[c] = *reinterpret_cast<const u32x4 *>(wk + koff[c]);
        __builtin_amdgcn_s_waitcnt(WAIT_LDS);
        __builtin_amdgcn_sched_barrier(0);
        if (NEXT) load_k(t + step, base1);                 // into the buffer that has just been read
        __builtin_amdgcn_sched_barrier(0);
        f32x16 sc;
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
        for (int c = 0; c < KCH; ++c)
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kop[c]), qop[c], sc, 0, 0, 0);
        if (!full) {
            const uint32_t w = sees >> (4 * half);
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = (w >> (8 * (r / 4) + r % 4)) & 1u ? sc[r] : -INFINITY;
        }
        float tmx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; r += 2) tmx = max_or_nan(max_or_nan(tmx, sc[r]), sc[r + 1]);
        raise_reference(half_rows_max(tmx) * a.scale_log2e, m_run, l_run, oacc);
        uint32_t part[TREE_PARTS][8];
        l_run += tree_weights(sc, a.scale_log2e, m_run, part);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(NEXT ? WAIT_OLDER : 0x0F70);        // V
        __asm__ volatile("" ::: "memory");
        bool odd = false;
        if (drafted) {
#pragma unroll
            for (int i = 0; i < TILE_LDS / 16 / 64; ++i) odd |= take_out_odd_values(wvl + (i * 64 + lane) * 16);
            odd = __ballot(odd) != 0;
        }
        u32x2 vop[2][DT][2];
#pragma unroll
        for (int kc = 0; kc < 2; ++kc)
#pragma unroll
            for (int c = 0; c < DT; ++c)
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    vop[kc][c][g] = read_transposed16(wvl + vrd[c] + (16 * kc + 8 * g) * ROW_BYTES);
        __builtin_amdgcn_s_waitcnt(WAIT_LDS);
        __builtin_amdgcn_sched_barrier(0);
        if (NEXT) {
            load_v(t + step, base1);
            base1 = tile_base(t + 2 * step);
        }
        __builtin_amdgcn_sched_barrier(0);
        add_products(vop, part, oacc);
        if (odd) {
            const int first = chunk * TREE_MT, count = nd - first < TREE_MT ? nd - first : TREE_MT;
            add_odd_values(a.v_draft + draft_at + (size_t)first * draft_row, draft_row, count, sees, oacc);
        }
    };
    if (t < tiles) {
        while (t + step < tiles) {
            tile_step(t, std::true_type{});
            t += step;
        }
        tile_step(t, std::false_type{});
    }

    // ---- join the waves: O of every wave in its own part of the buffers, 16-byte piece p of row r at slot p ^ r, rows 0-15 where
    // K was, the others where V was ----
    {
        const float l = half_rows_sum(l_run);
        if (half == 0) { red_m[wv][li] = m_run; red_l[wv][li] = l; }
        unsigned char *mine = (li < 16 ? wk : wvl) + (li & 15) * (D * 4);
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {   // register (c, 4g + i) holds d = 32 c + 8 g + 4 half + i
                const int piece = 8 * c + 2 * g + half;
                *reinterpret_cast<f32x4 *>(mine + ((piece ^ li) & (OP - 1)) * 16) =
                    f32x4{oacc[c][4 * g], oacc[c][4 * g + 1], oacc[c][4 * g + 2], oacc[c][4 * g + 3]};
            }
    }
    __syncthreads();
    constexpr int ROWS = TREE_WAVES * 64 / OP;             // rows per workgroup-wide store
    const int piece = threadIdx.x % OP;
    auto joined = [&](int i, float &m_all, float &l_all) {
        m_all = red_m[0][i];
#pragma unroll
        for (int w = 1; w < TREE_WAVES; ++w) m_all = fmaxf(m_all, red_m[w][i]);
        l_all = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < TREE_WAVES; ++w) {
            const float f = fast_exp2(red_m[w][i] - m_all);
            l_all += red_l[w][i] * f;
            o += *reinterpret_cast<const f32x4 *>((i < 16 ? lds_k : lds_v) + w * TILE_LDS + (i & 15) * (D * 4) +
                                                  ((piece ^ i) & (OP - 1)) * 16) * f;
        }
        return o;
    };
    float m_all, l_all;
    if (parts > 1) {                                       // a second launch joins the partials
        const size_t first = ((size_t)s.seg_local * a.S + split) * (size_t)(a.W * G) + row_base;
        for (int row = threadIdx.x / OP; row < R; row += ROWS) {
            const f32x4 o = joined(row, m_all, l_all);
            *(reinterpret_cast<f32x4 *>(a.part_o + (first + row) * D) + piece) = o;
            if (piece == 0) *reinterpret_cast<f32x2 *>(a.part_ml + (first + row) * 2) = f32x2{m_all, l_all};
        }
        return;
    }
    auto write = [&](int row, f32x4 o) {
        const size_t at = (s.seq * a.W + (row_base + row) / G) * Hq + s.h * G + (row_base + row) % G;
        *(reinterpret_cast<f32x4 *>(a.out + at * D) + piece) = o;
        if (a.lse_out && piece == 0) a.lse_out[at] = (m_all + __log2f(l_all)) * 0.6931471805599453f;
    };
    bool odd = false;
    for (int row = threadIdx.x / OP; row < R; row += ROWS) {
        const f32x4 o = joined(row, m_all, l_all) * (1.0f / l_all);
        odd |= is_odd(o, m_all);
        write(row, o);
    }
    if (__ballot(odd) == 0) return;
    for (int row = threadIdx.x / OP; row < R; row += ROWS) {
        const f32x4 o = joined(row, m_all, l_all) * (1.0f / l_all);
        if (row_is_odd<D>(is_odd(o, m_all))) write(row, odd_row<D>(s.seg_local, row_base + row, piece, o, m_all, l_all));
    }
}

// Joins the partials of a segment: out = sum_s O_s 2^(m_s - M) / sum_s l_s 2^(m_s - M).  D / 4 threads per query row.
constexpr int TREE_MERGE_THREADS = 256;
template <int D>
__global__ __launch_bounds__(TREE_MERGE_THREADS) void tree_merge_kernel(TreeArgs a, TreeTiles tl)
{
    constexpr int OP = D / 4;
    TreeSegment s(a, (int)blockIdx.x);
    s.clamp(a, false);
    const int row = (int)blockIdx.y * (TREE_MERGE_THREADS / OP) + (int)threadIdx.x / OP;
    const int piece = (int)threadIdx.x % OP;
    if (row >= s.nd * a.G) return;
    const int tiles = tl.groups(s.n, s.nd);
    const int parts = tiles < a.S ? tiles : a.S;
    if (parts == 1) return;                                // the only workgroup with tiles has written the output
    const size_t rows = (size_t)a.W * a.G;
    const size_t first = (size_t)s.seg_local * a.S * rows + row;
    constexpr int BATCH = 8;
    float M = TREE_M_INIT, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < parts; p0 += BATCH) {
        f32x4 o[BATCH];
        f32x2 ml[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const size_t at = first + (size_t)(p0 + u < parts ? p0 + u : parts - 1) * rows;
            o[u] = *(reinterpret_cast<const f32x4 *>(a.part_o + at * D) + piece);
            ml[u] = *reinterpret_cast<const f32x2 *>(a.part_ml + at * 2);
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < BATCH; ++u) top = fmaxf(top, ml[u][0]);
        const float old = fast_exp2(M - top);
        den *= old;
        num *= old;
        M = top;
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const float f = p0 + u < parts ? fast_exp2(ml[u][0] - top) : 0.f;
            den += ml[u][1] * f;
            num += o[u] * f;
        }
    }
    const size_t at = (s.seq * a.W + row / a.G) * (a.G * a.Hkv) + s.h * a.G + row % a.G;
    f32x4 o = num * (1.0f / den);
    if (row_is_odd<D>(is_odd(o, M))) o = odd_row<D>(s.seg_local, row, piece, o, M, den);
    *(reinterpret_cast<f32x4 *>(a.out + at * D) + piece) = o;
    if (a.lse_out && piece == 0) a.lse_out[at] = (M + __log2f(den)) * 0.6931471805599453f;
}

}  // namespace ngc

// ============================================================ host side ====

using namespace ngc;

namespace {
constexpr int TREE_MAX_NODES = 64;          // a word of ancestor bits
constexpr int TREE_MAX_SPLITS = 64;
constexpr int TREE_RESIDENT = 512;          // workgroups that the chip holds at once
constexpr int TREE_CUS = 256;

struct TreeShape {
    int wq, blocks, splits;             // row blocks of 32 in a workgroup (1: tree_narrow_kernel), workgroups for the rows, and for the keys
    TreeTiles tiles;
};

size_t tree_partial_bytes(const ngc_cache *c, int nseg, int W, int S)
{
    const size_t rows = (size_t)nseg * S * W * (c->Hq / c->Hkv);
    return S > 1 ? align256(rows * c->D * sizeof(float)) + align256(rows * 2 * sizeof(float)) : 0;
}

int tree_most_splits(int nseg, int blocks, int groups)
{
    long long most = TREE_RESIDENT / ((long long)nseg * blocks);
    most = most < groups ? most : groups;
    most = most < TREE_MAX_SPLITS ? most : TREE_MAX_SPLITS;
    return most > 1 ? (int)most : 1;
}

// How many workgroups share a segment's keys, and how long that takes: a model whose numbers were fitted to 325 geometries, each
// at up to 11 splits in workgroups of 32, 64 and 128 query rows.  A workgroup works through rounds of tiles, 128 keys (32 rows: 32 a
// wave) or 64, of `round` us; several on a CU take `crowd` of their sum.  Rows come from memory at 6.2 TB/s, less where the last
// workgroups have a CU to themselves, and again for every row block from L2, 13.6 TB/s in all.  Of work and rows the longer counts
// whole, the other by 0.3.  Sharing costs a launch that joins the partials and their way to memory and back.  Microseconds at S workgroups
// (HIP graph), best in brackets, * what the rule takes (over 80 other drawn geometries 1.02 times the best of all):
//     segments x rows, query rows     S=1     2      3      4       6      8      12     16     24
//         8 x 4000,  32              42.5   27.1   21.6   18.5    16.5   14.0   13.7  [12.6]* 13.4
//        64 x  800,  24              15.0   14.2   13.5  [12.6]*  13.5   14.5
//       256 x 2000,  16 (D = 64)    [25.5]* 28.6   28.3   28.9    29.5   32.0
//        16 x 8000,  63, in 32       77.1   46.4   34.0   28.7    23.4  [21.6]* 23.9   23.8
//       128 x 1493,  48, in 32      [27.3]* 32.2   34.1   36.7    42.5
//                        in 64       35.9   33.5*  33.7  [32.2]
//        32 x  525,  96, in 32       14.3  [14.3]* 15.1   14.6    18.6
//                        in 128      29.0   21.5   18.6   17.9   [16.1]* 16.7   18.9
//       128 x 4096, 112, in 128     124.9   89.3   93.2  [86.0]*
int tree_splits(int nseg, int rows, int blocks, int row_bytes, int max_len, int groups, int wq, float *us_out)
{
    const int most = tree_most_splits(nseg, blocks, groups);
    const bool d128 = row_bytes == 256;
    const float round = wq == 1 ? (d128 ? 1.2f : 0.78f) : wq == 2 ? (d128 ? 1.f : 0.85f) : (d128 ? 2.3f : 1.5f);
    const float crowd = wq == 1 ? 0.62f : wq == 2 ? 0.3f : 0.8f;
    const float bytes = (float)nseg * (float)max_len * 2.f * (float)row_bytes;
    const float read = fmaxf(bytes / 6.2e6f, bytes * (float)blocks / 13.6e6f);
    int best = 1;
    float best_us = 3.0e38f;
    for (int s = 1, rounds; s <= most; s = rounds > 1 ? (groups + rounds - 2) / (rounds - 1) : most + 1) {     // the next with fewer rounds
        rounds = (groups + s - 1) / s;
        const int wg = nseg * blocks * s, per_cu = (wg + TREE_CUS - 1) / TREE_CUS;
        const float work = round * (float)rounds * (per_cu == 1 ? 1.f : (float)per_cu * crowd);
        const float wait = read * (per_cu == 1 ? 1.f : sqrtf((float)(per_cu * TREE_CUS) / (float)wg));
        const float shared = s == 1 ? 0.f : 2.4f * (float)per_cu + (float)wg * (float)rows * (float)row_bytes * 4.f / 6.4e6f;
        const float us = (work > wait ? work + 0.3f * wait : wait + 0.3f * work) + shared;
        if (us < best_us) { best_us = us; best = s; }
    }
    *us_out = best_us;
    return best;
}

// wq row blocks of 32 in a workgroup, and how long the rule says it takes
TreeShape tree_shape_of(const ngc_cache *c, int nseg, int W, int max_len, int wq, float *us)
{
    const int R = W * (c->Hq / c->Hkv), rows = wq * TREE_QW;
    TreeShape s;
    s.wq = wq;
    s.blocks = (R + rows - 1) / rows;
    s.tiles = wq == 1 ? TreeTiles{TREE_MT, TREE_WAVES} : TreeTiles{64, 1};
    s.splits = tree_splits(nseg, R < rows ? R : rows, s.blocks, c->D * 2, max_len, s.tiles.groups(max_len, W), wq, us);
    return s;
}

int tree_widest(int R) { return R <= TREE_QW ? 1 : R <= 2 * TREE_QW ? 2 : 4; }

// Row blocks of 32 in workgroups of their own, or several in one: whichever the rule says is faster, as long as not many more than the
// chip holds at once are at work on the former.  Microseconds at the best split of each, * what is taken:
//     segments x rows, query rows   32     64     128 in a workgroup
//        32 x  525,  96            14.3*  15.4   16.1
//        32 x 1500,  48            14.1*  15.3   16.8
//        64 x 1500, 112            22.5*  29.7   31.2
//       128 x 1493,  48            27.3*  32.2   32.8
//        60 x 2000, 256            42.1*  46.7   48.7
//         4 x 16000, 140           24.6*  30.1   36.4
//       120 x 2000,  80            46.2*  47.1   45.7
//        64 x 3000, 128            40.8*  42.4   41.7
//       128 x 4096, 112            88.8   88.4   86.0*
//       200 x 1000, 120            52.5   44.8   42.4*
//       226 x   38,  84            19.8   15.2   13.5*
//       512 x 2713,  56           167    143*   166
TreeShape tree_shape(const ngc_cache *c, int nseg, int W, int max_len)
{
    const int R = W * (c->Hq / c->Hkv), wq = tree_widest(R);
    float us, us_narrow;
    const TreeShape s = tree_shape_of(c, nseg, W, max_len, wq, &us);
    if (wq == 1 || (long long)nseg * ((R + TREE_QW - 1) / TREE_QW) > (c->D == 128 ? TREE_RESIDENT : 3 * TREE_RESIDENT)) return s;
    const TreeShape narrow = tree_shape_of(c, nseg, W, max_len, 1, &us_narrow);
    return us_narrow < us ? narrow : s;
}

bool tree_geometry_ok(const ngc_cache *c, int32_t W)
{
    return c && c->L > 0 && c->B > 0 && c->Hkv > 0 && c->Hq > 0 && c->cap > 0 && c->Hq % c->Hkv == 0 && W >= 1 && W <= TREE_MAX_NODES;
}

int launch_tree(const ngc_cache *c, const ngc_paged_cache *pc, int32_t layer, const void *k_draft, const void *v_draft,
                const int32_t *parent, const int32_t *n_draft, int32_t W, const void *q, float scale, int32_t max_len_hint,
                float *out, float *lse_out, void *ws, size_t ws_bytes, void *stream)
{
    if (!c->k || !c->v || !c->len || !k_draft || !v_draft || !parent || !q || !out || !ws) return NGC_EINVAL;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(k_draft) || !aligned16(v_draft) || !aligned16(q) || !aligned16(out) ||
        !aligned16(ws))
        return NGC_EINVAL;
    if (c->L <= 0 || c->B <= 0 || c->Hkv <= 0 || c->Hq <= 0 || c->cap <= 0 || W < 1) return NGC_EINVAL;
    if (c->D != 64 && c->D != 128) return NGC_EINVAL;
    if (c->Hq % c->Hkv != 0 || c->Hq / c->Hkv > 16) return NGC_EINVAL;
    if (layer < -1 || layer >= c->L || max_len_hint < 0) return NGC_EINVAL;
    const float scale_log2e = scale * 1.4426950408889634f;
    if (!(scale > 0.f) || !(scale_log2e <= FLT_MAX)) return NGC_EINVAL;       // maxima are taken before scaling
    if (W > TREE_MAX_NODES) return NGC_EUNSUPPORTED;
    if ((long long)c->cap * c->D * 2 > 0x7FFFFFFFLL) return NGC_EUNSUPPORTED;                       // 32-bit byte offsets
    if ((long long)W * c->Hkv * c->D * 2 > 0x7FFFFFFFLL) return NGC_EUNSUPPORTED;
    const int per_layer = c->B * c->Hkv;
    const int nseg = layer < 0 ? c->L * per_layer : per_layer;
    const int max_len = (max_len_hint > 0 && max_len_hint < c->cap) ? max_len_hint : c->cap;
    const size_t off = scratch_offset(c);
    if (ws_bytes < off) return NGC_ENOSPC;
    const TreeShape shape = tree_shape(c, nseg, W, max_len);
    int S = shape.splits;
    while (S > 1 && ws_bytes < off + tree_partial_bytes(c, nseg, W, S)) --S;      // fewer workgroups: less scratch

    const int G = c->Hq / c->Hkv;
    TreeArgs a{};
    a.k = reinterpret_cast<const unsigned char *>(c->k);
    a.v = reinterpret_cast<const unsigned char *>(c->v);
    a.len = c->len;
    a.k_draft = reinterpret_cast<const unsigned char *>(k_draft);
    a.v_draft = reinterpret_cast<const unsigned char *>(v_draft);
    a.parent = parent;
    a.n_draft = n_draft;
    a.q = reinterpret_cast<const unsigned char *>(q);
    a.out = out;
    a.lse_out = lse_out;
    a.part_o = reinterpret_cast<float *>(reinterpret_cast<unsigned char *>(ws) + off);
    a.part_ml = reinterpret_cast<float *>(reinterpret_cast<unsigned char *>(ws) + off +
                                          align256((size_t)nseg * S * W * G * c->D * sizeof(float)));
    a.status = reinterpret_cast<int32_t *>(ws);
    a.seg0 = layer < 0 ? 0 : layer * per_layer;
    a.nseg = nseg; a.blocks = shape.blocks; a.S = S; a.W = W; a.G = G; a.B = c->B; a.Hkv = c->Hkv; a.cap = c->cap;
    a.scale_log2e = scale_log2e;
    if (pc) {
        a.table = pc->table; a.max_pages = pc->max_pages; a.num_pages = pc->num_pages;
        a.page_shift = __builtin_ctz((unsigned)pc->page_rows);
    }
    hipStream_t st = (hipStream_t)stream;
#define NGC_TREE(KERNEL, ...) (pc ? reinterpret_cast<const void *>(&KERNEL<__VA_ARGS__, true>) \
                                  : reinterpret_cast<const void *>(&KERNEL<__VA_ARGS__, false>))
#define NGC_TREE_D(D) (shape.wq == 1 ? (shape.blocks == 1 ? NGC_TREE(tree_narrow_kernel, D, true) : NGC_TREE(tree_narrow_kernel, D, false)) : shape.wq == 2 ? NGC_TREE(tree_attn_kernel, D, 2, true) \
                       : shape.blocks == 1 ? NGC_TREE(tree_attn_kernel, D, 4, true) : NGC_TREE(tree_attn_kernel, D, 4, false))
    const void *fn = c->D == 128 ? NGC_TREE_D(128) : NGC_TREE_D(64);
#undef NGC_TREE_D
#undef NGC_TREE
    const int rc = launch(fn, dim3(nseg * shape.blocks, S), dim3(TREE_WAVES * 64), 0, st, a);
    if (rc || S == 1) return rc;
    const int rows_per = TREE_MERGE_THREADS / (c->D / 4);
    const dim3 grid(nseg, (W * G + rows_per - 1) / rows_per);
    if (c->D == 128) hipLaunchKernelGGL(tree_merge_kernel<128>, grid, dim3(TREE_MERGE_THREADS), 0, st, a, shape.tiles);
    else hipLaunchKernelGGL(tree_merge_kernel<64>, grid, dim3(TREE_MERGE_THREADS), 0, st, a, shape.tiles);
    NGC_HIP_CHECK(hipGetLastError());
    return NGC_OK;
}
}  // namespace

extern "C" size_t ngc_tree_workspace_bytes(const ngc_cache *c, int32_t W)
{
    if (!tree_geometry_ok(c, W)) return 0;
    const int per_layer = c->B * c->Hkv;
    // one layer or all layers, any length hint: the most workgroups a segment can be shared by
    auto most = [&](int nseg) {
        float us;
        const TreeShape s = tree_shape_of(c, nseg, W, c->cap, tree_widest(W * (c->Hq / c->Hkv)), &us);
        return tree_partial_bytes(c, nseg, W, tree_most_splits(nseg, s.blocks, s.tiles.groups(c->cap, W)));
    };
    const size_t one = most(per_layer), all = most(per_layer * c->L);
    const size_t own = scratch_offset(c) + (one > all ? one : all), others = ngc_workspace_bytes(c, 0);
    return own > others ? own : others;
}

extern "C" size_t ngc_paged_tree_workspace_bytes(const ngc_paged_cache *pc, int32_t W)
{
    if (check_paged(pc) != NGC_OK) return 0;
    const ngc_cache c = logical_geometry(pc);
    return ngc_tree_workspace_bytes(&c, W);
}

extern "C" int ngc_tree_attn(const ngc_cache *c, int32_t layer, const void *k_draft, const void *v_draft,
                             const int32_t *parent, const int32_t *n_draft, int32_t W, const void *q, float scale,
                             int32_t max_len_hint, float *out, float *lse_out, void *ws, size_t ws_bytes, void *stream)
{
    if (!c) return NGC_EINVAL;
    return launch_tree(c, nullptr, layer, k_draft, v_draft, parent, n_draft, W, q, scale, max_len_hint, out, lse_out, ws, ws_bytes,
                       stream);
}

extern "C" int ngc_paged_tree_attn(const ngc_paged_cache *pc, int32_t layer, const void *k_draft, const void *v_draft,
                                   const int32_t *parent, const int32_t *n_draft, int32_t W, const void *q, float scale,
                                   int32_t max_len_hint, float *out, float *lse_out, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check_paged(pc);
    if (rc) return rc;
    const ngc_cache c = logical_geometry(pc);
    return launch_tree(&c, pc, layer, k_draft, v_draft, parent, n_draft, W, q, scale, max_len_hint, out, lse_out, ws, ws_bytes, stream);
}
