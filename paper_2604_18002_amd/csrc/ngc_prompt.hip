// Many new rows at once for the sequences of a paged cache, from their number for each sequence: pages, page tables, lengths and the
// slots of the packed tokens (extend), and the rows themselves (fill), on gfx950.
//
// extend   Two prefix sums: over the sequences, where the tokens of each begin among the packed ones, and over the segments, how many
//          pages are granted before each (the order of every grant of this layout, see ngc.h).  One workgroup makes them, a few
//          integers per segment; a workgroup per segment then writes its table entries and slots.  Bound by round trips: 28 x 16 x 2
//          segments that grow by a token 3.9 and 3.5 us (10.4 a call), 28 x 64 x 2 of 300 to 1000 tokens 6.1 and 9.2.  Lengths, pages and
//          slots go in batches of four, all of a batch on their way together (one by one 8.7 and 14.5).
// fill     A copy: row (token, head) to the slot that the map names.  Bound by the memory: 64 x 2 x 300 to 1000 rows of 128, K and V
//          (85 MB), 16.5 us, 5.2 TB/s; 8 x 1000 to 4096 rows of 576 (47 MB) 11.3.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ngc.h"
#include "ngc_device.h"
#include "ngc_workspace.h"

namespace ngc {

struct ExtendArgs {
    int32_t *table, *len, *free_stack, *free_count;
    const int32_t *n_new;                   // [B] or nullptr: 1
    int32_t *slot;                          // [launch layers][Hkv][T]
    int32_t *start;                         // [B + 1]
    int32_t *first;                         // workspace, per segment: where its first granted page lies on the stack
    int32_t *rows;                          // workspace, per segment: rows that got a page
    int32_t *status;
    int seg0, nseg, B, Hkv, T;
    int page_rows, page_shift, max_pages, num_pages;
};

constexpr int EXTEND_THREADS = 1024, EXTEND_BATCH = 4;
// Sums over all threads stay in 32 bits when each adds at most this.
constexpr int EXTEND_MOST_TOKENS = 1 << 20;

// One workgroup; consecutive sequences, then consecutive segments, per thread.
__global__ __launch_bounds__(EXTEND_THREADS) void extend_plan_kernel(ExtendArgs a)
{
    __shared__ int tmp[32];
    const int count_raw = *a.free_count;
    const int count = count_raw < 0 ? 0 : (count_raw > a.num_pages ? a.num_pages : count_raw);
    auto at_most = [&](int x) { return x < a.T ? x : a.T; };
    {
        const int per = (a.B + EXTEND_THREADS - 1) / EXTEND_THREADS;
        const int lo = (int)threadIdx.x * per, hi = lo + per < a.B ? lo + per : a.B;
        auto asked = [&](int b) { return a.n_new ? a.n_new[b] : 1; };
        int mine = 0;                       // no more than T
        for (int b = lo; b < hi; ++b) {
            const int x = asked(b);
            mine = x > 0 ? at_most(mine + at_most(x)) : mine;
        }
        int total;
        int at = at_most(block_excl_scan_i<EXTEND_THREADS>(mine, tmp, &total));
        int odd = 0;
        for (int b = lo; b < hi; ++b) {
            a.start[b] = at;
            const int x = asked(b), next = x > 0 ? at_most(at + at_most(x)) : at;
            odd += x != next - at;
            at = next;
        }
        if (odd) atomicAdd(&a.status[NGC_STATUS_LEN_CLAMPED], odd);
        if (threadIdx.x == 0) a.start[a.B] = at_most(total);
    }
    __syncthreads();                        // start[] of all sequences is there
    const int per = (a.nseg + EXTEND_THREADS - 1) / EXTEND_THREADS;
    const int lo = (int)threadIdx.x * per, hi = lo + per < a.nseg ? lo + per : a.nseg;
    const int cap = a.page_rows * a.max_pages;
    auto pages = [&](int rows) { return (rows + a.page_rows - 1) >> a.page_shift; };
    // lengths of a batch of segments and rows asked for: all of them on their way together
    int n[EXTEND_BATCH], w[EXTEND_BATCH];
    auto load = [&](int i0) {
#pragma unroll
        for (int u = 0; u < EXTEND_BATCH; ++u) {
            const int i = i0 + u < a.nseg ? i0 + u : a.nseg - 1, b = (i / a.Hkv) % a.B;
            n[u] = a.len[a.seg0 + i];
            w[u] = a.start[b + 1] - a.start[b];
        }
    };
    // rows there is room for (-1: no length), and pages that are missing for them
    auto wants = [&](int n_, int w_, int &m) {
        if (n_ < 0 || n_ > cap) { m = -1; return 0; }
        m = w_ < cap - n_ ? w_ : cap - n_;
        return pages(n_ + m) - pages(n_);
    };
    int m, mine = 0;
    for (int i0 = lo; i0 < hi; i0 += EXTEND_BATCH) {
        load(i0);
#pragma unroll
        for (int u = 0; u < EXTEND_BATCH; ++u)
            if (i0 + u < hi) mine += wants(n[u], w[u], m);
    }
    int total;
    int rank = block_excl_scan_i<EXTEND_THREADS>(mine, tmp, &total);       // (and everybody has read the height of the stack)
    for (int i0 = lo; i0 < hi; i0 += EXTEND_BATCH) {
        if (per > EXTEND_BATCH) load(i0);                  // (or they are here still)
#pragma unroll
        for (int u = 0; u < EXTEND_BATCH; ++u) {
            const int i = i0 + u;
            if (i >= hi) break;
            const int need = wants(n[u], w[u], m);
            int got = count - rank;
            got = got < 0 ? 0 : got < need ? got : need;
            if (got < need) m = ((pages(n[u]) + got) << a.page_shift) - n[u];
            if (m < 0) {                    // no length
                atomicAdd(&a.status[NGC_STATUS_LEN_CLAMPED], 1);
                m = 0;
            } else if (m > 0) {
                a.len[a.seg0 + i] = n[u] + m;
            }
            if (w[u] > m) atomicAdd(&a.status[NGC_STATUS_APPEND_FULL], w[u] - m);
            a.first[a.seg0 + i] = count - 1 - rank;
            a.rows[a.seg0 + i] = m;
            rank += need;
        }
    }
    if (threadIdx.x == 0) {
        if (count != count_raw) atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], 1);
        *a.free_count = count > total ? count - total : 0;
    }
}

constexpr int SLOT_THREADS = 256, SLOT_BATCH = 4;
__global__ __launch_bounds__(SLOT_THREADS) void extend_slots_kernel(ExtendArgs a)
{
    const int i = (int)blockIdx.x, seg = a.seg0 + i;
    const int h = i % a.Hkv, b = (i / a.Hkv) % a.B, layer = i / (a.Hkv * a.B);
    const int m = a.rows[seg], n = a.len[seg] - m, first = a.first[seg];
    const int start = a.start[b], w = a.start[b + 1] - start;
    int32_t *tab = a.table + (size_t)seg * a.max_pages;
    int32_t *slot = a.slot + ((size_t)layer * a.Hkv + h) * a.T;
    const int have = (n + a.page_rows - 1) >> a.page_shift, want = (n + m + a.page_rows - 1) >> a.page_shift;
    if (m > 0)
        for (int j = have + (int)threadIdx.x; j < want; j += SLOT_THREADS) tab[j] = a.free_stack[first - (j - have)];
    int outside = 0;
    for (int t0 = threadIdx.x; t0 < w; t0 += SLOT_BATCH * SLOT_THREADS) {
        int page[SLOT_BATCH];               // (all on their way together)
#pragma unroll
        for (int u = 0; u < SLOT_BATCH; ++u) {
            const int t = t0 + u * SLOT_THREADS, p = (n + t) >> a.page_shift;
            page[u] = t < m ? (p < have ? tab[p] : a.free_stack[first - (p - have)]) : 0;
        }
#pragma unroll
        for (int u = 0; u < SLOT_BATCH; ++u) {
            const int t = t0 + u * SLOT_THREADS;
            const bool in_pool = page[u] >= 0 && page[u] < a.num_pages;
            outside += !in_pool;
            if (t < w) slot[start + t] = t < m && in_pool ? (page[u] << a.page_shift) + ((n + t) & (a.page_rows - 1)) : -1;
        }
    }
    if (outside) atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], outside);
    // behind the last sequence's tokens: a part for each
    const int end = a.start[a.B], per = (a.T - end + a.B - 1) / a.B, lo = end + b * per, hi = lo + per < a.T ? lo + per : a.T;
    for (int t = lo + (int)threadIdx.x; t < hi; t += SLOT_THREADS) slot[t] = -1;
}

// ------------------------------------------------------------------ fill ------

struct FillArgs {
    unsigned char *k_pool, *v_pool;         // v_pool: nullptr for a cache of one pool
    int32_t *pos_pool;
    const unsigned char *k_new, *v_new;     // [launch layers][T][Hkv][D]
    const int32_t *new_pos;                 // [T] or nullptr
    const int32_t *slot;                    // [launch layers][Hkv][T]
    int32_t *status;
    int T, Hkv, slots;                      // slots: num_pages * page_rows
};

constexpr int FILL_THREADS = 256;
// 16-byte pieces of K (and V) per thread: 1 17.3 us for those 85 MB, 2 16.5, 4 18.9, 8 41.  The rows are read once, past the caches (through
// them 20.2); written through the L2 like any others, they are read soon (past it 20.3, with 4).
constexpr int FILL_BATCH = 2;
template <int PIECES, bool V>
__global__ __launch_bounds__(FILL_THREADS) void fill_kernel(FillArgs a)
{
    const size_t layer_rows = (size_t)a.T * a.Hkv;
    const unsigned char *k_new = a.k_new + (size_t)blockIdx.y * layer_rows * PIECES * 16;
    const unsigned char *v_new = V ? a.v_new + (size_t)blockIdx.y * layer_rows * PIECES * 16 : nullptr;
    const int32_t *slot = a.slot + (size_t)blockIdx.y * layer_rows;
    const size_t first = (size_t)blockIdx.x * (FILL_THREADS * FILL_BATCH) + threadIdx.x;
    int to[FILL_BATCH], piece[FILL_BATCH];
    u32x4 k[FILL_BATCH], v[FILL_BATCH];
    int outside = 0;
#pragma unroll
    for (int u = 0; u < FILL_BATCH; ++u) {
        const size_t at = first + u * FILL_THREADS, row = at / PIECES;
        piece[u] = (int)(at % PIECES);
        to[u] = -1;
        if (row < layer_rows) {
            const int token = (int)(row / (unsigned)a.Hkv), h = (int)(row % (unsigned)a.Hkv);
            to[u] = slot[(size_t)h * a.T + token];
            if (to[u] >= a.slots) { outside += piece[u] == 0; to[u] = -1; }
            if (piece[u] == 0 && to[u] >= 0 && a.pos_pool && a.new_pos) a.pos_pool[to[u]] = a.new_pos[token];
        }
        if (to[u] >= 0) {
            k[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(k_new) + at);
            if constexpr (V) v[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(v_new) + at);
        }
    }
#pragma unroll
    for (int u = 0; u < FILL_BATCH; ++u)
        if (to[u] >= 0) {
            const size_t at = (size_t)to[u] * PIECES + piece[u];
            reinterpret_cast<u32x4 *>(a.k_pool)[at] = k[u];
            if constexpr (V) reinterpret_cast<u32x4 *>(a.v_pool)[at] = v[u];
        }
    if (outside) atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], outside);
}

}  // namespace ngc

// ============================================================ host side ====

using namespace ngc;

extern "C" int ngc_paged_extend(const ngc_paged_cache *pc, int32_t layer, const int32_t *n_new, int32_t T, int32_t *slot_out,
                                int32_t *start_out, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_pages(pc);
    if (rc) return rc;
    if (!slot_out || !start_out || !ws || !aligned16(ws) || T < 1) return NGC_EINVAL;
    if ((long long)pc->B * pc->Hkv > MOST_SEGMENTS / pc->L) return NGC_EUNSUPPORTED;
    int seg0, nseg;
    rc = paged_layer_range(pc, layer, &seg0, &nseg);
    if (rc) return rc;
    const size_t segments = (size_t)pc->L * pc->B * pc->Hkv;
    if (ws_bytes < STATUS_BYTES + segments * 8) return NGC_ENOSPC;
    if (T > EXTEND_MOST_TOKENS || (long long)nseg * pc->max_pages + pc->num_pages > 0x7FFFFFFFLL ||
        (long long)pc->num_pages * pc->page_rows > 0x7FFFFFFFLL)
        return NGC_EUNSUPPORTED;
    ExtendArgs a{};
    a.table = pc->table; a.len = pc->len; a.free_stack = pc->free_stack; a.free_count = pc->free_count;
    a.n_new = n_new; a.slot = slot_out; a.start = start_out;
    a.first = reinterpret_cast<int32_t *>(reinterpret_cast<unsigned char *>(ws) + STATUS_BYTES);
    a.rows = a.first + segments;
    a.status = reinterpret_cast<int32_t *>(ws);
    a.seg0 = seg0; a.nseg = nseg; a.B = pc->B; a.Hkv = pc->Hkv; a.T = T;
    a.page_rows = pc->page_rows; a.page_shift = __builtin_ctz((unsigned)pc->page_rows);
    a.max_pages = pc->max_pages; a.num_pages = pc->num_pages;
    hipStream_t st = (hipStream_t)stream;
    rc = launch(reinterpret_cast<const void *>(&extend_plan_kernel), dim3(1), dim3(EXTEND_THREADS), 0, st, a);
    if (rc) return rc;
    return launch(reinterpret_cast<const void *>(&extend_slots_kernel), dim3((unsigned)nseg), dim3(SLOT_THREADS), 0, st, a);
}

extern "C" int ngc_paged_fill(const ngc_paged_cache *pc, int32_t layer, const void *k_new, const void *v_new, const int32_t *new_pos,
                              const int32_t *slot, int32_t T, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_pages(pc);
    if (rc) return rc;
    if (!k_new || !slot || !ws || !aligned16(k_new) || !aligned16(v_new) || !aligned16(ws) || T < 1) return NGC_EINVAL;
    if (!v_new != !pc->v_pool) return NGC_EINVAL;          // one pool, one tensor
    int seg0, nseg;
    rc = paged_layer_range(pc, layer, &seg0, &nseg);
    if (rc) return rc;
    if (ws_bytes < STATUS_BYTES) return NGC_ENOSPC;
    const int pieces = pc->D * 2 / 16;
    const long long groups = ((long long)T * pc->Hkv * pieces + FILL_THREADS * FILL_BATCH - 1) / (FILL_THREADS * FILL_BATCH);
    if ((long long)T * pc->Hkv > 0x7FFFFFFFLL || !launchable(groups * (layer < 0 ? pc->L : 1), FILL_THREADS) || (long long)pc->num_pages * pc->page_rows > 0x7FFFFFFFLL)
        return NGC_EUNSUPPORTED;
    FillArgs a{};
    a.k_pool = reinterpret_cast<unsigned char *>(pc->k_pool);
    a.v_pool = reinterpret_cast<unsigned char *>(pc->v_pool);
    a.pos_pool = pc->pos_pool;
    a.k_new = reinterpret_cast<const unsigned char *>(k_new);
    a.v_new = reinterpret_cast<const unsigned char *>(v_new);
    a.new_pos = new_pos; a.slot = slot;
    a.status = reinterpret_cast<int32_t *>(ws);
    a.T = T; a.Hkv = pc->Hkv; a.slots = pc->num_pages * pc->page_rows;
    const void *fn = pc->D == 576   ? reinterpret_cast<const void *>(&fill_kernel<72, false>)
                     : pc->D == 288 ? reinterpret_cast<const void *>(&fill_kernel<36, false>)
                     : pc->D == 128 ? reinterpret_cast<const void *>(&fill_kernel<16, true>)
                                    : reinterpret_cast<const void *>(&fill_kernel<8, true>);
    return launch(fn, dim3((unsigned)groups, (unsigned)(layer < 0 ? pc->L : 1)), dim3(FILL_THREADS), 0, (hipStream_t)stream, a);
}
