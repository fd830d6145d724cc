// Drafted rows that become rows of a cache, and the pages of sequences that fork, end or are packed, on gfx950.
//
// commit   rows path[0 .. m) of the drafted K and V are appended to every segment.  A workgroup per segment: it reads the
//          length, copies the rows and stores the new length.  Paged: a first launch grants the pages that are missing, in
//          segment order (a prefix sum over the segments by one workgroup).
// free     a prefix sum over the segments gives every dropped segment its place on the stack; a wave per segment pushes.
// fork     the destinations' own pages are released, then every destination is granted as many pages as its source has (same
//          prefix sums), then the pages are copied: workgroups take equal runs of them whatever the segments' lengths, and
//          find the segment of their first page by bisection.
// compact  with U pages in use, the i-th page in use beyond the first U moves to the i-th free place among them.  Movers and
//          holes are disjoint, so all pages move at once.  Pages in use are marked in a bitmap; one workgroup scans its words.
//
// Copies are bound by the memory; everything else is a few integers per segment or page and bound by launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ngc.h"
#include "ngc_device.h"
#include "ngc_workspace.h"

namespace ngc {

struct CommitArgs {
    unsigned char *k, *v;                   // the cache's rows, or the pools
    int32_t *pos;                           // or nullptr
    int32_t *len;
    const unsigned char *k_draft, *v_draft; // [launch layers][B][W][Hkv][D]
    const int32_t *draft_pos;               // [B][W] or nullptr
    const int32_t *path, *n_path;           // [B][W], [B]
    int32_t *status;
    int seg0, nseg, B, Hkv, W, cap;
    // paged layout only
    int32_t *table, *free_stack, *free_count;
    int32_t *rows;                          // workspace, per segment: rows that got a page
    int page_rows, page_shift, max_pages, num_pages;
};

__device__ __forceinline__ int path_length(const CommitArgs &a, int b)
{
    const int m = a.n_path[b];
    return m < 0 ? 0 : m > a.W ? a.W : m;
}

// Pages that missing rows need, granted in segment order from the top of the stack.  One workgroup.
constexpr int POOL_THREADS = 1024;
__global__ __launch_bounds__(POOL_THREADS) void commit_grant_kernel(CommitArgs a)
{
    __shared__ int tmp[32];
    const int count_raw = *a.free_count;
    const int count = count_raw < 0 ? 0 : (count_raw > a.num_pages ? a.num_pages : count_raw);
    const int per = (a.nseg + POOL_THREADS - 1) / POOL_THREADS;
    const int lo = (int)threadIdx.x * per, hi = lo + per < a.nseg ? lo + per : a.nseg;
    auto pages = [&](int rows) { return (rows + a.page_rows - 1) >> a.page_shift; };
    // length, rows to append if there is room, and pages that are missing for them
    auto wants = [&](int i, int &n, int &m) {
        n = a.len[a.seg0 + i];
        m = path_length(a, (i / a.Hkv) % a.B);
        if (n < 0 || n > a.cap) { m = 0; return 0; }
        m = m < a.cap - n ? m : a.cap - n;
        return pages(n + m) - pages(n);
    };
    int n, m, mine = 0;
    for (int i = lo; i < hi; ++i) mine += wants(i, n, m);
    int total;
    int rank = block_excl_scan_i<POOL_THREADS>(mine, tmp, &total);
    for (int i = lo; i < hi; ++i) {
        const int need = wants(i, n, m);
        int got = count - rank;
        got = got < 0 ? 0 : got < need ? got : need;
        if (need) {
            int32_t *entry = a.table + (size_t)(a.seg0 + i) * a.max_pages + pages(n);
            for (int j = 0; j < got; ++j) entry[j] = a.free_stack[count - 1 - rank - j];
            if (got < need) m = (pages(n) + got) * a.page_rows - n;
        }
        a.rows[a.seg0 + i] = m;
        rank += need;
    }
    __syncthreads();   // every thread has read the old count
    if (threadIdx.x == 0) {
        if (count != count_raw) atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], 1);
        *a.free_count = count > total ? count - total : 0;
    }
}

constexpr int COMMIT_THREADS = 256;
template <int ROW_BYTES, bool PAGED>
__global__ __launch_bounds__(COMMIT_THREADS) void commit_kernel(CommitArgs a)
{
    constexpr int PIECES = ROW_BYTES / 16;
    constexpr int ROWS = COMMIT_THREADS / (2 * PIECES);     // rows (K and V) per step
    const int seg = a.seg0 + (int)blockIdx.x;
    const int seq = (int)blockIdx.x / a.Hkv, h = (int)blockIdx.x % a.Hkv, b = seq % a.B;
    const int n = a.len[seg];
    const int asked = a.n_path[b];
    const int wanted = path_length(a, b);
    const bool valid = n >= 0 && n <= a.cap;
    int m = PAGED ? a.rows[seg] : wanted;
    m = !valid || m < 0 ? 0 : m < a.cap - n ? m : a.cap - n;
    if constexpr (PAGED) {
        // a page outside the pool ends what is appended
        for (int p = n >> a.page_shift; m > 0 && (p << a.page_shift) < n + m; ++p) {
            const int page = a.table[(size_t)seg * a.max_pages + p];
            if (page >= 0 && page < a.num_pages) continue;
            const int start = p << a.page_shift;
            m = start > n ? start - n : 0;
            if (threadIdx.x == 0) atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], 1);
        }
    }
    const int sub = (int)threadIdx.x / (2 * PIECES), lane = (int)threadIdx.x % (2 * PIECES);
    const bool is_v = lane >= PIECES;
    const int piece = is_v ? lane - PIECES : lane;
    int bad = 0;
    for (int i = sub; i < m; i += ROWS) {
        int node = a.path[(size_t)b * a.W + i];
        if (node < 0 || node >= a.W) {      // counted; some drafted row stands in
            node = 0;
            bad += lane == 0;
        }
        const size_t from = (((size_t)seq * a.W + node) * a.Hkv + h) * ROW_BYTES + piece * 16;
        size_t row;
        if constexpr (PAGED) {
            const int at = n + i;
            row = ((size_t)a.table[(size_t)seg * a.max_pages + (at >> a.page_shift)] << a.page_shift) + (at & (a.page_rows - 1));
        } else {
            row = (size_t)seg * a.cap + n + i;
        }
        *reinterpret_cast<u32x4 *>((is_v ? a.v : a.k) + row * ROW_BYTES + piece * 16) =
            *reinterpret_cast<const u32x4 *>((is_v ? a.v_draft : a.k_draft) + from);
        if (lane == 0 && a.pos && a.draft_pos) a.pos[row] = a.draft_pos[(size_t)b * a.W + node];
    }
    if (bad && h == 0) atomicAdd(&a.status[NGC_STATUS_BAD_TREE], bad);
    __syncthreads();                        // everybody has read the length
    if (threadIdx.x == 0) {
        if (!valid) atomicAdd(&a.status[NGC_STATUS_LEN_CLAMPED], 1);
        if (wanted > m) atomicAdd(&a.status[NGC_STATUS_APPEND_FULL], wanted - m);
        if (asked != wanted && h == 0) atomicAdd(&a.status[NGC_STATUS_BAD_TREE], 1);
        if (m > 0) a.len[seg] = n + m;
    }
}

// ------------------------------------------------------------ fork, free ------

struct PoolArgs {
    unsigned char *k_pool, *v_pool;
    int32_t *pos_pool;
    int32_t *table, *len, *free_stack, *free_count;
    const int32_t *mark;                    // [B]: fork: the sequence to copy, or below 0; free: whether it goes
    int32_t *freed, *push_base;             // workspace, per segment
    int32_t *first;                         // workspace, per segment: pages granted before it
    int32_t *head;                          // workspace: [0] pages granted, [1] height of the stack when they were
    int32_t *status;
    int seg0, nseg, B, Hkv;
    int page_rows, page_shift, max_pages, num_pages;
};

// The segment that launch segment i is to become a copy of, -1 if none; *invalid: its sequence names one that is none or
// is itself replaced.
__device__ __forceinline__ int fork_source(const PoolArgs &a, int i, bool *invalid)
{
    const int b = (i / a.Hkv) % a.B;
    const int s = a.mark[b];
    *invalid = false;
    if (s < 0 || s == b) return -1;
    if (s < a.B) {
        const int ss = a.mark[s];
        if (ss < 0 || ss == s) return i + (s - b) * a.Hkv;
    }
    *invalid = true;
    return -1;
}

template <bool FORK>
__global__ __launch_bounds__(POOL_THREADS) void pool_plan_kernel(PoolArgs a)
{
    __shared__ int tmp[32];
    const int count_raw = *a.free_count;
    const int count = count_raw < 0 ? 0 : (count_raw > a.num_pages ? a.num_pages : count_raw);
    const int per = (a.nseg + POOL_THREADS - 1) / POOL_THREADS;
    const int lo = (int)threadIdx.x * per, hi = lo + per < a.nseg ? lo + per : a.nseg;
    const int cap = a.page_rows * a.max_pages;
    auto rows_of = [&](int i) {
        const int n = a.len[a.seg0 + i];
        return n < 0 ? 0 : n > cap ? cap : n;
    };
    auto pages = [&](int rows) { return (rows + a.page_rows - 1) >> a.page_shift; };
    // pages that the segment gives back and takes
    auto plan = [&](int i, int &back, int &rows, bool &invalid) {
        invalid = false;
        back = 0;
        rows = -1;
        if constexpr (FORK) {
            const int src = fork_source(a, i, &invalid);
            if (src < 0) return;
            rows = rows_of(src);
        } else {
            if (a.mark[(i / a.Hkv) % a.B] == 0) return;
            rows = 0;
        }
        back = pages(rows_of(i));
    };
    int back, rows, sum_back = 0, sum_take = 0;
    bool invalid;
    for (int i = lo; i < hi; ++i) {
        plan(i, back, rows, invalid);
        sum_back += back;
        sum_take += rows > 0 ? pages(rows) : 0;
    }
    int total_back, total_take = 0, take_at = 0;
    int back_at = block_excl_scan_i<POOL_THREADS>(sum_back, tmp, &total_back);
    if constexpr (FORK) take_at = block_excl_scan_i<POOL_THREADS>(sum_take, tmp, &total_take);
    int height = count + total_back;
    if (height > a.num_pages) height = a.num_pages;
    // Nobody's length has been stored yet; a thread's sources belong to others, but no source is stored to.
    __syncthreads();
    int granted = 0;
    for (int i = lo; i < hi; ++i) {
        const int n = a.len[a.seg0 + i];
        plan(i, back, rows, invalid);
        if (FORK && invalid && i < a.B * a.Hkv && i % a.Hkv == 0) atomicAdd(&a.status[NGC_STATUS_BAD_FORK], 1);
        a.freed[a.seg0 + i] = back;
        a.push_base[a.seg0 + i] = count + back_at;
        back_at += back;
        if constexpr (FORK) a.first[i] = take_at < height ? take_at : height;
        if (rows < 0) continue;
        if (n < 0 || n > cap) atomicAdd(&a.status[NGC_STATUS_LEN_CLAMPED], 1);
        const int take = pages(rows);
        if (take && take_at + take > height) {      // not all of its pages are there: it gets none, nor does anybody behind it
            atomicAdd(&a.status[NGC_STATUS_APPEND_FULL], 1);
            rows = 0;
        } else {
            granted += take;
        }
        take_at += take;
        a.len[a.seg0 + i] = rows;
    }
    int all;
    (void)block_excl_scan_i<POOL_THREADS>(granted, tmp, &all);
    if (threadIdx.x == 0) {
        if (count != count_raw || count + total_back > a.num_pages) atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], 1);
        *a.free_count = height - all;
        if constexpr (FORK) { a.head[0] = all; a.head[1] = height; }
    }
}

// A wave per segment: all of its pages go onto the stack.
__global__ __launch_bounds__(64) void pool_push_kernel(PoolArgs a)
{
    const int seg = a.seg0 + (int)blockIdx.x;
    const int f = a.freed[seg], base = a.push_base[seg];
    const int32_t *tab = a.table + (size_t)seg * a.max_pages;
    for (int r = threadIdx.x; r < f; r += 64)
        if (base + r >= 0 && base + r < a.num_pages) a.free_stack[base + r] = tab[r];
}

// Copies page `from` to page `to`, by all threads of a workgroup.
template <int THREADS>
__device__ __forceinline__ void copy_page(const PoolArgs &a, int from, int to, int page_bytes)
{
    const u32x4 *ks = reinterpret_cast<const u32x4 *>(a.k_pool + (size_t)from * page_bytes);
    const u32x4 *vs = reinterpret_cast<const u32x4 *>(a.v_pool + (size_t)from * page_bytes);
    u32x4 *kd = reinterpret_cast<u32x4 *>(a.k_pool + (size_t)to * page_bytes);
    u32x4 *vd = reinterpret_cast<u32x4 *>(a.v_pool + (size_t)to * page_bytes);
    for (int i = threadIdx.x; i < page_bytes / 16; i += THREADS) {
        const u32x4 x = __builtin_nontemporal_load(ks + i), y = __builtin_nontemporal_load(vs + i);
        __builtin_nontemporal_store(x, kd + i);
        __builtin_nontemporal_store(y, vd + i);
    }
    if (a.pos_pool)
        for (int i = threadIdx.x; i < a.page_rows; i += THREADS)
            a.pos_pool[(size_t)to * a.page_rows + i] = a.pos_pool[(size_t)from * a.page_rows + i];
}

constexpr int COPY_THREADS = 256;
constexpr int COPY_GROUPS = 2048;           // workgroups that share the pages

__global__ __launch_bounds__(COPY_THREADS) void fork_copy_kernel(PoolArgs a, int page_bytes)
{
    const int total = a.head[0], height = a.head[1];
    const int lo = (int)((long long)total * blockIdx.x / gridDim.x), hi = (int)((long long)total * (blockIdx.x + 1) / gridDim.x);
    if (lo >= hi) return;
    // the segment that page lo is granted to: the last with first <= lo (later ones of the same value take no page)
    int i = 0;
    for (int span = a.nseg; span > 1;) {
        const int halfway = span / 2;
        if (a.first[i + halfway] <= lo) i += halfway;
        span -= halfway;
    }
    for (int g = lo; g < hi; ++g) {
        while (i + 1 < a.nseg && a.first[i + 1] <= g) ++i;
        bool invalid;
        const int src = fork_source(a, i, &invalid);
        const int j = g - a.first[i];
        const int to = a.free_stack[height - 1 - g];
        const int from = src >= 0 ? a.table[(size_t)(a.seg0 + src) * a.max_pages + j] : -1;
        if (threadIdx.x == 0) a.table[(size_t)(a.seg0 + i) * a.max_pages + j] = to;
        if (from < 0 || from >= a.num_pages || to < 0 || to >= a.num_pages) {
            if (threadIdx.x == 0) atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], 1);
            continue;
        }
        copy_page<COPY_THREADS>(a, from, to, page_bytes);
    }
}

// ---------------------------------------------------------------- compact ------

struct CompactArgs {
    PoolArgs p;
    uint32_t *used;                         // [words] bit per page
    int32_t *owner;                         // [num_pages] segment * max_pages + logical page; where `used`
    int32_t *holes_before, *movers_before;  // [words]
    int32_t *hole, *mover;                  // [num_pages]
    int words;
};

__global__ __launch_bounds__(256) void compact_clear_kernel(CompactArgs a)
{
    for (int i = (int)(blockIdx.x * 256 + threadIdx.x); i < a.words; i += (int)gridDim.x * 256) a.used[i] = 0;
}

// A wave per segment.
__global__ __launch_bounds__(64) void compact_mark_kernel(CompactArgs a)
{
    const int seg = (int)blockIdx.x;
    const int cap = a.p.page_rows * a.p.max_pages;
    int n = a.p.len[seg];
    if (n < 0 || n > cap) {
        if (threadIdx.x == 0) atomicAdd(&a.p.status[NGC_STATUS_LEN_CLAMPED], 1);
        n = n < 0 ? 0 : cap;
    }
    const int pages = (n + a.p.page_rows - 1) >> a.p.page_shift;
    for (int j = threadIdx.x; j < pages; j += 64) {
        const int page = a.p.table[(size_t)seg * a.p.max_pages + j];
        if (page < 0 || page >= a.p.num_pages) {
            atomicAdd(&a.p.status[NGC_STATUS_POOL_BOUNDS], 1);
            continue;
        }
        a.owner[page] = seg * a.p.max_pages + j;
        atomicOr(&a.used[page >> 5], 1u << (page & 31));
    }
}

// Pages below U that are free, and pages from U on that are in use, among the 32 of a word.
__device__ __forceinline__ void compact_word(const CompactArgs &a, int w, int U, uint32_t &holes, uint32_t &movers)
{
    const int first = w * 32;
    uint32_t real = first + 32 <= a.p.num_pages ? 0xFFFFFFFFu : (1u << (a.p.num_pages - first)) - 1u;
    const uint32_t inside = U >= first + 32 ? 0xFFFFFFFFu : U <= first ? 0u : (1u << (U - first)) - 1u;
    const uint32_t used = a.used[w];
    holes = ~used & inside & real;
    movers = used & ~inside & real;
}

__device__ __forceinline__ int compact_used(const CompactArgs &a, int *free_pages)
{
    const int raw = *a.p.free_count;
    const int f = raw < 0 ? 0 : raw > a.p.num_pages ? a.p.num_pages : raw;
    *free_pages = f;
    return a.p.num_pages - f;
}

__global__ __launch_bounds__(POOL_THREADS) void compact_scan_kernel(CompactArgs a)
{
    __shared__ int tmp[32];
    int f;
    const int U = compact_used(a, &f);
    const int per = (a.words + POOL_THREADS - 1) / POOL_THREADS;
    const int lo = (int)threadIdx.x * per, hi = lo + per < a.words ? lo + per : a.words;
    int nh = 0, nm = 0;
    uint32_t holes, movers;
    for (int w = lo; w < hi; ++w) {
        compact_word(a, w, U, holes, movers);
        nh += __popc(holes);
        nm += __popc(movers);
    }
    int all_h, all_m;
    int h = block_excl_scan_i<POOL_THREADS>(nh, tmp, &all_h);
    int m = block_excl_scan_i<POOL_THREADS>(nm, tmp, &all_m);
    for (int w = lo; w < hi; ++w) {
        a.holes_before[w] = h;
        a.movers_before[w] = m;
        compact_word(a, w, U, holes, movers);
        h += __popc(holes);
        m += __popc(movers);
    }
    if (threadIdx.x == 0) {
        a.p.head[0] = all_h < all_m ? all_h : all_m;
        // as many free places as pages that want one, or a page is in two places or in none
        if (all_h != all_m || *a.p.free_count != f) atomicAdd(&a.p.status[NGC_STATUS_POOL_BOUNDS], 1);
    }
}

// A thread per word: its holes and movers enter the lists; the free stack becomes the pages from U on, the lowest on top.
__global__ __launch_bounds__(256) void compact_list_kernel(CompactArgs a)
{
    const int w = (int)(blockIdx.x * 256 + threadIdx.x);
    if (w >= a.words) return;
    int f;
    const int U = compact_used(a, &f);
    uint32_t holes, movers;
    compact_word(a, w, U, holes, movers);
    for (int at = a.holes_before[w]; holes; holes &= holes - 1, ++at) a.hole[at] = w * 32 + __builtin_ctz(holes);
    for (int at = a.movers_before[w]; movers; movers &= movers - 1, ++at) a.mover[at] = w * 32 + __builtin_ctz(movers);
    for (int i = w * 32; i < w * 32 + 32 && i < f; ++i) a.p.free_stack[i] = a.p.num_pages - 1 - i;
}

__global__ __launch_bounds__(COPY_THREADS) void compact_move_kernel(CompactArgs a, int page_bytes)
{
    const int total = a.p.head[0];
    for (int i = (int)blockIdx.x; i < total; i += (int)gridDim.x) {
        const int from = a.mover[i], to = a.hole[i];
        copy_page<COPY_THREADS>(a.p, from, to, page_bytes);
        if (threadIdx.x == 0) a.p.table[a.owner[from]] = to;
    }
}

}  // namespace ngc

// ============================================================ host side ====

using namespace ngc;

namespace {

int check_commit(const ngc_cache *c, int32_t layer, const void *k_draft, const void *v_draft, const int32_t *path,
                 const int32_t *n_path, int32_t W, const void *ws)
{
    if (!c->k || !c->v || !c->len || !k_draft || !v_draft || !path || !n_path || !ws) return NGC_EINVAL;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(k_draft) || !aligned16(v_draft) || !aligned16(ws)) return NGC_EINVAL;
    if (c->L <= 0 || c->B <= 0 || c->Hkv <= 0 || c->cap <= 0 || W < 1) return NGC_EINVAL;
    if (c->D != 64 && c->D != 128) return NGC_EINVAL;
    if (layer < -1 || layer >= c->L) return NGC_EINVAL;
    if (W > 64) return NGC_EUNSUPPORTED;
    return NGC_OK;
}

CommitArgs commit_args(const ngc_cache *c, int32_t layer, const void *k_draft, const void *v_draft, const int32_t *draft_pos,
                       const int32_t *path, const int32_t *n_path, int32_t W, void *ws)
{
    CommitArgs a{};
    a.k = reinterpret_cast<unsigned char *>(c->k);
    a.v = reinterpret_cast<unsigned char *>(c->v);
    a.pos = c->pos;
    a.len = c->len;
    a.k_draft = reinterpret_cast<const unsigned char *>(k_draft);
    a.v_draft = reinterpret_cast<const unsigned char *>(v_draft);
    a.draft_pos = draft_pos;
    a.path = path; a.n_path = n_path;
    a.status = reinterpret_cast<int32_t *>(ws);
    const int per_layer = c->B * c->Hkv;
    a.seg0 = layer < 0 ? 0 : layer * per_layer;
    a.nseg = layer < 0 ? c->L * per_layer : per_layer;
    a.B = c->B; a.Hkv = c->Hkv; a.W = W; a.cap = c->cap;
    return a;
}

PoolArgs pool_args(const ngc_paged_cache *pc, const int32_t *mark, int seg0, int nseg, void *ws)
{
    const ngc_cache c = logical_geometry(pc);
    unsigned char *base = reinterpret_cast<unsigned char *>(ws);
    const size_t segments = (size_t)pc->L * pc->B * pc->Hkv;
    PoolArgs a{};
    a.k_pool = reinterpret_cast<unsigned char *>(pc->k_pool);
    a.v_pool = reinterpret_cast<unsigned char *>(pc->v_pool);
    a.pos_pool = pc->pos_pool;
    a.table = pc->table; a.len = pc->len;
    a.free_stack = pc->free_stack; a.free_count = pc->free_count;
    a.mark = mark;
    a.freed = reinterpret_cast<int32_t *>(base + STATUS_BYTES);
    a.push_base = a.freed + segments;
    a.head = reinterpret_cast<int32_t *>(base + scratch_offset(&c));
    a.first = a.head + 4;
    a.status = reinterpret_cast<int32_t *>(ws);
    a.seg0 = seg0; a.nseg = nseg; a.B = pc->B; a.Hkv = pc->Hkv;
    a.page_rows = pc->page_rows; a.page_shift = __builtin_ctz((unsigned)pc->page_rows);
    a.max_pages = pc->max_pages; a.num_pages = pc->num_pages;
    return a;
}

// Sums of pages, and heights of the stack, in 32 bits.
bool page_sums_fit(const ngc_paged_cache *pc, long long nseg) { return nseg * pc->max_pages + pc->num_pages <= 0x7FFFFFFFLL; }

size_t fork_scratch_bytes(const ngc_paged_cache *pc) { return 16 + (size_t)pc->L * pc->B * pc->Hkv * sizeof(int32_t); }
size_t compact_scratch_bytes(const ngc_paged_cache *pc)
{
    const size_t words = ((size_t)pc->num_pages + 31) / 32;
    return 16 + 3 * words * sizeof(int32_t) + 3 * (size_t)pc->num_pages * sizeof(int32_t);
}

}  // namespace

extern "C" size_t ngc_paged_pool_workspace_bytes(const ngc_paged_cache *pc)
{
    if (check_paged(pc) != NGC_OK) return 0;
    const ngc_cache c = logical_geometry(pc);
    const size_t fork = fork_scratch_bytes(pc), compact = compact_scratch_bytes(pc);
    const size_t own = scratch_offset(&c) + (fork > compact ? fork : compact), others = ngc_paged_workspace_bytes(pc);
    return own > others ? own : others;
}

extern "C" int ngc_tree_commit(const ngc_cache *c, int32_t layer, const void *k_draft, const void *v_draft, const int32_t *draft_pos,
                               const int32_t *path, const int32_t *n_path, int32_t W, void *ws, size_t ws_bytes, void *stream)
{
    if (!c) return NGC_EINVAL;
    const int rc = check_commit(c, layer, k_draft, v_draft, path, n_path, W, ws);
    if (rc) return rc;
    if (ws_bytes < STATUS_BYTES) return NGC_ENOSPC;
    CommitArgs a = commit_args(c, layer, k_draft, v_draft, draft_pos, path, n_path, W, ws);
    const void *fn = c->D == 128 ? reinterpret_cast<const void *>(&commit_kernel<256, false>)
                                 : reinterpret_cast<const void *>(&commit_kernel<128, false>);
    return launch(fn, dim3(a.nseg), dim3(COMMIT_THREADS), 0, (hipStream_t)stream, a);
}

extern "C" int ngc_paged_tree_commit(const ngc_paged_cache *pc, int32_t layer, const void *k_draft, const void *v_draft,
                                     const int32_t *draft_pos, const int32_t *path, const int32_t *n_path, int32_t W, void *ws,
                                     size_t ws_bytes, void *stream)
{
    int rc = check_paged(pc);
    if (rc) return rc;
    ngc_cache c = logical_geometry(pc);
    c.pos = pc->pos_pool;
    rc = check_commit(&c, layer, k_draft, v_draft, path, n_path, W, ws);
    if (rc) return rc;
    if (ws_bytes < STATUS_BYTES + (size_t)pc->L * pc->B * pc->Hkv * 8) return NGC_ENOSPC;
    CommitArgs a = commit_args(&c, layer, k_draft, v_draft, draft_pos, path, n_path, W, ws);
    a.table = pc->table; a.free_stack = pc->free_stack; a.free_count = pc->free_count;
    a.rows = reinterpret_cast<int32_t *>(reinterpret_cast<unsigned char *>(ws) + STATUS_BYTES);
    a.page_rows = pc->page_rows; a.page_shift = __builtin_ctz((unsigned)pc->page_rows);
    a.max_pages = pc->max_pages; a.num_pages = pc->num_pages;
    hipStream_t st = (hipStream_t)stream;
    rc = launch(reinterpret_cast<const void *>(&commit_grant_kernel), dim3(1), dim3(POOL_THREADS), 0, st, a);
    if (rc) return rc;
    const void *fn = pc->D == 128 ? reinterpret_cast<const void *>(&commit_kernel<256, true>)
                                  : reinterpret_cast<const void *>(&commit_kernel<128, true>);
    return launch(fn, dim3(a.nseg), dim3(COMMIT_THREADS), 0, st, a);
}

extern "C" int ngc_paged_free(const ngc_paged_cache *pc, int32_t layer, const int32_t *drop, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_paged(pc);
    if (rc) return rc;
    if (!drop || !ws || !aligned16(ws)) return NGC_EINVAL;
    int seg0, nseg;
    rc = paged_layer_range(pc, layer, &seg0, &nseg);
    if (rc) return rc;
    if (ws_bytes < STATUS_BYTES + (size_t)pc->L * pc->B * pc->Hkv * 8) return NGC_ENOSPC;
    if (!page_sums_fit(pc, nseg)) return NGC_EUNSUPPORTED;
    PoolArgs a = pool_args(pc, drop, seg0, nseg, ws);
    hipStream_t st = (hipStream_t)stream;
    rc = launch(reinterpret_cast<const void *>(&pool_plan_kernel<false>), dim3(1), dim3(POOL_THREADS), 0, st, a);
    if (rc) return rc;
    return launch(reinterpret_cast<const void *>(&pool_push_kernel), dim3(nseg), dim3(64), 0, st, a);
}

extern "C" int ngc_paged_fork(const ngc_paged_cache *pc, int32_t layer, const int32_t *source, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_paged(pc);
    if (rc) return rc;
    if (!source || !ws || !aligned16(ws)) return NGC_EINVAL;
    int seg0, nseg;
    rc = paged_layer_range(pc, layer, &seg0, &nseg);
    if (rc) return rc;
    const ngc_cache c = logical_geometry(pc);
    if (ws_bytes < scratch_offset(&c) + fork_scratch_bytes(pc)) return NGC_ENOSPC;
    if (!page_sums_fit(pc, nseg)) return NGC_EUNSUPPORTED;
    PoolArgs a = pool_args(pc, source, seg0, nseg, ws);
    hipStream_t st = (hipStream_t)stream;
    rc = launch(reinterpret_cast<const void *>(&pool_plan_kernel<true>), dim3(1), dim3(POOL_THREADS), 0, st, a);
    if (rc) return rc;
    rc = launch(reinterpret_cast<const void *>(&pool_push_kernel), dim3(nseg), dim3(64), 0, st, a);
    if (rc) return rc;
    const int page_bytes = pc->page_rows * pc->D * 2;
    void *kargs[] = {&a, const_cast<int *>(&page_bytes)};
    NGC_HIP_CHECK(hipLaunchKernel(reinterpret_cast<const void *>(&fork_copy_kernel), dim3(COPY_GROUPS), dim3(COPY_THREADS), kargs, 0, st));
    return NGC_OK;
}

extern "C" int ngc_paged_compact(const ngc_paged_cache *pc, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check_paged(pc);
    if (rc) return rc;
    if (!ws || !aligned16(ws)) return NGC_EINVAL;
    const ngc_cache c = logical_geometry(pc);
    const long long segments = (long long)pc->L * pc->B * pc->Hkv;
    if (segments * pc->max_pages > 0x7FFFFFFFLL) return NGC_EUNSUPPORTED;              // 32-bit names of table entries
    if (ws_bytes < scratch_offset(&c) + compact_scratch_bytes(pc)) return NGC_ENOSPC;
    CompactArgs a{};
    a.p = pool_args(pc, nullptr, 0, (int)segments, ws);
    a.words = (pc->num_pages + 31) / 32;
    a.used = reinterpret_cast<uint32_t *>(a.p.head + 4);
    a.holes_before = reinterpret_cast<int32_t *>(a.used) + a.words;
    a.movers_before = a.holes_before + a.words;
    a.owner = a.movers_before + a.words;
    a.hole = a.owner + pc->num_pages;
    a.mover = a.hole + pc->num_pages;
    hipStream_t st = (hipStream_t)stream;
    const int blocks = (a.words + 255) / 256;
    const int page_bytes = pc->page_rows * pc->D * 2;
    hipLaunchKernelGGL(compact_clear_kernel, dim3(blocks < 256 ? blocks : 256), dim3(256), 0, st, a);
    NGC_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(compact_mark_kernel, dim3((unsigned)segments), dim3(64), 0, st, a);
    NGC_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(compact_scan_kernel, dim3(1), dim3(POOL_THREADS), 0, st, a);
    NGC_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(compact_list_kernel, dim3(blocks), dim3(256), 0, st, a);
    NGC_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(compact_move_kernel, dim3(COPY_GROUPS), dim3(COPY_THREADS), 0, st, a, page_bytes);
    NGC_HIP_CHECK(hipGetLastError());
    return NGC_OK;
}
