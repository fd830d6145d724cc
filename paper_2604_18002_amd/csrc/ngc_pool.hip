// Drafted rows that become rows of a cache, and the pages of sequences that fork, end or are packed, on gfx950.
//
// commit   rows path[0 .. m) of the drafted K and V are appended to every segment.  A workgroup per segment: it reads the
//          length, copies the rows and stores the new length.  Paged: a first launch grants the pages that are missing, in
//          segment order (a prefix sum over the segments by one workgroup).
// free     a prefix sum over the segments gives every dropped segment its place on the stack; a wave per segment pushes.
// fork     the destinations' own pages are released, then every destination is granted as many pages as its source has (same
//          prefix sums); a wave per destination writes its table and what is to be copied where; then the pages are copied, a
//          page read once for up to four copies.
// compact  with U pages in use, the i-th page in use beyond the first U moves to the i-th free place among them.  Movers and
//          holes are disjoint, so all pages move at once.  Pages in use are marked in a bitmap; one workgroup scans its words.
//
// Copies are bound by the memory, everything else is a few integers per segment or page and bound by launches (~2 us each, the
// plan of a fork of 3584 segments 10).  Forks of 28 x 2 segments of 300-500 rows (256 bytes each), all launches: 15 copies of 48 MB
// 163 us (715 MB written; a fill runs at 5.7 TB/s: 125), one copy of 360 MB 168 us; packing a pool after half of 64 sequences have
// ended (611 MB moved) 138 us, the copy of it at 5.4 TB/s, the best copy shape of this card 5.9.  Rows appended to 3584 dense segments
// (4.5 each on average) 5.3-5.8 us, to 896 paged ones 6.4 (two launches).
// Measured and not kept: tiles of 64 KB, 256 or 1024 workgroups for the moves (0.98-1.02); plain stores (1.1); 8 or 16 copies from one
// read (15 copies 181-188 us without caching the reads, four copies 163 with).
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
    const int sub = (int)threadIdx.x / (2 * PIECES), lane = (int)threadIdx.x % (2 * PIECES);
    const bool is_v = lane >= PIECES;
    const int piece = is_v ? lane - PIECES : lane;
    const int n = a.len[seg];
    const int asked = a.n_path[b];
    const int wanted = path_length(a, b);
    // The first rows are asked for before it is known how many there are: a path has W entries, and node 0 stands in for those
    // that name none.
    const unsigned char *drafts = (is_v ? a.v_draft : a.k_draft) + ((size_t)seq * a.W * a.Hkv + h) * ROW_BYTES + piece * 16;
    int node, named;
    u32x4 x;
    auto ask = [&](int i) {
        named = a.path[(size_t)b * a.W + i];
        node = named < 0 || named >= a.W ? 0 : named;
        x = *reinterpret_cast<const u32x4 *>(drafts + (size_t)node * a.Hkv * ROW_BYTES);
    };
    ask(sub < a.W ? sub : 0);
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
    int bad = 0;
    for (int i = sub; i < m; i += ROWS) {
        if (i != sub) ask(i);
        bad += lane == 0 && named != node;
        size_t row;
        if constexpr (PAGED) {
            const int at = n + i;
            row = ((size_t)a.table[(size_t)seg * a.max_pages + (at >> a.page_shift)] << a.page_shift) + (at & (a.page_rows - 1));
        } else {
            row = (size_t)seg * a.cap + n + i;
        }
        *reinterpret_cast<u32x4 *>((is_v ? a.v : a.k) + row * ROW_BYTES + piece * 16) = x;
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

constexpr int FORK_COPIES = 4;              // copies of a page that are written from one read of it
constexpr int FORK_SEQUENCES = 8192;        // whose sources fit in LDS

struct PoolArgs {
    unsigned char *k_pool, *v_pool;
    int32_t *pos_pool;
    int32_t *table, *len, *free_stack, *free_count;
    const int32_t *mark;                    // [B]: fork: the sequence to copy, or below 0; free: whether it goes
    int32_t *freed, *push_base;             // workspace, per segment
    // fork: workspace.  head: [0] pages to move, [1] height of the stack when pages were granted, [2] whether all were, [3] whether
    // pages are read more than once
    int32_t *head;
    int32_t *first, *work;                  // per segment: pages granted before it; pieces of work before it
    int32_t *copies, *rank;                 // per sequence: copies of it; which of its source's copies it is
    int32_t *from, *to;                     // per piece of work: a page, and FORK_COPIES places (-1: none)
    int32_t *status;
    int seg0, nseg, B, Hkv;
    int page_rows, page_shift, max_pages, num_pages;
};

constexpr int FORK_NONE = -1, FORK_INVALID = -2;
// The sequence that b is to become a copy of; it must be one, and must not be replaced itself.
__device__ __forceinline__ int fork_source(const PoolArgs &a, int b)
{
    const int s = a.mark[b];
    if (s < 0 || s == b) return FORK_NONE;
    if (s >= a.B) return FORK_INVALID;
    const int ss = a.mark[s];
    return ss < 0 || ss == s ? s : FORK_INVALID;
}

// Exclusive prefix sums of three numbers at once.
template <int THREADS>
__device__ __forceinline__ void block_excl_scan3(int (&v)[3], int (*tmp)[THREADS / NGC_WAVE], int (&total)[3])
{
    int incl[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        incl[k] = wave_incl_scan_i(v[k]);
        if (lane_id() == NGC_WAVE - 1) tmp[k][wave_id()] = incl[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] = below_waves<THREADS / NGC_WAVE, 1>(tmp[k], &total[k]) + incl[k] - v[k];
    __syncthreads();
}

// What every segment gives back, is granted and is copied to; the new lengths and the new height of the stack.  One workgroup;
// consecutive segments per thread, four at a time so that their lengths are asked for together.
template <bool FORK>
__global__ __launch_bounds__(POOL_THREADS) void pool_plan_kernel(PoolArgs a)
{
    __shared__ int tmp[3][POOL_THREADS / NGC_WAVE];
    __shared__ int copies[FORK ? FORK_SEQUENCES : 1];
    __shared__ short source[FORK ? FORK_SEQUENCES : 1];
    const int count_raw = *a.free_count;
    const int count = count_raw < 0 ? 0 : (count_raw > a.num_pages ? a.num_pages : count_raw);
    const int per = (a.nseg + POOL_THREADS - 1) / POOL_THREADS;
    const int lo = (int)threadIdx.x * per, hi = lo + per < a.nseg ? lo + per : a.nseg;
    const int cap = a.page_rows * a.max_pages;
    auto pages = [&](int rows) { return (rows + a.page_rows - 1) >> a.page_shift; };
    [[maybe_unused]] bool shared = false;   // whether a page is read for more than one piece of work
    if constexpr (FORK) {
        int invalid = 0;
        for (int b = threadIdx.x; b < a.B; b += POOL_THREADS) {
            copies[b] = 0;
            const int s = fork_source(a, b);
            source[b] = (short)s;
            invalid += s == FORK_INVALID;
        }
        if (invalid) atomicAdd(&a.status[NGC_STATUS_BAD_FORK], invalid);
        __syncthreads();
        for (int b = threadIdx.x; b < a.B; b += POOL_THREADS)
            if (source[b] >= 0) a.rank[b] = atomicAdd(&copies[source[b]], 1);
        __syncthreads();
        for (int b = threadIdx.x; b < a.B; b += POOL_THREADS) {
            a.copies[b] = copies[b];
            shared |= copies[b] > FORK_COPIES;
        }
        shared = __syncthreads_or(shared) != 0;
    }
    struct Plan {
        int back, rows, take, work;         // pages given back; new length (-1: stays), pages granted; pieces of work as a source
        bool clamped;
    };
    constexpr int STEP = 4;
    auto plan = [&](int i0, Plan (&p)[STEP]) {
        int n[STEP], m[STEP];
#pragma unroll
        for (int u = 0; u < STEP; ++u) {    // all lengths first
            const int i = i0 + u < hi ? i0 + u : hi - 1, b = (i / a.Hkv) % a.B;
            n[u] = a.len[a.seg0 + i];
            m[u] = 0;
            if constexpr (FORK) {
                const int s = source[b];
                m[u] = s >= 0 ? a.len[a.seg0 + i + (s - b) * a.Hkv] : -1;
                if (s >= 0 && m[u] < 0) m[u] = 0;
                m[u] = m[u] > cap ? cap : m[u];
            } else {
                m[u] = a.mark[b] != 0 ? 0 : -1;
            }
        }
#pragma unroll
        for (int u = 0; u < STEP; ++u) {
            const int i = i0 + u < hi ? i0 + u : hi - 1, b = (i / a.Hkv) % a.B;
            const int held = pages(n[u] < 0 ? 0 : n[u] > cap ? cap : n[u]);
            p[u].rows = m[u];
            p[u].clamped = (m[u] >= 0 || (FORK && copies[b] > 0)) && (n[u] < 0 || n[u] > cap);      // given back, or copied
            p[u].back = m[u] >= 0 ? held : 0;
            p[u].take = m[u] > 0 ? pages(m[u]) : 0;
            p[u].work = FORK ? held * ((copies[b] + FORK_COPIES - 1) / FORK_COPIES) : 0;
        }
    };
    Plan p[STEP];
    int at[3] = {0, 0, 0}, total[3];        // of pages given back, of pages granted, of pieces of work
    for (int i0 = lo; i0 < hi; i0 += STEP) {
        plan(i0, p);
#pragma unroll
        for (int u = 0; u < STEP; ++u)
            if (i0 + u < hi) { at[0] += p[u].back; at[1] += p[u].take; at[2] += p[u].work; }
    }
    block_excl_scan3<POOL_THREADS>(at, tmp, total);       // (and everybody has read the lengths and the stack's height)
    const int height = count + total[0] < a.num_pages ? count + total[0] : a.num_pages;
    [[maybe_unused]] int granted = 0;
    for (int i0 = lo; i0 < hi; i0 += STEP) {
        if (per > STEP) plan(i0, p);        // (what is stored to meanwhile is nobody's source, and every segment is one thread's)
#pragma unroll
        for (int u = 0; u < STEP; ++u) {
            const int i = i0 + u;
            if (i >= hi) break;
            a.freed[a.seg0 + i] = p[u].back;
            a.push_base[a.seg0 + i] = count + at[0];
            if constexpr (FORK) {
                a.first[i] = at[1];
                a.work[i] = at[2];
            }
            if (p[u].clamped) atomicAdd(&a.status[NGC_STATUS_LEN_CLAMPED], 1);
            // not all of its pages are there: it gets none, nor does anybody behind it
            const bool dry = p[u].take && at[1] + p[u].take > height;
            if (dry) atomicAdd(&a.status[NGC_STATUS_APPEND_FULL], 1);
            else granted += p[u].take;
            if (p[u].rows >= 0) a.len[a.seg0 + i] = dry ? 0 : p[u].rows;
            at[0] += p[u].back;
            at[1] += p[u].take;
            at[2] += p[u].work;
        }
    }
    const bool enough = total[1] <= height;
    int all = total[1];
    if (!enough) (void)block_excl_scan_i<POOL_THREADS>(granted, tmp[0], &all);
    if (threadIdx.x == 0) {
        if (count != count_raw || count + total[0] > a.num_pages) atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], 1);
        *a.free_count = height - all;
        if constexpr (FORK) {
            a.head[0] = enough ? total[2] : all;           // either way no more than there are pages
            a.head[1] = height;
            a.head[2] = enough;
            a.head[3] = shared;
        }
    }
}

// A wave per segment: all of its pages go onto the stack.
constexpr int WAVES = 4;                    // per workgroup, where a wave takes a segment
__global__ __launch_bounds__(WAVES * 64) void pool_push_kernel(PoolArgs a)
{
    const int i = (int)blockIdx.x * WAVES + wave_id();
    if (i >= a.nseg) return;
    const int seg = a.seg0 + i;
    const int f = a.freed[seg], base = a.push_base[seg];
    const int32_t *tab = a.table + (size_t)seg * a.max_pages;
    for (int r = lane_id(); r < f; r += 64)
        if (base + r >= 0 && base + r < a.num_pages) a.free_stack[base + r] = tab[r];
}

// A wave per segment that becomes a copy: its pages, in its table and in the list of what is to be moved.  A piece of work is a
// page and up to FORK_COPIES of its copies; where the stack did not hold enough pages, one granted page each.
__global__ __launch_bounds__(WAVES * 64) void fork_list_kernel(PoolArgs a)
{
    const int i = (int)blockIdx.x * WAVES + wave_id();
    if (i >= a.nseg) return;
    const int b = (i / a.Hkv) % a.B, s = fork_source(a, b);
    if (s < 0) return;
    const int src = i + (s - b) * a.Hkv;
    const bool enough = a.head[2] != 0;
    const int height = a.head[1], first = a.first[i], rank = a.rank[b], copies = a.copies[s];
    const int pages = (a.len[a.seg0 + i] + a.page_rows - 1) >> a.page_shift;      // 0 where none were granted
    const int chunks = (copies + FORK_COPIES - 1) / FORK_COPIES;
    for (int j = lane_id(); j < pages; j += 64) {
        int to = a.free_stack[height - 1 - first - j];
        const int from = a.table[(size_t)(a.seg0 + src) * a.max_pages + j];
        a.table[(size_t)(a.seg0 + i) * a.max_pages + j] = to;
        if (from < 0 || from >= a.num_pages || to < 0 || to >= a.num_pages) {
            atomicAdd(&a.status[NGC_STATUS_POOL_BOUNDS], 1);
            to = -1;
        }
        const size_t piece = enough ? (size_t)a.work[src] + (size_t)j * chunks + rank / FORK_COPIES : (size_t)first + j;
        const int slot = enough ? rank % FORK_COPIES : 0;
        a.to[piece * FORK_COPIES + slot] = to;
        if (slot == 0) a.from[piece] = from;
        if (!enough || rank == copies - 1)                 // the piece's last copy
            for (int u = slot + 1; u < FORK_COPIES; ++u) a.to[piece * FORK_COPIES + u] = -1;
    }
}

// Moves pages: page from[x] to COPIES places to[x * COPIES ..].  Tiles of up to 128 KB of K and V: all of a tile's reads, a
// barrier, all of its writes, a barrier (a CU whose waves mix both moves less).  Compaction (COPIES = 1) updates the tables.
constexpr int MOVE_THREADS = 1024;
constexpr int MOVE_GROUPS = 512;
constexpr int MOVE_BATCH = 8;               // 16-byte pieces per thread
constexpr int MOVE_PIECES = MOVE_THREADS * MOVE_BATCH;
constexpr int MOVE_PAGES = MOVE_PIECES * 16 / (2 * 32 * 128);         // per tile, of the smallest kind

template <int COPIES>
__global__ __launch_bounds__(MOVE_THREADS) void move_pages_kernel(PoolArgs a, const int32_t *from_list, const int32_t *to_list,
                                                                  const int32_t *owner, int page_bytes)
{
    __shared__ int from[MOVE_PAGES], to[COPIES][MOVE_PAGES];
    const int total = a.head[0];
    const bool again = COPIES > 1 && a.head[3] != 0;        // (15 copies of 48 MB take 192 us if asked for as read once,
                                                            // 163 if not; one copy of 360 MB 176 and 182)
    const int pieces = page_bytes / 8, shift = 31 - __builtin_clz((unsigned)pieces);     // of a page's K and V
    // a tile holds `per` pages, or a `parts`-th of one; fewer pages where there are too few for two rounds of workgroups
    const int most = pieces < MOVE_PIECES ? MOVE_PIECES / pieces : 1, share = total / (2 * (int)gridDim.x);
    const int per = share < 1 ? 1 : share < most ? share : most;
    const int parts = pieces > MOVE_PIECES ? pieces / MOVE_PIECES : 1;
    const long long tiles = (long long)((total + per - 1) / per) * parts;
    for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int first = (int)(t / parts) * per, part = (int)(t % parts);
        const int here = total - first < per ? total - first : per;
        if ((int)threadIdx.x < here * COPIES) {
            const int x = (int)threadIdx.x / COPIES, u = (int)threadIdx.x % COPIES;
            const int hole = to_list[(size_t)(first + x) * COPIES + u];
            to[u][x] = hole;
            if (u == 0) {
                const int page = from_list[first + x];
                from[x] = page;
                if (COPIES == 1 && part == 0) a.table[owner[page]] = hole;
            }
        }
        __syncthreads();
        auto place = [&](int x, int page) {
            const int at = x & (pieces - 1);
            return reinterpret_cast<u32x4 *>((at < pieces / 2 ? a.k_pool : a.v_pool) + (size_t)page * page_bytes) + (at & (pieces / 2 - 1));
        };
        const int end = here << shift;
        u32x4 x[MOVE_BATCH];
        // a page whose copies' places are all outside the pool is not read: its number may be outside too
        auto wanted = [&](int q) {
            bool any = false;
#pragma unroll
            for (int u = 0; u < COPIES; ++u) any |= to[u][q] >= 0;
            return any;
        };
        auto read = [&](auto load) {
#pragma unroll
            for (int v = 0; v < MOVE_BATCH; ++v) {
                const int i = part * MOVE_PIECES + v * MOVE_THREADS + (int)threadIdx.x;
                if (i < end && wanted(i >> shift)) x[v] = load(place(i, from[i >> shift]));
            }
        };
        if (again) read([](const u32x4 *p) { return *p; });
        else read([](const u32x4 *p) { return __builtin_nontemporal_load(p); });
        __syncthreads();
#pragma unroll
        for (int u = 0; u < COPIES; ++u)
#pragma unroll
            for (int v = 0; v < MOVE_BATCH; ++v) {
                const int i = part * MOVE_PIECES + v * MOVE_THREADS + (int)threadIdx.x;
                if (i < end && to[u][i >> shift] >= 0) __builtin_nontemporal_store(x[v], place(i, to[u][i >> shift]));
            }
        if (a.pos_pool && part == 0)
            for (int i = threadIdx.x; i < here * a.page_rows; i += MOVE_THREADS) {
                const int q = i / a.page_rows, r = i % a.page_rows;
                if (!wanted(q)) continue;
                const int32_t pos = a.pos_pool[(size_t)from[q] * a.page_rows + r];
#pragma unroll
                for (int u = 0; u < COPIES; ++u)
                    if (to[u][q] >= 0) a.pos_pool[(size_t)to[u][q] * a.page_rows + r] = pos;
            }
        __syncthreads();
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
__global__ __launch_bounds__(WAVES * 64) void compact_mark_kernel(CompactArgs a)
{
    const int seg = (int)blockIdx.x * WAVES + wave_id();
    if (seg >= a.p.nseg) return;
    const int cap = a.p.page_rows * a.p.max_pages;
    int n = a.p.len[seg];
    if (n < 0 || n > cap) {
        if (lane_id() == 0) atomicAdd(&a.p.status[NGC_STATUS_LEN_CLAMPED], 1);
        n = n < 0 ? 0 : cap;
    }
    const int pages = (n + a.p.page_rows - 1) >> a.p.page_shift;
    for (int j = lane_id(); j < pages; j += 64) {
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

// A thread per page: holes and movers enter the lists; the free stack becomes the pages from U on, the lowest on top.
__global__ __launch_bounds__(256) void compact_list_kernel(CompactArgs a)
{
    const int page = (int)(blockIdx.x * 256 + threadIdx.x);
    if (page >= a.p.num_pages) return;
    int f;
    const int U = compact_used(a, &f);
    const int w = page / 32, bit = page % 32;
    uint32_t holes, movers;
    compact_word(a, w, U, holes, movers);
    const uint32_t below = (1u << bit) - 1u;
    if ((holes >> bit) & 1u) a.hole[a.holes_before[w] + __popc(holes & below)] = page;
    if ((movers >> bit) & 1u) a.mover[a.movers_before[w] + __popc(movers & below)] = page;
    if (page < f) a.p.free_stack[page] = a.p.num_pages - 1 - page;
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
    a.work = a.first + segments;
    a.copies = a.work + segments;
    a.rank = a.copies + pc->B;
    a.from = a.rank + pc->B;
    a.to = a.from + pc->num_pages;
    a.status = reinterpret_cast<int32_t *>(ws);
    a.seg0 = seg0; a.nseg = nseg; a.B = pc->B; a.Hkv = pc->Hkv;
    a.page_rows = pc->page_rows; a.page_shift = __builtin_ctz((unsigned)pc->page_rows);
    a.max_pages = pc->max_pages; a.num_pages = pc->num_pages;
    return a;
}

// Sums of pages, and heights of the stack, in 32 bits.
bool page_sums_fit(const ngc_paged_cache *pc, long long nseg) { return nseg * pc->max_pages + pc->num_pages <= 0x7FFFFFFFLL; }

size_t fork_scratch_bytes(const ngc_paged_cache *pc)
{
    return 16 + ((size_t)pc->L * pc->B * pc->Hkv * 2 + (size_t)pc->B * 2 + (size_t)pc->num_pages * (1 + FORK_COPIES)) * sizeof(int32_t);
}
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
    return launch(reinterpret_cast<const void *>(&pool_push_kernel), dim3((nseg + WAVES - 1) / WAVES), dim3(WAVES * 64), 0, st, a);
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
    if (!page_sums_fit(pc, nseg) || pc->B > FORK_SEQUENCES) return NGC_EUNSUPPORTED;
    PoolArgs a = pool_args(pc, source, seg0, nseg, ws);
    hipStream_t st = (hipStream_t)stream;
    rc = launch(reinterpret_cast<const void *>(&pool_plan_kernel<true>), dim3(1), dim3(POOL_THREADS), 0, st, a);
    if (rc) return rc;
    const dim3 waves((nseg + WAVES - 1) / WAVES), threads(WAVES * 64);
    rc = launch(reinterpret_cast<const void *>(&pool_push_kernel), waves, threads, 0, st, a);
    if (rc) return rc;
    rc = launch(reinterpret_cast<const void *>(&fork_list_kernel), waves, threads, 0, st, a);
    if (rc) return rc;
    hipLaunchKernelGGL(move_pages_kernel<FORK_COPIES>, dim3(MOVE_GROUPS), dim3(MOVE_THREADS), 0, st, a, a.from, a.to, nullptr,
                       pc->page_rows * pc->D * 2);
    NGC_HIP_CHECK(hipGetLastError());
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
    hipLaunchKernelGGL(compact_clear_kernel, dim3(blocks < 256 ? blocks : 256), dim3(256), 0, st, a);
    NGC_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(compact_mark_kernel, dim3((unsigned)((segments + WAVES - 1) / WAVES)), dim3(WAVES * 64), 0, st, a);
    NGC_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(compact_scan_kernel, dim3(1), dim3(POOL_THREADS), 0, st, a);
    NGC_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(compact_list_kernel, dim3((pc->num_pages + 255) / 256), dim3(256), 0, st, a);
    NGC_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(move_pages_kernel<1>, dim3(MOVE_GROUPS), dim3(MOVE_THREADS), 0, st, a.p, a.mover, a.hole, a.owner,
                       pc->page_rows * pc->D * 2);
    NGC_HIP_CHECK(hipGetLastError());
    return NGC_OK;
}
