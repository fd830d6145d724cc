// Layout of a cache's workspace, shared by the units that keep something in it:
//   [status words][per segment: 2 int32 of the paged layout's pool bookkeeping][per segment: ticket][scratch of the call]
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/ngc.h"

namespace ngc {

constexpr size_t STATUS_BYTES = NGC_STATUS_WORDS * sizeof(int32_t);

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline size_t ticket_offset(const ngc_cache *c)
{
    return STATUS_BYTES + (size_t)c->L * c->B * c->Hkv * 2 * sizeof(int32_t);
}
// Where the scratch begins: nothing in it has to be zero before a call.
inline size_t scratch_offset(const ngc_cache *c)
{
    return align256(ticket_offset(c) + (size_t)c->L * c->B * c->Hkv * sizeof(int32_t));
}

// Words between the tickets of two segments.  Atomics on one cache line are served one after the other, so a launch's
// tickets lie as far apart as the words at hand allow, up to a line of 128 bytes.  A workspace has a word for every
// segment of the cache, so the launches of a model of L layers, one layer each, have L words for a segment; a launch
// over all layers has one, as does a cache of a single layer.  Microseconds per layer from a HIP graph of 28 layers, words
// next to each other -> 28 apart, D = 128 (no difference below 16 segments, where at most 64 atomics meet):
//     16 x 1500 rows   8.27 -> 6.69      32 x 1500   8.83 -> 8.11      64 x 1500        11.56 -> 11.06
//     32 x  300        5.70 -> 5.47      64 x  525   8.06 -> 7.79      128 x 525        10.18 ->  9.55
//     32 x  525        6.31 -> 5.74      48 x 676-1352 8.91 -> 8.64    64 x 3000-10000  41.18 -> 39.89
inline int ticket_step(size_t words, int nseg_launch)
{
    const size_t apart = words / (size_t)nseg_launch;
    return apart > 32 ? 32 : apart > 1 ? (int)apart : 1;
}

// The geometry of a paged cache as if its rows were held contiguously.
inline ngc_cache logical_geometry(const ngc_paged_cache *pc)
{
    ngc_cache c{};
    c.k = pc->k_pool; c.v = pc->v_pool; c.len = pc->len; c.pos = nullptr;
    c.L = pc->L; c.B = pc->B; c.Hkv = pc->Hkv; c.Hq = pc->Hq; c.D = pc->D;
    c.cap = pc->max_pages * pc->page_rows;
    return c;
}

inline int check_paged(const ngc_paged_cache *pc)
{
    if (!pc || !pc->k_pool || !pc->v_pool || !pc->table || !pc->len || !pc->free_stack || !pc->free_count)
        return NGC_EINVAL;
    if (!aligned16(pc->k_pool) || !aligned16(pc->v_pool)) return NGC_EINVAL;
    if (pc->L <= 0 || pc->B <= 0 || pc->Hkv <= 0 || pc->Hq <= 0 || pc->max_pages <= 0 || pc->num_pages <= 0)
        return NGC_EINVAL;
    if (pc->D != 64 && pc->D != 128) return NGC_EINVAL;
    if (pc->Hq % pc->Hkv != 0 || pc->Hq / pc->Hkv > 16) return NGC_EINVAL;
    if (pc->L > 65535 || pc->Hkv > 65534) return NGC_EINVAL;
    if (pc->page_rows < 32 || (pc->page_rows & (pc->page_rows - 1)) != 0) return NGC_EINVAL;
    if (pc->max_pages > 16384) return NGC_EUNSUPPORTED;
    if ((long long)pc->max_pages * pc->page_rows > 0x7FFFFFFFLL / 256) return NGC_EUNSUPPORTED;
    return NGC_OK;
}

inline int paged_layer_range(const ngc_paged_cache *pc, int layer, int *seg0, int *nseg)
{
    if (layer < -1 || layer >= pc->L) return NGC_EINVAL;
    const int per_layer = pc->B * pc->Hkv;
    *seg0 = layer < 0 ? 0 : layer * per_layer;
    *nseg = layer < 0 ? pc->L * per_layer : per_layer;
    return NGC_OK;
}

}  // namespace ngc
