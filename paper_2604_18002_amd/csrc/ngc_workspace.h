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
