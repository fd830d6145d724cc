// How a call of attention over latent rows is dealt to workgroups: host code, and the constants of the kernels that it counts with.
#pragma once
#include <stddef.h>

namespace ngc {

constexpr int LT_ROWS = 16;                 // query rows of a wave
// Rows of a tile.  The waves of one row group are key groups, each with tiles of its own: small ones, the next on its way while one is
// worked on.  Four row groups are as much bound by the products, whose full rate takes 32.
constexpr int latent_keys(int RG) { return RG == 1 ? 16 : 32; }
constexpr int LT_MOST_SPLITS = 64;          // a lane of the join each

// How M query rows are dealt to waves and workgroups: one row group a workgroup, or four.
struct LatentShape {
    int waves, groups, blocks, key_groups;
};
inline LatentShape latent_shape(int groups, int M)
{
    LatentShape s;
    s.groups = groups;
    s.waves = groups == 1 ? 4 : 8;
    s.blocks = (M + LT_ROWS * groups - 1) / (LT_ROWS * groups);
    s.key_groups = s.waves / groups;
    return s;
}

// Workgroups that the chip holds at once: one a CU, for LDS; two of one row group with R = 256.
inline int latent_at_once(const LatentShape &s, int R) { return R == 512 || s.groups > 1 ? 256 : 512; }

// How many workgroups may share a sequence's rows: as many as the chip holds at once, a round of rows for each.
inline int latent_most_splits(const LatentShape &s, int nseg, int rows, int R)
{
    const int keys = latent_keys(s.groups) * s.key_groups, rounds = (rows + keys - 1) / keys;
    long long S = latent_at_once(s, R) / ((long long)nseg * s.blocks);
    if (S > rounds) S = rounds;
    if (S > LT_MOST_SPLITS) S = LT_MOST_SPLITS;
    return S < 1 ? 1 : (int)S;
}

// Microseconds that a call takes, about: what a workgroup needs besides its rounds (64 rows, in either shape), a round (as it is bound by
// products, LDS and its own loads, or by the memory), and partials written, read and joined in another launch, by their number and bytes.
// The constants are fitted to calls with 16 to 256 query rows and 1 to 300 sequences of 60 to 6000 rows, R = 512 and 256, layer after
// layer over more rows than the caches hold, lengths between half the hint and all of it: what they choose takes 1.007 times the best
// choice's time in the mean of those 180 geometries, 1.10 at most, and 1.012 (1.18) in 174 others.  Both sides, 64 query rows of R = 512, one row group and four, warm:
// 32 sequences of 400 rows 17.0 and 23.6 us, 32 of 1500 30.7 and 29.0, 128 of 1000 61.7 and 43.6.
inline float latent_cost(const LatentShape &s, int S, int nseg, int rows, int M, int R)
{
    const bool wide = s.groups > 1;
    const float start = R == 512 ? (wide ? 8.2f : 7.3f) : wide ? 6.6f : 6.4f;
    const float products = R == 512 ? (wide ? 2.95f : s.blocks == 1 ? 1.91f : 1.44f) : wide ? 0.91f : 0.85f;      // (rows that nobody shares come late)
    const long long groups = (long long)nseg * s.blocks * S;
    const int chip = latent_at_once(s, R), rounds = (rows + 63) / 64;
    const float at_once = (float)(groups < chip ? groups : chip), row_bytes = (float)(R / 8 * 9 * 2);
    const float memory = at_once / (float)s.blocks * 64.0f * row_bytes / 11.9e6f;
    const float turns = (float)((groups + chip - 1) / chip), mine = (float)((rounds + S - 1) / S);
    const float joined = S == 1 ? 0.f : 2.4f + 0.54f * (float)((S + 7) / 8) + 0.37e-6f * (float)nseg * (float)S * (float)M * (float)R * 4.0f;
    return turns * (start + mine * (products > memory ? products : memory)) + joined;
}

// The shape of a call, and how many workgroups share a sequence.  One row group reads every row once for 16 query rows, four for 64; but its
// workgroups start and end sooner and leave a quarter of the sums to join.
inline LatentShape latent_shape(int M, int nseg, int rows, int R, int *splits)
{
    LatentShape best{};
    float least = 0.f;
    for (int groups = 1; groups <= (M <= LT_ROWS ? 1 : 4); groups += 3) {
        const LatentShape s = latent_shape(groups, M);
        for (int S = latent_most_splits(s, nseg, rows, R); S >= 1; --S) {
            const float cost = latent_cost(s, S, nseg, rows, M, R);
            if (best.waves && cost >= least) continue;
            best = s;
            least = cost;
            *splits = S;
        }
    }
    return best;
}

inline size_t latent_partial_bytes(int nseg, int S, int M, int R) { return S == 1 ? 0 : (size_t)nseg * S * M * (R + 2) * sizeof(float); }

}  // namespace ngc
