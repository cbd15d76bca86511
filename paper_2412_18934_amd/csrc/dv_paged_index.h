// What the paged cache's kernels take from device memory, checked, and where it leads them:
// sequences, row numbers, shares of the work, paths, ranks.  Plain functions of their arguments,
// which compile for the host too, so that they can be tested there.
#pragma once

#include "dv_paged.h"

#ifdef __HIPCC__
#define PAGED_FN __host__ __device__ __forceinline__
#else
#define PAGED_FN static inline
#endif

PAGED_FN uint32_t float_bits(float x)
{
    uint32_t u;
    __builtin_memcpy(&u, &x, 4);
    return u;
}

constexpr uint32_t NONE = 0xffffffffu;  // no such row

struct Seq {
    int first, n, len;  // first new row, new rows (0: nothing to do), committed slots
};

// Sequence s of the call, n = 0 if its numbers cannot be (bad) or it has no rows.
PAGED_FN Seq seq_of(const PagedView &c, const int32_t *start, int n_rows, int s, int most, bool &bad)
{
    const int64_t first = start ? start[s] : s, end = start ? start[s + 1] : s + 1;
    const int len = c.lens[s];
    const int64_t n = end - first;
    Seq q = {(int)first, (int)n, len};
    if (n == 0) return q;
    if (first < 0 || n < 0 || end > n_rows || n > most || len < 0 || len + n > (int64_t)c.width * c.page) {
        bad = true;
        q.n = 0;
    }
    return q;
}

// Row number of slot `slot` of sequence s, NONE if its page is not in the pool.
PAGED_FN uint32_t row_of(const PagedView &c, int s, int h, int slot, bool &bad)
{
    const uint32_t p = (uint32_t)slot / (uint32_t)c.page;
    const uint32_t id = (uint32_t)c.table[(int64_t)s * c.width + p];
    if (id >= (uint32_t)c.n_pages) {
        bad = true;
        return NONE;
    }
    return (id * (uint32_t)c.H + (uint32_t)h) * (uint32_t)c.page + ((uint32_t)slot - p * (uint32_t)c.page);
}

// The work of a call is its 32-slot tiles in one line: sequences in order, of each its
// units (KV heads times row blocks of `block` rows) in order, of each the tiles.
struct Load {
    int units, tiles;
};
PAGED_FN Load load_of(const PagedView &c, const Seq &q, int G, int block)
{
    if (q.n == 0) return {0, 0};
    return {c.H * (int)(((int64_t)q.n * G + block - 1) / block), (q.len + q.n + PAGED_TILE - 1) / PAGED_TILE};
}

// Shares of a line: no more than tiles, so that none is empty (a joined unit's shares all have a part).
PAGED_FN int shares_of(int64_t total, int groups) { return total < groups ? (int)total : groups; }

// Workgroup g of `groups` has the tiles [share_start(g), share_start(g + 1)): total g / groups,
// rounded down, without a product that leaves 64 bits.
PAGED_FN int64_t share_start(int64_t total, int g, int groups)
{
    return total / groups * g + total % groups * g / groups;
}
PAGED_FN int share_of(int64_t total, int64_t tile, int groups)
{
    int g = (int)((double)tile / (double)total * groups);
    g = g < groups ? g : groups - 1;
    while (share_start(total, g + 1, groups) <= tile) ++g;
    while (share_start(total, g, groups) > tile) --g;
    return g;
}

// Whether entry i of sequence s's path of n can be, and whether its length can
PAGED_FN bool path_ok(const PagedMoveArgs &a, int s, int i, int n)
{
    const int32_t *p = a.path + s * a.path_stride;
    return p[i] >= 0 && p[i] < PAGED_MAX_NEW && (i == 0 || p[i] > p[i - 1]) &&
           (i < n - 1 || (int64_t)a.c.lens[s] + p[i] < (int64_t)a.c.width * a.c.page);
}
PAGED_FN bool commit_fits(const PagedMoveArgs &a, int s)
{
    const int64_t len = a.c.lens[s], n = a.path_len[s];
    return len >= 0 && n >= 0 && len + n <= (int64_t)a.c.width * a.c.page && (!a.path || (n <= PAGED_MAX_NEW && n <= a.path_stride));
}

// Masses as numbers of the same order: NaN above all, 0 and -0 equal.
PAGED_FN uint32_t rank_of(float m)
{
    const uint32_t u = float_bits(m + 0.f);  // (-0 becomes 0)
    if (m != m) return 0xffffffffu;
    return u >> 31 ? ~u : u | 0x80000000u;
}
