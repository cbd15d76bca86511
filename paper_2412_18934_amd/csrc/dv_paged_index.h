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

// The sequence that row `row` belongs to, at least s (n_seqs: none), by steps that double and then halve: mostly
// it is s or near, but any number of empty sequences may lie between.
PAGED_FN int seq_from(const int32_t *start, int n_seqs, int s, int row)
{
    int step = 1;
    for (; s + step <= n_seqs && start[s + step] <= row; step *= 2) s += step;
    for (step /= 2; step > 0; step /= 2)
        if (s + step <= n_seqs && start[s + step] <= row) s += step;
    return s;
}

// The work of a call on a sequence: units (KV heads times row blocks of `block` rows), each of
// them 32-slot tiles.
struct Load {
    int units, tiles;
};
PAGED_FN Load load_of(const PagedView &c, const Seq &q, int G, int block)
{
    if (q.n == 0) return {0, 0};
    return {c.H * (int)(((int64_t)q.n * G + block - 1) / block), (q.len + q.n + PAGED_TILE - 1) / PAGED_TILE};
}

// a / b for numbers that are hardly ever over 32 bits (a 64-bit division is some 100 instructions)
PAGED_FN int64_t quotient(int64_t a, int64_t b)
{
    return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// Units are cut into pieces of about `size` tiles, equal ones of a unit, so that all are `most`
// pieces at most: a unit has less than tiles / size + 1.  With `most` units or more none is cut.
PAGED_FN int piece_size(int64_t units, int64_t tiles, int most, int least)
{
    if (units >= most) return 1 << 30;
    const int64_t size = quotient(tiles + most - units - 1, most - units);
    return size < least ? least : size > (1 << 30) ? 1 << 30 : (int)size;  // (no unit has more than 2^25 tiles)
}
PAGED_FN int pieces_of(int tiles, int size) { return (int)(((uint32_t)tiles + (uint32_t)size - 1) / (uint32_t)size); }
PAGED_FN int piece_start(int tiles, int pieces, int i) { return (int)((uint64_t)tiles * i / pieces); }

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
