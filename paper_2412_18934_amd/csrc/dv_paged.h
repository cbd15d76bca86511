// Internal interface of the paged KV cache: what dv_paged.cpp (entry points) hands to
// the kernels of dv_paged.hip.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime_api.h>
#include <hip/hip_vector_types.h>
#include <stddef.h>
#include <stdint.h>

#define PAGED_TILE 32        // slots of a V tile, and of a step of attention
#define PAGED_MAX_NEW 64     // new rows of a sequence that a mask names
#define PAGED_MAX_EVICT 262144  // slots of a sequence that an eviction marks in LDS, a bit each

// The cache; layer-wise calls have k, v and mass at their layer.
struct PagedView {
    uint16_t *k, *v;
    float *mass;
    const int32_t *table, *lens;
    int32_t *fault;
    int32_t L, H, hd, n_pages, page, n_seqs, width;  // width: table entries of a sequence
};

// The new rows as attention and mass take them.
struct PagedRowsView {
    const void *q;
    int64_t ldq;
    const int32_t *start;
    const uint64_t *mask;
    float scale, cap;
    int32_t G, n_rows;  // query heads per KV head
};

struct PagedAppendArgs {
    PagedView c;
    const int32_t *start, *positions;
    void *q;
    const void *k, *v;
    int64_t ldq, ldk, ldv;
    int32_t Hq, n_rows;         // Hq 0: no queries
    int32_t rot, interleaved;   // rot 0: nothing turned
    float magnitude;
    double freq[64];
};

struct PagedAttnArgs {
    PagedView c;
    PagedRowsView r;
    void *out;
    int64_t ldo;
    float2 *stats;
    int32_t groups;              // workgroups that share all tiles, or 0: one per row block
    float *part_o;               // [2 groups][16 rt][hd] unnormalised sums
    float2 *part_ml;             // [2 groups][16 rt]: largest score and sum of weights
};

// How attention is cut.  rt: 16-row tiles of a row block.
struct PagedCut {
    int rt, blocks, groups;      // blocks: row blocks of the sequence with the most rows
    bool whole;                  // a workgroup per row block and KV head, no joining
};
inline PagedCut paged_cut(int n_seqs, int heads, int group, int max_rows, int max_len, int n_cu)
{
    PagedCut c;
    const int64_t rows = (int64_t)max_rows * group, tiles = max_len / PAGED_TILE + 1;
    c.rt = rows > 16 ? 2 : 1;
    c.blocks = (int)((rows + 16 * c.rt - 1) / (16 * c.rt));
    const int64_t all = (int64_t)n_seqs * heads * c.blocks * tiles;
    c.whole = tiles <= 24;
    const int64_t most = (all + 7) / 8;  // a tile for each wave
    c.groups = c.whole ? 0 : (int)(most < n_cu ? most : n_cu);
    return c;
}
inline size_t paged_attention_bytes(const PagedCut &c, int hd)
{
    return c.whole ? 0 : (size_t)2 * c.groups * 16 * c.rt * (hd + 2) * 4;
}

// Workgroups that share mass's tiles
inline int paged_mass_groups(int n_seqs, int heads, int max_len, int n_cu)
{
    const int64_t most = ((int64_t)n_seqs * heads * (max_len / PAGED_TILE + 1) + 7) / 8;
    return (int)(most < 2 * n_cu ? most : 2 * n_cu);
}

struct PagedMassArgs {
    PagedView c;
    PagedRowsView r;
    const float2 *stats;
    const uint64_t *count;
    int32_t groups;
};

struct PagedMoveArgs {
    PagedView c;
    const int32_t *path, *path_len;  // commit
    int64_t path_stride;
    int32_t budget, recent;          // evict
    int32_t *new_lens;
};

hipError_t launch_paged_append(const PagedAppendArgs &a, bool bf, hipStream_t s);
hipError_t launch_paged_attention(const PagedAttnArgs &a, bool bf, const PagedCut &cut, hipStream_t s);
hipError_t launch_paged_mass(const PagedMassArgs &a, bool bf, hipStream_t s);
// new_lens == c.lens: a second launch writes it
hipError_t launch_paged_commit(const PagedMoveArgs &a, hipStream_t s);
hipError_t launch_paged_evict(const PagedMoveArgs &a, hipStream_t s);
