// Internal interface of the paged KV cache: what dv_paged.cpp (entry points) hands to
// the kernels of dv_paged.hip.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime_api.h>
#include <hip/hip_vector_types.h>
#include <stddef.h>
#include <stdint.h>

#define PAGED_TILE 32        // slots of a V tile, and of a step of attention
#define PAGED_MAX_NEW 64     // new rows of a sequence that a mask names
#define PAGED_MAX_LINE 1024    // sequences among which a workgroup looks for its piece (64 at a time, about 1 us)
#define PAGED_MAX_RANKS 10240   // slots of a table row that an eviction keeps the ranks of in LDS
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
    float scale, cap, cap_in[2];  // capped: cap tanh(q.k cap_in[0] cap_in[1])
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
    float *part_o;               // [groups][16 rt][hd] unnormalised sums
    float2 *part_ml;             // [groups][16 rt]: largest score and sum of weights
    int2 *line;                  // [n_seqs]: first piece, and pieces of each unit
};

// How attention is cut.  A unit is a row block (rt row tiles of 16) of a KV head.  Where there are many units, or short
// ones, each has one workgroup that writes the output (whole).  Otherwise units are cut into pieces
// of equal length, whose number follows the lengths in device memory, and a second launch combines them:
// about as many pieces as workgroups fit the chip at once (two per CU), and half of that (rt 2) or all of it (rt 1)
// beyond the units where these alone come near it, so that the longest of a ragged batch are cut.
//
// us as pieces / whole (fp32 but for the third and fourth, 40 KV heads, 16 rows a unit, but for the last two):
//   34 tiles, 40 units 17.1 / 19.5      22 tiles, 40 units 15.0 / 16.0       13 tiles, 40 units 13.9 / 12.6
//   34 tiles, 160 units 23.8 / 20.9     34 tiles, 320 units 35.9 / 30.6      47 tiles, 320 units 42.1 / 40.5
//   66 tiles, 320 units 55.9 / 56.0     34 tiles, 1280 units 90 / 81         66 tiles, 1280 units 152 / 143
//   63 tiles, 384 units of 4 rows 51 / 53    32 tiles, 128 units of 32 rows 25.4 / 21.7
// Pieces beyond 384 units of up to 130 tiles, 4 rows: none 103, half the chip's 95, all of it 89.7, 1.5 times 91;
// 256 units of 32 rows: half 62.8, all 67.
// rt 2 reads a tile once for 32 rows: 8 units of 64 rows, 4063 tiles 160 (rt 1: 290); 40 of 60, 67 tiles 32 (37).
struct PagedCut {
    int rt, blocks;     // blocks: row blocks of the sequence with the most rows, about
    bool whole;
    int groups;         // pieces at most, unless there are more units
    int64_t grid;       // workgroups, enough for both
};
inline PagedCut paged_cut(int n_seqs, int heads, int group, int n_rows, int max_rows, int max_len, int n_cu)
{
    PagedCut c;
    const int64_t rows = (int64_t)max_rows * group, tiles = max_len / PAGED_TILE + 1, slots = 2 * n_cu;
    c.rt = rows > 16 ? 2 : 1;
    const int block = 16 * c.rt;
    c.blocks = (int)((rows + block - 1) / block);
    const int64_t units = (int64_t)n_seqs * heads * c.blocks, limit = units >= 2 * slots ? 96 : 48;
    c.whole = tiles <= (16 + units / 4 < limit ? 16 + units / 4 : limit) || n_seqs > PAGED_MAX_LINE ||
              units >= 8 * slots;  // (pieces of so many would be dozens of MB of sums, for the longest's sake)
    // units of any rows: a sequence has at most 64, and all together n_rows
    const int64_t most = ((int64_t)PAGED_MAX_NEW * group + block - 1) / block * n_seqs, sum = (int64_t)n_rows * group / block + n_seqs;
    const int64_t bound = heads * (most < sum ? most : sum);
    const int64_t pieces = units >= slots / 2 ? units + (c.rt == 1 ? slots : slots / 2) : slots;
    c.groups = c.whole ? 0 : (int)pieces;
    c.grid = c.groups > bound ? c.groups : bound;
    return c;
}
inline size_t paged_attention_bytes(const PagedCut &c, int n_seqs, int hd)
{
    return c.whole ? 0 : (size_t)c.groups * 16 * c.rt * (hd + 2) * 4 + (size_t)n_seqs * 8;
}

// Mass: a workgroup per sequence and KV head where these are many, else pieces as above, three workgroups per CU.
struct PagedMassCut {
    bool whole;
    int64_t grid;
};
inline PagedMassCut paged_mass_cut(int n_seqs, int heads, int max_len, int n_cu)
{
    const int64_t units = (int64_t)n_seqs * heads, slots = 3 * n_cu, most = (units * (max_len / PAGED_TILE + 1) + 3) / 4;
    const int64_t pieces = most < slots ? most : slots;
    return {units >= 8 * slots || n_seqs > PAGED_MAX_LINE, pieces > units ? pieces : units};
}

struct PagedMassArgs {
    PagedView c;
    PagedRowsView r;
    const float2 *stats;
    const uint64_t *count;
    int32_t whole, groups;  // groups: workgroups
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
