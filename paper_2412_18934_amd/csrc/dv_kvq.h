// Internal interface of the 8-bit KV cache: what dv_kvq.cpp (entry points, the
// step and prompt paths) hands to the kernels of dv_kvq.hip.  Not part of the
// public ABI.
#pragma once

#include <hip/hip_runtime_api.h>
#include <hip/hip_vector_types.h>
#include <stddef.h>
#include <stdint.h>

#define KVQ_BLOCK 32      // slots that share a scale
#define KVQ_TAIL 96       // bf16 slots per head behind the last whole block: 31 committed + 64 new
#define KVQ_MAX_NEW 64    // new rows of one call

// Consecutive layers of a cache (L of them, from the pointers' layer on).
struct KvqLayers {
    uint8_t *k, *v;              // codes [L][H][nb] blocks of 32 hd bytes (order: dv.h)
    float *scale;                // [L][H][nb][2]
    uint16_t *k_tail, *v_tail;   // [L][H][96][hd], [L][H][3][hd][32]
    int32_t L, H, hd, nb;        // nb: blocks per head (capacity / 32)
    int32_t f8;                  // e4m3 codes (else int8)
    int32_t len;                 // committed slots
};

// bf16 rows in dv_kv's layouts, the same layers.
struct KvqRows {
    uint16_t *k, *v;             // [L][H][cap][hd], [L][H][cap/32][hd][32]
    int32_t cap;
};

// Append rows [len, len + n) of `from` (whole blocks become codes, the rest the tail).
hipError_t launch_kvq_store(const KvqLayers &c, const KvqRows &from, int n, hipStream_t s);
// Read slots [0, len) back into `to`.
hipError_t launch_kvq_load(const KvqLayers &c, const KvqRows &to, hipStream_t s);
// Tail rows r + path[0..n) (r = len % 32, path increasing) follow the r committed
// ones; blocks that are full become codes, the rest moves to the tail's start.
hipError_t launch_kvq_advance(const KvqLayers &c, const int32_t *path, int n, hipStream_t s);

// How a call's keys are cut: row tiles of up to 16 rt query rows (a KV head's
// n x group rows), n_split ranges of per_split 32-key tiles each.
struct KvqCut {
    int rt, z, per_split, n_split;
};
inline int kvq_row_tiles(int rows) { return rows <= 16 ? 1 : 2; }
inline int kvq_row_groups(int rows) { return (rows + 16 * kvq_row_tiles(rows) - 1) / (16 * kvq_row_tiles(rows)); }
// the most ranges of any cache length: about one workgroup per CU
inline int kvq_max_split(int heads, int rows, int n_cu)
{
    const int most = n_cu / (heads * kvq_row_groups(rows));
    return most > 1 ? most : 1;
}
inline KvqCut kvq_cut(int heads, int rows, int tiles, int n_cu)
{
    KvqCut c;
    c.rt = kvq_row_tiles(rows);
    c.z = kvq_row_groups(rows);
    const int most = kvq_max_split(heads, rows, n_cu);
    c.per_split = (tiles + most - 1) / most;
    if (c.per_split < 8) c.per_split = 8;  // a tile for each wave
    c.n_split = (tiles + c.per_split - 1) / c.per_split;
    return c;
}
// Workspace of n_split ranges (one writes the output itself): partial sums, and a
// reference and sum of weights for each.
inline size_t kvq_attention_bytes(int heads, int rows, int hd, int n_split)
{
    return n_split == 1 ? 0 : (size_t)heads * n_split * rows * (hd + 2) * 4;
}

// Where attention's sums go: the output, or ranges to be combined.
struct KvqOut {
    float *out;                  // [n][H G][hd], row stride ldo, or
    int64_t ldo;
    uint16_t *split;             // the split layout of a step's activations (Mpad, half)
    int32_t Mpad, half;
    int32_t H, G;                // KV heads, query heads per KV head
    int32_t rows, rows_out;      // n G; those to write: with the split layout its padding too (zeros)
    int32_t n_split;
    float *part_o;               // [H][n_split][rows][hd] unnormalised sums
    float2 *part_ml;             // [H][n_split][rows]: reference (base 2) and sum of weights
};
struct KvqAttnArgs {
    const uint8_t *k, *v;        // this layer's codes, scales, tail
    const float *scale;
    const uint16_t *kt, *vt;
    int32_t nb;                  // blocks per head (the stride)
    int32_t blocks;              // whole blocks committed
    int32_t r, n;                // committed and new rows of the tail
    const float *q;              // [n][H G][hd], row stride ldq
    int64_t ldq;
    int32_t tiles, per_split;
    KvqOut o;
    uint64_t mask[KVQ_MAX_NEW];  // bit j: new row i sees new row j
};
hipError_t launch_kvq_attention(const KvqAttnArgs &a, int hd, int f8, const KvqCut &cut, hipStream_t s);
