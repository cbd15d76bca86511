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

// How a call's keys are cut: row tiles of up to 16 rt query rows (a KV head's n x
// group rows) in z groups, n_split shares of the 32-key tiles.  A workgroup's 8 waves take
// a tile each at a time, and z n_split heads is as many of the CUs as whole shares make (129
// of 256 at worst).  Shares are dealt in groups of 8 tiles in turn, so that the workgroups of
// a head read side by side: where each has a range of its own, their distances can fall
// on the same memory channels (8 heads x 32 rows, 130001 slots, weights in two parts: 61
// to 66 us as ranges, by where the cache lies, 55 to 56 dealt).
//
// rt 2 reads and converts a tile once for 32 rows, rt 1 has twice the workgroups and no
// waiting for the longer sums: rt 1 up to 12 tiles a wave, counted as if rt 1 kept every CU
// at work (one share of 129 to 255 workgroups has up to twice that).  us by that count,
// rt 1 / 2, calls in a row:
//   2.0 (8 heads x 32 rows, 8192 slots) 12.3 / 16.2     5.2 (40 x 60, 2077) 16.7 / 18.9
//   8.0 (8 x 64, 16384) 20.2 / 21.4                     9.8 (40 x 60, 4000) 26.6 / 27.2
//   12.0 (40 x 60, 4900) 28.9 / 26.9, int8 31.0 / 27.5  16 (32 x 32, 16384) 35.0 / 34.0
//   32 (8 x 32, 130001) 72 / 60
// (At 160 workgroups, the 40 x 60 ones, the better limit lies between 10 and 12.)
//
// Shares of less than 8 tiles leave waves idle, and several shares cost a second launch,
// so up to 24 tiles stay one, us as one share and as several, calls in a row: 17 tiles of 32
// heads 8.5 and 9.3; 22 of 8 heads 9.7 and 8.8; 34 of 40 heads 11.2 and 9.9; 32 of 8 heads
// 11.1 and 8.8.  (In a step the second launch takes up to 1.7 us more.)
struct KvqCut {
    int rt, z, n_split;
};
inline int kvq_row_groups(int rows, int rt) { return (rows + 16 * rt - 1) / (16 * rt); }
// the most shares of any cache length
inline int kvq_max_split(int heads, int rows, int n_cu)
{
    const int most = n_cu / (heads * kvq_row_groups(rows, 2));
    return most > 1 ? most : 1;
}
inline KvqCut kvq_cut(int heads, int rows, int tiles, int n_cu)
{
    KvqCut c;
    c.rt = (double)tiles * heads * kvq_row_groups(rows, 1) > 12. * 8 * n_cu && rows > 16 ? 2 : 1;
    c.z = kvq_row_groups(rows, c.rt);
    const int most = tiles <= 24 ? 1 : n_cu / (heads * c.z) > 1 ? n_cu / (heads * c.z) : 1, groups = (tiles + 7) / 8;
    c.n_split = most < groups ? most : groups;
    return c;
}
// Workspace of n_split shares (one writes the output itself): partial sums, and a
// reference and sum of weights for each.
inline size_t kvq_attention_bytes(int heads, int rows, int hd, int n_split)
{
    return n_split == 1 ? 0 : (size_t)heads * n_split * rows * (hd + 2) * 4;
}

// Where attention's sums go: the output, or shares to be combined.
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
    int32_t tiles;
    KvqOut o;
    uint64_t mask[KVQ_MAX_NEW];  // bit j: new row i sees new row j
};
hipError_t launch_kvq_attention(const KvqAttnArgs &a, int hd, int f8, const KvqCut &cut, hipStream_t s);
