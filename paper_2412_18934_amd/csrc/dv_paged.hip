// HIP kernels (gfx950) of the paged KV cache: rotary positions and the write of new rows,
// attention over the pages, accumulated attention weights, commit and eviction.
//
// A (page, KV head, slot) has the row number (page H + head) page_slots + slot, below
// 2^32: row r is K's elements r hd .. + hd, V's column r % 32 of the 32-slot tile
// r / 32 (hd x 32, dim-major), and mass's element r.  A 32-slot tile of keys and its tile of
// values start at the same element.
#include <algorithm>
#include <type_traits>

#include "dv_device.h"
#include "dv_paged_index.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// ---------------------------------------------------------------------------
// sequences, rows and shares

__device__ __forceinline__ void report(const PagedView &c, bool bad)
{
    if (bad && c.fault) *c.fault = 1;  // (every writer writes the same)
}

// Consecutive tiles of a unit
struct Segment {
    Seq q;
    int s, h, b, t0, t1;
    bool whole;  // all of the unit's tiles
};

// Sums over the lanes below `n` (a power of two or more than they are; the others hold 0): all, and up
// to each.  A step is two trips through LDS, so there are no more than n needs.
__device__ __forceinline__ int64_t wave_sum(int64_t x, int n)
{
    for (int off = 1; off < 64 && off < n; off <<= 1) x += __shfl_xor((long long)x, off);
    return (int64_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x);
}
__device__ __forceinline__ int64_t wave_prefix(int64_t x, int n)
{
    for (int off = 1; off < 64 && off < n; off <<= 1) {
        const int64_t y = __shfl_up((long long)x, off);
        if ((int)(threadIdx.x & 63) >= off) x += y;
    }
    return x;
}

// All pieces of a call in one line: sequences in order, of each its units, of each its pieces.
// The waves of a workgroup go through the sequences side by side, 64 at a time, a lane each, so up to
// that many are read once.
struct Pieces {
    const PagedView &c;
    const PagedRowsView &r;
    const int block;
    int size;       // tiles of a piece, about
    int base;       // the lanes' first sequence
    int64_t before, all;  // pieces before the lanes' sequences, and with them
    Seq mine;       // the lane's sequence, its load and the pieces of its units
    Load load;
    int cut;

    __device__ __forceinline__ void read(int first, bool &bad)
    {
        const int i = first + (threadIdx.x & 63);
        base = first;
        mine = {0, 0, 0};
        if (i < c.n_seqs) mine = seq_of(c, r.start, r.n_rows, i, PAGED_MAX_NEW, bad);
        load = load_of(c, mine, r.G, block);
    }
    __device__ __forceinline__ void count()
    {
        cut = load.units ? pieces_of(load.tiles, size) : 0;
        all = before + wave_sum((int64_t)load.units * cut, c.n_seqs - base);
    }
    __device__ __forceinline__ Pieces(const PagedView &c_, const PagedRowsView &r_, int block_, int most, int least, bool &bad)
        : c(c_), r(r_), block(block_), before(0)
    {
        int64_t units = 0, tiles = 0;
        for (int first = 0; first < c.n_seqs; first += 64) {
            read(first, bad);
            units += load.units;
            tiles += (int64_t)load.units * load.tiles;
        }
        size = piece_size(wave_sum(units, c.n_seqs), wave_sum(tiles, c.n_seqs), most, least);
        if (c.n_seqs > 64) read(0, bad);
        count();
    }
    // the lanes come to the next 64 sequences; false if there are none
    __device__ __forceinline__ bool on(bool &bad)
    {
        if (base + 64 >= c.n_seqs) return false;
        before = all;
        read(base + 64, bad);
        count();
        return true;
    }
    // every sequence's first piece, and the pieces of its units
    __device__ __forceinline__ void publish(int2 *line, bool &bad)
    {
        do {
            const int64_t sum = (int64_t)load.units * cut, first = before + wave_prefix(sum, c.n_seqs - base) - sum;
            const int i = base + (int)(threadIdx.x & 63);
            if (i < c.n_seqs) line[i] = make_int2((int)first, cut);
        } while (on(bad));
    }
    // piece number `at`; false if there are not so many
    __device__ __forceinline__ bool take(int64_t at, Segment &x, bool &bad)
    {
        while (at >= all)
            if (!on(bad)) return false;
        const int64_t sum = (int64_t)load.units * cut, up = before + wave_prefix(sum, c.n_seqs - base);
        const int lane = __builtin_ctzll(__ballot(at < up));
        const int units = __builtin_amdgcn_readlane(load.units, lane), tiles = __builtin_amdgcn_readlane(load.tiles, lane);
        const int n = __builtin_amdgcn_readlane(cut, lane), i = (int)(at - __shfl((long long)(up - sum), lane));
        const int unit = (uint32_t)i / (uint32_t)n, p = i - unit * n, blocks = (uint32_t)units / (uint32_t)c.H;
        x.q = {__builtin_amdgcn_readlane(mine.first, lane), __builtin_amdgcn_readlane(mine.n, lane),
               __builtin_amdgcn_readlane(mine.len, lane)};
        x.s = base + lane;
        x.h = __builtin_amdgcn_readfirstlane((uint32_t)unit / (uint32_t)blocks);
        x.b = __builtin_amdgcn_readfirstlane(unit - x.h * blocks);
        x.t0 = __builtin_amdgcn_readfirstlane(piece_start(tiles, n, p));
        x.t1 = __builtin_amdgcn_readfirstlane(piece_start(tiles, n, p + 1));
        x.whole = n == 1;
        return true;
    }
};

// Piece number `at`, false if there is none.  (A workgroup has one: in a loop over pieces the compiler
// keeps 42 registers more.)
__device__ __forceinline__ bool piece_at(const PagedView &c, const PagedRowsView &r, int block, int most, int least, int64_t at,
                                         Segment &x, bool &bad)
{
    Pieces p(c, r, block, most, least, bad);
    return p.take(at, x, bad);
}

// ---------------------------------------------------------------------------
// conversions

// Eight fp32 numbers as three bf16 each, by truncation: their sum is the number
// (unless it is near the smallest ones).
__device__ __forceinline__ void split3(const float *v, u32x4 (&t)[3])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[3][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float x = v[2 * i + j];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                w[p][j] = __float_as_uint(x);
                x -= __uint_as_float(w[p][j] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) t[p][i] = __builtin_amdgcn_perm(w[p][1], w[p][0], 0x07060302u);
    }
}

// Eight bf16, infinities and NaN as 0
__device__ __forceinline__ u32x4 finite(u32x4 x)
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if ((x[w] & 0x7f80u) == 0x7f80u) x[w] &= 0xffff0000u;
        if ((x[w] & 0x7f800000u) == 0x7f800000u) x[w] &= 0xffffu;
    }
    return x;
}

__device__ __forceinline__ f32x4 mfma_bf16(const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight numbers of a row
template <bool BF> __device__ __forceinline__ void load8(const void *p, int64_t at, float (&v)[8])
{
    if constexpr (BF) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(i & 1 ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16);
    } else {
        const float *f = static_cast<const float *>(p) + at;
        const float4 x = *reinterpret_cast<const float4 *>(f), y = *reinterpret_cast<const float4 *>(f + 4);
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
    }
}
__device__ __forceinline__ u32x4 bf16x8_of(const float (&v)[8])
{
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (uint32_t)f2bf(v[2 * i]) | (uint32_t)f2bf(v[2 * i + 1]) << 16;
    return x;
}
template <bool BF> __device__ __forceinline__ void store8(void *p, int64_t at, const float (&v)[8])
{
    if constexpr (BF) {
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(p) + at) = bf16x8_of(v);
    } else {
        float *f = static_cast<float *>(p) + at;
        *reinterpret_cast<float4 *>(f) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(f + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// f(0), .. f(N - 1) with constant arguments: a row tile's registers are never indexed
template <int N, typename F> __device__ __forceinline__ void each(F f)
{
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// ---------------------------------------------------------------------------
// Append: x' = m (x cos - y sin), y' = m (y cos + x sin) for a pair (x, y) at angle position
// * freq.  Angles are reduced in 64 bits (a position of 10^6 times a frequency of 1 leaves
// fp32 seven bits behind the point); sin and cos are those of the angle's fp32 number with the
// rest as a first-order term; products and sums are fp32, and a result is rounded once.
//
// Two ways, by the rows per sequence.  Few (decoding, small trees): a workgroup has 16 or 32 heads of a row, one
// load and one store each; what bounds it is V, where each number of a new slot is 2 bytes of a line of its
// own (64 rows of 40 + 40 + 40 heads: 8.2 us; with the rows and not the head groups as the grid's slow dimension
// 12.8).  Many (8 rows a sequence and more): all heads of 4 rows, so that a row's place and turns are found once, and
// V by way of LDS (3800 rows of 32 + 8 + 8 heads, bf16, 90 MB: 22.3 us, 4.0 TB/s; a workgroup for 16 heads of a row
// 37; the values' workgroups ahead of the others, or in turn with them, 5 to 7 more).

// cos and sin of angle, times m
__device__ __forceinline__ float2 turn_of(double angle, float m)
{
    const double k = rint(angle * 0.15915494309189535);  // whole turns; 2 pi in two parts
    double r = fma(-k, 6.283185307179586, angle);
    r = fma(-k, 2.4492935982947064e-16, r);
    const float hi = (float)r, lo = (float)(r - hi);
    float s, c;
    sincosf(hi, &s, &c);
    return make_float2(m * fmaf(-lo, s, c), m * fmaf(lo, c, s));
}

// The sequence that row `row` belongs to: how many of start[1 ..] are at most row.  All 64 lanes.
__device__ __forceinline__ int seq_of_row(const int32_t *start, int n_seqs, int row)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n_seqs;
    while (hi > lo) {
        const int step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step - 1;
        const int below = __popcll(__ballot(at < hi && start[at + 1] <= row));
        lo = min(lo + below * step, hi);
        if (step == 1) break;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}

// The values of 32 rows and one KV head: V's slots are its fastest dimension, so the rows are turned
// over in LDS, and 8 that stand in 8 aligned slots are one store per dim.
constexpr int V_ROWS = 32;
template <bool BF, int HD> __device__ __forceinline__ void append_values(const PagedAppendArgs &a, int row0, int h)
{
    constexpr int LD = HD + 8;
    __shared__ __align__(16) uint16_t sm_v[V_ROWS][LD];
    __shared__ uint32_t sm_row[V_ROWS];
    __shared__ uint8_t sm_kind[V_ROWS];  // 0: nothing to store, 1: a number per dim, 8: eight, of the rows from here on
    const int tid = threadIdx.x;
    constexpr int U = V_ROWS * (HD / 8) / 256;
    float x[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int e = tid + u * 256, row = row0 + e / (HD / 8);
        if (row < a.n_rows) load8<BF>(a.v, row * a.ldv + (int64_t)h * HD + e % (HD / 8) * 8, x[u]);
    }
    if (tid < 64) {
        bool bad = false;
        int s = seq_of_row(a.start, a.c.n_seqs, row0);
        const int row = row0 + tid;
        if (tid < V_ROWS) {
            s = seq_from(a.start, a.c.n_seqs, s, row);
            sm_row[tid] = NONE;
            if (row < a.n_rows && s < a.c.n_seqs) {
                const Seq q = seq_of(a.c, a.start, a.n_rows, s, 1 << 30, bad);
                if (row >= q.first && row - q.first < q.n) sm_row[tid] = row_of(a.c, s, h, q.len + row - q.first, bad);
            }
        }
        report(a.c, bad);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int e = tid + u * 256;
        *reinterpret_cast<u32x4 *>(&sm_v[e / (HD / 8)][e % (HD / 8) * 8]) = bf16x8_of(x[u]);
    }
    __syncthreads();
    if (tid < V_ROWS) {
        // the first of the 8 aligned slots that a row is among stands in row lead, if all 8 are here
        const uint32_t r = sm_row[tid];
        const int lead = tid - (int)(r % 8);
        bool all = lead >= 0 && lead + 8 <= V_ROWS;
#pragma unroll
        for (int u = 0; u < 8; ++u) all = all && sm_row[lead + u] == r - r % 8 + u;
        sm_kind[tid] = r == NONE ? 0 : !all ? 1 : lead == tid ? 8 : 0;
    }
    __syncthreads();
    for (int e = tid; e < V_ROWS * HD; e += 256) {
        const int i = e / HD, d = e % HD, kind = sm_kind[i];  // (i is the same in a wave)
        if (!kind) continue;
        const uint32_t r = sm_row[i];
        uint16_t *to = a.c.v + ((size_t)(r / PAGED_TILE) * HD + d) * PAGED_TILE + r % PAGED_TILE;
        if (kind == 1) {
            *to = sm_v[i][d];
        } else {
            u32x4 y;
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] = sm_v[i + 2 * u][d] | (uint32_t)sm_v[i + 2 * u + 1][d] << 16;
            *reinterpret_cast<u32x4 *>(to) = y;
        }
    }
}

// 8 dims of a head, from d0 on, turned.  at: the head's numbers in LDS, needed where pairs are half a turn
// apart (they are read in fours where the halves begin at a multiple of 8: one by one costs 8 conflicts a read).
__device__ __forceinline__ void turn8(const PagedAppendArgs &a, const float *at, const float2 *turn, int d0, float (&x)[8])
{
    if (d0 >= a.rot) return;
    const int half = a.rot / 2;
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            if (d0 + i >= a.rot) break;
            const float2 t = turn[(d0 + i) / 2];
            const float u = x[i], w = x[i + 1];
            x[i] = fmaf(u, t.x, -(w * t.y));
            x[i + 1] = fmaf(w, t.x, u * t.y);
        }
    } else if (half % 8 == 0) {
        const bool second = d0 >= half;
        const float *other = at + (second ? d0 - half : d0 + half);
        const float4 *t4 = reinterpret_cast<const float4 *>(turn + (second ? d0 - half : d0));
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 o = *reinterpret_cast<const float4 *>(other + i);
            y[i] = o.x, y[i + 1] = o.y, y[i + 2] = o.z, y[i + 3] = o.w;
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float4 t = t4[i / 2];
            x[i] = fmaf(x[i], t.x, second ? y[i] * t.y : -(y[i] * t.y));
            x[i + 1] = fmaf(x[i + 1], t.z, second ? y[i + 1] * t.w : -(y[i + 1] * t.w));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = d0 + i;
            if (d >= a.rot) break;
            const bool second = d >= half;
            const float y = at[second ? d - half : d + half];
            const float2 t = turn[second ? d - half : d];
            x[i] = fmaf(x[i], t.x, second ? y * t.y : -(y * t.y));
        }
    }
}

// The queries and keys of 4 rows, all heads: a wave finds a row's place and turns, then HD / 8 threads
// have a head at a time and ask for the next one's numbers before they turn its.
template <bool BF, int HD> __device__ __forceinline__ void append_rows(const PagedAppendArgs &a, int row0)
{
    constexpr int R = 4, PER = HD / 8, AT_ONCE = 256 / PER;
    __shared__ __align__(16) float2 sm_turn[R][64];
    __shared__ __align__(16) float sm_x[AT_ONCE][HD];
    __shared__ uint32_t sm_row[R];  // of KV head 0
    __shared__ bool sm_own[R];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, d0 = 8 * (tid % PER), heads = a.Hq + a.c.H, mine = tid / PER;
    float x[8] = {};
    auto fetch = [&](int it) {
        const int i = (uint32_t)it / (uint32_t)heads, head = it - i * heads, row = row0 + i;
        if (i >= R || row >= a.n_rows) return;
        const bool is_q = head < a.Hq;
        load8<BF>(is_q ? a.q : a.k, row * (is_q ? a.ldq : a.ldk) + (int64_t)(is_q ? head : head - a.Hq) * HD + d0, x);
    };
    fetch(mine);
    {
        const int row = row0 + wave;
        bool own = false, bad = false;
        uint32_t r = NONE;
        if (row < a.n_rows) {
            int pos = a.positions ? a.positions[row] : 0;
            const int s = seq_of_row(a.start, a.c.n_seqs, row);
            if (s < a.c.n_seqs) {
                const Seq q = seq_of(a.c, a.start, a.n_rows, s, 1 << 30, bad);
                own = row >= q.first && row - q.first < q.n;
                if (own) {
                    r = row_of(a.c, s, 0, q.len + row - q.first, bad);
                    if (!a.positions) pos = q.len + row - q.first;
                    if (lane < a.rot / 2) sm_turn[wave][lane] = turn_of(pos * a.freq[lane], a.magnitude);
                }
            }
        }
        if (lane == 0) {
            sm_row[wave] = r;
            sm_own[wave] = own;
        }
        report(a.c, bad);
    }
    __syncthreads();
    for (int it = mine; it < R * heads; it += AT_ONCE) {
        const int i = (uint32_t)it / (uint32_t)heads, head = it - i * heads;
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j];
#pragma unroll
        for (int j = 0; j < 8; j += 4) *reinterpret_cast<float4 *>(&sm_x[mine][d0 + j]) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
        fetch(it + AT_ONCE);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a head's threads are of one wave)
        if (sm_own[i]) {
            turn8(a, sm_x[mine], sm_turn[i], d0, y);
            if (head < a.Hq) {
                store8<BF>(a.q, (row0 + i) * a.ldq + (int64_t)head * HD + d0, y);
            } else if (sm_row[i] != NONE) {
                const uint32_t r = sm_row[i] + (uint32_t)(head - a.Hq) * (uint32_t)a.c.page;
                *reinterpret_cast<u32x4 *>(a.c.k + (size_t)r * HD + d0) = bf16x8_of(y);
                if (d0 == 0 && a.c.mass) a.c.mass[r] = 0.f;
            }
        }
        asm volatile("" ::: "memory");
    }
}

// Many rows of a sequence (so there is a start): workgroups of 4 rows' queries and keys, behind them those of 32 rows' values.
template <bool BF, int HD> __global__ __launch_bounds__(256) void k_paged_append_rows(PagedAppendArgs a)
{
    const int groups = (a.n_rows + 3) / 4, b = blockIdx.x - groups;
    if (b < 0)
        append_rows<BF, HD>(a, blockIdx.x * 4);
    else
        append_values<BF, HD>(a, b / a.c.H * V_ROWS, b % a.c.H);
}

// Few rows: workgroup (row, group of heads), 8 dims of a head per thread.
template <bool BF, int HD> __global__ __launch_bounds__(256) void k_paged_append(PagedAppendArgs a)
{
    constexpr int PER = HD / 8, HEADS = 256 / PER;
    __shared__ __align__(16) float2 sm_turn[64];
    __shared__ __align__(16) float sm_x[HEADS][HD];
    const int tid = threadIdx.x, d0 = 8 * (tid % PER), H = a.c.H;
    const int row = blockIdx.x, heads = a.Hq + 2 * H, head = blockIdx.y * HEADS + tid / PER, kv = head - a.Hq;
    // (asked for first: nothing else is needed for these)
    const bool there = head < heads, is_q = kv < 0, is_k = !is_q && kv < H;
    int pos = a.positions ? a.positions[row] : 0;
    float x[8] = {};
    if (there)
        load8<BF>(is_q ? a.q : is_k ? a.k : a.v,
                  row * (is_q ? a.ldq : is_k ? a.ldk : a.ldv) + (int64_t)(is_q ? head : is_k ? kv : kv - H) * HD + d0, x);
    const int s = a.start ? seq_of_row(a.start, a.c.n_seqs, row) : row;
    if (s >= a.c.n_seqs) return;
    bool bad = false;
    const Seq q = seq_of(a.c, a.start, a.n_rows, s, 1 << 30, bad);
    if (row < q.first || row - q.first >= q.n) {
        report(a.c, bad);
        return;
    }
    const int slot = q.len + row - q.first;
    if (!a.positions) pos = slot;
    const uint32_t r = there && !is_q ? row_of(a.c, s, is_k ? kv : kv - H, slot, bad) : NONE;
    if (tid < a.rot / 2) sm_turn[tid] = turn_of(pos * a.freq[tid], a.magnitude);
    if (there && (is_q || is_k))
#pragma unroll
        for (int i = 0; i < 8; i += 4) *reinterpret_cast<float4 *>(&sm_x[tid / PER][d0 + i]) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    __syncthreads();
    report(a.c, bad);
    if (!there) return;
    if (is_q || is_k) turn8(a, sm_x[tid / PER], sm_turn, d0, x);
    if (is_q) {
        store8<BF>(a.q, row * a.ldq + (int64_t)head * HD + d0, x);
        return;
    }
    if (r == NONE) return;
    if (is_k) {
        *reinterpret_cast<u32x4 *>(a.c.k + (size_t)r * HD + d0) = bf16x8_of(x);
        if (d0 == 0 && a.c.mass) a.c.mass[r] = 0.f;
    } else {
        uint16_t *to = a.c.v + ((size_t)(r / PAGED_TILE) * HD + d0) * PAGED_TILE + r % PAGED_TILE;
#pragma unroll
        for (int i = 0; i < 8; ++i) to[i * PAGED_TILE] = f2bf(x[i]);
    }
}

// ---------------------------------------------------------------------------
// Attention of new rows over pages, split over the slots and combined.
//
//   z_ij = scale (q_i . k_j), capped: cap tanh(z / cap); over the slots that row i sees
//   o_i = sum_j exp(z_ij - m_i) v_j / sum_j exp(z_ij - m_i), m_i the largest z: one pass,
//   m and the sums rescaled when a larger z comes.
//
// Rows are a sequence's new tokens times the G query heads of a KV head, 16 rt to a block.
//   S^T = K Q^T: A = 16 keys x dims, B = queries; the A rows of the two products of a tile
//   are keys 8 (i / 4) + 4 t + i % 4, so D gives lane (n, g) the scores of row n for the keys
//   8 g .. + 8, which are the B operand of O^T = V^T P^T; its D has 4 consecutive dims of
//   row n.  A row's numbers belong to lanes n + 16 g, only its maximum crosses lanes.
//
// Roundings: weights and fp32 queries enter as three bf16 parts (all 24 bits), bf16 queries as one.  Scores, maxima
// and sums are fp32.
//
// A wave has a tile of its own, so no barrier stands between tiles; K's registers take the next
// tile when the last row tile's scores are made, V's after the products: up to 128 KB per CU in flight.
// What bounds it: the pages' bytes, once per 16 or 32 rows of a KV head.  532 MB of one sequence 92 us, 5.8 TB/s, 6 of
// them the combining launch; 48 ragged ones (438 MB) 87 us, 5.0 TB/s, 5 of them that launch; short calls 2.5 us
// until a workgroup knows its piece, 3 to 6 until its first tile is there, 2 for the waves' sums.  64 rows of a KV
// head: those 48 143 us, 145 with weights of three parts and not two.
// Measured and taken: 4 waves twice per CU for 8 once (93 for 101 us, 48 ragged sequences); V's loads past
// the caches where a tile is read once (92 for 102, one sequence; K's too: its lines are read in halves, 36 to
// 41 us for eight 16-node trees); queries from LDS and not from 48 registers.
// Not taken: equal shares of all tiles that run over units' ends (the eight trees 39 to 50 for 31 us: each end
// costs a workgroup 4 us); 12 waves per CU (spills with fp32 rows, no gain with bf16); pieces in a loop per workgroup
// (42 registers more); a whole tile ahead in registers of its own (96 for 90 us, 48 ragged sequences; 33 for 31, the
// trees); a whole unit's first pages asked for before its length is known (no difference).

// A 32-slot tile in registers, 16 bytes per lane and load
template <int HD> struct Tile {
    u32x4 k[HD / 16], v[HD / 16];
    // (k: the two products' operands, HD / 32 each)
    __device__ __forceinline__ void load_k(const uint16_t *base, uint32_t row, int lane)
    {
        const uint16_t *p = base + (size_t)row * HD + (8 * ((lane & 15) >> 2) + (lane & 3)) * HD + 8 * (lane >> 4);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < HD / 32; ++c)
                k[t * (HD / 32) + c] = *reinterpret_cast<const u32x4 *>(p + 4 * t * HD + 32 * c);
    }
    template <bool ONCE> __device__ __forceinline__ void load_v(const uint16_t *base, uint32_t row, int lane)
    {
        const uint16_t *p = base + (size_t)row * HD + (lane & 15) * PAGED_TILE + 8 * (lane >> 4);
#pragma unroll
        for (int dt = 0; dt < HD / 16; ++dt) {
            const u32x4 *at = reinterpret_cast<const u32x4 *>(p + dt * 16 * PAGED_TILE);
            v[dt] = ONCE ? __builtin_nontemporal_load(at) : *at;
        }
    }
};

// Row numbers of a wave's next 64 tiles, lane i that of tile t + i step; NONE from `end` on.
__device__ __forceinline__ uint32_t tile_rows(const PagedView &c, int s, int h, int t, int step, int end, int lane, bool &bad)
{
    const int64_t mine = t + (int64_t)lane * step;
    return mine < end ? row_of(c, s, h, (int)mine * PAGED_TILE, bad) : NONE;
}

// Queries of a row block as B operands in LDS, NP parts: [rt][dims / 32][part][lane]
template <int HD, bool BF, int RT, int NW>
__device__ __forceinline__ void stage_queries(const PagedRowsView &r, const Seq &q, int h, int row0, u32x4 *to)
{
    constexpr int NP = BF ? 1 : 3, NC = HD / 32;
    const int rows = q.n * r.G;
    for (int e = threadIdx.x; e < RT * 16 * (HD / 8); e += 64 * NW) {
        const int d8 = e % (HD / 8), row = e / (HD / 8), mine = row0 + row;
        const int at = ((row / 16 * NC + (d8 >> 2)) * NP) * 64 + 16 * (d8 & 3) + row % 16;
        const int64_t from = (int64_t)(q.first + mine / r.G) * r.ldq + ((int64_t)h * r.G + mine % r.G) * HD + 8 * d8;
        if constexpr (BF) {
            u32x4 x = {};
            if (mine < rows) x = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(r.q) + from);
            to[at] = x;
        } else {
            float v[8] = {};
            if (mine < rows) load8<false>(r.q, from, v);
            u32x4 t[3];
            split3(v, t);
            bool odd = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) odd |= !__builtin_isfinite(v[i]);
            if (odd) {  // an infinity or NaN is its first part, the others 0
                t[0] = bf16x8_of(v);
                t[1] = finite(t[1]);
                t[2] = finite(t[2]);
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) to[at + p * 64] = t[p];
        }
    }
}

// Scores of a lane's 8 keys for the row tile at qs.  With a key's infinity the parts of a query that
// are 0 (or of the other sign) make NaN of what is an infinity: where there is a NaN the infinities
// and NaN of K meet the first part alone, which is 0 only where the query is.
template <int HD, bool BF> __device__ __forceinline__ void scores8(const u32x4 *k, const u32x4 *qs, int lane, float (&s)[8])
{
    constexpr int NP = BF ? 1 : 3, NC = HD / 32;
    f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = sa;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const u32x4 q = qs[(c * NP + p) * 64 + lane];
            sa = mfma_bf16(k[c], q, sa);
            sb = mfma_bf16(k[NC + c], q, sb);
        }
    if constexpr (!BF) {
        const float all = ((sa[0] + sa[1]) + (sa[2] + sa[3])) + ((sb[0] + sb[1]) + (sb[2] + sb[3]));
        if (__any(all != all)) {
            sa = sb = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const u32x4 q = qs[(c * NP + p) * 64 + lane];
                    sa = mfma_bf16(p ? finite(k[c]) : k[c], q, sa);
                    sb = mfma_bf16(p ? finite(k[NC + c]) : k[NC + c], q, sb);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = sa[i], s[4 + i] = sb[i];
}

__device__ __forceinline__ void scaled(const PagedRowsView &r, float (&s)[8])
{
    if (r.cap != 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = r.cap * tanhf(s[i] * r.cap_in[0] * r.cap_in[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] *= r.scale;
    }
}

// Mask of a block row, and which of the lane's 8 keys from slot `slot` on it sees
__device__ __forceinline__ uint64_t mask_of(const PagedRowsView &r, const Seq &q, int row)
{
    if (row >= q.n * r.G) return 0ull;
    const int i = row / r.G;
    return r.mask ? r.mask[q.first + i] : ~0ull >> (63 - i);
}
__device__ __forceinline__ uint32_t sees(uint64_t mask, const Seq &q, int slot)
{
    const int first = slot - q.len, mine = min(max(q.len + q.n - slot, 0), 8);
    return (first >= 0 ? (uint32_t)(mask >> (first & 63))
            : first > -8 ? (uint32_t)mask << -first | ((1u << -first) - 1) : 0xffu) & ((1u << mine) - 1);
}

template <bool BF> __device__ __forceinline__ void write_out(const PagedAttnArgs &a, int64_t at, const float (&o)[4])
{
    if constexpr (BF)
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) =
            make_uint2((uint32_t)f2bf(o[0]) | (uint32_t)f2bf(o[1]) << 16, (uint32_t)f2bf(o[2]) | (uint32_t)f2bf(o[3]) << 16);
    else
        *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = make_float4(o[0], o[1], o[2], o[3]);
}

// A finished row: sums over the sum of weights, 0 if it saw nothing
template <int HD, bool BF>
__device__ __forceinline__ void finish(const PagedAttnArgs &a, const Seq &q, int h, int row, int d0, float m, float l, float (&o)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = l == 0.f ? 0.f : o[j] / l;
    const int64_t token = q.first + row / a.r.G, head = (int64_t)h * a.r.G + row % a.r.G;
    write_out<BF>(a, token * a.ldo + head * HD + d0, o);
    if (d0 == 0 && a.stats) a.stats[token * ((int64_t)a.c.H * a.r.G) + head] = make_float2(m, l);
}

template <int HD, bool BF, int RT, int NW, bool WHOLE> __global__ __launch_bounds__(64 * NW, 2) void k_paged_attn(PagedAttnArgs a)
{
    constexpr int NC = HD / 32, ND = HD / 16, NP = BF ? 1 : 3;
    constexpr int SUMS = NW * 16 * RT * (HD + 4) * 4, PARTS = RT * NC * NP * 1024;
    __shared__ __align__(16) char sm[SUMS > PARTS ? SUMS : PARTS];  // queries, then the waves' sums
    __shared__ float sm_m[NW][16 * RT], sm_l[NW][16 * RT];
    u32x4 *qs = reinterpret_cast<u32x4 *>(sm);
    float(*sm_o)[16 * RT][HD + 4] = reinterpret_cast<float(*)[16 * RT][HD + 4]>(sm);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    bool bad = false;

    // piece: where partial sums go
    auto segment = [&](const Segment &x, int piece) {
        const Seq q = x.q;
        const int row0 = x.b * 16 * RT, rows = q.n * a.r.G, t1 = x.t1;
        const int plain = q.len / PAGED_TILE;  // tiles below: all slots committed
        uint32_t ids = tile_rows(a.c, x.s, x.h, x.t0 + wave, NW, t1, lane, bad);
        Tile<HD> kv;
        uint32_t row = __builtin_amdgcn_readlane(ids, 0);
        // (loads never branch: where there is no tile they read the pool's first)
        kv.load_k(a.c.k, row == NONE ? 0 : row, lane);
        kv.template load_v<RT == 1>(a.c.v, row == NONE ? 0 : row, lane);
        stage_queries<HD, BF, RT, NW>(a.r, q, x.h, row0, qs);
        uint64_t mask[RT];
        float m_run[RT], l_run[RT];  // (l_run: of the lane's own keys)
        f32x4 o[RT][ND];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            mask[rt] = t1 > plain ? mask_of(a.r, q, row0 + 16 * rt + n) : 0ull;
            m_run[rt] = -INFINITY;
            l_run[rt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[rt][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
        __syncthreads();
        int at = 0;
        for (int t = x.t0 + wave; t < t1; t += NW) {
            if (!BF || RT > 1) asm volatile("" ::: "memory");  // (queries stay in LDS: in registers they take too many)
            if (++at == 64) {
                ids = tile_rows(a.c, x.s, x.h, t + NW, NW, t1, lane, bad);
                at = 0;
            }
            const uint32_t next = __builtin_amdgcn_readlane(ids, at), from = next == NONE ? 0 : next;
            const bool part = t >= plain;
            bool odd = false;
            uint32_t see[RT];
            if (part) {
                // V without the slots past the last row, which hold anything; infinities and NaN of
                // new rows are taken out as well, and come after, for the rows that see them
                const int mine = min(max(q.len + q.n - (t * PAGED_TILE + 8 * g), 0), 8);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) see[rt] = sees(mask[rt], q, t * PAGED_TILE + 8 * g);
                bool any = false;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        kv.v[dt][i] &= (2 * i < mine ? 0xffffu : 0u) | (2 * i + 1 < mine ? 0xffff0000u : 0u);
                        any |= (kv.v[dt][i] & 0x7f80u) == 0x7f80u || (kv.v[dt][i] & 0x7f800000u) == 0x7f800000u;
                    }
                odd = __any(any);
                if (odd)
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) kv.v[dt] = finite(kv.v[dt]);
            }
            each<RT>([&](auto rt_) {
                constexpr int rt = decltype(rt_)::value;
                const bool none = row == NONE || (RT > 1 && row0 + 16 * rt >= rows);
                float s8[8];
                if (!none) scores8<HD, BF>(kv.k, qs + rt * NC * NP * 64, lane, s8);
                if (rt == RT - 1) kv.load_k(a.c.k, from, lane);
                if (none) return;
                scaled(a.r, s8);
                if (part)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s8[i] = see[rt] >> i & 1 ? s8[i] : -INFINITY;
                float mt = s8[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) mt = fmaxf(mt, s8[i]);
                if (__any(mt > m_run[rt])) {
                    mt = fmaxf(mt, __shfl_xor(mt, 16));
                    mt = fmaxf(mt, __shfl_xor(mt, 32));
                    const float mnew = fmaxf(m_run[rt], mt);
                    const float alpha = m_run[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run[rt] - mnew) * LOG2E);
                    l_run[rt] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[rt][dt][j] *= alpha;
                    m_run[rt] = mnew;
                }
                float ps = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s8[i] = s8[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s8[i] - m_run[rt]) * LOG2E);
                    ps += s8[i];
                }
                l_run[rt] += ps;
                u32x4 p[3];
                split3(s8, p);
#pragma unroll
                for (int i = 0; i < 3; ++i)
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) o[rt][dt] = mfma_bf16(kv.v[dt], p[i], o[rt][dt]);
                if (!odd) return;
                // an infinity or NaN counts for the rows that see its key, however small its weight
                const uint16_t *vt = a.c.v + (size_t)row * HD;
                const int left = min(PAGED_TILE, q.len + q.n - t * PAGED_TILE);
#pragma unroll 1
                for (int key = 0; key < left; ++key) {
                    float pk = s8[0];
#pragma unroll
                    for (int i = 1; i < 8; ++i) pk = (key & 7) == i ? s8[i] : pk;
                    pk = __shfl(pk, 16 * (key >> 3) + n);
                    const bool seen = __shfl((int)see[rt], 16 * (key >> 3) + n) >> (key & 7) & 1;
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float y = bf2f(vt[(dt * 16 + 4 * g + j) * PAGED_TILE + key]);
                            if (!__builtin_isfinite(y) && seen) o[rt][dt][j] += pk * y;
                        }
                }
            });
            kv.template load_v<RT == 1>(a.c.v, from, lane);
            row = next;
        }

        // combine the waves, in their order
        const int rows_here = min(16 * RT, rows - row0), active = min(NW, t1 - x.t0);
        __syncthreads();
        if (wave < active)
            each<RT>([&](auto rt_) {
                constexpr int rt = decltype(rt_)::value;
                float l = l_run[rt];
                l += __shfl_xor(l, 16);
                l += __shfl_xor(l, 32);
                if (16 * rt + n >= rows_here) return;
                if (g == 0) {
                    sm_m[wave][16 * rt + n] = m_run[rt];
                    sm_l[wave][16 * rt + n] = l;
                }
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
                    *reinterpret_cast<f32x4 *>(&sm_o[wave][16 * rt + n][dt * 16 + 4 * g]) = o[rt][dt];
            });
        __syncthreads();
        for (int e = tid; e < rows_here * (HD / 4); e += 64 * NW) {
            const int i = e / (HD / 4), d0 = 4 * (e % (HD / 4));
            float m = -INFINITY, l = 0.f, ov[4] = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < active; ++w) m = fmaxf(m, sm_m[w][i]);
            for (int w = 0; w < active; ++w) {
                // (a wave whose every score is NaN has a largest of -infinity and a sum of NaN)
                const float mw = sm_m[w][i], f = mw == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mw - m) * LOG2E);
                l = fmaf(f, sm_l[w][i], l);
                const f32x4 o4 = *reinterpret_cast<const f32x4 *>(&sm_o[w][i][d0]);
#pragma unroll
                for (int j = 0; j < 4; ++j) ov[j] = fmaf(f, o4[j], ov[j]);
            }
            if (x.whole) {
                finish<HD, BF>(a, q, x.h, row0 + i, d0, m, l, ov);
            } else {
                const int64_t p = (int64_t)piece * 16 * RT + i;
                *reinterpret_cast<float4 *>(a.part_o + p * HD + d0) = make_float4(ov[0], ov[1], ov[2], ov[3]);
                if (d0 == 0) a.part_ml[p] = make_float2(m, l);
            }
        }
    };

    Segment x{};
    if constexpr (WHOLE) {
        x.s = blockIdx.x / a.c.H;
        x.h = blockIdx.x % a.c.H;
        x.q = seq_of(a.c, a.r.start, a.r.n_rows, x.s, PAGED_MAX_NEW, bad);
        const Load w = load_of(a.c, x.q, a.r.G, 16 * RT);
        x.t1 = w.tiles;
        x.whole = true;
        for (x.b = blockIdx.y; x.b < w.units / a.c.H; x.b += gridDim.y) {
            segment(x, 0);
            __syncthreads();
        }
    } else {
        // (the last workgroup writes down for the combining launch how the sequences are cut)
        if (blockIdx.x == gridDim.x - 1) {
            Pieces pieces(a.c, a.r, 16 * RT, a.groups, NW, bad);
            if (wave == 0) pieces.publish(a.line, bad);
        } else if (piece_at(a.c, a.r, 16 * RT, a.groups, NW, blockIdx.x, x, bad)) {
            segment(x, blockIdx.x);
        }
    }
    report(a.c, bad);
}

// The pieces of a row block combined in a launch of its own (5 to 6 us; 7 where it works out again how the
// sequences are cut, in place of finding it in the workspace).  Workgroup (sequence and KV head, rows):
// HD / 4 threads have 4 dims of a row each, and LANES such groups every LANES-th piece; they are
// combined in LDS.  The order is fixed, so are the results.
template <int HD, bool BF, int RT, int LANES> __global__ __launch_bounds__(256) void k_paged_merge(PagedAttnArgs a)
{
    constexpr int PER = HD / 4, AT_ONCE = 256 / PER / LANES, STEP = LANES == 1 ? 2 : 4;
    __shared__ __align__(16) float sm_o[AT_ONCE][LANES][HD];
    __shared__ float2 sm_ml[AT_ONCE][LANES];
    const int tid = threadIdx.x, s = blockIdx.x / a.c.H, h = blockIdx.x % a.c.H, d0 = 4 * (tid % PER);
    const int part = tid / PER % LANES, mine = tid / PER / LANES;
    bool bad = false;
    const Seq q = seq_of(a.c, a.r.start, a.r.n_rows, s, PAGED_MAX_NEW, bad);
    const int2 cut = a.line[s];
    const int n = cut.y;
    if (n < 2) return;  // (nothing, or one workgroup had it all)
    const int64_t before = cut.x;
    const int rows = q.n * a.r.G, blocks = (rows + 16 * RT - 1) / (16 * RT);
    for (int row0 = blockIdx.y * AT_ONCE; row0 < rows; row0 += gridDim.y * AT_ONCE) {
        const int row = row0 + mine, b = row / (16 * RT), i = row % (16 * RT);
        const int64_t first = before + ((int64_t)h * blocks + b) * n;
        float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        if (row < rows)
            for (int g = part; g < n; g += LANES * STEP) {
                float2 ml[STEP];
                float4 x[STEP];
#pragma unroll
                for (int u = 0; u < STEP; ++u) {
                    const int64_t p = (first + min(g + u * LANES, n - 1)) * 16 * RT + i;
                    ml[u] = a.part_ml[p];
                    x[u] = *reinterpret_cast<const float4 *>(a.part_o + p * HD + d0);
                }
                float top = m;
#pragma unroll
                for (int u = 0; u < STEP; ++u) top = g + u * LANES < n ? fmaxf(top, ml[u].x) : top;
                const float f0 = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * LOG2E);
                l *= f0;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] *= f0;
#pragma unroll
                for (int u = 0; u < STEP; ++u) {
                    if (g + u * LANES >= n) break;
                    const float f = ml[u].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((ml[u].x - top) * LOG2E);
                    l = fmaf(f, ml[u].y, l);
                    o[0] = fmaf(f, x[u].x, o[0]);
                    o[1] = fmaf(f, x[u].y, o[1]);
                    o[2] = fmaf(f, x[u].z, o[2]);
                    o[3] = fmaf(f, x[u].w, o[3]);
                }
                m = top;
            }
        __syncthreads();
        *reinterpret_cast<float4 *>(&sm_o[mine][part][d0]) = make_float4(o[0], o[1], o[2], o[3]);
        if (d0 == 0) sm_ml[mine][part] = make_float2(m, l);
        __syncthreads();
        if (part == 0 && row < rows) {
            float top = -INFINITY, ov[4] = {0.f, 0.f, 0.f, 0.f};
            l = 0.f;
#pragma unroll
            for (int k = 0; k < LANES; ++k) top = fmaxf(top, sm_ml[mine][k].x);
#pragma unroll
            for (int k = 0; k < LANES; ++k) {
                const float2 ml = sm_ml[mine][k];
                const float f = ml.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((ml.x - top) * LOG2E);
                const float4 x = *reinterpret_cast<const float4 *>(&sm_o[mine][k][d0]);
                l = fmaf(f, ml.y, l);
                ov[0] = fmaf(f, x.x, ov[0]);
                ov[1] = fmaf(f, x.y, ov[1]);
                ov[2] = fmaf(f, x.z, ov[2]);
                ov[3] = fmaf(f, x.w, ov[3]);
            }
            finish<HD, BF>(a, q, h, row, d0, top, l, ov);
        }
    }
}

// ---------------------------------------------------------------------------
// Mass: mass_j += sum over counted rows of exp(z_ij - m_i) / l_i.  The scores are made again
// from K alone, half of what attention read; a tile belongs to one wave, which adds its
// rows in order, so nothing is atomic.  K and the masses are read again for every 64 rows of a KV head, also for rows
// that do not count.  A tile's masses are asked for with its keys: read where they are added to, they
// hold up the keys behind them (loads return in order; 29 us for 37 of 16 ragged sequences, 4 rows a KV head).
// Now 20.2 us for those (80 MB, 4.0 TB/s), 25.0 for two of up to 8191 slots with 16 fp32 rows of 32 heads (98 MB); with
// 8 waves a workgroup, of which one fits a CU where rows are fp32, 22.0 and 28.7.

// Sum over the 16 lanes of a row of lanes, in all of them: rotations inside the row
__device__ __forceinline__ float row_sum(float x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int y = i == 0   ? __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, false)
                      : i == 1 ? __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xf, 0xf, false)
                      : i == 2 ? __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x122, 0xf, 0xf, false)
                               : __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x121, 0xf, 0xf, false);
        x += __int_as_float(y);
    }
    return x;
}

template <int HD, bool BF> __global__ __launch_bounds__(256, 3) void k_paged_mass(PagedMassArgs a)
{
    constexpr int NC = HD / 32, NP = BF ? 1 : 3, RT = 4, NW = 4;  // row tiles at a time
    __shared__ __align__(16) u32x4 qs[RT * NC * NP * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    bool bad = false;

    auto segment = [&](const Seq &q, int s, int h, int t0, int t1) {
        const int rows = q.n * a.r.G, plain = q.len / PAGED_TILE;
        const uint64_t count = a.count ? a.count[s] : ~0ull;
        for (int row0 = 0; row0 < rows; row0 += 16 * RT) {
            uint32_t ids = tile_rows(a.c, s, h, t0 + wave, NW, t1, lane, bad);
            __syncthreads();
            stage_queries<HD, BF, RT, NW>(a.r, q, h, row0, qs);
            uint64_t mask[RT];
            float m[RT], f[RT];  // a row that does not count: f < 0
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int row = row0 + 16 * rt + n, i = row / a.r.G;
                mask[rt] = mask_of(a.r, q, row);
                m[rt] = 0.f;
                f[rt] = -1.f;
                if (row < rows && count >> i & 1) {
                    const float2 ml = a.stats[(int64_t)(q.first + i) * ((int64_t)a.c.H * a.r.G) + (int64_t)h * a.r.G + row % a.r.G];
                    m[rt] = ml.x;
                    if (ml.y != 0.f) f[rt] = 1.f / ml.y;
                }
            }
            Tile<HD> x;
            int at = 0;
            uint32_t row = __builtin_amdgcn_readlane(ids, 0);
            // (lane (n, g): key 8 g + n % 8)
            float had = a.c.mass[(size_t)(row == NONE ? 0 : row) + 8 * g + (n & 7)];
            x.load_k(a.c.k, row == NONE ? 0 : row, lane);
            __syncthreads();
            for (int t = t0 + wave; t < t1; t += NW) {
                asm volatile("" ::: "memory");  // (queries stay in LDS: in registers they take too many)
                if (++at == 64) {
                    ids = tile_rows(a.c, s, h, t + NW, NW, t1, lane, bad);
                    at = 0;
                }
                const uint32_t next = __builtin_amdgcn_readlane(ids, at), from = next == NONE ? 0 : next;
                float sum[8] = {};
                each<RT>([&](auto rt_) {
                    constexpr int rt = decltype(rt_)::value;
                    if (row0 + 16 * rt >= rows) return;
                    float z[8];
                    scores8<HD, BF>(x.k, qs + rt * NC * NP * 64, lane, z);
                    scaled(a.r, z);
                    const uint32_t see = t < plain ? 0xffu : sees(mask[rt], q, t * PAGED_TILE + 8 * g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float w = __builtin_amdgcn_exp2f((z[i] - m[rt]) * LOG2E) * f[rt];
                        // (f of a NaN sum is NaN, and shows)
                        sum[i] += (see >> i & 1) && !(f[rt] < 0.f) ? w : 0.f;
                    }
                });
                const float old = had;
                had = a.c.mass[(size_t)from + 8 * g + (n & 7)];
                x.load_k(a.c.k, from, lane);
                float mine = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float all = row_sum(sum[i]);
                    mine = (n & 7) == i ? all : mine;
                }
                if (row != NONE && n < 8 && t * PAGED_TILE + 8 * g + n < q.len + q.n)
                    a.c.mass[(size_t)row + 8 * g + n] = old + mine;
                row = next;
            }
        }
    };

    Segment x;
    if (a.whole) {
        const int s = blockIdx.x / a.c.H;
        const Seq q = seq_of(a.c, a.r.start, a.r.n_rows, s, PAGED_MAX_NEW, bad);
        segment(q, s, blockIdx.x % a.c.H, 0, load_of(a.c, q, a.r.G, 1 << 30).tiles);
    } else if (piece_at(a.c, a.r, 1 << 30, gridDim.x, NW, blockIdx.x, x, bad)) {
        segment(x.q, x.s, x.h, x.t0, x.t1);
    }
    report(a.c, bad);
}

// ---------------------------------------------------------------------------
// Commit moves rows of a (layer, sequence, KV head) to lower slots, in order.  Source slots increase, and
// each is at least its destination; so a wave that always has the same columns of K (or dims of V) can
// go through the list by itself: what it overwrites is no later row's source, and a step's loads stand before
// its stores.  What bounds it is V, whose lines hold 32 slots of a dim: five rows of 8 sequences, 40 layers
// of 40 heads 48 us (63 MB of rows; counted 115 MB read and 70 written, 3.8 TB/s), 38 of 16 sequences, 32 of 32, 114
// (501 MB of rows, of which some stay where they are; 247 read and 200 written, 3.9 TB/s).
// Workgroups are small, so that many wait for their chain of lengths, path, table and rows at once: 4 waves
// 52 and 112, 8 waves 70 and 124.

// Rows list[i].x to list[i].y, i < count; NONE in either: not moved.  NW waves.
template <int HD, int NW> __device__ __forceinline__ void move_rows(const PagedView &c, int layer, const uint2 *list, int count)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t base = (size_t)layer * c.n_pages * c.H * c.page;
    if (wave < NW / 2) {  // K: a share of the columns
        constexpr int CH = HD / 4 / NW, ROWS = 64 / CH, U = 4;  // 16 bytes each
        uint16_t *k = c.k + base * HD + (wave * CH + lane % CH) * 8;
        for (int i0 = 0; i0 < count; i0 += ROWS * U) {
            u32x4 x[U];
            uint2 at[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * ROWS + lane / CH;
                at[u] = i < count ? list[i] : make_uint2(NONE, NONE);
                if (at[u].x == NONE || at[u].y == NONE) at[u].y = NONE;
                else x[u] = *reinterpret_cast<const u32x4 *>(k + (size_t)at[u].x * HD);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at[u].y != NONE) *reinterpret_cast<u32x4 *>(k + (size_t)at[u].y * HD) = x[u];
        }
        if (wave == 0 && c.mass) {
            float *mass = c.mass + base;
            for (int i = lane; i < count; i += 64) {
                const uint2 e = list[i];
                if (e.x == NONE || e.y == NONE) continue;
                const float m = mass[e.x];
                mass[e.y] = m;
            }
        }
    } else {  // V: a share of the dims, two of them and 32 rows a load
        constexpr int U = HD / NW;
        uint16_t *v = c.v + base * HD + ((wave - NW / 2) * (2 * HD / NW) + lane / 32) * PAGED_TILE;
        for (int i0 = 0; i0 < count; i0 += 32) {
            const int i = i0 + lane % 32;
            const uint2 e = i < count ? list[i] : make_uint2(NONE, NONE);
            if (e.x == NONE || e.y == NONE) continue;
            uint16_t x[U], *to = v + (size_t)(e.y / PAGED_TILE) * HD * PAGED_TILE + e.y % PAGED_TILE;
            const uint16_t *from = v + (size_t)(e.x / PAGED_TILE) * HD * PAGED_TILE + e.x % PAGED_TILE;
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = from[2 * u * PAGED_TILE];
#pragma unroll
            for (int u = 0; u < U; ++u) to[2 * u * PAGED_TILE] = x[u];
        }
    }
}

template <int HD, int NW> __global__ __launch_bounds__(64 * NW) void k_paged_commit(PagedMoveArgs a)
{
    __shared__ uint2 list[PAGED_MAX_NEW];
    const int h = blockIdx.x % a.c.H, s = blockIdx.x / a.c.H, layer = blockIdx.y;
    const int len = a.c.lens[s], n = a.path_len[s], i = threadIdx.x;
    const bool first = h == 0 && layer == 0 && i == 0, apart = a.new_lens != a.c.lens;
    const bool fits = commit_fits(a, s);
    if (__syncthreads_or(!fits || (i < n && !path_ok(a, s, i, n)))) {
        if (first) report(a.c, true);
        if (first && apart) a.new_lens[s] = len;
        return;
    }
    if (first && apart) a.new_lens[s] = len + n;
    bool bad = false;
    if (i < n) {
        const int from = a.path[s * a.path_stride + i];
        list[i] = from == i ? make_uint2(NONE, NONE)
                            : make_uint2(row_of(a.c, s, h, len + from, bad), row_of(a.c, s, h, len + i, bad));
    }
    __syncthreads();
    report(a.c, bad);
    move_rows<HD, NW>(a.c, layer, list, n);
}

__global__ __launch_bounds__(256) void k_paged_commit_lens(PagedMoveArgs a)
{
    const int s = blockIdx.x * 256 + threadIdx.x;
    if (s >= a.c.n_seqs) return;
    const int len = a.c.lens[s], n = a.path_len[s];
    bool ok = commit_fits(a, s);
    if (a.path)
        for (int i = 0; ok && i < n; ++i) ok = path_ok(a, s, i, n);
    report(a.c, !ok);
    a.new_lens[s] = ok ? len + n : len;
}

// ---------------------------------------------------------------------------
// Eviction, a workgroup for each (layer, sequence, KV head).  The mass that separates what stays is found digit by
// digit from the top, counted in LDS; then every slot's bit is made (equal masses: the lower
// slots), and the slots whose bit is set move up, 24 tiles of source slots at a time: K's rows as they are;
// of V, whose slots are its fastest dimension, 32 dims of all 24 tiles are laid into LDS and
// gathered there, 8 slots of a dim to a store.  Source slots increase and each is at least its
// destination: what a step overwrites is in registers or LDS by then, and no later step's source.
// What bounds it is that V's tiles are read whole for the slots that stay, and the rate of one CU where heads are few:
// 128 heads, 2049 slots to 1024 63 us (1.35 MB a workgroup at 25 GB/s, 10 us before the first row moves);
// 16 ragged sequences of up to 4500 slots to 1500, 64 heads and layers, 389 us (counted 0.93 GB read and 0.61 written,
// 4.0 TB/s).  With V gathered 2 bytes a lane from memory 73 and 460.

constexpr int MOVE_TILES = 24, MOVE = MOVE_TILES * PAGED_TILE, DIMS = 32, V_DIM = 72;  // V_DIM: bytes of a dim's tile in LDS

template <int HD, bool RANKS> __global__ __launch_bounds__(512, 4) void k_paged_evict(PagedMoveArgs a)
{
    constexpr int NT = 512, BITS = 11, BINS = 1 << BITS, BUF = MOVE_TILES * DIMS * V_DIM;
    static_assert(PAGED_MAX_RANKS * 4 + BINS * 4 <= BUF, "ranks and counts stand where V's tiles come");
    extern __shared__ uint32_t sm_bits[];
    __shared__ __align__(16) char sm[BUF];
    __shared__ uint2 list[MOVE];
    __shared__ __align__(16) uint16_t off[MOVE + 16];  // of the rows' numbers in sm, from the 8 slots that hold the first row on
    __shared__ uint32_t sm_wave[NT / 64], sm_bin, sm_above, sm_word[MOVE_TILES + 1], from_tile[MOVE_TILES], to_tile[MOVE_TILES + 2];
    __shared__ int sm_first;
    uint32_t *hist = reinterpret_cast<uint32_t *>(sm), *ranks = hist + BINS;
    const int h = blockIdx.x % a.c.H, s = blockIdx.x / a.c.H, layer = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), N = a.c.lens[s];
    const bool first = h == 0 && layer == 0 && tid == 0, apart = a.new_lens != a.c.lens;
    if (N < 0 || N > (int64_t)a.c.width * a.c.page || N <= a.budget) {
        if (first) report(a.c, N < 0 || N > (int64_t)a.c.width * a.c.page);
        if (first && apart) a.new_lens[s] = N;
        return;
    }
    if (first && apart) a.new_lens[s] = a.budget;
    bool bad = false;
    const int M = N - a.recent, keep = a.budget - a.recent;  // keep < M
    const size_t base = (size_t)layer * a.c.n_pages * a.c.H * a.c.page;
    float *mass = a.c.mass + base;
    auto look = [&](int slot) {
        const uint32_t r = row_of(a.c, s, h, slot, bad);
        return r == NONE ? 0u : rank_of(mass[r]);
    };
    if (RANKS && keep > 0) {
        constexpr int U = 4;
        for (int i0 = tid; i0 < M; i0 += U * NT) {
            uint32_t r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = i0 + u * NT < M ? row_of(a.c, s, h, i0 + u * NT, bad) : NONE;
            float m[U];
#pragma unroll
            for (int u = 0; u < U; ++u) m[u] = mass[r[u] == NONE ? 0 : r[u]];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * NT < M) ranks[i0 + u * NT] = r[u] == NONE ? 0u : rank_of(m[u]);
        }
    }
    auto rank = [&](int slot) { return RANKS ? ranks[slot] : look(slot); };

    // the keep-th largest rank, and how many of that rank stay
    uint32_t want = 0, left = keep;
    if (keep > 0) {
#pragma unroll 1
        for (int shift = 21; shift >= 0; shift -= shift > 10 ? 11 : 10) {
            // digits: bits 31..21, 20..10, 9..0
            const uint32_t mask = shift == 0 ? 0x3ffu : 0x7ffu, above = shift == 21 ? 0u : shift == 10 ? 0xffe00000u : 0xfffffc00u;
            for (int i = tid; i < BINS; i += NT) hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < M; i += NT) {
                const uint32_t r = rank(i);
                if ((r & above) == want) atomicAdd(&hist[r >> shift & mask], 1u);
            }
            __syncthreads();
            // bins from the top, 4 a thread: the one where the count reaches `left`
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += c[i] = hist[BINS - 1 - 4 * tid - i];
            uint32_t up = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t x = __shfl_up(up, o);
                if (lane >= o) up += x;
            }
            if (lane == 63) sm_wave[wave] = up;
            __syncthreads();
            uint32_t before = up - sum;
            for (int i = 0; i < wave; ++i) before += sm_wave[i];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (before < left && left <= before + c[i]) {
                    sm_bin = BINS - 1 - 4 * tid - i;
                    sm_above = before;
                }
                before += c[i];
            }
            __syncthreads();
            want |= sm_bin << shift;
            left -= sm_above;
        }
    }
    // `left` slots of rank `want` stay (the lowest); each wave has a run of slots
    const int run = (N + NT - 1) / NT * 64, lo = min(wave * run, N), hi = min(lo + run, N);
    uint32_t ties = 0;
    if (keep > 0)
        for (int i0 = lo; i0 < hi; i0 += 64) {
            const int i = i0 + lane;
            ties += __popcll(__ballot(i < hi && i < M && rank(i) == want));
        }
    __syncthreads();  // (sm_wave's last readers)
    if (lane == 0) sm_wave[wave] = ties;
    if (tid == 0) sm_first = N;
    __syncthreads();
    uint32_t before = 0;
    for (int i = 0; i < wave; ++i) before += sm_wave[i];
    int mine = N;  // the wave's first slot that goes
    for (int i0 = lo; i0 < hi; i0 += 64) {
        const int i = i0 + lane;
        const uint32_t r = keep > 0 && i < hi && i < M ? rank(i) : 0u;
        const uint64_t tie = __ballot(keep > 0 && i < hi && i < M && r == want);
        const bool stays = i < hi && (i >= M || (keep > 0 && (r > want || (r == want && before + __popcll(tie & ((1ull << lane) - 1)) < left))));
        const uint64_t bits = __ballot(stays);
        before += __popcll(tie);
        if (~bits && mine == N) mine = i0 + __builtin_ctzll(~bits);
        if (lane == 0) sm_bits[i0 >> 5] = (uint32_t)bits;
        if (lane == 32 && i0 + 32 < N) sm_bits[(i0 >> 5) + 1] = (uint32_t)(bits >> 32);
    }
    if (lane == 0) atomicMin(&sm_first, mine);
    __syncthreads();
    // (all ranks are read: mass may move now)

    constexpr int PASSES = HD / DIMS, ROWS = MOVE / PASSES, U = 6;
    static_assert(MOVE_TILES * DIMS * 4 == U * NT && ROWS * (HD / 8) == U * NT, "16 bytes a thread, U times");
    uint16_t *k = a.c.k + base * HD, *v = a.c.v + base * HD;
    const int words = (N + 31) / 32;
    int done = sm_first / 32 * 32;  // (slots before it stay where they are)
    // the next tile from w on with a slot that stays
    auto from = [&](int w) {
        uint64_t any = 0;
        for (; w < words; w += 64)
            if ((any = __ballot(w + lane < words && sm_bits[min(w + lane, words - 1)] != 0))) return w + (int)__builtin_ctzll(any);
        return words;
    };
    for (int w0 = from(done / 32); w0 < words; w0 = from(w0 + MOVE_TILES)) {
        if (wave == 0) {
            const uint32_t c = lane < MOVE_TILES && w0 + lane < words ? __popc(sm_bits[w0 + lane]) : 0u;
            uint32_t up = c;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t x = __shfl_up(up, o);
                if (lane >= o) up += x;
            }
            if (lane <= MOVE_TILES) sm_word[lane] = up - c;
            if (lane < MOVE_TILES) from_tile[lane] = c ? row_of(a.c, s, h, (w0 + lane) * 32, bad) : NONE;
        } else if (wave == 1 && lane < MOVE_TILES + 2) {
            const int to = (done / 32 + lane) * 32;
            to_tile[lane] = to < a.budget ? row_of(a.c, s, h, to, bad) : NONE;
        }
        for (int i = tid; i < MOVE + 16; i += NT) off[i] = 0xffff;
        __syncthreads();
        const int count = sm_word[MOVE_TILES];
        for (int i = tid; i < MOVE; i += NT) {
            if (w0 + (i >> 5) >= words) break;
            const uint32_t w = sm_bits[w0 + (i >> 5)];
            if (!(w >> (i & 31) & 1)) continue;
            const int j = sm_word[i >> 5] + __popc(w & ((1u << (i & 31)) - 1)), to = done + j;
            const uint32_t x = from_tile[i >> 5], y = to_tile[(to >> 5) - (done >> 5)];
            const bool moves = x != NONE && y != NONE && to != w0 * 32 + i;
            list[j] = moves ? make_uint2(x + (i & 31), y + (to & 31)) : make_uint2(NONE, NONE);
            if (x != NONE && y != NONE) off[(done & 7) + j] = (uint16_t)((i >> 5) * DIMS * V_DIM + (i & 31) * 2);
        }
        __syncthreads();
        u32x4 xv[U], xk[U];
        float xm[MOVE / NT + 1];
        auto fetch = [&](int p) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = tid + u * NT, row = p * ROWS + e / (HD / 8);
                const uint32_t x = row < count ? list[row].x : NONE;
                if (x != NONE) xk[u] = *reinterpret_cast<const u32x4 *>(k + (size_t)x * HD + e % (HD / 8) * 8);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = tid + u * NT;
                const uint32_t x = from_tile[e / (DIMS * 4)];
                if (x != NONE)
                    xv[u] = *reinterpret_cast<const u32x4 *>(v + (size_t)x * HD + (p * DIMS + e / 4 % DIMS) * PAGED_TILE + e % 4 * 8);
            }
        };
#pragma unroll
        for (int u = 0; u < MOVE / NT + 1; ++u) {
            const int i = tid + u * NT;
            const uint32_t x = i < count ? list[i].x : NONE;
            if (x != NONE) xm[u] = mass[x];
        }
        fetch(0);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = tid + u * NT;
                uint2 *to = reinterpret_cast<uint2 *>(sm + e / 4 * V_DIM + e % 4 * 16);
                to[0] = make_uint2(xv[u][0], xv[u][1]);
                to[1] = make_uint2(xv[u][2], xv[u][3]);
            }
            // everything that this step's stores may overwrite has been read, by all waves
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = tid + u * NT, row = p * ROWS + e / (HD / 8);
                const uint32_t y = row < count ? list[row].y : NONE;
                if (y != NONE) *reinterpret_cast<u32x4 *>(k + (size_t)y * HD + e % (HD / 8) * 8) = xk[u];
            }
            if (p + 1 < PASSES) fetch(p + 1);
            if (p == 0)
#pragma unroll
                for (int u = 0; u < MOVE / NT + 1; ++u) {
                    const int i = tid + u * NT;
                    const uint32_t y = i < count ? list[i].y : NONE;
                    if (y != NONE) mass[y] = xm[u];
                }
            for (int e = tid; e < ((done & 7) + count + 7) / 8 * DIMS; e += NT) {
                const int dim = e % DIMS, c = e / DIMS, to = (done & ~7) + 8 * c;
                const uint32_t y = to_tile[(to >> 5) - (done >> 5)];
                if (y == NONE) continue;
                uint16_t *at = v + (size_t)y * HD + (p * DIMS + dim) * PAGED_TILE + (to & 31);
                const u32x4 o = *reinterpret_cast<const u32x4 *>(off + 8 * c);
                uint32_t n[8];
                bool all = true;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    n[i] = o[i / 2] >> (16 * (i & 1)) & 0xffff;
                    all &= n[i] != 0xffff;
                }
                if (all) {
                    u32x4 x;
#pragma unroll
                    for (int i = 0; i < 8; i += 2)
                        x[i / 2] = *reinterpret_cast<const uint16_t *>(sm + n[i] + dim * V_DIM) |
                                   (uint32_t)*reinterpret_cast<const uint16_t *>(sm + n[i + 1] + dim * V_DIM) << 16;
                    *reinterpret_cast<u32x4 *>(at) = x;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (n[i] != 0xffff) at[i] = *reinterpret_cast<const uint16_t *>(sm + n[i] + dim * V_DIM);
                }
            }
            __syncthreads();
        }
        done += count;
    }
    report(a.c, bad);
}

__global__ __launch_bounds__(256) void k_paged_evict_lens(PagedMoveArgs a)
{
    const int s = blockIdx.x * 256 + threadIdx.x;
    if (s >= a.c.n_seqs) return;
    const int N = a.c.lens[s];
    if (N <= (int64_t)a.c.width * a.c.page && N > a.budget) a.new_lens[s] = a.budget;
}

// ---------------------------------------------------------------------------
// launches

template <bool BF, int HD> void append(const PagedAppendArgs &a, hipStream_t s)
{
    constexpr int HEADS = 256 / (HD / 8);
    if (a.n_rows >= 8ll * a.c.n_seqs)
        k_paged_append_rows<BF, HD><<<(a.n_rows + 3) / 4 + (a.n_rows + V_ROWS - 1) / V_ROWS * a.c.H, 256, 0, s>>>(a);
    else
        k_paged_append<BF, HD><<<dim3(a.n_rows, (a.Hq + 2 * a.c.H + HEADS - 1) / HEADS), 256, 0, s>>>(a);
}

template <int HD, bool BF, int RT, int NW> void attention(const PagedAttnArgs &a, const PagedCut &cut, hipStream_t s)
{
    const unsigned units = (unsigned)a.c.n_seqs * a.c.H;
    if (cut.whole) {
        k_paged_attn<HD, BF, RT, NW, true><<<dim3(units, cut.blocks), 64 * NW, 0, s>>>(a);
    } else {
        k_paged_attn<HD, BF, RT, NW, false><<<(unsigned)cut.grid + 1, 64 * NW, 0, s>>>(a);
        // (rows beyond the grid's are looped over)
        auto merge = [&](auto lanes_) {
            constexpr int LANES = decltype(lanes_)::value, AT_ONCE = 256 / (HD / 4) / LANES;
            const int groups = std::min((cut.blocks * 16 * RT + AT_ONCE - 1) / AT_ONCE, 4096);
            k_paged_merge<HD, BF, RT, LANES><<<dim3(units, groups), 256, 0, s>>>(a);
        };
        // pieces of a unit, about: with many, 8 groups of threads share them
        if (cut.groups > 4 * (int64_t)units * cut.blocks)
            merge(std::integral_constant<int, 8>{});
        else
            merge(std::integral_constant<int, 1>{});
    }
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs &a, bool bf, hipStream_t s)
{
    if (a.c.hd == 64)
        bf ? append<true, 64>(a, s) : append<false, 64>(a, s);
    else
        bf ? append<true, 128>(a, s) : append<false, 128>(a, s);
    return hipGetLastError();
}

hipError_t launch_paged_attention(const PagedAttnArgs &a, bool bf, const PagedCut &cut, hipStream_t s)
{
    auto of = [&](auto hd_, auto bf_) {
        constexpr int HD = decltype(hd_)::value;
        constexpr bool BF = decltype(bf_)::value;
        cut.rt == 1 ? attention<HD, BF, 1, 4>(a, cut, s) : attention<HD, BF, 2, 4>(a, cut, s);
    };
    using I64 = std::integral_constant<int, 64>;
    using I128 = std::integral_constant<int, 128>;
    if (a.c.hd == 64)
        bf ? of(I64{}, std::true_type{}) : of(I64{}, std::false_type{});
    else
        bf ? of(I128{}, std::true_type{}) : of(I128{}, std::false_type{});
    return hipGetLastError();
}

hipError_t launch_paged_mass(const PagedMassArgs &a, bool bf, hipStream_t s)
{
    if (a.c.hd == 64)
        bf ? k_paged_mass<64, true><<<a.groups, 256, 0, s>>>(a) : k_paged_mass<64, false><<<a.groups, 256, 0, s>>>(a);
    else
        bf ? k_paged_mass<128, true><<<a.groups, 256, 0, s>>>(a) : k_paged_mass<128, false><<<a.groups, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_commit(const PagedMoveArgs &a, hipStream_t s)
{
    if (a.path) {
        const dim3 units((unsigned)a.c.n_seqs * a.c.H, a.c.L);
        a.c.hd == 64 ? k_paged_commit<64, 2><<<units, 128, 0, s>>>(a) : k_paged_commit<128, 2><<<units, 128, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || a.new_lens != a.c.lens) return e;
    }
    k_paged_commit_lens<<<(a.c.n_seqs + 255) / 256, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_evict(const PagedMoveArgs &a, hipStream_t s)
{
    const dim3 units((unsigned)a.c.n_seqs * a.c.H, a.c.L);
    // Ranks are in LDS where all slots of a table row fit; else every pass reads them from memory by way of the table,
    // for short sequences in wide tables too: 66 for 62 us (2049 slots to 1024 in tables of 10368 and 10240),
    // 412 for 389 (16 ragged sequences of up to 4500, tables of 10304 and 10240), 276 for 256 (9000 to 4500).  Widest
    // tables leave room for one workgroup per CU: 449.
    const size_t slots = (size_t)a.c.width * a.c.page;
    if (slots <= PAGED_MAX_RANKS)
        a.c.hd == 64 ? k_paged_evict<64, true><<<units, 512, slots / 8, s>>>(a) : k_paged_evict<128, true><<<units, 512, slots / 8, s>>>(a);
    else
        a.c.hd == 64 ? k_paged_evict<64, false><<<units, 512, slots / 8, s>>>(a) : k_paged_evict<128, false><<<units, 512, slots / 8, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.new_lens != a.c.lens) return e;
    k_paged_evict_lens<<<(a.c.n_seqs + 255) / 256, 256, 0, s>>>(a);
    return hipGetLastError();
}
