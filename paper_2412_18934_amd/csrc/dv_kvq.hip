// HIP kernels (gfx950) of the 8-bit KV cache: quantising rows into blocks, reading
// them back, advancing the tail, and attention over codes and tail.
//
// A block is 32 slots of one KV head, K and V apart, one byte per number and one
// fp32 scale.  The bytes stand in the order in which the attention's matrix
// instructions take them, so that every load there is 16 bytes per lane and 1 KB
// contiguous per wave; lane l = 16 g + n:
//   K: for each 64 dims p and tile t (0, 1), 1 KB: lane l holds slot
//      8 (n / 4) + 4 t + n % 4, dims 64 p + 8 g .. +8, then 64 p + 32 + 8 g .. +8;
//   V: for each 32 dims p, 1 KB: lane l holds slots 8 g .. +8 of dim 32 p + n, then
//      of dim 32 p + 16 + n.
#include <type_traits>

#include "dv_device.h"
#include "dv_internal.h"
#include "dv_kvq.h"

namespace {

// ---------------------------------------------------------------------------
// codes

// The largest magnitude of a block as bf16 bits: without the sign they order like
// the numbers, infinities and NaN above all finite ones.
__device__ __forceinline__ uint32_t max_bits(uint32_t m, const u32x4 &x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
    return m;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t m)
{
#pragma unroll
    for (int off = 32; off; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
    return m;
}

// A block's scale and the factor of its codes.  Below 2^-100 the factor could leave
// fp32: such a block is zero.  A block with an infinity or NaN has no scale, and
// reads as NaN.
struct BlockScale {
    float scale, inv;
};
template <bool F8> __device__ __forceinline__ BlockScale block_scale(uint32_t bits)
{
    constexpr float top = F8 ? 448.f : 127.f;
    const float most = bf2f((uint16_t)bits);
    if (bits >= 0x7f80u) return {__uint_as_float(0x7fc00000u), 0.f};
    if (most < 0x1p-100f) return {0.f, 0.f};
    return {most / top, top / most};
}

// Codes of eight bf16 numbers, x inv rounded to fp32, then to the nearest code,
// ties to even.  |x inv| is at most top (1 + 2^-23), which rounds to top.  (inv 0
// makes NaN of an infinity: such a block's codes are 0 by choice.)
template <bool F8> __device__ __forceinline__ uint2 codes8(const u32x4 &x, float inv)
{
#pragma clang fp contract(off)
    if (inv == 0.f) return make_uint2(0u, 0u);
    uint32_t d[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f[2 * i] = __uint_as_float(x[2 * h + i] << 16) * inv;
            f[2 * i + 1] = __uint_as_float(x[2 * h + i] & 0xffff0000u) * inv;
        }
        if constexpr (F8) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
            d[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
        } else {
            // 1.5 2^23 + y: the sum's low byte is y rounded to nearest even
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(f[i] + 12582912.f);
            const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u);
            const uint32_t hi = __builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u);
            d[h] = lo | hi << 16;
        }
    }
    return make_uint2(d[0], d[1]);
}

template <bool F8> __device__ __forceinline__ void put_codes(const u32x4 &x, const u32x4 &y, float inv, uint8_t *to)
{
    const uint2 lo = codes8<F8>(x, inv), hi = codes8<F8>(y, inv);
    __builtin_nontemporal_store((u32x4){lo.x, lo.y, hi.x, hi.y}, reinterpret_cast<u32x4 *>(to));
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// scale x code of eight codes, rounded to fp32, then to bf16 (nearest even)
template <bool F8> __device__ __forceinline__ u32x4 scaled_bf16(uint32_t lo, uint32_t hi, float scale)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? lo : hi;
        f32x2 x;
        if constexpr (F8)
            x = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(w, true) : __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
        else
            x = (f32x2){(float)(int8_t)(w >> (16 * (i & 1))), (float)(int8_t)(w >> (16 * (i & 1) + 8))};
        const f32x2 y = {x[0] * scale, x[1] * scale};
        r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
    }
    return r;
}

// The numbers of a lane's share of a block, 8 to a vector: pieces 2 j and 2 j + 1 are
// the two halves of the lane's 16 bytes in the block's j-th KB.
__device__ __forceinline__ int k_slot(int lane, int t) { return 8 * ((lane & 15) >> 2) + 4 * t + (lane & 3); }

// A lane's K numbers are two 64-byte pieces of its row.  For loads and stores of whole
// 128-byte lines, lanes n and n ^ 8 exchange: the first halves of both rows become lane
// n < 8's and the second ones lane n + 8's.  (Its own inverse.)
__device__ __forceinline__ void swap_halves(u32x4 &x0, u32x4 &x1, bool upper)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t give = upper ? x0[i] : x1[i];
        const uint32_t get = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)give, 0x128 /* rotate 16 lanes by 8 */, 0xf, 0xf, false);
        if (upper) x0[i] = get;
        else x1[i] = get;
    }
}
// Where piece `half` of KB j is then: row n & 7 (half 0) or that + 8, its dims by the lane.
__device__ __forceinline__ int k_line(int lane, int j, int half, int hd)
{
    return k_slot((lane & 55) | 8 * half, j & 1) * hd + 64 * (j >> 1) + 4 * (lane & 8) + 8 * (lane >> 4);
}

// Quantise one block by one wave: x[j][half] are its numbers.
template <bool F8, int HD>
__device__ __forceinline__ void quantise(const u32x4 (&x)[HD / 32][2], uint8_t *codes, float *scale, int lane)
{
    constexpr int NJ = HD / 32;
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) m = max_bits(max_bits(m, x[j][0]), x[j][1]);
    const BlockScale b = block_scale<F8>(wave_max(m));
#pragma unroll
    for (int j = 0; j < NJ; ++j)
        put_codes<F8>(x[j][0], x[j][1], b.inv, codes + (j * 64 + lane) * 16);
    if (lane == 0) *scale = b.scale;
}

// Eight slots of a dim of V: x's from slot `first` on, y's before
__device__ __forceinline__ u32x4 join(const u32x4 &x, const u32x4 &y, int first)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t old = (2 * i < first ? 0xffffu : 0u) | (2 * i + 1 < first ? 0xffff0000u : 0u);
        r[i] = (y[i] & old) | (x[i] & ~old);
    }
    return r;
}

// Slots [s0, s1) of 32 slots of one head by one wave, K rows or a V tile; the others stay.
// All is read before anything is written, so that one latency is paid, not eight.
template <int HD> struct CopySlots {
    static constexpr int N = HD / 16;
    u32x4 x[N];
    // K: rows, slot by slot.  V: octets of slots, those at the ends joined with what is there
    __device__ __forceinline__ void read(const uint16_t *to, const uint16_t *from, bool is_v, int s0, int s1, int lane)
    {
        if (is_v) {
            u32x4 y[N];
            const int s = 8 * (lane & 3);
            const bool some = s < s1 && s + 8 > s0, whole = s >= s0 && s + 8 <= s1;
            if (some) {
#pragma unroll
                for (int k = 0; k < N; ++k) x[k] = *reinterpret_cast<const u32x4 *>(from + (lane + 64 * k) * 8);
            }
            if (some && !whole) {
#pragma unroll
                for (int k = 0; k < N; ++k) y[k] = *reinterpret_cast<const u32x4 *>(to + (lane + 64 * k) * 8);
#pragma unroll
                for (int k = 0; k < N; ++k) x[k] = join(y[k], join(x[k], y[k], s0 - s), s1 - s);
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int e = lane + 64 * k, s = e / (HD / 8);
                if (s >= s0 && s < s1) x[k] = *reinterpret_cast<const u32x4 *>(from + e * 8);
            }
        }
    }
    __device__ __forceinline__ void write(uint16_t *to, bool is_v, int s0, int s1, int lane) const
    {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int e = lane + 64 * k, s = is_v ? 8 * (lane & 3) : e / (HD / 8);
            if (s < s1 && s + (is_v ? 8 : 1) > s0) *reinterpret_cast<u32x4 *>(to + e * 8) = x[k];
        }
    }
};

// ---------------------------------------------------------------------------
// Store: a wave per block and per K or V (blockIdx.y), four to a workgroup.  The
// wave of a head's first block also writes the new tail, after it has read the old
// one (both by the same wave, in that order).
//
// A block is a wave's registers: 16 bytes per lane and load, one maximum over the
// wave, 16 bytes of codes per lane and store, in the operands' order.  So nothing goes
// through LDS and the rows are read once, K by whole lines (by half ones 3% longer).
// Bound by memory: 2 bytes read and 1 written per number, none of them used again here, so
// they go past the caches (through them 6% longer).  1024 rows of a 13B model's 1600 heads
// (1.26 GB) 195 us, 6.5 TB/s, where the same bytes moved by nothing but loads and stores
// take 191; 160 rows of 1024 heads (126 MB) 24 us, 5.2 TB/s (21).  Rows that begin and end
// inside a block cost the old tail, which is read, and V's tiles, whose lines hold all 32
// slots: 150 rows behind 333 30 us.  Few rows take a launch, 3.5 us.

struct StoreArgs {
    KvqLayers c;
    KvqRows from;
    int32_t n, full;  // rows, whole blocks that they complete
    int32_t jobs;     // blocks per head, at least one
};

template <bool F8, int HD> __global__ __launch_bounds__(256) void k_kvq_store(StoreArgs a)
{
    constexpr int NJ = HD / 32;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= (int64_t)a.c.L * a.c.H * a.jobs) return;
    const int64_t lh = w / a.jobs;
    const int job = (int)(w - lh * a.jobs);
    const bool is_v = blockIdx.y != 0;
    const int b0 = a.c.len / KVQ_BLOCK, r = a.c.len % KVQ_BLOCK;
    uint16_t *tail = (is_v ? a.c.v_tail : a.c.k_tail) + lh * KVQ_TAIL * HD;
    const uint16_t *rows = (is_v ? a.from.v : a.from.k) + lh * a.from.cap * HD;
    u32x4 x[NJ][2];
    if (job < a.full) {
        const int old = job == 0 ? r : 0;  // rows that the tail holds
        const uint16_t *block = rows + (size_t)(b0 + job) * KVQ_BLOCK * HD;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int s = is_v ? 8 * g : k_slot(lane & 55 | 8 * half, j & 1);
                const int e = is_v ? (32 * j + 16 * half + n) * 32 + s : s * HD + 64 * (j >> 1) + 4 * (n & 8) + 8 * g;
                x[j][half] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>((s < old ? tail : block) + e));
            }
        if (!is_v)
#pragma unroll
            for (int j = 0; j < NJ; ++j) swap_halves(x[j][0], x[j][1], n & 8);
        if (is_v && old > 8 * g && old < 8 * g + 8) {  // old and new slots in one octet
            u32x4 y[NJ][2];
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    y[j][half] = *reinterpret_cast<const u32x4 *>(block + (32 * j + 16 * half + n) * 32 + 8 * g);
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int half = 0; half < 2; ++half) x[j][half] = join(y[j][half], x[j][half], old - 8 * g);
        }
    }
    // tail slots [s0, s1): the rows behind the last whole block
    const int b1 = b0 + a.full, s0 = a.full ? 0 : r, s1 = job == 0 ? a.c.len + a.n - b1 * KVQ_BLOCK : 0;
    CopySlots<HD> rest;
    if (s1 > s0) rest.read(tail, rows + (size_t)b1 * KVQ_BLOCK * HD, is_v, s0, s1, lane);
    if (job < a.full) {
        const int64_t at = lh * a.c.nb + b0 + job;
        quantise<F8, HD>(x, (is_v ? a.c.v : a.c.k) + at * KVQ_BLOCK * HD, a.c.scale + at * 2 + is_v, lane);
    }
    if (s1 > s0) rest.write(tail, is_v, s0, s1, lane);
}

// ---------------------------------------------------------------------------
// Load: a wave per block, the tail's committed rows as one more; store backwards, 1 byte
// read and 2 written per number.  Bound by memory: 8191 slots of 320 heads (2.0 GB)
// 336 us, 6.0 TB/s; 333 slots of 1024 heads (265 MB) 46.5 us, 5.7 TB/s.  K is written by
// whole lines (by half ones 12% longer), all of it past the caches (through them 10%
// longer); the conversion is 2.5 instructions a number (with a rounding to bf16 by
// integers four times that, and 4% longer).
//
// A number is its code x scale, rounded to fp32 and then to bf16, the cache's type: two
// roundings of 2^-24 and 2^-8, beside a code's own of up to half a step.

struct LoadArgs {
    KvqLayers c;
    KvqRows to;
    int32_t jobs;  // whole blocks, and one for the tail
};

template <bool F8, int HD> __global__ __launch_bounds__(256) void k_kvq_load(LoadArgs a)
{
    constexpr int NJ = HD / 32;
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= (int64_t)a.c.L * a.c.H * a.jobs) return;
    const int64_t lh = w / a.jobs;
    const int b = (int)(w - lh * a.jobs), blocks = a.c.len / KVQ_BLOCK, r = a.c.len % KVQ_BLOCK;
    const bool is_v = blockIdx.y != 0;
    const int n = lane & 15, g = lane >> 4;
    // K rows, or the V tile, of the block
    uint16_t *to = (is_v ? a.to.v : a.to.k) + (lh * a.to.cap + (int64_t)b * KVQ_BLOCK) * HD;
    if (b < blocks) {
        const int64_t at = lh * a.c.nb + b;
        const uint8_t *codes = (is_v ? a.c.v : a.c.k) + at * KVQ_BLOCK * HD;
        const float scale = a.c.scale[at * 2 + is_v];
        u32x4 x[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes + (j * 64 + lane) * 16));
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            u32x4 y[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) y[half] = scaled_bf16<F8>(x[j][2 * half], x[j][2 * half + 1], scale);
            if (is_v) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    __builtin_nontemporal_store(y[half], reinterpret_cast<u32x4 *>(to + (32 * j + 16 * half + n) * 32 + 8 * g));
            } else {
                swap_halves(y[0], y[1], n & 8);
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    __builtin_nontemporal_store(y[half], reinterpret_cast<u32x4 *>(to + k_line(lane, j, half, HD)));
            }
        }
        return;
    }
    CopySlots<HD> x;
    x.read(to, (is_v ? a.c.v_tail : a.c.k_tail) + lh * KVQ_TAIL * HD, is_v, 0, r, lane);
    x.write(to, is_v, 0, r, lane);
}

// ---------------------------------------------------------------------------
// Advance: a workgroup per (layer, head) and V or K.  New row j is accepted where bit j
// of `mask` is set, and follows those below it, so a row's place is a count of bits.
// Every row that is needed is in LDS, in its new order, before any is written.  A
// block's hd / 32 KB are quantised by different waves, which share its maximum.
//
// Moves a few KB per head, so it is bound by the latency of one read, LDS and write
// chain: all loads of a thread are in flight at once, V is written in whole octets of
// slots, and 6 workgroups share a CU, so that the 3200 of a 13B model are about two
// rounds.  5 of 16 rows of its 1600 heads (8.2 MB) 8.2 us; 38 of 64 rows of 1024 heads,
// two blocks filled (52 MB), 14.7 us, 3.6 TB/s.  A wave for each block of a head and one
// for the rest took 16 us.

struct AdvanceArgs {
    KvqLayers c;
    uint64_t mask;
    int32_t total, full, first;  // rows, whole blocks among them, first row whose slot changes
    int32_t last;                // last accepted row's slot
};
// V in LDS: slots of a dim from the octet of the first needed row on, an odd number of
// 16 bytes apart
__host__ __device__ constexpr int advance_stride(int total, int lo) { return ((total - lo / 8 * 8 + 7) / 8 | 1) * 8; }
__host__ __device__ constexpr int advance_lds(int hd, int total, int lo)  // 16-bit numbers
{
    return (total - lo) * hd > advance_stride(total, lo) * hd ? (total - lo) * hd : advance_stride(total, lo) * hd;
}

template <bool F8, int HD> __global__ __launch_bounds__(256, 6) void k_kvq_advance(AdvanceArgs a)
{
    constexpr int NJ = HD / 32, nt = 256;
    extern __shared__ __align__(16) uint16_t buf[];
    __shared__ uint32_t sm_top[2][NJ];
    __shared__ __align__(8) uint8_t sm_row[KVQ_TAIL];  // the row that a slot becomes, 255: none
    const int64_t lh = blockIdx.x;
    const bool is_v = blockIdx.y == 0;  // (the longer ones first)
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int r = a.c.len % KVQ_BLOCK;
    uint16_t *tail = (is_v ? a.c.v_tail : a.c.k_tail) + lh * KVQ_TAIL * HD;
    const int lo = a.full ? 0 : a.first, lo8 = lo / 8 * 8;  // rows from here on are needed
    const int vs = advance_stride(a.total, lo);
    if (tid < KVQ_TAIL) {
        const uint64_t bit = 1ull << ((tid - r) & 63);
        sm_row[tid] = tid < r ? tid : tid <= a.last && a.mask & bit ? r + __popcll(a.mask & (bit - 1)) : 255;
    }
    constexpr int IN = 3 * HD * 4 / nt;  // 16 bytes each of at most three tiles, all in flight
    u32x4 x[IN];
    auto slot = [&](int e) { return (lo / 32 + e / (HD * 4)) * 32 + 8 * (e & 3); };  // V: first of eight
    if (is_v) {
        const int end = (a.last / 32 + 1 - lo / 32) * HD * 4;
        auto skip = [&](int e) { return e >= end || slot(e) < lo8 || slot(e) > a.last; };
#pragma unroll
        for (int k = 0; k < IN; ++k) {
            const int e = tid + k * nt, s = slot(e), d = e / 4 % HD;
            if (!skip(e)) x[k] = *reinterpret_cast<const u32x4 *>(tail + ((s >> 5) * HD + d) * 32 + (s & 31));
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < IN; ++k) {
            const int e = tid + k * nt;
            if (skip(e)) continue;
            const uint2 row = *reinterpret_cast<const uint2 *>(sm_row + slot(e));
            uint16_t *to = buf + e / 4 % HD * vs - lo8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t t = ((i < 4 ? row.x : row.y) >> (8 * (i & 3))) & 0xff;
                if (t != 255) to[t] = (uint16_t)(x[k][i >> 1] >> (16 * (i & 1)));
            }
        }
    } else {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < IN; ++k) {
            const int e = tid + k * nt, s = lo + e / (HD / 8);
            if (s <= a.last && sm_row[s] != 255) x[k] = *reinterpret_cast<const u32x4 *>(tail + s * HD + e % (HD / 8) * 8);
        }
#pragma unroll
        for (int k = 0; k < IN; ++k) {
            const int e = tid + k * nt, s = lo + e / (HD / 8);
            if (s <= a.last && sm_row[s] != 255) *reinterpret_cast<u32x4 *>(buf + (sm_row[s] - lo) * HD + e % (HD / 8) * 8) = x[k];
        }
    }
    __syncthreads();
    if (a.full) {
        // unit (block, KB), 4 waves: at most two each
        constexpr int MOST = 2 * NJ / 4;
        u32x4 x[MOST][2];
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            const int u = (tid >> 6) + 4 * k, b = u / NJ, j = u % NJ;
            if (u >= a.full * NJ) break;
#pragma unroll
            for (int half = 0; half < 2; ++half)
                x[k][half] = *reinterpret_cast<const u32x4 *>(
                    is_v ? buf + (32 * j + 16 * half + n) * vs + b * KVQ_BLOCK + 8 * g
                         : buf + (b * KVQ_BLOCK + k_slot(lane, j & 1)) * HD + 64 * (j >> 1) + 32 * half + 8 * g);
            const uint32_t top = wave_max(max_bits(max_bits(0, x[k][0]), x[k][1]));
            if (lane == 0) sm_top[b][j] = top;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            const int u = (tid >> 6) + 4 * k, b = u / NJ, j = u % NJ;
            if (u >= a.full * NJ) break;
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < NJ; ++i) top = max(top, sm_top[b][i]);
            const BlockScale s = block_scale<F8>(top);
            const int64_t at = lh * a.c.nb + a.c.len / KVQ_BLOCK + b;
            put_codes<F8>(x[k][0], x[k][1], s.inv, (is_v ? a.c.v : a.c.k) + at * KVQ_BLOCK * HD + (j * 64 + lane) * 16);
            if (j == 0 && lane == 0) a.c.scale[at * 2 + is_v] = s.scale;
        }
    }
    // the rows behind the whole blocks, from the tail's start; slots [s0, s1) change
    const int base = a.full * KVQ_BLOCK, s0 = a.full ? 0 : lo8, s1 = a.total - base;
    if (is_v) {
#pragma unroll
        for (int k = 0; k < IN; ++k) {
            const int e = tid + k * nt, s = slot(e), d = e / 4 % HD;
            if (s < s0 || s >= s1) continue;
            // (slots behind the rows keep what the same thread read from them)
            u32x4 y = *reinterpret_cast<const u32x4 *>(buf + d * vs + base + s - lo8);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t keep = (s + 2 * i < s1 ? 0u : 0xffffu) | (s + 2 * i + 1 < s1 ? 0u : 0xffff0000u);
                y[i] = (y[i] & ~keep) | (x[k][i] & keep);
            }
            *reinterpret_cast<u32x4 *>(tail + ((s >> 5) * HD + d) * 32 + (s & 31)) = y;
        }
    } else {
        const int k0 = a.full ? 0 : lo;
        for (int e = k0 * (HD / 8) + tid; e < s1 * (HD / 8); e += nt)
            *reinterpret_cast<u32x4 *>(tail + e * 8) = *reinterpret_cast<const u32x4 *>(buf + (base - lo) * HD + e * 8);
    }
}

// ---------------------------------------------------------------------------
// Attention of a tree's new rows over codes and tail, split over keys.
//
//   s_ij = (q_i . k_j) / sqrt(hd) over the keys that row i sees: all committed
//   ones, and new row j where bit j of its mask is set;
//   o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i), 0 if it sees none.
//
// Workgroup (split, KV head, row group): its share of the 32-key tiles (blocks of codes,
// then up to three tiles of the tail) is groups of eight in turn, a tile a wave, each with
// a running reference m and sum per query row.  The waves are combined in LDS; a second
// launch combines the shares, in their order.  Rows are the n new tokens x the G query
// heads that share the KV head.
//
//   S^T = K Q^T: A = 16 keys x dims, B = queries; D gives lane (n, g) the scores of
//   row n for the 8 consecutive keys 8 g .. +8 of the tile, which are the B operand
//   of O^T = V^T P^T; its D has 4 consecutive dims of row n.  So a row's numbers all
//   belong to lanes n + 16 g, and only its reference ever crosses lanes.
//
// Codes enter the matrix instructions as codes, scales go onto scores and weights.
// Each query and weight is one fp32 number in parts:
//   int8 K: q as a 23-bit integer relative to its row's largest, in three signed bytes;
//     the products are exact integers, and K's bytes are operands as they stand;
//   e4m3 K: q in two fp16 (11 + 11 bits and a sign between), its row scaled to a largest of
//     2^10 .. 2^11 so that the low part stays normal; e4m3 is exact in fp16;
//   V: weights in three bf16 (8 + 8 + 8 bits: all of them); int8 and e4m3 are exact in bf16;
//   tail: q and weights in three bf16.
// Weights are exp2(s - m) with m a reference that a row's scores exceed by at most
// LAZY (in base 2): it moves, and the sums are rescaled, only when a score is further
// above it, which after the first tiles is rare.  V's scales likewise: the sums are
// in units of the largest scale so far, and 2^-32 of that (W_UNIT), so that a weight times its
// scale is a normal number while scales differ by up to 2^126, and the sums stay far
// below fp32's end.
//
// Roundings: a query to 2^-22 of its row's largest (int8: half a step of an integer of at
// least 2^21) or 2^-23 of itself and 2^-35 of its row's largest (e4m3);
// weights, products and sums are fp32 (int8 scores integers).  Against 64 bits the outputs
// are about as near as a plain fp32 computation's.  (Weights in two fp16, which have 22 bits
// and an end at 2^-24 of the unit, lost those of small weights and of blocks whose
// scale is small beside an earlier one's: 23% of an output at a ratio of 2^36.  Three bf16
// cost nothing with few rows, 8 to 11% with many.)
//
// What bounds it: with few rows the codes' bytes (2 hd + 8 / 32 per key and head); with
// more, the conversion of V and the parts' matrix instructions, which come per tile and
// per row.  8 waves of a workgroup take tiles of their own, so no barrier stands between
// tiles, and each asks for its next tile when the scores of the last row tile have used
// K (V is converted by then): 64 KB per CU in flight while weights and sums are made.
// Times of calls in a row, with the merge where there is one; in brackets what two tiles in
// flight, in two sets of registers and twice the code, took more or less (with weights in
// two parts, as all that was not taken):
//   8 heads x 32 rows, 130001 slots (267 MB)  57 to 61.5 us (+3), 4.5 TB/s; reading alone,
//                                             this way cut, 41 to 45, and the merge 4.5
//   32 heads x 1 row, 8191 slots (67 MB)      17.5 (+0.5): reading alone 12.4, merge
//   40 heads x 60 rows, 2077 slots, e4m3      16.6 (+1): 160 workgroups, 9 tiles a wave
//   40 heads x 16 rows, 1037 slots (12 MB)    9.5 (-0.1): latencies of 1 tile a wave, merge
// Measured and not taken: 4 waves a workgroup (1 to 6 per CU), 12 and 16 waves per CU
// (spills), 64 rows a workgroup, workgroups of a head on one XCD, a higher wave priority
// at the matrix instructions, more independent chains of them, V asked for before the
// scores: each equal or slower.

constexpr float LAZY = 4.f, W_UNIT = 0x1p32f;

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t bits_of(f16x2 x) { return __builtin_bit_cast(uint32_t, x); }

// Eight e4m3 codes as fp16
__device__ __forceinline__ u32x4 f16_of(uint32_t lo, uint32_t hi)
{
    return (u32x4){bits_of((f16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false)),
                   bits_of((f16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true)),
                   bits_of((f16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false)),
                   bits_of((f16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true))};
}

// Eight codes as bf16: at most 8 bits each, so exact
template <bool F8> __device__ __forceinline__ u32x4 bf16_of(uint32_t lo, uint32_t hi)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? lo : hi;
        if constexpr (F8) {
            r[i] = __builtin_bit_cast(uint32_t, i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)
                                                      : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
        } else {
            const f32x2 x = {(float)(int8_t)(w >> (16 * (i & 1))), (float)(int8_t)(w >> (16 * (i & 1) + 8))};
            r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
        }
    }
    return r;
}

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

// Eight fp32 numbers of at most 2^15 as two fp16 each, to the nearest: off by at most 2^-23
// of the number, or 2^-25 (half of fp16's smallest).
__device__ __forceinline__ void split2(const float *v, u32x4 (&t)[2])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f16x2 h = {(_Float16)v[2 * i], (_Float16)v[2 * i + 1]};
        t[0][i] = bits_of(h);
        t[1][i] = bits_of((f16x2){(_Float16)(v[2 * i] - (float)h[0]), (_Float16)(v[2 * i + 1] - (float)h[1])});
    }
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
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
__device__ __forceinline__ f32x4 mfma_f16(const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ i32x4 mfma_i8(const u32x4 &a, const u32x4 &b, const i32x4 &c)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// Row `row` of KV head h is query head h G + row % G of token row / G.
__device__ __forceinline__ void write_out(const KvqOut &a, int hd, int h, int row, int d0, const float (&o)[4])
{
    const int i = (uint32_t)row / (uint32_t)a.G, col = (h * a.G + row - i * a.G) * hd + d0;
    if (a.split)
        store_split4(a.split, i, col, split_mt(a.Mpad, a.half), make_float4(o[0], o[1], o[2], o[3]));
    else
        *reinterpret_cast<float4 *>(a.out + i * a.ldo + col) = make_float4(o[0], o[1], o[2], o[3]);
}

// f(0), .. f(N - 1) with constant arguments: a row tile's registers are never indexed
template <int N, typename F> __device__ __forceinline__ void each(F f)
{
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

template <int HD, bool F8, int RT, int NW> __global__ __launch_bounds__(64 * NW) void k_kvq_attn(KvqAttnArgs a)
{
    constexpr int NC = HD / 32, ND = HD / 16;
    constexpr int NQ = F8 ? 2 * NC : 3 * (HD / 64);  // KB of a row tile's query parts for codes
    constexpr int NT = 3 * NC;                       // and for the tail
    const int split = blockIdx.x, h = blockIdx.y, row0 = blockIdx.z * 16 * RT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    const int rows = a.n * a.o.G;
    constexpr float scale2 = HD == 128 ? 1.4426950408889634f / 11.313708498984761f : 1.4426950408889634f / 8.f;

    // query parts as operands; later the waves' sums
    constexpr int SUMS = NW * 16 * RT * (HD + 4) * 4, PARTS = RT * (NQ + NT) * 1024;
    __shared__ __align__(16) char sm[SUMS > PARTS ? SUMS : PARTS];
    __shared__ float sm_m[NW][16 * RT], sm_l[NW][16 * RT], sm_c[16 * RT];
    u32x4(*qc)[NQ * 64] = reinterpret_cast<u32x4(*)[NQ * 64]>(sm);
    u32x4(*qt)[NT * 64] = reinterpret_cast<u32x4(*)[NT * 64]>(sm + RT * NQ * 1024);
    float(*sm_o)[16 * RT][HD + 4] = reinterpret_cast<float(*)[16 * RT][HD + 4]>(sm);

    struct Raw {
        u32x4 k[NC], v[NC];
        float s;  // K's scale in even lanes, V's in odd ones
    };
    auto load = [&](int t, Raw &x) {
        const int64_t at = (int64_t)h * a.nb + t;
        const uint8_t *kp = a.k + at * KVQ_BLOCK * HD + lane * 16, *vp = a.v + at * KVQ_BLOCK * HD + lane * 16;
        x.s = a.scale[at * 2 + (lane & 1)];
#pragma unroll
        for (int j = 0; j < NC; ++j) x.k[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kp + j * 1024));
#pragma unroll
        for (int j = 0; j < NC; ++j) x.v[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vp + j * 1024));
    };
    // the wave's tiles: every step-th from t0 on, codes below a.blocks and then at most one of
    // the tail's (there are three, in two groups)
    const int t0 = split * NW + wave, step = a.o.n_split * NW;
    const bool has_tail = a.blocks / NW % a.o.n_split == split || (a.tiles - 1) / NW % a.o.n_split == split;
    Raw buf0, buf1;  // (buf1: a tail tile's other half, which is twice a tile of codes)

    // 8 dims of one row per thread; a row's threads are neighbours.  (Loads return in
    // order: the queries' go ahead of the first tile's.)
    static_assert(RT * 16 * (HD / 8) <= 64 * NW, "a thread per 8 query numbers");
    const int d8 = tid % (HD / 8), qrow = tid / (HD / 8);
    float4 qx = make_float4(0.f, 0.f, 0.f, 0.f), qy = qx;
    if (qrow < RT * 16 && row0 + qrow < rows) {
        const float *p = a.q + ((row0 + qrow) / a.o.G) * a.ldq + (h * a.o.G + (row0 + qrow) % a.o.G) * HD + d8 * 8;
        qx = *reinterpret_cast<const float4 *>(p);
        qy = *reinterpret_cast<const float4 *>(p + 4);
    }
    // a tile of the tail in the same registers: 16 bytes per lane and load, strides k_step
    // (K) and 1 KB (V)
    auto tail_at = [&](int t, const char *&k0, const char *&k1, const char *&v0) {
        const int s0 = (t - a.blocks) * KVQ_BLOCK;
        const uint16_t *kp = a.kt + ((int64_t)h * KVQ_TAIL + s0) * HD + 8 * g;
        k0 = reinterpret_cast<const char *>(kp + k_slot(lane, 0) * HD);
        k1 = reinterpret_cast<const char *>(kp + k_slot(lane, 1) * HD);
        v0 = reinterpret_cast<const char *>(a.vt + ((int64_t)h * KVQ_TAIL + s0) * HD + n * 32 + 8 * g);
    };
    auto fetch = [&](const char *kp, int k_step, const char *vp, Raw &x) {
#pragma unroll
        for (int j = 0; j < NC; ++j) x.k[j] = *reinterpret_cast<const u32x4 *>(kp + j * k_step);
#pragma unroll
        for (int j = 0; j < NC; ++j) x.v[j] = *reinterpret_cast<const u32x4 *>(vp + j * 1024);
    };
    auto load_tail = [&](int t) {
        const char *k0, *k1, *v0;
        tail_at(t, k0, k1, v0);
        fetch(k0, 64, v0, buf0);
        fetch(k1, 64, v0 + NC * 1024, buf1);
    };
    // The wave's first tile, codes or tail, without a branch: the queries' wait then leaves
    // these loads in flight.  (A wave without a tile takes one that is there and
    // does not use it.)
    const bool tail_first = t0 >= a.blocks;
    {
        const char *k0, *k1, *v0;
        tail_at(max(min(t0, a.tiles - 1), a.blocks), k0, k1, v0);
        const int64_t at = (int64_t)h * a.nb + (tail_first ? 0 : t0);
        const char *kc = reinterpret_cast<const char *>(a.k + at * KVQ_BLOCK * HD + lane * 16);
        const char *vc = reinterpret_cast<const char *>(a.v + at * KVQ_BLOCK * HD + lane * 16);
        buf0.s = a.scale[at * 2 + (lane & 1)];
        fetch(tail_first ? k0 : kc, tail_first ? 64 : 1024, tail_first ? v0 : vc, buf0);
    }
    if (qrow < RT * 16) {
        const int row = qrow, c = d8 >> 2, at = 16 * (d8 & 3) + row % 16;
        const float v[8] = {qx.x, qx.y, qx.z, qx.w, qy.x, qy.y, qy.z, qy.w};
        // the row's largest, as bits (NaN is above infinity)
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
        for (int off = 1; off < HD / 8; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
        // 2^ex is at most the largest, and at least 2^-100 (below, a row has fewer bits)
        const int ex = max((int)(top >> 23) - 127, -100), to = F8 ? 10 : 21;
        const float f = __uint_as_float((uint32_t)(127 + to - ex) << 23);  // (ex 128: 2^-118 or 2^-107)
        if (d8 == 0) sm_c[row] = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : scale2 * __uint_as_float((uint32_t)(127 - to + ex) << 23);
        if constexpr (F8) {
            float y[8];
            u32x4 t[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[i] * f;
            split2(y, t);
            qc[row / 16][(2 * c) * 64 + at] = t[0];
            qc[row / 16][(2 * c + 1) * 64 + at] = t[1];
        } else {
            uint32_t d[3][2] = {};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int y = (int)rintf(v[i] * f);  // at most 2^22
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    const int low = (int)(int8_t)y;
                    d[p][i >> 2] |= (uint32_t)(low & 0xff) << (8 * (i & 3));
                    y = (y - low) >> 8;
                }
            }
#pragma unroll
            for (int p = 0; p < 3; ++p)
                reinterpret_cast<uint2 *>(&qc[row / 16][(p * (HD / 64) + (c >> 1)) * 64 + at])[c & 1] = make_uint2(d[p][0], d[p][1]);
        }
        if (has_tail) {
            u32x4 t[3];
            split3(v, t);
#pragma unroll
            for (int p = 0; p < 3; ++p) qt[row / 16][(c * 3 + p) * 64 + at] = t[p];
        }
    }
    if (tail_first && t0 < a.tiles) {
        const char *k0, *k1, *v0;
        tail_at(t0, k0, k1, v0);
        fetch(k1, 64, v0 + NC * 1024, buf1);
    }
    uint64_t mask[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = row0 + 16 * rt + n;
        mask[rt] = has_tail && row < rows ? a.mask[row / a.o.G] : 0ull;
    }
    __syncthreads();

    float m_run[RT], l_run[RT], coef[RT];  // (l_run: of the lane's own keys)
    f32x4 o[RT][ND];
    float v_unit = 0x1p-64f, v_inv = 0x1p64f;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_run[rt] = -INFINITY;
        l_run[rt] = 0.f;
        coef[rt] = sm_c[16 * rt + n];
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[rt][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    // moves row tile rt's reference to at least mt (one lane's maximum of the row)
    auto move = [&](auto rt_, float mt) {
        constexpr int rt = decltype(rt_)::value;
        mt = fmaxf(mt, __shfl_xor(mt, 16));
        mt = fmaxf(mt, __shfl_xor(mt, 32));
        const float mnew = fmaxf(m_run[rt], mt);
        const float alpha = m_run[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[rt] - mnew);
        l_run[rt] *= alpha;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[rt][dt][j] *= alpha;
        m_run[rt] = mnew;
    };

    // the unit of the sums at least u
    auto grow = [&](float u) {
        if (!(u > v_unit)) return;
        const float r = v_unit / u;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[rt][dt][j] *= r;
        v_unit = u;
        v_inv = 1.f / u;
    };
    // one tile, whose registers take tile `next` as soon as they are free
    auto codes = [&](Raw &x, int next) {
        const float k_scale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x.s), 0));
        const float v_scale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x.s), 1));
        grow(v_scale);
        const float vs = v_scale * v_inv * W_UNIT;
        u32x4 v[ND];
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int half = 0; half < 2; ++half) v[2 * j + half] = bf16_of<F8>(x.v[j][2 * half], x.v[j][2 * half + 1]);
        u32x4 ka[NC], kb[NC];  // e4m3 as fp16
        if constexpr (F8)
#pragma unroll
            for (int j = 0; j < NC / 2; ++j)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    ka[2 * j + half] = f16_of(x.k[2 * j][2 * half], x.k[2 * j][2 * half + 1]);
                    kb[2 * j + half] = f16_of(x.k[2 * j + 1][2 * half], x.k[2 * j + 1][2 * half + 1]);
                }
        each<RT>([&](auto rt_) {
            constexpr int rt = decltype(rt_)::value;
            if (RT > 1 && row0 + 16 * rt >= rows) {
                if (rt == RT - 1 && next < a.blocks) load(next, x);
                return;
            }
            float s[8];
            if constexpr (F8) {
                f32x4 sa = (f32x4){0.f, 0.f, 0.f, 0.f}, sb = sa;
#pragma unroll
                for (int c = 0; c < 2 * NC; ++c) {
                    const u32x4 q = qc[rt][c * 64 + lane];
                    sa = mfma_f16(ka[c >> 1], q, sa);
                    sb = mfma_f16(kb[c >> 1], q, sb);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = sa[i], s[4 + i] = sb[i];
            } else {
                i32x4 sa[3] = {}, sb[3] = {};
#pragma unroll
                for (int c = 0; c < HD / 64; ++c)
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        const u32x4 q = qc[rt][(p * (HD / 64) + c) * 64 + lane];
                        sa[p] = mfma_i8(x.k[2 * c], q, sa[p]);
                        sb[p] = mfma_i8(x.k[2 * c + 1], q, sb[p]);
                    }
                // the low two digits' sums are below 2^30 together
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[i] = fmaf((float)sa[2][i], 65536.f, (float)(sa[1][i] * 256 + sa[0][i]));
                    s[4 + i] = fmaf((float)sb[2][i], 65536.f, (float)(sb[1][i] * 256 + sb[0][i]));
                }
            }
            if (rt == RT - 1 && next < a.blocks) load(next, x);
            const float c = coef[rt] * k_scale;
            float mt = s[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) mt = fmaxf(mt, s[i]);
            mt *= c;
            if (__any(mt > m_run[rt] + LAZY)) move(rt_, mt);
            float w[8], ps = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -m_run[rt]));
                ps += w[i];
                w[i] *= vs;
            }
            l_run[rt] += ps;
            u32x4 p3[3];
            split3(w, p3);
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) o[rt][dt] = mfma_bf16(v[dt], p3[p], o[rt][dt]);
        });
    };
    int t = __builtin_amdgcn_readfirstlane(t0);
    for (; t < a.blocks; t += step) codes(buf0, t + step);

    if (t < a.tiles) {  // a tile of the tail
        const int s0 = (t - a.blocks) * KVQ_BLOCK, left = min(KVQ_BLOCK, a.r + a.n - s0);
        const uint16_t *vt = a.vt + ((int64_t)h * KVQ_TAIL + s0) * HD;
        if (!tail_first) load_tail(t);
        u32x4 v[ND];
        // V without the slots past the last row, which hold anything
        const int mine = min(max(left - 8 * g, 0), 8);  // of the lane's 8 keys
        uint32_t keep[4], top = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) keep[w] = (2 * w < mine ? 0xffffu : 0u) | (2 * w + 1 < mine ? 0xffff0000u : 0u);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            v[dt] = dt < NC ? buf0.v[dt % NC] : buf1.v[dt % NC];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                v[dt][w] &= keep[w];
                top = max_u16x2(top, v[dt][w] & 0x7fff7fffu);
            }
        }
        // infinities and NaN are taken out as well, and come after
        const bool odd = __any((top & 0xffffu) >= 0x7f80u || top >= 0x7f800000u);
        if (odd)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) v[dt] = finite(v[dt]);
        // the sums' unit holds these numbers too (2^64: up to 2^128 they stay far from fp32's end)
        grow(__any((top & 0xffffu) >= 0x5f80u || top >= 0x5f800000u) ? 0x1p64f : 1.f);
        const float vs = v_inv * W_UNIT;
        // Scores of part p of the queries.  A query's first part is 0 only where the query is, its
        // others often: so infinities and NaN of K meet the first part only.
        f32x4 sa_[RT], sb_[RT];
        auto scores = [&](int p) {
            each<RT>([&](auto rt_) {
                constexpr int rt = decltype(rt_)::value;
                if (row0 + 16 * rt >= rows) return;
                if (p == 0) sa_[rt] = sb_[rt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const u32x4 q = qt[rt][(3 * c + p) * 64 + lane];
                    sa_[rt] = mfma_bf16(buf0.k[c], q, sa_[rt]);
                    sb_[rt] = mfma_bf16(buf1.k[c], q, sb_[rt]);
                }
            });
        };
        scores(0);
        top = 0;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int w = 0; w < 4; ++w) top = max_u16x2(top, max_u16x2(buf0.k[c][w] & 0x7fff7fffu, buf1.k[c][w] & 0x7fff7fffu));
        if (__any((top & 0xffffu) >= 0x7f80u || top >= 0x7f800000u)) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                buf0.k[c] = finite(buf0.k[c]);
                buf1.k[c] = finite(buf1.k[c]);
            }
        }
        scores(1);
        scores(2);
        each<RT>([&](auto rt_) {
            constexpr int rt = decltype(rt_)::value;
            if (row0 + 16 * rt >= rows) return;
            const f32x4 sa = sa_[rt], sb = sb_[rt];
            // bit i: the row sees the lane's key i, committed or new row first + i
            const int first = s0 + 8 * g - a.r;
            const uint32_t see = (first >= 0 ? (uint32_t)(mask[rt] >> (first & 63))
                                  : first > -8 ? (uint32_t)mask[rt] << -first | (1u << -first) - 1 : 0xffu) & ((1u << mine) - 1);
            float s[8], mt = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[i] = see >> i & 1 ? (i < 4 ? sa[i] : sb[i - 4]) * scale2 : -INFINITY;
                mt = fmaxf(mt, s[i]);
            }
            if (__any(mt > m_run[rt] + LAZY)) move(rt_, mt);
            float w[8], ps = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = s[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s[i] - m_run[rt]);
                ps += w[i];
                w[i] *= vs;
            }
            l_run[rt] += ps;
            u32x4 p3[3];
            split3(w, p3);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int p = 0; p < 3; ++p) o[rt][dt] = mfma_bf16(v[dt], p3[p], o[rt][dt]);
            if (!odd) return;
            // an infinity or NaN counts for the rows that see its key, however small its weight,
            // and is nothing (not 0 x infinity) for the others
#pragma unroll 1
            for (int key = 0; key < left; ++key) {
                float p = w[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) p = (key & 7) == i ? w[i] : p;
                p = __shfl(p, 16 * (key >> 3) + n);
                const bool seen = __shfl((int)see, 16 * (key >> 3) + n) >> (key & 7) & 1;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x = bf2f(vt[(dt * 16 + 4 * g + j) * 32 + key]);
                        if (!__builtin_isfinite(x) && seen) o[rt][dt][j] += p * x;
                    }
            }
        });
    }

    // combine the waves, in their order
    const int rows_here = min(16 * RT, rows - row0);
    const int rows_end = row0 + rows_here == rows ? a.o.rows_out - row0 : rows_here;  // with padding
    __syncthreads();
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
        const float u = v_unit / W_UNIT;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
#pragma unroll
            for (int j = 0; j < 4; ++j) o[rt][dt][j] *= u;
            *reinterpret_cast<f32x4 *>(&sm_o[wave][16 * rt + n][dt * 16 + 4 * g]) = o[rt][dt];
        }
    });
    __syncthreads();
#pragma unroll
    for (int e0 = 0; e0 < 16 * RT * (HD / 4); e0 += 64 * NW) {
        const int i = (e0 + tid) / (HD / 4), d0 = 4 * (tid % (HD / 4));
        if (i >= (a.o.n_split == 1 ? rows_end : rows_here)) break;
        float mx = -INFINITY, ls = 0.f, ov[4] = {0.f, 0.f, 0.f, 0.f};
        if (i < rows_here) {
#pragma unroll
            for (int w = 0; w < NW; ++w) mx = fmaxf(mx, sm_m[w][i]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float mw = sm_m[w][i], wgt = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mx);
                ls = fmaf(wgt, sm_l[w][i], ls);
                const f32x4 o4 = *reinterpret_cast<const f32x4 *>(&sm_o[w][i][d0]);
#pragma unroll
                for (int j = 0; j < 4; ++j) ov[j] = fmaf(wgt, o4[j], ov[j]);
            }
        }
        if (a.o.n_split == 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) ov[j] = ls == 0.f ? 0.f : ov[j] / ls;
            write_out(a.o, HD, h, row0 + i, d0, ov);
        } else {
            const int64_t p = ((int64_t)h * a.o.n_split + split) * rows + row0 + i;
            *reinterpret_cast<float4 *>(a.o.part_o + p * HD + d0) = make_float4(ov[0], ov[1], ov[2], ov[3]);
            if (d0 == 0) a.o.part_ml[p] = make_float2(mx, ls);
        }
    }
}

// The shares combined, in a launch of its own: 4 threads share a row's 4 dims, each with
// every fourth share, and are combined in LDS.  The order is fixed, so are the results.
// 3 to 4.7 us in a loop of calls, 4.7 to 4.9 in a step of a 13B model (16 nodes, 1037 slots),
// a launch's start and end and one chain of reads.  The last workgroup of a head doing
// it in place of a launch was slower everywhere: it waits for its own writes and for a
// counter, then merges alone (32 heads x 1 row, 8191 slots 18.7 us for 17.9; 8 x 32, 130001
// slots 67 for 58, at the time).
template <int HD> __global__ __launch_bounds__(256) void k_kvq_merge(KvqOut a)
{
    constexpr int D4 = HD / 4, NR = 64 / D4;  // rows of a workgroup
    __shared__ __align__(16) f32x4 sm_o[4][64];
    __shared__ float sm_m[4][64], sm_l[4][64];
    const int part = threadIdx.x >> 6, lane = threadIdx.x & 63, d0 = 4 * (lane % D4);
    const int rows = a.rows, h = blockIdx.y, row = blockIdx.x * NR + lane / D4;
    const bool real = row < rows;
    float m = -INFINITY, l = 0.f, ov[4] = {0.f, 0.f, 0.f, 0.f};
    if (real)
#pragma unroll 2  // (8: longer code to fetch, 0.3 us more for few shares, 0.6 us less for 32)
        for (int s = part; s < a.n_split; s += 4) {
            const int64_t p = ((int64_t)h * a.n_split + s) * rows + row;
            const float2 ml = a.part_ml[p];
            const f32x4 o4 = *reinterpret_cast<const f32x4 *>(a.part_o + p * HD + d0);
            const float ms = ml.x, ls = ml.y;
            const float mx = fmaxf(m, ms);  // (a share that saw nothing, or only NaN, has no reference)
            const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mx);
            const float w = ms == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ms - mx);
            l = l * f + w * ls;
#pragma unroll
            for (int j = 0; j < 4; ++j) ov[j] = ov[j] * f + w * o4[j];
            m = mx;
        }
    sm_m[part][lane] = m;
    sm_l[part][lane] = l;
    sm_o[part][lane] = (f32x4){ov[0], ov[1], ov[2], ov[3]};
    __syncthreads();
    if (part || row >= a.rows_out) return;
#pragma unroll
    for (int p = 1; p < 4; ++p) {
        const float ms = sm_m[p][lane], mx = fmaxf(m, ms);
        const f32x4 o4 = sm_o[p][lane];
        const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mx);
        const float w = ms == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ms - mx);
        l = l * f + w * sm_l[p][lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) ov[j] = ov[j] * f + w * o4[j];
        m = mx;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) ov[j] = l == 0.f ? 0.f : ov[j] / l;
    write_out(a, HD, h, row, d0, ov);
}

template <int HD, bool F8> hipError_t attention(const KvqAttnArgs &a, const KvqCut &cut, hipStream_t s)
{
    const dim3 grid(cut.n_split, a.o.H, cut.z);
    if (cut.rt == 1)
        hipLaunchKernelGGL((k_kvq_attn<HD, F8, 1, 8>), grid, dim3(512), 0, s, a);
    else
        hipLaunchKernelGGL((k_kvq_attn<HD, F8, 2, 8>), grid, dim3(512), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || cut.n_split == 1) return e;
    constexpr int NR = 256 / HD;
    hipLaunchKernelGGL(k_kvq_merge<HD>, dim3((a.o.rows_out + NR - 1) / NR, a.o.H), dim3(256), 0, s, a.o);
    return hipGetLastError();
}

template <bool F8, int HD> hipError_t store(const StoreArgs &a, unsigned grid, hipStream_t s)
{
    hipLaunchKernelGGL((k_kvq_store<F8, HD>), dim3(grid, 2), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <bool F8, int HD> hipError_t load(const LoadArgs &a, unsigned grid, hipStream_t s)
{
    hipLaunchKernelGGL((k_kvq_load<F8, HD>), dim3(grid, 2), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <bool F8, int HD> hipError_t advance(const AdvanceArgs &a, hipStream_t s)
{
    const int lds = advance_lds(HD, a.total, a.full ? 0 : a.first) * 2;
    hipLaunchKernelGGL((k_kvq_advance<F8, HD>), dim3((unsigned)(a.c.L * a.c.H), 2), dim3(256), lds, s, a);
    return hipGetLastError();
}

// workgroups of four jobs; a grid's work-items are counted in 32 bits
bool grid_of(int64_t jobs, unsigned *grid)
{
    *grid = (unsigned)((jobs + 3) / 4);
    return jobs > 0 && (jobs + 3) / 4 < (1ll << 24);
}

}  // namespace

#define KVQ_DISPATCH(c, fn, ...)                                                                                   \
    ((c).hd == 128 ? ((c).f8 ? fn<true, 128>(__VA_ARGS__) : fn<false, 128>(__VA_ARGS__))                           \
                   : (c).hd == 64 ? ((c).f8 ? fn<true, 64>(__VA_ARGS__) : fn<false, 64>(__VA_ARGS__)) : hipErrorInvalidValue)

hipError_t launch_kvq_store(const KvqLayers &c, const KvqRows &from, int n, hipStream_t s)
{
    StoreArgs a{c, from, n, (c.len % KVQ_BLOCK + n) / KVQ_BLOCK, 1};
    if (a.full > 1) a.jobs = a.full;
    unsigned grid;
    if (!grid_of((int64_t)c.L * c.H * a.jobs, &grid)) return hipErrorInvalidValue;
    return KVQ_DISPATCH(c, store, a, grid, s);
}

hipError_t launch_kvq_load(const KvqLayers &c, const KvqRows &to, hipStream_t s)
{
    if (c.len == 0) return hipSuccess;
    const LoadArgs a{c, to, (c.len + KVQ_BLOCK - 1) / KVQ_BLOCK};
    unsigned grid;
    if (!grid_of((int64_t)c.L * c.H * a.jobs, &grid)) return hipErrorInvalidValue;
    return KVQ_DISPATCH(c, load, a, grid, s);
}

hipError_t launch_kvq_advance(const KvqLayers &c, const int32_t *path, int n, hipStream_t s)
{
    AdvanceArgs a{};
    const int r = c.len % KVQ_BLOCK;
    a.c = c;
    a.total = r + n;
    a.full = a.total / KVQ_BLOCK;
    a.first = a.total;
    for (int i = n - 1; i >= 0; --i) {
        a.mask |= 1ull << path[i];
        if (path[i] != i) a.first = r + i;
    }
    a.last = r + path[n - 1];
    if (!a.full && a.first == a.total) return hipSuccess;  // every row stays where it is
    return KVQ_DISPATCH(c, advance, a, s);
}

hipError_t launch_kvq_attention(const KvqAttnArgs &a, int hd, int f8, const KvqCut &cut, hipStream_t s)
{
    if (hd == 128) return f8 ? attention<128, true>(a, cut, s) : attention<128, false>(a, cut, s);
    if (hd == 64) return f8 ? attention<64, true>(a, cut, s) : attention<64, false>(a, cut, s);
    return hipErrorInvalidValue;
}
