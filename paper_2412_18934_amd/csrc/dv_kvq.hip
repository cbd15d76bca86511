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

// Eight codes as bf16, exact: int8 has 8 significant bits, e4m3 four and exponents
// of -9 to 8.
template <bool F8> __device__ __forceinline__ u32x4 bf16_of(uint32_t lo, uint32_t hi)
{
    u32x4 r;
    if constexpr (F8) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        r[0] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
        r[1] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
        r[2] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
        r[3] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
    } else {
        const uint2 a = i8x4_to_bf16(lo), b = i8x4_to_bf16(hi);
        r = (u32x4){a.x, a.y, b.x, b.y};
    }
    return r;
}

// scale x code rounded to fp32, then to bf16
__device__ __forceinline__ u32x4 scaled_bf16(const u32x4 &codes, float scale)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __uint_as_float(codes[i] << 16) * scale, hi = __uint_as_float(codes[i] & 0xffff0000u) * scale;
        r[i] = (uint32_t)f2bf(lo) | (uint32_t)f2bf(hi) << 16;
    }
    return r;
}

// The numbers of a lane's share of a block, 8 to a vector: pieces 2 j and 2 j + 1 are
// the two halves of the lane's 16 bytes in the block's j-th KB.
__device__ __forceinline__ int k_slot(int lane, int t) { return 8 * ((lane & 15) >> 2) + 4 * t + (lane & 3); }

// Quantise one block by one wave; get(j, half) gives eight bf16 numbers.
template <bool F8, int HD, typename Get>
__device__ __forceinline__ void quantise(Get get, uint8_t *codes, float *scale, int lane)
{
    constexpr int NJ = HD / 32;
    u32x4 x[NJ][2];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        x[j][0] = get(j, 0);
        x[j][1] = get(j, 1);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) m = max_bits(max_bits(m, x[j][0]), x[j][1]);
    const BlockScale b = block_scale<F8>(wave_max(m));
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const uint2 lo = codes8<F8>(x[j][0], b.inv), hi = codes8<F8>(x[j][1], b.inv);
        *reinterpret_cast<u32x4 *>(codes + (j * 64 + lane) * 16) = (u32x4){lo.x, lo.y, hi.x, hi.y};
    }
    if (lane == 0) *scale = b.scale;
}

// ---------------------------------------------------------------------------
// Store: a wave per block and per K or V (blockIdx.y), four to a workgroup.  The
// wave of a head's first block also writes the new tail, after it has read the old
// one (both by the same wave, in that order).  Moves 3 bytes per number.

struct StoreArgs {
    KvqLayers c;
    KvqRows from;
    int32_t n, full;  // rows, whole blocks that they complete
    int32_t jobs;     // blocks per head, at least one
};

template <bool F8, int HD> __global__ __launch_bounds__(256) void k_kvq_store(StoreArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= (int64_t)a.c.L * a.c.H * a.jobs) return;
    const int64_t lh = w / a.jobs;
    const int job = (int)(w - lh * a.jobs);
    const bool is_v = blockIdx.y != 0;
    const int b0 = a.c.len / KVQ_BLOCK, r = a.c.len % KVQ_BLOCK, n = lane & 15, g = lane >> 4;
    uint16_t *tail = (is_v ? a.c.v_tail : a.c.k_tail) + lh * KVQ_TAIL * HD;
    const uint16_t *rows = (is_v ? a.from.v : a.from.k) + lh * a.from.cap * HD;
    if (job < a.full) {
        const int64_t at = lh * a.c.nb + b0 + job;
        uint8_t *codes = (is_v ? a.c.v : a.c.k) + at * KVQ_BLOCK * HD;
        float *scale = a.c.scale + at * 2 + is_v;
        const int old = job == 0 ? r : 0;  // rows that the tail holds
        if (is_v) {
            const uint16_t *tile = rows + (size_t)(b0 + job) * KVQ_BLOCK * HD;
            quantise<F8, HD>(
                [&](int j, int half) {
                    const int e = (32 * j + 16 * half + n) * 32 + 8 * g;
                    u32x4 x = *reinterpret_cast<const u32x4 *>(tile + e);
                    if (8 * g < old) {
                        const u32x4 y = *reinterpret_cast<const u32x4 *>(tail + e);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t keep = (8 * g + 2 * i < old ? 0xffffu : 0u) | (8 * g + 2 * i + 1 < old ? 0xffff0000u : 0u);
                            x[i] = (y[i] & keep) | (x[i] & ~keep);
                        }
                    }
                    return x;
                },
                codes, scale, lane);
        } else {
            quantise<F8, HD>(
                [&](int j, int half) {
                    const int s = k_slot(lane, j & 1), d = 64 * (j >> 1) + 32 * half + 8 * g;
                    const uint16_t *p = s < old ? tail + s * HD : rows + (size_t)((b0 + job) * KVQ_BLOCK + s) * HD;
                    return *reinterpret_cast<const u32x4 *>(p + d);
                },
                codes, scale, lane);
        }
    }
    if (job != 0) return;
    // tail slots [s0, s1): the rows behind the last whole block
    const int b1 = b0 + a.full, s0 = a.full ? 0 : r, s1 = a.c.len + a.n - b1 * KVQ_BLOCK;
    if (s1 <= s0) return;
    if (is_v) {
        const uint16_t *tile = rows + (size_t)b1 * KVQ_BLOCK * HD;
        for (int e = lane; e < HD * 4; e += 64) {
            const int s = 8 * (e & 3);
            if (s >= s1 || s + 8 <= s0) continue;
            u32x4 x = *reinterpret_cast<const u32x4 *>(tile + e * 8), y = *reinterpret_cast<const u32x4 *>(tail + e * 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t take = 0;
                if (s + 2 * i >= s0 && s + 2 * i < s1) take |= 0xffffu;
                if (s + 2 * i + 1 >= s0 && s + 2 * i + 1 < s1) take |= 0xffff0000u;
                x[i] = (x[i] & take) | (y[i] & ~take);
            }
            *reinterpret_cast<u32x4 *>(tail + e * 8) = x;
        }
    } else {
        const uint16_t *first = rows + (size_t)b1 * KVQ_BLOCK * HD;
        for (int e = s0 * HD / 8 + lane; e < s1 * HD / 8; e += 64)
            *reinterpret_cast<u32x4 *>(tail + e * 8) = *reinterpret_cast<const u32x4 *>(first + e * 8);
    }
}

// ---------------------------------------------------------------------------
// Load: a wave per block, the tail's committed rows as one more.

struct LoadArgs {
    KvqLayers c;
    KvqRows to;
    int32_t jobs;  // whole blocks, and one for the tail
};

template <bool F8, int HD> __global__ __launch_bounds__(256) void k_kvq_load(LoadArgs a)
{
    constexpr int NJ = HD / 32;
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
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
        for (int j = 0; j < NJ; ++j) x[j] = *reinterpret_cast<const u32x4 *>(codes + (j * 64 + lane) * 16);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const u32x4 y = scaled_bf16(bf16_of<F8>(x[j][2 * half], x[j][2 * half + 1]), scale);
                const int e = is_v ? (32 * j + 16 * half + n) * 32 + 8 * g
                                   : k_slot(lane, j & 1) * HD + 64 * (j >> 1) + 32 * half + 8 * g;
                *reinterpret_cast<u32x4 *>(to + e) = y;
            }
        return;
    }
    if (is_v) {
        const uint16_t *tail = a.c.v_tail + lh * KVQ_TAIL * HD;
        for (int e = lane; e < HD * 32; e += 64)
            if ((e & 31) < r) to[e] = tail[e];
    } else {
        const uint16_t *tail = a.c.k_tail + lh * KVQ_TAIL * HD;
        for (int e = lane; e < r * HD / 8; e += 64)
            *reinterpret_cast<u32x4 *>(to + e * 8) = *reinterpret_cast<const u32x4 *>(tail + e * 8);
    }
}

// ---------------------------------------------------------------------------
// Advance: a workgroup per (layer, head) and K or V.  Logical row t of the new tail
// is old slot src[t]; every row is in LDS before any is written.

struct AdvanceArgs {
    KvqLayers c;
    int32_t total, full, first;  // rows, whole blocks among them, first row whose slot changes
    int32_t src[KVQ_TAIL];
};

template <bool F8, int HD> __global__ __launch_bounds__(256) void k_kvq_advance(AdvanceArgs a)
{
    __shared__ __align__(16) uint16_t buf[KVQ_TAIL * HD];
    __shared__ int src[KVQ_TAIL];
    const int64_t lh = blockIdx.x;
    const bool is_v = blockIdx.y != 0;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    uint16_t *tail = (is_v ? a.c.v_tail : a.c.k_tail) + lh * KVQ_TAIL * HD;
    const int lo = a.full ? 0 : a.first;  // rows from here on are needed
    if (tid < a.total) src[tid] = a.src[tid];
    if (is_v) {
        // the tiles from the first needed row's to the last source's, as they are
        const int e1 = (a.src[a.total - 1] / 32 + 1) * HD * 4;
        for (int e = lo / 32 * HD * 4 + tid; e < e1; e += 256)
            *reinterpret_cast<u32x4 *>(buf + e * 8) = *reinterpret_cast<const u32x4 *>(tail + e * 8);
    } else {
        // rows in their new order
        for (int e = lo * HD / 8 + tid; e < a.total * HD / 8; e += 256) {
            const int t = e / (HD / 8), d = e % (HD / 8);
            *reinterpret_cast<u32x4 *>(buf + e * 8) = *reinterpret_cast<const u32x4 *>(tail + a.src[t] * HD + d * 8);
        }
    }
    __syncthreads();
    // eight slots of a dim of V, in the new order
    auto v8 = [&](int t, int d) {
        u32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = src[t + 2 * i], s2 = src[t + 2 * i + 1];
            x[i] = (uint32_t)buf[((s >> 5) * HD + d) * 32 + (s & 31)] | (uint32_t)buf[((s2 >> 5) * HD + d) * 32 + (s2 & 31)] << 16;
        }
        return x;
    };
    if (wave < a.full) {
        const int64_t at = lh * a.c.nb + a.c.len / KVQ_BLOCK + wave;
        uint8_t *codes = (is_v ? a.c.v : a.c.k) + at * KVQ_BLOCK * HD;
        float *scale = a.c.scale + at * 2 + is_v;
        if (is_v)
            quantise<F8, HD>([&](int j, int half) { return v8(wave * KVQ_BLOCK + 8 * g, 32 * j + 16 * half + n); }, codes, scale,
                             lane);
        else
            quantise<F8, HD>(
                [&](int j, int half) {
                    const int s = wave * KVQ_BLOCK + k_slot(lane, j & 1), d = 64 * (j >> 1) + 32 * half + 8 * g;
                    return *reinterpret_cast<const u32x4 *>(buf + s * HD + d);
                },
                codes, scale, lane);
    }
    // the rows behind the whole blocks, from the tail's start
    const int base = a.full * KVQ_BLOCK, s0 = a.full ? 0 : a.first, s1 = a.total - base;
    if (is_v) {
        for (int e = tid; e < HD * 32 * ((s1 + 31) / 32); e += 256) {
            const int d = e / 32 % HD, s = e / (32 * HD) * 32 + e % 32;
            if (s < s0 || s >= s1) continue;
            const int o = src[base + s];
            tail[e] = buf[((o >> 5) * HD + d) * 32 + (o & 31)];
        }
    } else {
        for (int e = s0 * HD / 8 + tid; e < s1 * HD / 8; e += 256)
            *reinterpret_cast<u32x4 *>(tail + e * 8) = *reinterpret_cast<const u32x4 *>(buf + base * HD + e * 8);
    }
}

// ---------------------------------------------------------------------------
// Attention of a tree's new rows over codes and tail, split over keys.
//
//   s_ij = (q_i . k_j) / sqrt(hd) over the keys that row i sees: all committed
//   ones, and new row j where bit j of its mask is set;
//   o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i), 0 if it sees none.
//
// Workgroup (split, KV head, row tile): its 4 waves take interleaved 32-key tiles
// of the range (blocks of codes, then up to three tiles of the tail) with a
// running maximum and sum per query row, and are combined in LDS; a second launch
// combines the ranges.  Rows are the n new tokens x the G query heads that share
// the KV head.  Scores are in base-2 units.
//
//   S^T = K Q^T: A = 16 keys x 32 dims; D gives lane (n, g) the scores of row n for
//   the 8 consecutive keys 8 g .. +8 of the tile; O = P V takes those as A.
// Codes are exact in bf16, so K and V go into the matrix instructions as codes and
// their scales onto the scores and the weights, in fp32.  Queries and weights
// are fp32 numbers, each cut into three bf16 (8 + 8 + 8 bits, nothing lost).

// fp32 -> three bf16 by truncation: their sum is the number (unless it is near the
// smallest ones)
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

__device__ __forceinline__ f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// What a tile is made of.
struct Codes {
    static constexpr bool value = false;
};
struct Tail {
    static constexpr bool value = true;
};

// Row `row` of KV head h is query head h G + row % G of token row / G.
__device__ __forceinline__ void write_out(const KvqAttnArgs &a, int hd, int h, int row, int d0, const float (&o)[4])
{
    const int i = row / a.G, col = (h * a.G + row % a.G) * hd + d0;
    if (a.out_split)
        store_split4(a.out_split, i, col, split_mt(a.Mpad, a.half), make_float4(o[0], o[1], o[2], o[3]));
    else
        *reinterpret_cast<float4 *>(a.out + i * a.ldo + col) = make_float4(o[0], o[1], o[2], o[3]);
}

template <int HD, bool F8, int RT> __global__ __launch_bounds__(256) void k_kvq_attn(KvqAttnArgs a)
{
    constexpr int NW = 4, NC = HD / 32, ND = HD / 16;
    const int split = blockIdx.x, h = blockIdx.y, row0 = blockIdx.z * 16 * RT;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const int rows = a.n * a.G;
    const float scale2 = 1.4426950408889634f / sqrtf((float)HD);
    __shared__ u32x4 sm_q[RT][NC * 3 * 64];
    __shared__ float sm_m[NW][16], sm_l[NW][16];
    __shared__ __align__(16) float sm_o[NW][16][HD + 4];

    // queries into LDS as B operands: 8 dims of one row per thread and pass
    for (int e = threadIdx.x; e < RT * 16 * (HD / 8); e += 256) {
        const int d8 = e % (HD / 8), row = e / (HD / 8), c = d8 >> 2, qg = d8 & 3;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (row0 + row < rows) {
            const float *p = a.q + ((row0 + row) / a.G) * a.ldq + (h * a.G + (row0 + row) % a.G) * HD + d8 * 8;
            const float4 x = *reinterpret_cast<const float4 *>(p), y = *reinterpret_cast<const float4 *>(p + 4);
            v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
        }
        u32x4 t[3];
        split3(v, t);
#pragma unroll
        for (int p = 0; p < 3; ++p) sm_q[row / 16][(c * 3 + p) * 64 + 16 * qg + row % 16] = t[p];
    }
    uint64_t mask[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = row0 + 16 * rt + n;
        mask[rt] = row < rows ? a.mask[row / a.G] : 0ull;
    }
    __syncthreads();

    float m_run[RT], l_run[RT];
    f32x4 o[RT][ND];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_run[rt] = -INFINITY;
        l_run[rt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[rt][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    // one tile of 32 keys as bf16 operands.  From the tail (slots from tail0 on): `left`
    // of them exist, and new rows are seen by the rows whose mask says so; `odd`: the
    // tile of V where numbers are infinite or NaN (taken out of the operand), or null.
    auto process = [&](auto from_tail, const u32x4 (&ka)[NC], const u32x4 (&kb)[NC], const u32x4 (&v)[ND], float ks, float vs,
                       int tail0, int left, const uint16_t *odd) {
        constexpr bool tail = decltype(from_tail)::value;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (row0 + 16 * rt >= rows) break;
            f32x4 sa = (f32x4){0.f, 0.f, 0.f, 0.f}, sb = sa;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    const u32x4 q = sm_q[rt][(c * 3 + p) * 64 + lane];
                    sa = mfma(ka[c], q, sa);
                    sb = mfma(kb[c], q, sb);
                }
            float sv[8], mt = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sv[i] = (i < 4 ? sa[i] : sb[i - 4]) * (ks * scale2);
                if constexpr (tail) {
                    const int j = tail0 + 8 * g + i - a.r;  // new row of the key, or committed
                    if (8 * g + i >= left || (j >= 0 && !((mask[rt] >> (j & 63)) & 1ull))) sv[i] = -INFINITY;
                }
                mt = fmaxf(mt, sv[i]);
            }
            mt = fmaxf(mt, __shfl_xor(mt, 16));
            mt = fmaxf(mt, __shfl_xor(mt, 32));
            const float mnew = fmaxf(m_run[rt], mt);
            const float alpha = m_run[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[rt] - mnew);
            float ps = 0.f, pv[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                pv[i] = sv[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sv[i] - mnew);
                ps += pv[i];
                pv[i] *= vs;
            }
            ps += __shfl_xor(ps, 16);
            ps += __shfl_xor(ps, 32);
            l_run[rt] = l_run[rt] * alpha + ps;
            m_run[rt] = mnew;
            float al[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) al[j] = __shfl(alpha, 4 * g + j);
            u32x4 p3[3];
            split3(pv, p3);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
#pragma unroll
                for (int j = 0; j < 4; ++j) o[rt][dt][j] *= al[j];
#pragma unroll
                for (int p = 0; p < 3; ++p) o[rt][dt] = mfma(p3[p], v[dt], o[rt][dt]);
            }
            if constexpr (tail) {
                if (!odd) continue;
                // such a number counts for the rows that see its key, and is nothing (not
                // 0 x infinity) for the others
                for (int kg = 0; kg < 4; ++kg)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (8 * kg + i >= left) break;
                        float pr[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) pr[j] = __shfl(pv[i], 16 * kg + 4 * g + j);
#pragma unroll
                        for (int dt = 0; dt < ND; ++dt) {
                            const float x = bf2f(odd[(dt * 16 + n) * 32 + 8 * kg + i]);
                            if (__builtin_isfinite(x)) continue;
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (pr[j] != 0.f) o[rt][dt][j] += pr[j] * x;
                        }
                    }
            }
        }
    };

    const int t0 = split * a.per_split, t1 = min(a.tiles, t0 + a.per_split);
    const int c1 = min(t1, a.blocks);
    u32x4 ka[NC], kb[NC], v[ND];
    for (int t = t0 + wave; t < c1; t += NW) {
        const int64_t at = (int64_t)h * a.nb + t;
        const uint8_t *kp = a.k + at * KVQ_BLOCK * HD + lane * 16, *vp = a.v + at * KVQ_BLOCK * HD + lane * 16;
        const float2 sc = *reinterpret_cast<const float2 *>(a.scale + at * 2);
        u32x4 kr[NC], vr[NC];
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            kr[j] = *reinterpret_cast<const u32x4 *>(kp + j * 1024);
            vr[j] = *reinterpret_cast<const u32x4 *>(vp + j * 1024);
        }
#pragma unroll
        for (int j = 0; j < NC / 2; ++j)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                ka[2 * j + half] = bf16_of<F8>(kr[2 * j][2 * half], kr[2 * j][2 * half + 1]);
                kb[2 * j + half] = bf16_of<F8>(kr[2 * j + 1][2 * half], kr[2 * j + 1][2 * half + 1]);
            }
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int half = 0; half < 2; ++half) v[2 * j + half] = bf16_of<F8>(vr[j][2 * half], vr[j][2 * half + 1]);
        process(Codes{}, ka, kb, v, sc.x, sc.y, 0, KVQ_BLOCK, nullptr);
    }
    // tail tiles of the range
    for (int t = max(t0, a.blocks) + (wave + NW - (max(t0, a.blocks) - t0) % NW) % NW; t < t1; t += NW) {
        const int s0 = (t - a.blocks) * KVQ_BLOCK, left = min(KVQ_BLOCK, a.r + a.n - s0);
        const uint16_t *kp = a.kt + ((int64_t)h * KVQ_TAIL + s0) * HD + 8 * g;
        const uint16_t *vp = a.vt + ((int64_t)h * KVQ_TAIL + s0) * HD + n * 32 + 8 * g;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            ka[c] = *reinterpret_cast<const u32x4 *>(kp + k_slot(lane, 0) * HD + 32 * c);
            kb[c] = *reinterpret_cast<const u32x4 *>(kp + k_slot(lane, 1) * HD + 32 * c);
        }
        // slots past the last row hold anything
        bool odd = false;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            v[dt] = *reinterpret_cast<const u32x4 *>(vp + dt * 512);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if (8 * g + 2 * w >= left) v[dt][w] = 0u;
                else if (8 * g + 2 * w + 1 >= left) v[dt][w] &= 0xffffu;
                const uint32_t x = v[dt][w];
                const uint32_t is = ((x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                v[dt][w] = x & ~is;
                odd |= is != 0u;
            }
        }
        process(Tail{}, ka, kb, v, 1.f, 1.f, s0, left, __any(odd) ? a.vt + ((int64_t)h * KVQ_TAIL + s0) * HD : nullptr);
    }

    // combine the waves (fixed order), one row tile at a time
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (row0 + 16 * rt >= rows) break;  // (padding rows are of the last tile)
        if (g == 0) {
            sm_m[wave][n] = m_run[rt];
            sm_l[wave][n] = l_run[rt];
        }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) sm_o[wave][4 * g + j][dt * 16 + n] = o[rt][dt][j];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * (HD / 4); e += 256) {
            const int i = e / (HD / 4), d0 = 4 * (e % (HD / 4)), row = row0 + 16 * rt + i;
            if (row >= (a.n_split == 1 ? a.rows_out : rows)) continue;
            float mx = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w) mx = fmaxf(mx, sm_m[w][i]);
            float l = 0.f, ov[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float mw = sm_m[w][i], wgt = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mx);
                l = fmaf(wgt, sm_l[w][i], l);
                const f32x4 o4 = *reinterpret_cast<const f32x4 *>(&sm_o[w][i][d0]);
#pragma unroll
                for (int j = 0; j < 4; ++j) ov[j] = fmaf(wgt, o4[j], ov[j]);
            }
            if (a.n_split == 1) {
#pragma unroll
                for (int j = 0; j < 4; ++j) ov[j] = l == 0.f ? 0.f : ov[j] / l;
                write_out(a, HD, h, row, d0, ov);
            } else {
                const int64_t p = ((int64_t)h * a.n_split + split) * rows + row;
                *reinterpret_cast<float4 *>(a.part_o + p * HD + d0) = make_float4(ov[0], ov[1], ov[2], ov[3]);
                if (d0 == 0) {
                    a.part_m[p] = mx;
                    a.part_l[p] = l;
                }
            }
        }
        __syncthreads();
    }
}

// The ranges of a row combined in their order, 4 dims per thread.
template <int HD> __global__ __launch_bounds__(256) void k_kvq_merge(KvqAttnArgs a)
{
    const int rows = a.n * a.G, rows_out = a.rows_out;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int d0 = 4 * (int)(e % (HD / 4));
    const int64_t hr = e / (HD / 4);
    if (hr >= (int64_t)a.H * rows_out) return;
    const int h = (int)(hr / rows_out), row = (int)(hr - (int64_t)h * rows_out);
    float m = -INFINITY, l = 0.f, ov[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.n_split && row < rows; ++s) {
        const int64_t p = ((int64_t)h * a.n_split + s) * rows + row;
        const float ms = a.part_m[p], ls = a.part_l[p];
        const float4 o4 = *reinterpret_cast<const float4 *>(a.part_o + p * HD + d0);
        if (ms == -INFINITY) {
            // nothing seen in this range, or only NaN
            l += ls;
            continue;
        }
        const float mx = fmaxf(m, ms);
        const float sc = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mx), w = __builtin_amdgcn_exp2f(ms - mx);
        l = fmaf(w, ls, l * sc);
        ov[0] = fmaf(w, o4.x, ov[0] * sc);
        ov[1] = fmaf(w, o4.y, ov[1] * sc);
        ov[2] = fmaf(w, o4.z, ov[2] * sc);
        ov[3] = fmaf(w, o4.w, ov[3] * sc);
        m = mx;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) ov[j] = l == 0.f ? 0.f : ov[j] / l;
    write_out(a, HD, h, row, d0, ov);
}

template <int HD, bool F8> hipError_t attention(const KvqAttnArgs &a, const KvqCut &cut, hipStream_t s)
{
    const dim3 grid(cut.n_split, a.H, cut.z);
    switch (cut.rt) {
    case 1: hipLaunchKernelGGL((k_kvq_attn<HD, F8, 1>), grid, dim3(256), 0, s, a); break;
    case 2: hipLaunchKernelGGL((k_kvq_attn<HD, F8, 2>), grid, dim3(256), 0, s, a); break;
    case 4: hipLaunchKernelGGL((k_kvq_attn<HD, F8, 4>), grid, dim3(256), 0, s, a); break;
    default: return hipErrorInvalidValue;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || cut.n_split == 1) return e;
    const int64_t work = (int64_t)a.H * a.rows_out * (HD / 4);
    hipLaunchKernelGGL(k_kvq_merge<HD>, dim3((unsigned)((work + 255) / 256)), dim3(256), 0, s, a);
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
    hipLaunchKernelGGL((k_kvq_advance<F8, HD>), dim3((unsigned)(a.c.L * a.c.H), 2), dim3(256), 0, s, a);
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
    for (int t = 0; t < a.total; ++t) {
        a.src[t] = t < r ? t : r + path[t - r];
        if (a.src[t] != t && t < a.first) a.first = t;
    }
    if (!a.full && a.first == a.total) return hipSuccess;  // every row stays where it is
    return KVQ_DISPATCH(c, advance, a, s);
}

hipError_t launch_kvq_attention(const KvqAttnArgs &a, int hd, int f8, const KvqCut &cut, hipStream_t s)
{
    if (hd == 128) return f8 ? attention<128, true>(a, cut, s) : attention<128, false>(a, cut, s);
    if (hd == 64) return f8 ? attention<64, true>(a, cut, s) : attention<64, false>(a, cut, s);
    return hipErrorInvalidValue;
}
