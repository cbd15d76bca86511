// Entry points of the paged KV cache: argument checks and launches.  Contracts are in
// include/dv.h.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <limits>
#include <mutex>

#include "dv_engine.h"
#include "dv_paged.h"

namespace {

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// A dimension of a grid counts its work-items in 32 bits, so it has less than 2^23 workgroups of 512 (one for each
// head of a sequence at least) and 2^24 of 256: one for 4 rows of an append, and one for 32 rows of a KV head.  Those
// of attention and mass stay below that whatever the rows.  Layers are a dimension of their own.
constexpr int64_t MAX_HEADS = (1ll << 22) - 1, MAX_APPEND = 1ll << 28;  // of all sequences; rows times KV heads
constexpr int MAX_GROUP = 1024, MAX_SEQS = 65536, MAX_ROWS = 1 << 22, MAX_LAYERS = 65535;

int check_cache(const dv_paged *c)
{
    if (!c) return set_err(nullptr, DV_EINVAL, "null paged cache");
    if (!c->k || !c->v || !c->table || !c->lens) return set_err(nullptr, DV_EINVAL, "null buffer in the paged cache");
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->mass, 16) || !aligned(c->table, 4) || !aligned(c->lens, 4) ||
        !aligned(c->fault, 4))
        return set_err(nullptr, DV_EINVAL, "paged cache buffers must be 16-byte aligned (table, lens, fault: 4)");
    if (c->n_layers < 1 || c->n_layers > MAX_LAYERS || c->n_heads < 1 || c->n_heads > 65535 || (c->head_dim != 64 && c->head_dim != 128))
        return set_err(nullptr, DV_EINVAL, "bad paged cache shape (%d layers, %d heads, head_dim %d)", c->n_layers, c->n_heads,
                       c->head_dim);
    if (c->page < PAGED_TILE || c->page % PAGED_TILE || c->n_pages < 1 ||
        (double)c->n_pages * c->n_heads * c->page >= 4294967296.0)
        return set_err(nullptr, DV_EINVAL, "bad pages (%d of %d slots, %d heads): page must be a positive multiple of 32, all "
                                           "slots of all heads below 2^32", c->n_pages, c->page, c->n_heads);
    if (c->n_seqs < 1 || c->n_seqs > MAX_SEQS || c->table_stride < 1 || (int64_t)c->table_stride * c->page > (1ll << 30))
        return set_err(nullptr, DV_EINVAL, "bad table (%d sequences of %d pages of %d slots)", c->n_seqs, c->table_stride, c->page);
    if ((int64_t)c->n_heads * c->n_seqs > MAX_HEADS)
        return set_err(nullptr, DV_EINVAL, "paged cache has too many heads (%d of each of %d sequences)", c->n_heads, c->n_seqs);
    return DV_OK;
}

int check_layer(const dv_paged *c, int layer)
{
    if (layer < 0 || layer >= c->n_layers) return set_err(nullptr, DV_EINVAL, "layer %d outside [0, %d)", layer, c->n_layers);
    return DV_OK;
}

// a buffer of rows of `row` elements, which `stride` elements part
bool rows_ok(const void *p, int64_t stride, int64_t row, int size)
{
    return aligned(p, 16) && stride >= row && stride % (16 / size) == 0 && stride <= (1ll << 40);
}

// queries: whether q has to be there
int check_rows(const dv_paged *c, const dv_paged_rows *r, bool queries)
{
    if (!r) return set_err(nullptr, DV_EINVAL, "null rows");
    if (r->dtype != DV_F32 && r->dtype != DV_BF16) return set_err(nullptr, DV_EINVAL, "rows must be DV_F32 or DV_BF16");
    if (r->n_rows < 1 || r->n_rows > MAX_ROWS || (!r->start && r->n_rows != c->n_seqs))
        return set_err(nullptr, DV_EINVAL, "%d rows for %d sequences", r->n_rows, c->n_seqs);
    if (!aligned(r->start, 4)) return set_err(nullptr, DV_EINVAL, "start must be 4-byte aligned");
    if (!r->q && !queries) return DV_OK;
    if (!r->q) return set_err(nullptr, DV_EINVAL, "null queries");
    if (r->n_heads < 1 || r->n_heads > 65535 || r->n_heads % c->n_heads || r->n_heads / c->n_heads > MAX_GROUP)
        return set_err(nullptr, DV_EINVAL, "%d query heads do not share %d KV heads evenly, %d each at most", r->n_heads, c->n_heads,
                       MAX_GROUP);
    const int64_t row = (int64_t)r->n_heads * c->head_dim;
    if (!rows_ok(r->q, r->q_stride, row, r->dtype == DV_F32 ? 4 : 2))
        return set_err(nullptr, DV_EINVAL, "queries need 16-byte aligned rows of at least %lld numbers", (long long)row);
    return DV_OK;
}

// what attention and mass ask of rows beyond that
int check_scores(const dv_paged_rows *r)
{
    if (!std::isfinite(r->scale) || !std::isfinite(r->cap) || r->cap < 0.f)
        return set_err(nullptr, DV_EINVAL, "bad scale or cap (%g, %g)", r->scale, r->cap);
    if (!aligned(r->mask, 8)) return set_err(nullptr, DV_EINVAL, "mask must be 8-byte aligned");
    if (r->max_rows < 1 || r->max_rows > PAGED_MAX_NEW || r->max_len < 0 || r->max_len > (1 << 30))
        return set_err(nullptr, DV_EINVAL, "max_rows %d outside [1, %d], or max_len %d", r->max_rows, PAGED_MAX_NEW, r->max_len);
    return DV_OK;
}

PagedView view_of(const dv_paged *c, int layer)
{
    const size_t at = (size_t)layer * c->n_pages * c->n_heads * c->page;
    PagedView v{};
    v.k = static_cast<uint16_t *>(c->k) + at * c->head_dim;
    v.v = static_cast<uint16_t *>(c->v) + at * c->head_dim;
    v.mass = c->mass ? c->mass + at : nullptr;
    v.table = c->table;
    v.lens = c->lens;
    v.fault = c->fault;
    v.L = c->n_layers;
    v.H = c->n_heads;
    v.hd = c->head_dim;
    v.n_pages = c->n_pages;
    v.page = c->page;
    v.n_seqs = c->n_seqs;
    v.width = c->table_stride;
    return v;
}

PagedRowsView view_of(const dv_paged *c, const dv_paged_rows *r)
{
    PagedRowsView v{};
    v.q = r->q;
    v.ldq = r->q_stride;
    v.start = r->start;
    v.mask = r->mask;
    v.scale = r->scale != 0.f ? r->scale : 1.f / std::sqrt((float)c->head_dim);
    v.cap = r->cap;
    if (r->cap != 0.f) {
        // scale / cap; a factor that is too large is the largest number (a product of 0 stays 0), one that is too
        // small to have all its bits comes in two halves, of which the first is a power of 2
        const double f = (double)v.scale / r->cap, most = std::numeric_limits<float>::max();
        const bool small = std::fabs(f) < std::numeric_limits<float>::min();
        const double half = small ? std::exp2(std::floor(std::log2(std::fabs(f)) / 2)) : 1.;
        v.cap_in[0] = small ? (float)half : (float)std::fmax(-most, std::fmin(f, most));
        v.cap_in[1] = small ? (float)(f / half) : 1.f;
    }
    v.G = r->n_heads / c->n_heads;
    v.n_rows = r->n_rows;
    return v;
}

// compute units of the current device (looked up once per device)
hipError_t current_cus(int *n)
{
    static std::mutex mu;
    static int known[DV_NOALLOC_MAX_DEVICES];
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= DV_NOALLOC_MAX_DEVICES) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    if (!known[dev] && (e = hipDeviceGetAttribute(&known[dev], hipDeviceAttributeMultiprocessorCount, dev)) != hipSuccess)
        return e;
    *n = known[dev];
    return hipSuccess;
}

int cut_of(const dv_paged *c, const dv_paged_rows *r, PagedCut *cut)
{
    int n_cu = 0;
    const hipError_t e = current_cus(&n_cu);
    if (e != hipSuccess) return set_err(nullptr, DV_EHIP, "compute units: %s", hipGetErrorString(e));
    *cut = paged_cut(c->n_seqs, c->n_heads, r->n_heads / c->n_heads, r->n_rows, r->max_rows, r->max_len, n_cu);
    return DV_OK;
}

int launched(hipError_t e, const char *what)
{
    return e == hipSuccess ? DV_OK : set_err(nullptr, DV_EHIP, "%s launch: %s", what, hipGetErrorString(e));
}

}  // namespace

extern "C" {

int dv_rope_init(dv_rope *r)
{
    if (!r) return set_err(nullptr, DV_EINVAL, "null rotary positions");
    // (every comparison is false for a NaN)
    if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_dim > 128 || !(r->base > 1.) || !std::isfinite(r->base) ||
        !(r->magnitude > 0.) || !std::isfinite((float)r->magnitude))
        return set_err(nullptr, DV_EINVAL, "bad rotary positions (rot_dim %d, base %g, magnitude %g)", r->rot_dim, r->base,
                       r->magnitude);
    if (r->scaling < DV_ROPE_PLAIN || r->scaling > DV_ROPE_LOG_TURNS) return set_err(nullptr, DV_EINVAL, "scaling %d", r->scaling);
    if (r->scaling != DV_ROPE_PLAIN && (!(r->factor >= 1.) || !std::isfinite(r->factor)))
        return set_err(nullptr, DV_EINVAL, "factor %g below 1", r->factor);
    const bool turns = r->scaling == DV_ROPE_TURNS, log_turns = r->scaling == DV_ROPE_LOG_TURNS;
    if ((turns || log_turns) && (!(r->low > 0.) || !(r->high > r->low) || !std::isfinite(r->high) || r->original_ctx < 1))
        return set_err(nullptr, DV_EINVAL, "bad turns (%g to %g over %d)", r->low, r->high, r->original_ctx);
    for (int i = 0; i < r->rot_dim / 2; ++i) {
        double f = std::pow(r->base, -2. * i / r->rot_dim);
        if (r->scaling == DV_ROPE_LINEAR) f /= r->factor;
        if (turns || log_turns) {
            const double t = r->original_ctx * f / (2. * M_PI);
            // (bounds far apart have no quotient, those close together one logarithm)
            const double w = t <= r->low    ? 0.
                             : t >= r->high ? 1.
                             : turns        ? (t - r->low) / (r->high - r->low)
                             : r->high > 2. * r->low
                                 ? (std::log(t) - std::log(r->low)) / (std::log(r->high) - std::log(r->low))
                                 : std::log1p((t - r->low) / r->low) / std::log1p((r->high - r->low) / r->low);
            f *= w + (1. - w) / r->factor;
        }
        r->freq[i] = f;
    }
    return DV_OK;
}

int dv_paged_append(const dv_paged *c, int32_t layer, const dv_paged_rows *r, const dv_rope *rope, const int32_t *positions,
                    const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *stream)
{
    int rc = check_cache(c);
    if (rc || (rc = check_layer(c, layer)) || (rc = check_rows(c, r, false))) return rc;
    if (!k || !v) return set_err(nullptr, DV_EINVAL, "null keys or values");
    if ((int64_t)r->n_rows * c->n_heads > MAX_APPEND)
        return set_err(nullptr, DV_EINVAL, "%d rows of %d KV heads are too many for one call", r->n_rows, c->n_heads);
    const int64_t row = (int64_t)c->n_heads * c->head_dim;
    const int size = r->dtype == DV_F32 ? 4 : 2;
    if (!rows_ok(k, k_stride, row, size) || !rows_ok(v, v_stride, row, size))
        return set_err(nullptr, DV_EINVAL, "keys and values need 16-byte aligned rows of at least %lld numbers", (long long)row);
    if (!aligned(positions, 4)) return set_err(nullptr, DV_EINVAL, "positions must be 4-byte aligned");
    if (rope && (rope->rot_dim < 2 || rope->rot_dim % 2 || rope->rot_dim > c->head_dim))
        return set_err(nullptr, DV_EINVAL, "rot_dim %d is odd or outside [2, %d]", rope->rot_dim, c->head_dim);
    if (rope && (!(rope->magnitude > 0.) || !std::isfinite((float)rope->magnitude)))
        return set_err(nullptr, DV_EINVAL, "bad magnitude %g", rope->magnitude);
    PagedAppendArgs a{};
    a.c = view_of(c, layer);
    a.start = r->start;
    a.positions = positions;
    a.q = r->q;
    a.k = k;
    a.v = v;
    a.ldq = r->q_stride;
    a.ldk = k_stride;
    a.ldv = v_stride;
    a.Hq = r->q ? r->n_heads : 0;
    a.n_rows = r->n_rows;
    if (rope) {
        a.rot = rope->rot_dim;
        a.interleaved = rope->interleaved != 0;
        a.magnitude = (float)rope->magnitude;
        for (int i = 0; i < a.rot / 2; ++i) a.freq[i] = rope->freq[i];
    }
    return launched(launch_paged_append(a, r->dtype == DV_BF16, static_cast<hipStream_t>(stream)), "append");
}

int64_t dv_paged_attention_workspace(const dv_paged *c, const dv_paged_rows *r)
{
    int rc = check_cache(c);
    PagedCut cut;
    if (rc || (rc = check_rows(c, r, true)) || (rc = check_scores(r)) || (rc = cut_of(c, r, &cut))) return rc;
    return (int64_t)paged_attention_bytes(cut, c->n_seqs, c->head_dim);
}

int dv_paged_attention(const dv_paged *c, int32_t layer, const dv_paged_rows *r, void *out, int64_t out_stride, float *stats,
                       void *workspace, int64_t workspace_bytes, void *stream)
{
    int rc = check_cache(c);
    if (rc || (rc = check_layer(c, layer)) || (rc = check_rows(c, r, true)) || (rc = check_scores(r))) return rc;
    const int64_t row = (int64_t)r->n_heads * c->head_dim;
    if (!out || !rows_ok(out, out_stride, row, r->dtype == DV_F32 ? 4 : 2))
        return set_err(nullptr, DV_EINVAL, "outputs need 16-byte aligned rows of at least %lld numbers", (long long)row);
    // (another row's output would be written over queries that are still to be read)
    if (r->q == out && r->n_rows > 1 && r->q_stride != out_stride)
        return set_err(nullptr, DV_EINVAL, "outputs in place of the queries need their row stride");
    if (!aligned(stats, 8)) return set_err(nullptr, DV_EINVAL, "stats must be 8-byte aligned");
    PagedCut cut;
    if ((rc = cut_of(c, r, &cut))) return rc;
    const size_t need = paged_attention_bytes(cut, c->n_seqs, c->head_dim);
    if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < 0 || (size_t)workspace_bytes < need))
        return set_err(nullptr, DV_EINVAL, "attention needs a 16-byte aligned workspace of %zu bytes", need);
    PagedAttnArgs a{};
    a.c = view_of(c, layer);
    a.r = view_of(c, r);
    a.out = out;
    a.ldo = out_stride;
    a.stats = reinterpret_cast<float2 *>(stats);
    a.groups = cut.groups;
    a.part_o = static_cast<float *>(workspace);
    if (need) {
        a.part_ml = reinterpret_cast<float2 *>(a.part_o + (size_t)cut.groups * 16 * cut.rt * c->head_dim);
        a.line = reinterpret_cast<int2 *>(a.part_ml + (size_t)cut.groups * 16 * cut.rt);
    }
    return launched(launch_paged_attention(a, r->dtype == DV_BF16, cut, static_cast<hipStream_t>(stream)), "paged attention");
}

int dv_paged_mass(const dv_paged *c, int32_t layer, const dv_paged_rows *r, const float *stats, const uint64_t *count, void *stream)
{
    int rc = check_cache(c);
    if (rc || (rc = check_layer(c, layer)) || (rc = check_rows(c, r, true)) || (rc = check_scores(r))) return rc;
    if (!c->mass) return set_err(nullptr, DV_EINVAL, "the paged cache has no mass");
    if (!stats || !aligned(stats, 8) || !aligned(count, 8))
        return set_err(nullptr, DV_EINVAL, "null stats, or stats or count not 8-byte aligned");
    int n_cu = 0;
    const hipError_t e = current_cus(&n_cu);
    if (e != hipSuccess) return set_err(nullptr, DV_EHIP, "compute units: %s", hipGetErrorString(e));
    PagedMassArgs a{};
    a.c = view_of(c, layer);
    a.r = view_of(c, r);
    a.stats = reinterpret_cast<const float2 *>(stats);
    a.count = count;
    const PagedMassCut cut = paged_mass_cut(c->n_seqs, c->n_heads, r->max_len, n_cu);
    a.whole = cut.whole;
    a.groups = (int)cut.grid;
    return launched(launch_paged_mass(a, r->dtype == DV_BF16, static_cast<hipStream_t>(stream)), "mass");
}

int dv_paged_commit(const dv_paged *c, const int32_t *path, int64_t path_stride, const int32_t *path_len, int32_t *new_lens,
                    void *stream)
{
    const int rc = check_cache(c);
    if (rc) return rc;
    if (!path_len || !new_lens || !aligned(path, 4) || !aligned(path_len, 4) || !aligned(new_lens, 4))
        return set_err(nullptr, DV_EINVAL, "null path lengths or new lengths, or not 4-byte aligned");
    if (path && (path_stride < 1 || path_stride > (1ll << 40))) return set_err(nullptr, DV_EINVAL, "path stride %lld", (long long)path_stride);
    PagedMoveArgs a{};
    a.c = view_of(c, 0);
    a.path = path;
    a.path_len = path_len;
    a.path_stride = path_stride;
    a.new_lens = new_lens;
    return launched(launch_paged_commit(a, static_cast<hipStream_t>(stream)), "paged commit");
}

int dv_paged_evict(const dv_paged *c, int32_t budget, int32_t recent, int32_t *new_lens, void *stream)
{
    const int rc = check_cache(c);
    if (rc) return rc;
    if (!c->mass) return set_err(nullptr, DV_EINVAL, "the paged cache has no mass");
    if (budget < 1 || recent < 0 || recent > budget) return set_err(nullptr, DV_EINVAL, "budget %d, recent %d", budget, recent);
    if ((int64_t)c->table_stride * c->page > PAGED_MAX_EVICT)
        return set_err(nullptr, DV_EINVAL, "eviction from tables of more than %d slots", PAGED_MAX_EVICT);
    if (!new_lens || !aligned(new_lens, 4)) return set_err(nullptr, DV_EINVAL, "null new lengths, or not 4-byte aligned");
    PagedMoveArgs a{};
    a.c = view_of(c, 0);
    a.budget = budget;
    a.recent = recent;
    a.new_lens = new_lens;
    return launched(launch_paged_evict(a, static_cast<hipStream_t>(stream)), "eviction");
}

}  // extern "C"
