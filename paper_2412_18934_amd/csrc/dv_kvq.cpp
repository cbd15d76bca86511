// Entry points of the 8-bit KV cache: argument checks, the operators on it, and the
// handle's step, prompt and commit over it.  Contracts are in include/dv.h.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstring>
#include <mutex>

#include "dv_engine.h"
#include "dv_kvq.h"

namespace {

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// A grid's work-items are counted in 32 bits: 2^24 workgroups of 256.
constexpr int64_t MAX_GROUPS = (1ll << 24) - 1;
// Query heads of a KV head: 64 rows each, 16 to a row group, are a grid's z (65535 at most).
constexpr int MAX_GROUP = 1024;

int check_kvq(dv_handle *h, const dv_kvq *c)
{
    if (!c) return set_err(h, DV_EINVAL, "null 8-bit cache");
    if (!c->k || !c->v || !c->scale || !c->k_tail || !c->v_tail) return set_err(h, DV_EINVAL, "null buffer in the 8-bit cache");
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_tail, 16) || !aligned(c->v_tail, 16) || !aligned(c->scale, 8))
        return set_err(h, DV_EINVAL, "8-bit cache buffers must be 16-byte aligned (scale: 8)");
    if (c->n_layers < 1 || c->n_heads < 1 || c->n_heads > 65535 || (c->head_dim != 64 && c->head_dim != 128))
        return set_err(h, DV_EINVAL, "bad 8-bit cache shape (%d layers, %d heads, head_dim %d)", c->n_layers, c->n_heads,
                       c->head_dim);
    if (c->format != DV_I8 && c->format != DV_F8) return set_err(h, DV_EINVAL, "8-bit cache format must be DV_I8 or DV_F8");
    if (c->capacity < KVQ_BLOCK || c->capacity % KVQ_BLOCK || c->len < 0 || c->len > c->capacity)
        return set_err(h, DV_EINVAL, "bad 8-bit cache capacity/len (%d/%d); capacity must be a positive multiple of 32",
                       c->len, c->capacity);
    // one wave per block of a layer and head in the largest launch
    if ((int64_t)c->n_layers * c->n_heads > MAX_GROUPS ||
        (int64_t)c->n_layers * c->n_heads * (c->capacity / KVQ_BLOCK + 1) > 4 * MAX_GROUPS)
        return set_err(h, DV_EINVAL, "8-bit cache has too many blocks");
    return DV_OK;
}

int check_rows(const dv_kv *kv)
{
    if (!kv || !kv->k || !kv->v) return set_err(nullptr, DV_EINVAL, "null KV cache");
    if (!aligned(kv->k, 16) || !aligned(kv->v, 16)) return set_err(nullptr, DV_EINVAL, "KV cache buffers must be 16-byte aligned");
    if (kv->capacity < 32 || kv->capacity % 32 || kv->len < 0 || kv->len > kv->capacity)
        return set_err(nullptr, DV_EINVAL, "bad KV cache capacity/len (%d/%d); capacity must be a positive multiple of 32",
                       kv->len, kv->capacity);
    return DV_OK;
}

// layers [l, l + n) of a cache
KvqLayers layers_of(const dv_kvq *c, int l, int n)
{
    KvqLayers k{};
    const size_t heads = (size_t)l * c->n_heads, nb = c->capacity / KVQ_BLOCK, hd = c->head_dim;
    k.k = static_cast<uint8_t *>(c->k) + heads * nb * KVQ_BLOCK * hd;
    k.v = static_cast<uint8_t *>(c->v) + heads * nb * KVQ_BLOCK * hd;
    k.scale = c->scale + heads * nb * 2;
    k.k_tail = static_cast<uint16_t *>(c->k_tail) + heads * KVQ_TAIL * hd;
    k.v_tail = static_cast<uint16_t *>(c->v_tail) + heads * KVQ_TAIL * hd;
    k.L = n;
    k.H = c->n_heads;
    k.hd = c->head_dim;
    k.nb = (int32_t)nb;
    k.f8 = c->format == DV_F8;
    k.len = c->len;
    return k;
}

KvqRows rows_of(const dv_kv *kv) { return {static_cast<uint16_t *>(kv->k), static_cast<uint16_t *>(kv->v), kv->capacity}; }

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

// Attention's arguments over one layer of the cache, n new rows; queries, outputs,
// mask, cut and workspace are the caller's to set.
KvqAttnArgs attention_args(const dv_kvq *c, int layer, int n)
{
    const KvqLayers k = layers_of(c, layer, 1);
    KvqAttnArgs a{};
    a.k = k.k;
    a.v = k.v;
    a.scale = k.scale;
    a.kt = k.k_tail;
    a.vt = k.v_tail;
    a.nb = k.nb;
    a.blocks = c->len / KVQ_BLOCK;
    a.r = c->len % KVQ_BLOCK;
    a.n = n;
    a.o.H = c->n_heads;
    a.tiles = a.blocks + (a.r + n + KVQ_BLOCK - 1) / KVQ_BLOCK;
    return a;
}

// The cut, and its parts of the workspace.
void set_cut(KvqAttnArgs &a, const KvqCut &cut, int hd, void *ws)
{
    a.o.n_split = cut.n_split;
    a.o.part_o = static_cast<float *>(ws);
    a.o.part_ml = reinterpret_cast<float2 *>(a.o.part_o + (size_t)a.o.H * cut.n_split * a.o.rows * hd);
}

// The handle's step and prompts over an 8-bit cache: a step's nodes go to the tail
// and stay there until they are committed; a long prompt's layers are read back into
// one layer of bf16 rows, extended there, and appended to the cache.
struct KvqSeam final : CacheSeam {
    dv_handle *h;
    dv_kvq *c;
    KvqSeam(dv_handle *handle, dv_kvq *cache) : h(handle), c(cache) { at_tail(); }

    void at_tail()
    {
        rows = {c->k_tail, c->v_tail, KVQ_TAIL, 0};
        slot = c->len % KVQ_BLOCK;
    }
    hipError_t attend(const AttnArgs &s, int l) override
    {
        KvqAttnArgs a = attention_args(c, l, s.tm.M);
        a.q = s.q;
        a.ldq = (int64_t)s.H * s.hd;
        a.o.G = 1;
        a.o.rows = a.n;
        a.o.rows_out = s.out_split ? (s.tm.half ? 8 : s.tm.Mpad) : a.n;
        a.o.out = s.out;
        a.o.ldo = a.ldq;
        a.o.split = s.out_split;
        a.o.Mpad = s.tm.Mpad;
        a.o.half = s.tm.half;
        std::memcpy(a.mask, s.tm.anc, sizeof a.mask);
        // (the handle's partials hold 512 workgroups' sums of 64 rows)
        const KvqCut cut = kvq_cut(a.o.H, a.n, a.tiles, std::min(h->n_cu, 256));
        set_cut(a, cut, s.hd, h->part_o);
        return launch_kvq_attention(a, s.hd, c->format == DV_F8, cut, h->stream);
    }
    hipError_t committed(int n) override
    {
        int32_t path[DV_MAX_TREE];
        for (int i = 0; i < n; ++i) path[i] = i;
        const hipError_t e = launch_kvq_advance(layers_of(c, 0, c->n_layers), path, n, h->stream);
        if (e != hipSuccess) return e;
        c->len += n;
        at_tail();
        return hipSuccess;
    }
    hipError_t before(int l, int) override { return launch_kvq_load(layers_of(c, l, 1), rows_of(&rows), h->stream); }
    hipError_t after(int l, int n) override { return launch_kvq_store(layers_of(c, l, 1), rows_of(&rows), n, h->stream); }
    void chunk_done(int n) override { c->len += n; }
    int reserve(int slots) override
    {
        const int cap = (slots + 31) / 32 * 32;
        const size_t slot = (size_t)c->n_heads * c->head_dim * 2, one = cap * slot;
        if (h->kvq_rows_bytes < 2 * one) {
            // room for the turns behind this one too: every allocation and release of this size
            // waits for the device
            const int most = (std::min(c->capacity, h->cfg.max_ctx) + 31) / 32 * 32;
            size_t bytes = 2 * slot * std::max(cap, (int)std::min<int64_t>(2ll * cap, most));
            void *p = nullptr;
            if (hipMalloc(&p, bytes) != hipSuccess) {
                (void)hipGetLastError();  // or the next launch would report it
                bytes = 2 * one;
                if (hipMalloc(&p, bytes) != hipSuccess) {
                    (void)hipGetLastError();
                    return set_err(h, DV_ENOMEM, "no room for a layer of %d bf16 rows", cap);
                }
            }
            if (h->kvq_rows) (void)hipFree(h->kvq_rows);
            h->kvq_rows = p;
            h->kvq_rows_bytes = bytes;
        }
        rows = {h->kvq_rows, static_cast<char *>(h->kvq_rows) + one, cap, 0};
        return DV_OK;
    }
};

// The cache as the handle's checks and pending step see it.
int handle_view(dv_handle *h, const dv_kvq *c, dv_kv *view)
{
    if (!h) return set_err(nullptr, DV_EINVAL, "null handle");
    if (h->poisoned) return DV_EHIP;
    const int rc = check_kvq(h, c);
    if (rc) return rc;
    if (!h->bf16) return set_err(h, DV_EINVAL, "an 8-bit cache needs a model with bf16 or int8 weights");
    if (c->n_layers != h->cfg.n_layers || c->n_heads != h->cfg.n_heads || c->head_dim != h->cfg.head_dim)
        return set_err(h, DV_EINVAL, "the 8-bit cache (%d layers, %d heads, head_dim %d) is not this model's", c->n_layers,
                       c->n_heads, c->head_dim);
    *view = {c->k, c->v, c->capacity, c->len};
    return DV_OK;
}

int step(dv_handle *h, const int32_t *tokens, const int32_t *tree_parents, int32_t n_tree, dv_kvq *c, dv_kv *view,
         float *out_logits, dv_accept *out_accept, const float *draft_probs, float temperature, const float *u_accept,
         const float *u_bonus, bool sampled)
{
    KvqSeam seam(h, c);
    const int rc = verify_step_impl(h, tokens, tree_parents, n_tree, view, out_logits, out_accept, draft_probs, temperature,
                                    u_accept, u_bonus, sampled, &seam);
    if (rc == DV_OK) h->pend_cache = *c;
    return rc;
}

}  // namespace

extern "C" {

int dv_kvq_store(dv_kvq *c, const dv_kv *kv, int32_t n, void *stream)
{
    int rc = check_kvq(nullptr, c);
    if (rc || (rc = check_rows(kv))) return rc;
    if (n < 1) return set_err(nullptr, DV_EINVAL, "nothing to store (n = %d)", n);
    if ((int64_t)c->len + n > kv->len)
        return set_err(nullptr, DV_EINVAL, "rows [%d, %d + %d) are not committed in the bf16 cache (len %d)", c->len, c->len, n,
                       kv->len);
    if ((int64_t)c->len + n > c->capacity)
        return set_err(nullptr, DV_ECAPACITY, "len %d + %d exceeds the 8-bit cache's capacity %d", c->len, n, c->capacity);
    const hipError_t e = launch_kvq_store(layers_of(c, 0, c->n_layers), rows_of(kv), n, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_err(nullptr, DV_EHIP, "cache store launch: %s", hipGetErrorString(e));
    c->len += n;
    return DV_OK;
}

int dv_kvq_load(const dv_kvq *c, dv_kv *kv, void *stream)
{
    int rc = check_kvq(nullptr, c);
    if (rc || (rc = check_rows(kv))) return rc;
    if (c->len > kv->capacity)
        return set_err(nullptr, DV_ECAPACITY, "%d rows exceed the bf16 cache's capacity %d", c->len, kv->capacity);
    const hipError_t e = launch_kvq_load(layers_of(c, 0, c->n_layers), rows_of(kv), static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_err(nullptr, DV_EHIP, "cache read-back launch: %s", hipGetErrorString(e));
    kv->len = c->len;
    return DV_OK;
}

int dv_kvq_advance(dv_kvq *c, const int32_t *path, int32_t n, void *stream)
{
    const int rc = check_kvq(nullptr, c);
    if (rc) return rc;
    if (!path) return set_err(nullptr, DV_EINVAL, "null path");
    if (n < 1 || n > KVQ_MAX_NEW) return set_err(nullptr, DV_EINVAL, "path length %d outside [1, %d]", n, KVQ_MAX_NEW);
    for (int i = 0; i < n; ++i)
        if (path[i] < 0 || path[i] >= KVQ_MAX_NEW || (i && path[i] <= path[i - 1]))
            return set_err(nullptr, DV_EINVAL, "path must be increasing rows in [0, %d)", KVQ_MAX_NEW);
    if ((int64_t)c->len + n > c->capacity)
        return set_err(nullptr, DV_ECAPACITY, "len %d + %d exceeds the 8-bit cache's capacity %d", c->len, n, c->capacity);
    const hipError_t e = launch_kvq_advance(layers_of(c, 0, c->n_layers), path, n, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_err(nullptr, DV_EHIP, "cache advance launch: %s", hipGetErrorString(e));
    c->len += n;
    return DV_OK;
}

int64_t dv_kvq_attention_workspace(const dv_kvq *c, int32_t n, int32_t n_heads)
{
    const int rc = check_kvq(nullptr, c);
    if (rc) return rc;
    if (n < 1 || n > KVQ_MAX_NEW) return set_err(nullptr, DV_EINVAL, "n %d outside [1, %d]", n, KVQ_MAX_NEW);
    if (n_heads < 1 || n_heads > 65535 || n_heads % c->n_heads || n_heads / c->n_heads > MAX_GROUP)
        return set_err(nullptr, DV_EINVAL, "%d query heads do not share %d KV heads evenly, %d each at most", n_heads, c->n_heads,
                       MAX_GROUP);
    int n_cu = 0;
    const hipError_t e = current_cus(&n_cu);
    if (e != hipSuccess) return set_err(nullptr, DV_EHIP, "compute units: %s", hipGetErrorString(e));
    const int rows = n * (n_heads / c->n_heads), tiles = c->capacity / KVQ_BLOCK + KVQ_TAIL / KVQ_BLOCK;
    return (int64_t)kvq_attention_bytes(c->n_heads, rows, c->head_dim,
                                        std::min(kvq_max_split(c->n_heads, rows, n_cu), tiles));
}

int dv_kvq_attention(const dv_kvq *c, int32_t layer, const float *q, int64_t q_stride, int32_t n, int32_t n_heads,
                     const uint64_t *mask, float *out, int64_t out_stride, void *workspace, int64_t workspace_bytes,
                     void *stream)
{
    const int rc = check_kvq(nullptr, c);
    if (rc) return rc;
    if (layer < 0 || layer >= c->n_layers) return set_err(nullptr, DV_EINVAL, "layer %d outside [0, %d)", layer, c->n_layers);
    if (!q || !out) return set_err(nullptr, DV_EINVAL, "null queries or output");
    if (n < 1 || n > KVQ_MAX_NEW) return set_err(nullptr, DV_EINVAL, "n %d outside [1, %d]", n, KVQ_MAX_NEW);
    if (n_heads < 1 || n_heads > 65535 || n_heads % c->n_heads || n_heads / c->n_heads > MAX_GROUP)
        return set_err(nullptr, DV_EINVAL, "%d query heads do not share %d KV heads evenly, %d each at most", n_heads, c->n_heads,
                       MAX_GROUP);
    const int64_t row = (int64_t)n_heads * c->head_dim;
    if (!aligned(q, 16) || !aligned(out, 16) || q_stride < row || out_stride < row || q_stride % 4 || out_stride % 4 ||
        q_stride > (1ll << 40) || out_stride > (1ll << 40))
        return set_err(nullptr, DV_EINVAL, "queries and outputs need 16-byte aligned rows of at least %lld floats", (long long)row);
    // (another row's output would be written over queries that are still to be read)
    if (q == out && n > 1 && q_stride != out_stride)
        return set_err(nullptr, DV_EINVAL, "outputs in place of the queries need their row stride");
    if ((int64_t)c->len + n > c->capacity)
        return set_err(nullptr, DV_ECAPACITY, "len %d + %d exceeds the 8-bit cache's capacity %d", c->len, n, c->capacity);
    int n_cu = 0;
    hipError_t e = current_cus(&n_cu);
    if (e != hipSuccess) return set_err(nullptr, DV_EHIP, "compute units: %s", hipGetErrorString(e));
    KvqAttnArgs a = attention_args(c, layer, n);
    a.q = q;
    a.ldq = q_stride;
    a.o.G = n_heads / c->n_heads;
    a.o.rows = a.o.rows_out = n * a.o.G;
    a.o.out = out;
    a.o.ldo = out_stride;
    for (int i = 0; i < n; ++i) a.mask[i] = mask ? mask[i] : ~0ull >> (63 - i);
    const KvqCut cut = kvq_cut(a.o.H, a.o.rows, a.tiles, n_cu);
    const size_t need = kvq_attention_bytes(a.o.H, a.o.rows, c->head_dim, cut.n_split);
    if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < 0 || (size_t)workspace_bytes < need))
        return set_err(nullptr, DV_EINVAL, "attention needs a 16-byte aligned workspace of %zu bytes", need);
    set_cut(a, cut, c->head_dim, workspace);
    e = launch_kvq_attention(a, c->head_dim, c->format == DV_F8, cut, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_err(nullptr, DV_EHIP, "cache attention launch: %s", hipGetErrorString(e));
    return DV_OK;
}

int dv_verify_step_kvq(dv_handle *h, const int32_t *tokens, const int32_t *tree_parents, int32_t n_tree, dv_kvq *c,
                       float *out_logits, dv_accept *out_accept)
{
    dv_kv view;
    const int rc = handle_view(h, c, &view);
    if (rc) return rc;
    return step(h, tokens, tree_parents, n_tree, c, &view, out_logits, out_accept, nullptr, 0.f, nullptr, nullptr, false);
}

int dv_verify_step_kvq_sampled(dv_handle *h, const int32_t *tokens, const int32_t *tree_parents, int32_t n_tree, dv_kvq *c,
                               const float *draft_probs, float temperature, const float *u_accept, const float *u_bonus,
                               float *out_logits, dv_accept *out_accept)
{
    dv_kv view;
    const int rc = handle_view(h, c, &view);
    if (rc) return rc;
    return step(h, tokens, tree_parents, n_tree, c, &view, out_logits, out_accept, draft_probs, temperature, u_accept, u_bonus,
                true);
}

int dv_prefill_kvq(dv_handle *h, const int32_t *tokens, int32_t n, dv_kvq *c, int32_t *out_next_token)
{
    dv_kv view;
    const int rc = handle_view(h, c, &view);
    if (rc) return rc;
    KvqSeam seam(h, c);
    return prefill_impl(h, tokens, n, &view, out_next_token, &seam);
}

int dv_kvq_commit(dv_handle *h, dv_kvq *c, const dv_accept *acc)
{
    dv_kv view;
    int rc = handle_view(h, c, &view);
    if (rc) return rc;
    if (!acc) return set_err(h, DV_EINVAL, "null accept struct");
    bool identity;
    if ((rc = check_commit(h, &view, acc, true, &identity))) return rc;
    // (caches may share blocks and have tails of their own, where the step's rows are)
    if (std::memcmp(c, &h->pend_cache, sizeof *c))
        return set_err(h, DV_ESTATE, "the cache is not the pending step's in all its buffers and sizes");
    const hipError_t e = launch_kvq_advance(layers_of(c, 0, c->n_layers), acc->path, acc->accept_len, h->stream);
    if (e != hipSuccess) return hip_fail(h, e, "cache advance launch");
    c->len += acc->accept_len;
    h->pending = false;
    return DV_OK;
}

}  // extern "C"
