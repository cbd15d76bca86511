// The host engine's handle and the parts that other host files build on (the 8-bit
// cache's paths in dv_kvq.cpp).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime_api.h>

#include <string>
#include <vector>

#include "dv.h"
#include "dv_internal.h"

struct LayerW {
    const void *attn_norm, *wq, *wk, *wv, *wo, *ffn_norm, *w_gate, *w_up, *w_down;
    const float *sq = nullptr, *sk = nullptr, *sv = nullptr, *so = nullptr, *sg = nullptr, *su = nullptr,
                *sd = nullptr;  // int8: row scales as passed in
    uint16_t *pk_qkv = nullptr, *pk_o = nullptr, *pk_gu = nullptr, *pk_down = nullptr;
    float *ps_qkv = nullptr, *ps_o = nullptr, *ps_gu = nullptr, *ps_down = nullptr;  // int8: packed-order scales
};

struct GemmPlan {
    int n_tiles = 0;   // 32-row tiles
    int mfma = 0;      // packed weights and split-layout activations (bf16 and int8 weights, K % 32 == 0)
    int rb = 0;        // 16-row blocks per row group (0: the VALU kernel)
    int n_groups = 0;  // row groups (VALU: tiles)
    int ks = 1;        // K splits per row group (residual projections)
};

struct ProfEv {
    int cls;
    hipEvent_t a, b;
};

struct dv_handle {
    dv_config cfg{};
    hipStream_t stream = nullptr;
    int bf16 = 0;          // 16-bit embedding, gains and KV cache; MFMA projections
    int wkind = W_F32;     // projection weights: W_F32, W_BF16 or W_I8
    size_t esz = 4;
    const void *embed = nullptr, *final_norm = nullptr, *lm_head = nullptr;
    std::vector<LayerW> layers;

    // workspace (device)
    float *x = nullptr, *u = nullptr, *q = nullptr, *attn = nullptr, *hbuf = nullptr;
    float *ssq = nullptr;  // per-token partial sums of squares, [64][ssq_max]
    int ssq_max = 0;
    float *part_gemm = nullptr;  // split-K partials of the residual projections
    uint32_t *cnt = nullptr;     // their per-row-group arrival counters
    size_t part_elems = 0;       // floats in part_gemm
    int cnt_n = 0;               // counters in cnt
    uint16_t *u_s = nullptr, *attn_s = nullptr, *h_s = nullptr;  // split-layout activations
    float *part_o = nullptr, *part_m = nullptr, *part_l = nullptr;
    uint32_t *attn_cnt = nullptr;  // per-head arrivals of the attention splits
    int attn_split_max = 0;
    float *arg_val = nullptr;
    int32_t *arg_idx = nullptr;
    float *rope_cos = nullptr, *rope_sin = nullptr;
    uint16_t *pk_lm = nullptr;
    const float *lm_scale = nullptr;
    float *ps_lm = nullptr;
    StepDesc *h_sd = nullptr;  // the step's tree (kernels get it by value)
    DevAccept *d_acc = nullptr, *h_acc = nullptr;  // one pinned host struct, as the device and the host address it
    float *logits_ws = nullptr;  // [max_tree][vocab] logits of a sampled step without out_logits
    // large-M prefill (allocated at its first use, sized for pf_cap tokens,
    // a multiple of 128; pf_part and pf_cnt for the split-K units of any
    // chunk of up to that many): residual stream, rotated queries, the split-layout
    // operands (norm numerators, attention output, SwiGLU output) and the
    // norms' sums of squares over 64-row slices
    int pf_cap = 0;
    void *pf_block = nullptr;  // the allocation that holds them all
    int32_t *pf_tok = nullptr;
    float *pf_x = nullptr, *pf_q = nullptr, *pf_ssq = nullptr;
    uint16_t *pf_us = nullptr, *pf_as = nullptr, *pf_hs = nullptr;
    float *pf_part = nullptr;
    uint32_t *pf_cnt = nullptr;
    // draft side
    bool draft = false;
    const void *dgf_h = nullptr, *dgf_e = nullptr, *dgf_g = nullptr;  // W_h, W_e [d][d], W_g [d][2d]
    GemmPlan p_dgf_d, p_dgf_g;    // projections of W_h / W_e (K = d) and W_g (K = 2 d)
    uint16_t *pk_dh = nullptr, *pk_de = nullptr, *pk_dg = nullptr;  // their MFMA block order
    uint16_t *dgf_xf = nullptr, *dgf_xe = nullptr, *dgf_xg = nullptr;  // split-layout operands
    float *dgf_h1 = nullptr, *dgf_h2 = nullptr, *dgf_z = nullptr;       // [64][d] outputs
    const float *x_in = nullptr;  // stack input rows for the next forward (null: embeddings)
    float *feat_a = nullptr, *feat_b = nullptr;  // [DV_TREE_MAX + 1][d] draft features (row 64: the root's input)
    int32_t *tk_tok = nullptr, *tk_tok_h = nullptr;
    float *tk_p = nullptr, *tk_p_h = nullptr;
    float *p_ws = nullptr;       // [2][vocab] current / residual distribution of the one-workgroup sampling walk
    GemmPlan p_qkv, p_o, p_gu, p_down, p_lm;
    int n_cu = 256;

    // pending (uncommitted) step
    bool pending = false;
    int32_t pend_n = 0, pend_base = 0;
    int32_t pend_parents[DV_TREE_MAX];
    void *pend_k = nullptr, *pend_v = nullptr;
    bool pend_kvq = false;  // of an 8-bit cache (its codes),
    dv_kvq pend_cache{};    // which was this

    // prompts into an 8-bit cache: one layer's keys and values as bf16 (allocated at the
    // first such prompt)
    void *kvq_rows = nullptr;
    size_t kvq_rows_bytes = 0;

    bool poisoned = false;
    std::string err;

    // per-kernel-class event timing
    int prof = 0;  // class mask
    bool prof_open = false;
    std::vector<hipEvent_t> ev_pool;
    std::vector<ProfEv> ev_live;
    double prof_ms[DV_K_COUNT] = {0, 0, 0, 0};
    int64_t prof_n[DV_K_COUNT] = {0, 0, 0, 0};
};

// What a step or a prompt does around its attention when the cache is not a plain
// dv_kv: the QKV projections write to `rows`, and the calls below come in between.
// (A table of calls, so that the engine needs nothing of the caches that use it.)
struct CacheSeam {
    dv_kv rows{};          // where the new keys and values go, dv_kv's layouts
    int slot = 0;          // a step's: slot of its first node in `rows`
    virtual ~CacheSeam() = default;
    // a step's attention over layer l; a has its queries, masks and outputs
    virtual hipError_t attend(const AttnArgs &a, int l) = 0;
    // a chain's n nodes become committed
    virtual hipError_t committed(int n) = 0;
    // a prompt's chunk of n tokens on the causal pass: `rows` holds one layer, all of it
    // from slot 0 on; `before` fills in the committed ones, `after` takes the new ones
    virtual hipError_t before(int l, int n) = 0;
    virtual hipError_t after(int l, int n) = 0;
    virtual void chunk_done(int n) = 0;
    // room for a causal pass up to `slots` committed and new tokens; DV_ENOMEM: none
    virtual int reserve(int slots) = 0;
};

int set_err(dv_handle *h, int code, const char *fmt, ...);
int hip_fail(dv_handle *h, hipError_t e, const char *what);
// kv: pointers, capacity and len of the cache for the checks and the pending step
int verify_step_impl(dv_handle *h, const int32_t *tokens, const int32_t *tree_parents, int32_t n_tree, dv_kv *kv,
                     float *out_logits, dv_accept *out_accept, const float *draft_probs, float temperature,
                     const float *u_accept, const float *u_bonus, bool sampled, CacheSeam *seam);
int prefill_impl(dv_handle *h, const int32_t *tokens, int32_t n, dv_kv *kv, int32_t *out_next_token, CacheSeam *seam);
// DV_OK where acc is the pending step's and its path a chain of that tree; *identity:
// every node is at its place already
int check_commit(dv_handle *h, const dv_kv *kv, const dv_accept *acc, bool kvq, bool *identity);
