// Entry points of decoding with drafted tokens in a tree: attention over the tree and the gathered context, rules on
// logits, acceptance, and the accepted tokens' way into the contexts of all layers.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>

#include "en_internal.h"

static int fail(int code, const char *fmt, ...)
{
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof(text), fmt, ap);
    va_end(ap);
    en_set_error("%s", text);
    return code;
}
static int launched(int e, const char *who)
{
    return e == 0 ? EN_OK : fail(EN_ERR_DEVICE, "%s launch: %s", who, hipGetErrorString((hipError_t)e));
}
static bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Whether what lies in the plan's context buffers are values.
static int check_gathered(const en_plan *plan, const char *who)
{
    if (plan->values_from_pool)
        return fail(EN_ERR_UNSUPPORTED, "%s: the plan's values stay in the pool (en_plan_values_from_pool); drafted tokens "
                    "need a gathered context", who);
    if (plan->gathered_values_from_pool == 1)
        return fail(EN_ERR_INVALID_ARG, "%s: en_plan_values_from_pool was changed after the plan's last gather; gather again", who);
    return EN_OK;
}

static int check_nodes(int32_t n_nodes, const char *who)
{
    if (n_nodes < 1)
        return fail(EN_ERR_INVALID_ARG, "%s: n_nodes = %d", who, n_nodes);
    if (n_nodes > EN_TREE_MAX_NODES)
        return fail(EN_ERR_UNSUPPORTED, "%s: a tree of %d nodes, %d at most", who, n_nodes, EN_TREE_MAX_NODES);
    return EN_OK;
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
// How a step of n nodes is cut: waves of a workgroup with row blocks and the blocks that there are for them, workgroups
// over the rows of a KV head, splits of its keys.
struct TreeCut {
    int blocks, tile_blocks, n_ptiles, n_splits;
    int head_blocks;               // blocks of rows of a KV head
    int tree_tiles;                // key tiles that the tree's own counts as
};
static TreeCut tree_cut(const en_pool *pool, const en_plan *plan, int n)
{
    TreeCut c{1, 1, 1, 1, 1, 1};
    const int all = c.head_blocks = (pool->r * n + EN_ROWS_PER_WAVE - 1) / EN_ROWS_PER_WAVE;
    if (pool->d.dtype == EN_F32) {
        // As choose_splits for the fp32 attention: rounds of workgroups times the 16-key blocks that a wave of them takes,
        // and two for its start and end; splits cost the merge.
        c.n_ptiles = (pool->r * n + EN_F32_ROWS - 1) / EN_F32_ROWS;
        const long base = long(plan->B) * pool->d.n_kv_heads * c.n_ptiles;
        const int all_blocks = (plan->max_ctx_len + 15) / 16 + (n + 15) / 16;
        long best_cost = -1;
        for (int s = 1; s <= std::min((all_blocks + EN_WAVES - 1) / EN_WAVES, EN_MAX_SPLITS); ++s) {
            const long rounds = (base * s + pool->n_cu - 1) / pool->n_cu;
            const long blocks = ((all_blocks + s - 1) / s + EN_WAVES - 1) / EN_WAVES;
            const long cost = rounds * (blocks + 2) + (s > 1 ? 128 / pool->d.head_dim : 0);
            if (best_cost < 0 || cost < best_cost) {
                best_cost = cost;
                c.n_splits = s;
            }
        }
        return c;
    }
    while (c.blocks < EN_TREE_BLOCKS && c.blocks < all)
        c.blocks *= 2;
    c.n_ptiles = (all + c.blocks - 1) / c.blocks;
    c.tile_blocks = (all + c.n_ptiles - 1) / c.n_ptiles;
    // (Its start included, the tree's tile of eight blocks takes as long as two: counted as one / two, 64 nodes of 56 heads over
    // 8 K tokens 29.0 / 28.0 us, over 2 K 18.0 / 17.2, of 32 heads over 8 K 22.2 / 22.0.)
    c.tree_tiles = c.blocks == EN_TREE_BLOCKS ? 2 : 1;
    const long units = long(plan->B) * pool->d.n_kv_heads * c.n_ptiles;
    const int tiles = (plan->max_ctx_len + EN_KEY_TILE - 1) / EN_KEY_TILE + 1;
    // Workgroups: one to a compute unit; two where each would have more than twelve tiles, which then hide each other's starts
    // and ends (a workgroup of eight blocks has a compute unit to itself). Attention and merge, us, one / two to a compute
    // unit: 1 agent of 8 KV heads x 4 K tokens, 8 nodes 15.2 / 17.2, 16 nodes 16.3 / 20.0, x 12 K, 4 nodes 18.8 / 19.6, 4
    // agents x 4 K, 32 nodes 28.9 / 33.6, 2 x 3 K, 16 nodes of 64 values 13.4 / 14.6; 16 agents x 2 K (15 tiles), 13 nodes 37.1 /
    // 35.7, x 8 K (63), 8 nodes 126.8 / 124.3.
    const long all_tiles = units * tiles;
    const long slots = long(pool->n_cu) * (c.blocks < EN_TREE_BLOCKS && all_tiles > 12L * pool->n_cu ? 2 : 1);
    c.n_splits = int(std::max<long>(1, std::min<long>(std::min<long>(slots / std::max<long>(1, units), tiles), EN_MAX_SPLITS)));
    return c;
}
struct TreeWs {
    size_t opart_off, total;
};
static TreeWs tree_ws(const en_pool *pool, const en_plan *plan, const TreeCut &cut)
{
    TreeWs w{0, 0};
    if (cut.n_splits > 1) {
        const size_t parts = size_t(cut.n_splits) * plan->B * pool->d.n_kv_heads * cut.head_blocks * EN_ROWS_PER_WAVE;
        w.opart_off = (parts * 2 * sizeof(float) + 255) & ~size_t(255);
        w.total = w.opart_off + parts * pool->d.head_dim * sizeof(float);
    }
    return w;
}

extern "C" size_t en_tree_workspace_bytes(const en_pool *pool, const en_plan *plan, int32_t n_nodes)
{
    if (!pool || !plan || n_nodes < 1 || n_nodes > EN_TREE_MAX_NODES)
        return 0;
    return tree_ws(pool, plan, tree_cut(pool, plan, n_nodes)).total;
}

static int segmented_tree_attention_impl(en_pool *pool, en_plan *plan, int32_t n_nodes, const int32_t *done_dev,
                                         const int32_t *parent_dev, const void *q_dev, const void *k_rows_dev,
                                         const void *v_rows_dev, const void *kc_dev, const void *vt_dev,
                                         void *out_dev, void *ws_dev, size_t ws_bytes, void *stream)
{
    const char *who = "segmented_tree_attention";
    if (!pool || !plan || !done_dev || !parent_dev || !q_dev || !k_rows_dev || !v_rows_dev || !kc_dev || !vt_dev || !out_dev)
        return fail(EN_ERR_INVALID_ARG, "%s: null argument", who);
    if (plan->pool != pool)
        return fail(EN_ERR_INVALID_ARG, "%s: plan belongs to another pool", who);
    int rc = check_nodes(n_nodes, who);
    if (rc != EN_OK)
        return rc;
    if (!aligned(done_dev, 4) || !aligned(parent_dev, 4))
        return fail(EN_ERR_INVALID_ARG, "%s: int32 arrays must be 4-byte aligned", who);
    for (const void *p : {q_dev, k_rows_dev, v_rows_dev, kc_dev, vt_dev, (const void *)out_dev, (const void *)ws_dev})
        if (!aligned(p, 16))
            return fail(EN_ERR_INVALID_ARG, "%s: rows, contexts and scratch must be 16-byte aligned", who);
    if ((rc = check_gathered(plan, who)) != EN_OK)
        return rc;
    const size_t elem = pool->d.dtype == EN_F32 ? 4 : 2;
    if (size_t(plan->B) * pool->d.n_q_heads * size_t(n_nodes) > 0x7fffffffu)
        return fail(EN_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 (agent, head, node) rows", who);
    if (size_t(plan->ctx_stride) * pool->d.head_dim * elem > 0x7fffffffu)
        return fail(EN_ERR_UNSUPPORTED, "%s: a context of more than 2^31 - 1 bytes per KV head", who);
    const TreeCut cut = tree_cut(pool, plan, n_nodes);
    const TreeWs ws = tree_ws(pool, plan, cut);
    const size_t need = ws.total;
    if (need && !ws_dev)
        return fail(EN_ERR_INVALID_ARG, "%s: workspace of %zu bytes required", who, need);
    if (ws_bytes < need)
        return fail(EN_ERR_CAPACITY, "%s: workspace %zu < %zu bytes", who, ws_bytes, need);
    const size_t units = size_t(plan->B) * pool->d.n_kv_heads * cut.n_ptiles * cut.n_splits;
    if (units > EN_GRID_MAX / 2 || size_t(plan->B) * pool->d.n_kv_heads * cut.head_blocks > EN_GRID_MAX / 16)
        return fail(EN_ERR_UNSUPPORTED, "%s: a step of %zu workgroups", who, units);
    if ((rc = en_ready_on_device(pool, plan, stream)) != EN_OK)
        return rc;
    EnTreeArgs a;
    a.q = q_dev;
    a.k_rows = k_rows_dev;
    a.v_rows = v_rows_dev;
    a.kc = kc_dev;
    a.vt = vt_dev;
    a.out = out_dev;
    a.cos_tab = pool->d_cos;
    a.sin_tab = pool->d_sin;
    a.hdr = en_plan_headers(plan);
    a.done = done_dev;
    a.parent = parent_dev;
    a.B = plan->B;
    a.Hq = pool->d.n_q_heads;
    a.Hkv = pool->d.n_kv_heads;
    a.Nq = plan->Nq;
    a.n = n_nodes;
    a.T = plan->ctx_stride;
    a.scale_log2e = en_softmax_scale_log2e(pool);
    a.n_splits = cut.n_splits;
    a.n_ptiles = cut.n_ptiles;
    a.n_units = unsigned(units);
    a.by_ptiles = en_divisor(unsigned(cut.n_ptiles));
    a.by_splits = en_divisor(unsigned(cut.n_splits));
    a.by_hkv = en_divisor(unsigned(a.Hkv));
    a.by_n = en_divisor(unsigned(n_nodes));
    a.head_blocks = unsigned(cut.head_blocks);
    a.n_blocks = unsigned(size_t(plan->B) * pool->d.n_kv_heads * cut.head_blocks);
    a.by_blocks = en_divisor(a.head_blocks);
    a.by_r = en_divisor(unsigned(pool->r));
    a.tile_blocks = cut.tile_blocks;
    a.tree_tiles = cut.tree_tiles;
    a.ws_ml = need ? static_cast<float *>(ws_dev) : nullptr;
    a.ws_opart = need ? reinterpret_cast<float *>(static_cast<char *>(ws_dev) + ws.opart_off) : nullptr;
    const bool timed = en_timing_begin(pool, stream);
    const int e = en_launch_tree_attention(pool, a, cut.blocks, stream);
    if (timed)
        en_timing_end(pool, stream);
    if (e != 0 || cut.n_splits == 1)
        return launched(e, who);
    return launched(en_launch_tree_merge(pool, a, stream), "segmented_tree_attention merge");
}
extern "C" int segmented_tree_attention(en_pool *pool, en_plan *plan, int32_t n_nodes, const int32_t *done_dev,
                                        const int32_t *parent_dev, const void *q_dev, const void *k_rows_dev,
                                        const void *v_rows_dev, const void *kc_dev, const void *vt_dev, void *out_dev,
                                        void *ws_dev, size_t ws_bytes, void *stream)
{
    EN_GUARDED("segmented_tree_attention",
               segmented_tree_attention_impl(pool, plan, n_nodes, done_dev, parent_dev, q_dev, k_rows_dev, v_rows_dev, kc_dev,
                                             vt_dev, out_dev, ws_dev, ws_bytes, stream));
}

// ---------------------------------------------------------------------------
// commit
// ---------------------------------------------------------------------------
static int segmented_tree_commit_impl(en_pool *pool, en_plan *plan, int32_t n_nodes, int32_t n_layers,
                                      const int32_t *done_dev, const int32_t *n_accepted_dev, const int32_t *path_dev,
                                      const void *const *k_rows_dev, const void *const *v_rows_dev, void *const *kc_dev,
                                      void *const *vt_dev, void *stream)
{
    const char *who = "segmented_tree_commit";
    if (!pool || !plan || !done_dev || !n_accepted_dev || !path_dev || n_layers < 0 ||
        (n_layers > 0 && (!k_rows_dev || !v_rows_dev || !kc_dev || !vt_dev)))
        return fail(EN_ERR_INVALID_ARG, "%s: null argument or negative count", who);
    if (plan->pool != pool)
        return fail(EN_ERR_INVALID_ARG, "%s: plan belongs to another pool", who);
    int rc = check_nodes(n_nodes, who);
    if (rc != EN_OK)
        return rc;
    if (!aligned(done_dev, 4) || !aligned(n_accepted_dev, 4) || !aligned(path_dev, 4))
        return fail(EN_ERR_INVALID_ARG, "%s: int32 arrays must be 4-byte aligned", who);
    if (plan->B > EN_GRID_YZ_MAX)
        return fail(EN_ERR_UNSUPPORTED, "%s: more than %d agents", who, EN_GRID_YZ_MAX);
    for (int l = 0; l < n_layers; ++l) {
        if (!k_rows_dev[l] || !v_rows_dev[l] || !kc_dev[l] || !vt_dev[l])
            return fail(EN_ERR_INVALID_ARG, "%s: null pointer for layer %d", who, l);
        if (!aligned(k_rows_dev[l], 16) || !aligned(v_rows_dev[l], 16) || !aligned(kc_dev[l], 16) || !aligned(vt_dev[l], 16))
            return fail(EN_ERR_INVALID_ARG, "%s: rows and contexts must be 16-byte aligned (layer %d)", who, l);
    }
    if ((rc = check_gathered(plan, who)) != EN_OK)
        return rc;
    if ((rc = en_ready_on_device(pool, plan, stream)) != EN_OK)
        return rc;
    EnTreeCommitArgs a;
    a.cos_tab = pool->d_cos;
    a.sin_tab = pool->d_sin;
    a.hdr = en_plan_headers(plan);
    a.done = done_dev;
    a.accepted = n_accepted_dev;
    a.path = path_dev;
    a.B = plan->B;
    a.Hkv = pool->d.n_kv_heads;
    a.Nq = plan->Nq;
    a.n = n_nodes;
    a.T = plan->ctx_stride;
    a.by_hkv = en_divisor(unsigned(a.Hkv));
    for (int l0 = 0; l0 < n_layers; l0 += EN_TREE_COMMIT_LAYERS) {
        a.layers = n_layers - l0 < EN_TREE_COMMIT_LAYERS ? n_layers - l0 : EN_TREE_COMMIT_LAYERS;
        for (int l = 0; l < a.layers; ++l) {
            a.k_rows[l] = k_rows_dev[l0 + l];
            a.v_rows[l] = v_rows_dev[l0 + l];
            a.kc[l] = kc_dev[l0 + l];
            a.vt[l] = vt_dev[l0 + l];
        }
        if ((rc = launched(en_launch_tree_commit(pool, a, stream), who)) != EN_OK)
            return rc;
    }
    return EN_OK;
}
extern "C" int segmented_tree_commit(en_pool *pool, en_plan *plan, int32_t n_nodes, int32_t n_layers,
                                     const int32_t *done_dev, const int32_t *n_accepted_dev, const int32_t *path_dev,
                                     const void *const *k_rows_dev, const void *const *v_rows_dev, void *const *kc_dev,
                                     void *const *vt_dev, void *stream)
{
    EN_GUARDED("segmented_tree_commit",
               segmented_tree_commit_impl(pool, plan, n_nodes, n_layers, done_dev, n_accepted_dev, path_dev, k_rows_dev,
                                          v_rows_dev, kc_dev, vt_dev, stream));
}

// ---------------------------------------------------------------------------
// rules and acceptance
// ---------------------------------------------------------------------------
static int check_rules(const en_token_rules &r, int32_t vocab, const char *who)
{
    if (r.reserved != 0 || r.history_stride < 0 || (r.history_dev && !r.history_len_dev))
        return fail(EN_ERR_INVALID_ARG, "%s: rules with reserved != 0, a negative history_stride or a history without lengths", who);
    const int64_t words = (int64_t(vocab) + 31) / 32;
    if (r.bias_dev && r.bias_agent_stride != 0 && r.bias_agent_stride < vocab)
        return fail(EN_ERR_INVALID_ARG, "%s: bias_agent_stride %lld is neither 0 nor at least vocab", who, (long long)r.bias_agent_stride);
    if (r.mask_dev && ((r.mask_agent_stride != 0 && r.mask_agent_stride < words) || (r.mask_node_stride != 0 && r.mask_node_stride < words)))
        return fail(EN_ERR_INVALID_ARG, "%s: a mask stride that is neither 0 nor at least %lld words", who, (long long)words);
    for (const void *p : {(const void *)r.penalties_dev, (const void *)r.history_dev, (const void *)r.history_len_dev,
                          (const void *)r.bias_dev, (const void *)r.mask_dev})
        if (!aligned(p, 4))
            return fail(EN_ERR_INVALID_ARG, "%s: the rules' arrays must be 4-byte aligned", who);
    return EN_OK;
}
static int check_logits(int32_t vocab, int32_t dtype, const void *p, int64_t stride, const char *who)
{
    if (vocab < 1 || stride < vocab)
        return fail(EN_ERR_INVALID_ARG, "%s: vocab %d, rows %lld apart", who, vocab, (long long)stride);
    if (dtype != EN_F32 && dtype != EN_BF16)
        return fail(EN_ERR_UNSUPPORTED, "%s: logits of dtype %d (EN_F32 or EN_BF16)", who, dtype);
    if (!aligned(p, dtype == EN_F32 ? 4 : 2))
        return fail(EN_ERR_INVALID_ARG, "%s: logits not aligned to an element", who);
    return EN_OK;
}
// Rows of an agent that a workgroup takes: as many groups of them as give every compute unit its four workgroups, no more:
// each sets its tables up anew. (16 agents with 13 rows of 50021 tokens under all rules, 1, 2, 4 and 7 groups: 36.7, 24.1, 19.3
// and 22.0 us; of 128000 tokens, 1, 2, 3 and 4: 38.2, 26.7, 32.2 and 34.3.)
static int rules_nodes(const EnRulesArgs &a)
{
    const long groups = std::min<long>(a.n, std::max<long>(1, 4 * 256 / (long(a.B) * a.chunks)));
    return int((a.n + groups - 1) / groups);
}
static int check_grid(int32_t n_agents, int32_t chunks, const char *who)
{
    if (n_agents > EN_GRID_YZ_MAX || chunks > EN_GRID_YZ_MAX)
        return fail(EN_ERR_UNSUPPORTED, "%s: more than %d agents or %lld tokens", who, EN_GRID_YZ_MAX, (long long)EN_GRID_YZ_MAX * EN_RULES_CHUNK);
    return EN_OK;
}
static int chunks_of(int32_t vocab) { return int((int64_t(vocab) + EN_RULES_CHUNK - 1) / EN_RULES_CHUNK); }

static int token_rules_apply_impl(const en_token_rules *rules, int32_t n_agents, int32_t n_nodes, int32_t vocab,
                                  int32_t dtype, const int32_t *parent_dev, const int32_t *tokens_dev,
                                  const void *logits_dev, int64_t logits_stride, void *out_dev, int64_t out_stride,
                                  void *stream)
{
    const char *who = "token_rules_apply";
    if (!rules || !logits_dev || !out_dev || n_agents < 1 || !parent_dev != !tokens_dev)
        return fail(EN_ERR_INVALID_ARG, "%s: null argument, n_agents < 1 or one of parents and tokens without the other", who);
    int rc;
    if ((rc = check_nodes(n_nodes, who)) != EN_OK || (rc = check_logits(vocab, dtype, logits_dev, logits_stride, who)) != EN_OK ||
        (rc = check_logits(vocab, dtype, out_dev, out_stride, who)) != EN_OK || (rc = check_rules(*rules, vocab, who)) != EN_OK)
        return rc;
    if ((rc = check_grid(n_agents, chunks_of(vocab), who)) != EN_OK)
        return rc;
    if (out_dev == logits_dev && out_stride != logits_stride)
        return fail(EN_ERR_INVALID_ARG, "%s: in place with another stride", who);
    if (!aligned(parent_dev, 4) || !aligned(tokens_dev, 4))
        return fail(EN_ERR_INVALID_ARG, "%s: int32 arrays must be 4-byte aligned", who);
    EnRulesArgs a;
    a.rules = *rules;
    a.parent = parent_dev;
    a.tokens = tokens_dev;
    a.logits = logits_dev;
    a.out = out_dev;
    a.logits_stride = logits_stride;
    a.out_stride = out_stride;
    a.B = n_agents;
    a.n = n_nodes;
    a.vocab = vocab;
    a.chunks = chunks_of(vocab);
    a.best = nullptr;
    a.nodes = rules_nodes(a);
    return launched(en_launch_rules(a, dtype, stream), who);
}
extern "C" int token_rules_apply(const en_token_rules *rules, int32_t n_agents, int32_t n_nodes, int32_t vocab, int32_t dtype,
                                 const int32_t *parent_dev, const int32_t *tokens_dev, const void *logits_dev,
                                 int64_t logits_stride, void *out_dev, int64_t out_stride, void *stream)
{
    EN_GUARDED("token_rules_apply", token_rules_apply_impl(rules, n_agents, n_nodes, vocab, dtype, parent_dev, tokens_dev, logits_dev,
                                                           logits_stride, out_dev, out_stride, stream));
}

extern "C" size_t en_tree_accept_workspace_bytes(const en_plan *plan, int32_t n_nodes, int32_t vocab)
{
    if (!plan || n_nodes < 1 || n_nodes > EN_TREE_MAX_NODES || vocab < 1)
        return 0;
    return size_t(plan->B) * n_nodes * chunks_of(vocab) * sizeof(unsigned long long);
}

static int token_tree_accept_impl(const en_plan *plan, const en_token_rules *rules, int32_t n_nodes, int32_t vocab,
                                  int32_t dtype, const int32_t *done_dev, const int32_t *parent_dev,
                                  const int32_t *tokens_dev, const void *logits_dev, int64_t logits_stride,
                                  int32_t *choice_dev, int32_t *path_dev, int32_t *n_accepted_dev, int32_t *next_dev,
                                  int32_t *done_out_dev, void *ws_dev, size_t ws_bytes, void *stream)
{
    const char *who = "token_tree_accept";
    if (!plan || !done_dev || !parent_dev || !tokens_dev || !path_dev || !n_accepted_dev || !next_dev || !done_out_dev ||
        (!logits_dev && !choice_dev))
        return fail(EN_ERR_INVALID_ARG, "%s: null argument", who);
    if (!plan->pool)
        return fail(EN_ERR_INVALID_ARG, "%s: the plan's pool has been destroyed", who);
    int rc = check_nodes(n_nodes, who);
    if (rc != EN_OK)
        return rc;
    if ((rc = check_grid(plan->B, 0, who)) != EN_OK)
        return rc;
    for (const void *p : {(const void *)done_dev, (const void *)parent_dev, (const void *)tokens_dev, (const void *)choice_dev,
                          (const void *)path_dev, (const void *)n_accepted_dev, (const void *)next_dev, (const void *)done_out_dev})
        if (!aligned(p, 4))
            return fail(EN_ERR_INVALID_ARG, "%s: int32 arrays must be 4-byte aligned", who);
    EnRulesArgs c;
    EnAcceptArgs a;
    a.best = nullptr;
    a.choice_in = choice_dev;
    a.choice_out = nullptr;
    a.chunks = 0;
    if (logits_dev) {
        c.rules = rules ? *rules : en_token_rules{};
        if ((rc = check_logits(vocab, dtype, logits_dev, logits_stride, who)) != EN_OK || (rc = check_rules(c.rules, vocab, who)) != EN_OK ||
            (rc = check_grid(plan->B, chunks_of(vocab), who)) != EN_OK)
            return rc;
        const size_t need = en_tree_accept_workspace_bytes(plan, n_nodes, vocab);
        if (!ws_dev || !aligned(ws_dev, 8))
            return fail(EN_ERR_INVALID_ARG, "%s: an 8-byte aligned workspace of %zu bytes is required", who, need);
        if (ws_bytes < need)
            return fail(EN_ERR_CAPACITY, "%s: workspace %zu < %zu bytes", who, ws_bytes, need);
        c.parent = parent_dev;
        c.tokens = tokens_dev;
        c.logits = logits_dev;
        c.out = nullptr;
        c.logits_stride = logits_stride;
        c.out_stride = 0;
        c.B = plan->B;
        c.n = n_nodes;
        c.vocab = vocab;
        c.chunks = chunks_of(vocab);
        c.best = static_cast<unsigned long long *>(ws_dev);
        c.nodes = rules_nodes(c);
        if ((rc = launched(en_launch_choices(c, dtype, stream), who)) != EN_OK)
            return rc;
        a.best = c.best;
        a.choice_in = nullptr;
        a.choice_out = choice_dev;
        a.chunks = c.chunks;
    }
    a.done = done_dev;
    a.parent = parent_dev;
    a.tokens = tokens_dev;
    a.path = path_dev;
    a.accepted = n_accepted_dev;
    a.next = next_dev;
    a.done_out = done_out_dev;
    a.B = plan->B;
    a.n = n_nodes;
    a.Nq = plan->Nq;
    return launched(en_launch_accept(a, stream), who);
}
extern "C" int token_tree_accept(const en_plan *plan, const en_token_rules *rules, int32_t n_nodes, int32_t vocab, int32_t dtype,
                                 const int32_t *done_dev, const int32_t *parent_dev, const int32_t *tokens_dev,
                                 const void *logits_dev, int64_t logits_stride, int32_t *choice_dev, int32_t *path_dev,
                                 int32_t *n_accepted_dev, int32_t *next_dev, int32_t *done_out_dev, void *ws_dev,
                                 size_t ws_bytes, void *stream)
{
    EN_GUARDED("token_tree_accept",
               token_tree_accept_impl(plan, rules, n_nodes, vocab, dtype, done_dev, parent_dev, tokens_dev, logits_dev, logits_stride,
                                      choice_dev, path_dev, n_accepted_dev, next_dev, done_out_dev, ws_dev, ws_bytes, stream));
}
