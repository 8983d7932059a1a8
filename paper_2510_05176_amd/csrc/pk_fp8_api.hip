// Host side of the 8-bit cache's entry points (pk_fp8_* of include/patternkv.h): checks, sizes, launches.
#include <cfloat>
#include <cmath>
#include <cstring>

#include "pk_fp8.h"

using namespace pk;

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline uint64_t round_up(uint64_t v, uint64_t a) { return (v + a - 1) / a * a; }
// workgroups of 256 threads that one dimension of a launch can have (its threads are counted in 32 bits)
constexpr int64_t kMostGroups = ((int64_t)1 << 24) - 1;

pk_status check_config(const pk_fp8_config *c)
{
    if (!c) return PK_ERR_INVALID_ARG;
    if (c->n_seq < 1 || c->n_kv_heads < 1 || c->n_q_heads < 1 || c->t_capacity < 1) return PK_ERR_INVALID_ARG;
    if (c->dtype != PK_DTYPE_FP16 && c->dtype != PK_DTYPE_BF16) return PK_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256) return PK_ERR_UNSUPPORTED;
    if (c->block != 32 && c->block != 64 && c->block != 128) return PK_ERR_UNSUPPORTED;
    if (c->n_q_heads % c->n_kv_heads != 0) return PK_ERR_SHAPE;
    if (c->n_q_heads / c->n_kv_heads > 64) return PK_ERR_UNSUPPORTED;
    if ((int64_t)c->n_seq * c->n_kv_heads > 65535) return PK_ERR_UNSUPPORTED;
    if (c->t_capacity % c->block != 0 || c->t_capacity % 64 != 0) return PK_ERR_SHAPE;
    if (c->t_capacity > (1 << 25)) return PK_ERR_UNSUPPORTED;
    if (c->page_tokens < 0 || c->n_pages < 0) return PK_ERR_INVALID_ARG;
    if (c->page_tokens > 0) {
        if (c->page_tokens < 128 || (c->page_tokens & (c->page_tokens - 1)) != 0) return PK_ERR_UNSUPPORTED;
        if (c->t_capacity % c->page_tokens != 0) return PK_ERR_SHAPE;
        if (c->n_pages < 1) return PK_ERR_INVALID_ARG;
        if ((int64_t)c->n_pages * c->n_kv_heads * c->page_tokens > ((int64_t)1 << 36)) return PK_ERR_UNSUPPORTED;
    }
    return PK_OK;
}

pk_status check_cache(const pk_fp8_config *c, const pk_fp8_cache *k)
{
    if (!k || !k->k_codes || !k->v_codes || !k->k_scale || !k->v_scale || !k->pos) return PK_ERR_INVALID_ARG;
    if (!aligned16(k->k_codes) || !aligned16(k->v_codes) || !aligned16(k->k_scale) || !aligned16(k->v_scale) || !aligned16(k->pos) ||
        !aligned16(k->weight))
        return PK_ERR_ALIGNMENT;
    if (c->page_tokens > 0) {
        if (!k->page_table) return PK_ERR_INVALID_ARG;
        if (!aligned16(k->page_table)) return PK_ERR_ALIGNMENT;
    }
    return PK_OK;
}

pk_status check_strides(const pk_strides *s)
{
    if (!s) return PK_ERR_INVALID_ARG;
    return s->seq % 8 == 0 && s->token % 8 == 0 && s->head % 8 == 0 ? PK_OK : PK_ERR_ALIGNMENT;
}

Fp8View make_view(const pk_fp8_config *c, const pk_fp8_cache *k)
{
    Fp8View v;
    v.k_codes = static_cast<uint8_t *>(k->k_codes);
    v.v_codes = static_cast<uint8_t *>(k->v_codes);
    v.k_scale = k->k_scale;
    v.v_scale = k->v_scale;
    v.pos = k->pos;
    v.weight = k->weight;
    v.map.page_table = c->page_tokens > 0 ? k->page_table : nullptr;
    v.map.page_shift = 0;
    while (c->page_tokens > 0 && (1 << v.map.page_shift) < c->page_tokens) ++v.map.page_shift;
    v.map.pages_per_seq = c->page_tokens > 0 ? c->t_capacity / c->page_tokens : 0;
    v.map.n_pages = c->n_pages;
    v.map.n_kv_heads = c->n_kv_heads;
    v.map.t_capacity = c->t_capacity;
    v.log_block = c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
    v.t_capacity = c->t_capacity;
    v.n_kv_heads = c->n_kv_heads;
    return v;
}

bool overlap(const void *a, uint64_t na, const void *b, uint64_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + nb && y < x + na;
}

// indices of the kept tokens; a budget of the whole capacity or more keeps them all and writes none
uint64_t kept_bytes(const pk_fp8_config *c, int64_t budget)
{
    return budget < c->t_capacity ? round_up((uint64_t)c->n_seq * c->n_kv_heads * budget * 4, 256) : 0;
}

struct AttentionPlan {
    int64_t parts;
    uint64_t o_bytes, ml_bytes;
};
AttentionPlan plan_attention(const pk_fp8_config *c, int64_t n_query, int64_t bound)
{
    const int64_t r = c->n_q_heads / c->n_kv_heads;
    AttentionPlan p = {0, 0, 0};
    if (n_query < 1) return p;
    p.parts = fp8_attention_parts(c->n_seq, c->n_kv_heads, r, n_query, c->head_dim, bound);
    if (p.parts > 0) {
        const uint64_t results = (uint64_t)fp8_attention_slots(c->n_seq, p.parts) * c->n_kv_heads * r * n_query;
        p.o_bytes = round_up(results * c->head_dim * 4, 256);
        p.ml_bytes = round_up(results * 2 * 4, 256);
    }
    return p;
}

// what attention and weights check and hand on alike
pk_status take_queries(const pk_fp8_config *cfg, const pk_fp8_cache *cache, const int32_t *states, int32_t bound, const void *q, const pk_strides *qs,
                       int32_t n_query, const int32_t *counts, const pk_fp8_scores *scores, Fp8Queries &a)
{
    pk_status st = check_config(cfg);
    if (st != PK_OK) return st;
    if ((st = check_cache(cfg, cache)) != PK_OK) return st;
    if (!states || (!q && n_query > 0) || !scores || n_query < 0 || bound < 0) return PK_ERR_INVALID_ARG;
    if ((st = check_strides(qs)) != PK_OK) return st;
    if (!aligned16(states) || !aligned16(q) || !aligned16(counts) || !aligned16(scores->slopes)) return PK_ERR_ALIGNMENT;
    if (!(std::fabs(scores->softmax_scale) <= FLT_MAX)) return PK_ERR_INVALID_ARG;
    if (!(scores->cap == 0.f || (scores->cap >= 1e-30f && scores->cap <= 1e30f)) || scores->window < 0) return PK_ERR_INVALID_ARG;   // also a NaN
    if (n_query > cfg->t_capacity || bound > cfg->t_capacity) return PK_ERR_CAPACITY;
    if ((int64_t)n_query * (cfg->n_q_heads / cfg->n_kv_heads) > (1 << 28)) return PK_ERR_UNSUPPORTED;   // rows of a KV head, counted in 32 bits
    a.c = make_view(cfg, cache);
    a.states = states;
    a.q = q;
    a.qs = *qs;
    a.counts = counts;
    a.slopes = scores->slopes;
    a.scale = scores->softmax_scale;
    a.cap = scores->cap;
    a.window = scores->window;
    a.n_seq = cfg->n_seq;
    a.n_query = n_query;
    a.r = cfg->n_q_heads / cfg->n_kv_heads;
    a.d = cfg->head_dim;
    a.bf16 = cfg->dtype == PK_DTYPE_BF16;
    return PK_OK;
}

}  // namespace

extern "C" {

pk_status pk_fp8_cache_layout(const pk_fp8_config *cfg, pk_fp8_layout *out)
{
    const pk_status st = check_config(cfg);
    if (st != PK_OK) return st;
    if (!out) return PK_ERR_INVALID_ARG;
    const uint64_t N = (uint64_t)cfg->n_seq * cfg->n_kv_heads, tokens = N * cfg->t_capacity;
    const uint64_t slots = cfg->page_tokens > 0 ? (uint64_t)cfg->n_pages * cfg->n_kv_heads * cfg->page_tokens : tokens;
    out->align = 16;
    out->k_codes = out->v_codes = slots * cfg->head_dim;
    out->k_scale = out->v_scale = slots / cfg->block * 4;
    out->pos = out->weight = tokens * 4;
    const uint64_t parts[6] = {out->k_codes, out->v_codes, out->k_scale, out->v_scale, out->pos, out->weight};
    out->total = 0;
    for (uint64_t p : parts) out->total += round_up(p, out->align);
    return PK_OK;
}

size_t pk_fp8_workspace_bytes(const pk_fp8_config *cfg, pk_fp8_op op, int64_t a, int64_t b)
{
    if (check_config(cfg) != PK_OK || a < 0 || b < 0) return 0;
    if (op == PK_FP8_OP_ATTENTION) {
        if (a > cfg->t_capacity || b > cfg->t_capacity) return 0;
        const AttentionPlan p = plan_attention(cfg, a, b);
        return p.o_bytes + p.ml_bytes;
    }
    if (op == PK_FP8_OP_EVICT) return kept_bytes(cfg, a);
    return 0;
}

pk_status pk_fp8_append(const pk_fp8_config *cfg, const pk_fp8_cache *cache, int32_t *states, int32_t *states_out, const void *k_new,
                        const void *v_new, const pk_strides *ks, const pk_strides *vs, int32_t n_new, const int32_t *counts, void *stream)
{
    pk_status st = check_config(cfg);
    if (st != PK_OK) return st;
    if ((st = check_cache(cfg, cache)) != PK_OK) return st;
    if (!states || n_new < 0) return PK_ERR_INVALID_ARG;
    if (!states_out) states_out = states;
    if (n_new > 0) {
        if (!k_new || !v_new) return PK_ERR_INVALID_ARG;
        if ((st = check_strides(ks)) != PK_OK || (st = check_strides(vs)) != PK_OK) return st;
    }
    if (!aligned16(states) || !aligned16(states_out) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(counts)) return PK_ERR_ALIGNMENT;
    if (states_out != states && overlap(states, (uint64_t)cfg->n_seq * 16, states_out, (uint64_t)cfg->n_seq * 16)) return PK_ERR_INVALID_ARG;
    if (n_new > cfg->t_capacity) return PK_ERR_CAPACITY;
    if (n_new == 0 && states_out == states) return PK_OK;
    if (((int64_t)n_new / cfg->block + 2) * 2 * cfg->n_kv_heads > kMostGroups) return PK_ERR_UNSUPPORTED;
    Fp8AppendArgs a;
    std::memset(&a, 0, sizeof(a));
    a.c = make_view(cfg, cache);
    a.states = states;
    a.states_out = states_out;
    a.k_new = k_new;
    a.v_new = v_new;
    if (n_new > 0) {
        a.ks = *ks;
        a.vs = *vs;
    }
    a.counts = counts;
    a.n_seq = cfg->n_seq;
    a.n_new = n_new;
    a.d = cfg->head_dim;
    a.bf16 = cfg->dtype == PK_DTYPE_BF16;
    return launch_fp8_append(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_DEVICE;
}

pk_status pk_fp8_attention(const pk_fp8_config *cfg, const pk_fp8_cache *cache, const int32_t *states, int32_t bound, const void *q,
                           const pk_strides *qs, int32_t n_query, const int32_t *counts, const pk_fp8_scores *scores, void *out,
                           const pk_strides *os, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    Fp8AttentionArgs a;
    pk_status st = take_queries(cfg, cache, states, bound, q, qs, n_query, counts, scores, a.in);
    if (st != PK_OK) return st;
    if (!out && n_query > 0) return PK_ERR_INVALID_ARG;
    if ((st = check_strides(os)) != PK_OK) return st;
    // rows of the output do not lie within each other
    const auto within = [&](int64_t n, int64_t stride) { return n > 1 && stride > -cfg->head_dim && stride < cfg->head_dim; };
    if (within(cfg->n_seq, os->seq) || within(n_query, os->token) || within(cfg->n_q_heads, os->head)) return PK_ERR_SHAPE;
    if (!aligned16(out) || !aligned16(lse) || !aligned16(workspace)) return PK_ERR_ALIGNMENT;
    if (n_query == 0) return PK_OK;
    const AttentionPlan p = plan_attention(cfg, n_query, bound);
    // groups of at least 16 rows, and the merge's of at least 2
    const int64_t rows = (int64_t)a.in.r * n_query, slots = fp8_attention_slots(cfg->n_seq, p.parts) * cfg->n_kv_heads;
    if (slots * ((rows + 15) / 16) > kMostGroups || (p.parts > 0 && (int64_t)cfg->n_seq * cfg->n_kv_heads * ((rows + 1) / 2) > kMostGroups))
        return PK_ERR_UNSUPPORTED;
    if (p.parts > 0 && (!workspace || workspace_bytes < p.o_bytes + p.ml_bytes)) return PK_ERR_WORKSPACE;
    a.out = out;
    a.os = *os;
    a.lse = lse;
    a.parts = (int32_t)p.parts;
    a.groups = 0;
    a.bound = bound;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.o_bytes);
    return launch_fp8_attention(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_DEVICE;
}

pk_status pk_fp8_weights(const pk_fp8_config *cfg, const pk_fp8_cache *cache, const int32_t *states, int32_t bound, const void *q,
                         const pk_strides *qs, int32_t n_query, const int32_t *counts, const pk_fp8_scores *scores, const float *lse,
                         int32_t accumulate, void *stream)
{
    Fp8WeightsArgs a;
    const pk_status st = take_queries(cfg, cache, states, bound, q, qs, n_query, counts, scores, a.in);
    if (st != PK_OK) return st;
    if ((!lse && n_query > 0) || !cache->weight) return PK_ERR_INVALID_ARG;
    if (!aligned16(lse)) return PK_ERR_ALIGNMENT;
    if (n_query == 0 && accumulate) return PK_OK;
    a.lse = lse;
    a.accumulate = accumulate != 0;
    a.bound = bound;
    a.parts = 0;
    return launch_fp8_weights(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_DEVICE;
}

pk_status pk_fp8_evict(const pk_fp8_config *cfg, const pk_fp8_cache *cache, const int32_t *states, const pk_fp8_config *to_cfg,
                       const pk_fp8_cache *to, int32_t *to_states, int32_t budget, int32_t keep_first, int32_t keep_last, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    pk_status st;
    if ((st = check_config(cfg)) != PK_OK || (st = check_config(to_cfg)) != PK_OK) return st;
    if ((st = check_cache(cfg, cache)) != PK_OK || (st = check_cache(to_cfg, to)) != PK_OK) return st;
    if (!states || !to_states || !cache->weight || budget < 1 || keep_first < 0 || keep_last < 0) return PK_ERR_INVALID_ARG;
    if (!aligned16(states) || !aligned16(to_states) || !aligned16(workspace)) return PK_ERR_ALIGNMENT;
    if (cfg->n_seq != to_cfg->n_seq || cfg->n_kv_heads != to_cfg->n_kv_heads || cfg->head_dim != to_cfg->head_dim || cfg->block != to_cfg->block)
        return PK_ERR_SHAPE;
    if ((int64_t)keep_first + keep_last > budget) return PK_ERR_SHAPE;
    if (budget > to_cfg->t_capacity) return PK_ERR_CAPACITY;
    pk_fp8_layout x, y;
    if ((st = pk_fp8_cache_layout(cfg, &x)) != PK_OK || (st = pk_fp8_cache_layout(to_cfg, &y)) != PK_OK) return st;
    const void *p[6] = {cache->k_codes, cache->v_codes, cache->k_scale, cache->v_scale, cache->pos, cache->weight};
    const void *r[6] = {to->k_codes, to->v_codes, to->k_scale, to->v_scale, to->pos, to->weight};
    const uint64_t np[6] = {x.k_codes, x.v_codes, x.k_scale, x.v_scale, x.pos, x.weight};
    const uint64_t nr[6] = {y.k_codes, y.v_codes, y.k_scale, y.v_scale, y.pos, y.weight};
    for (int i = 0; i < 6; ++i)
        for (int j = 0; j < 6; ++j)
            if (overlap(p[i], np[i], r[j], nr[j])) return PK_ERR_INVALID_ARG;
    if (overlap(states, (uint64_t)cfg->n_seq * 16, to_states, (uint64_t)cfg->n_seq * 16)) return PK_ERR_INVALID_ARG;
    const uint64_t need = kept_bytes(cfg, budget);
    if (need > 0 && (!workspace || workspace_bytes < need)) return PK_ERR_WORKSPACE;
    if (2 * (((int64_t)budget + cfg->block - 1) / cfg->block) > kMostGroups) return PK_ERR_UNSUPPORTED;
    Fp8EvictArgs a;
    a.from = make_view(cfg, cache);
    a.to = make_view(to_cfg, to);
    a.states = states;
    a.to_states = to_states;
    a.n_seq = cfg->n_seq;
    a.d = cfg->head_dim;
    a.budget = budget;
    a.keep_first = keep_first;
    a.keep_last = keep_last;
    a.kept = static_cast<int32_t *>(workspace);
    return launch_fp8_evict(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_DEVICE;
}

}  // extern "C"
