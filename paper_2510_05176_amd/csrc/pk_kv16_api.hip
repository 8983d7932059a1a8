// Host side of the paged 16-bit cache, its pages and the attention of prompts (pk_pages_*, pk_kv16_*, pk_prompt_attention of
// include/patternkv.h): checks, sizes, launches.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>

#include "pk_kv16.h"

using namespace pk;

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline uint64_t round_up(uint64_t v, uint64_t a) { return (v + a - 1) / a * a; }
// workgroups that one dimension of a launch can have with up to 512 threads each (its threads are counted in 32 bits)
constexpr int64_t kMostGroups = ((int64_t)1 << 23) - 1;
constexpr int64_t kMostTokens = 1 << 25;   // of a sequence

bool power_of_two(int32_t x) { return x > 0 && (x & (x - 1)) == 0; }
int log2_of(int32_t x)
{
    int n = 0;
    while ((1 << n) < x) ++n;
    return n;
}

bool overlap(const void *a, uint64_t na, const void *b, uint64_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + nb && y < x + na;
}

pk_status check_pool(int32_t page_tokens, int32_t n_pages)
{
    if (page_tokens < 1 || n_pages < 1) return PK_ERR_INVALID_ARG;
    if (!power_of_two(page_tokens)) return PK_ERR_UNSUPPORTED;
    return (int64_t)n_pages * page_tokens < ((int64_t)1 << 31) ? PK_OK : PK_ERR_UNSUPPORTED;
}

pk_status check_pages(const pk_pages_config *c)
{
    if (!c || c->n_seq < 1 || c->pages_per_seq < 1) return PK_ERR_INVALID_ARG;
    const pk_status st = check_pool(c->page_tokens, c->n_pages);
    if (st != PK_OK) return st;
    return c->n_seq <= 65535 && (int64_t)c->pages_per_seq * c->page_tokens <= kMostTokens ? PK_OK : PK_ERR_UNSUPPORTED;
}

pk_status check_heads(int32_t n_seq, int32_t n_kv_heads, int32_t n_q_heads, int32_t head_dim, int32_t dtype)
{
    if (n_seq < 1 || n_kv_heads < 1 || n_q_heads < 1) return PK_ERR_INVALID_ARG;
    if (dtype != PK_DTYPE_FP16 && dtype != PK_DTYPE_BF16) return PK_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) return PK_ERR_UNSUPPORTED;
    if (n_q_heads % n_kv_heads != 0) return PK_ERR_SHAPE;
    return n_q_heads / n_kv_heads <= 64 && n_kv_heads <= 65535 ? PK_OK : PK_ERR_UNSUPPORTED;
}

pk_status check_kv16(const pk_kv16_config *c)
{
    if (!c || c->t_capacity < 1) return PK_ERR_INVALID_ARG;
    pk_status st = check_heads(c->n_seq, c->n_kv_heads, c->n_q_heads, c->head_dim, c->dtype);
    if (st != PK_OK || (st = check_pool(c->page_tokens, c->n_pages)) != PK_OK) return st;
    if (c->page_tokens < 16 || (int64_t)c->n_seq * c->n_kv_heads > 65535 || c->t_capacity > kMostTokens) return PK_ERR_UNSUPPORTED;
    return c->t_capacity % c->page_tokens == 0 ? PK_OK : PK_ERR_SHAPE;
}

pk_status check_cache(const pk_kv16_cache *k)
{
    if (!k || !k->k || !k->v) return PK_ERR_INVALID_ARG;
    return aligned16(k->k) && aligned16(k->v) ? PK_OK : PK_ERR_ALIGNMENT;
}

// first and second: the strides that are used
pk_status check_strides(const pk_strides *s, int64_t pk_strides::*first, int64_t pk_strides::*second)
{
    if (!s) return PK_ERR_INVALID_ARG;
    return s->*first % 8 == 0 && s->*second % 8 == 0 ? PK_OK : PK_ERR_ALIGNMENT;
}

// rows of an output do not lie within each other
bool within(int64_t n, int64_t stride, int d) { return n > 1 && stride > -d && stride < d; }

pk_status check_scores(const pk_fp8_scores *s)
{
    if (!s) return PK_ERR_INVALID_ARG;
    if (!(std::fabs(s->softmax_scale) <= FLT_MAX)) return PK_ERR_INVALID_ARG;   // also a NaN
    if (!(s->cap == 0.f || (s->cap >= 1e-30f && s->cap <= 1e30f)) || s->window < 0) return PK_ERR_INVALID_ARG;
    return aligned16(s->slopes) ? PK_OK : PK_ERR_ALIGNMENT;
}

struct AttentionPlan {
    int64_t parts;
    uint64_t o_bytes, ml_bytes;
};
AttentionPlan plan_attention(const pk_kv16_config *c, int64_t bound)
{
    const int64_t r = c->n_q_heads / c->n_kv_heads;
    AttentionPlan p = {0, 0, 0};
    p.parts = kv16_attention_parts(c->n_seq, c->n_kv_heads, r, c->head_dim, bound);
    if (p.parts > 0) {
        const uint64_t results = (uint64_t)fp8_attention_slots(c->n_seq, p.parts) * c->n_kv_heads * r;
        p.o_bytes = round_up(results * c->head_dim * 4, 256);
        p.ml_bytes = round_up(results * 2 * 4, 256);
    }
    return p;
}

}  // namespace

extern "C" {

size_t pk_pages_workspace_bytes(const pk_pages_config *cfg)
{
    return check_pages(cfg) == PK_OK ? round_up((uint64_t)cfg->n_seq * 4, 256) : 0;
}

pk_status pk_pages_update(const pk_pages_config *cfg, const pk_pages *pages, const int32_t *states, int32_t *states_out, const int32_t *counts,
                          int32_t n_tokens, int32_t *starts, int32_t *slots, int32_t *positions, int32_t *taken, void *workspace,
                          size_t workspace_bytes, void *stream)
{
    const pk_status st = check_pages(cfg);
    if (st != PK_OK) return st;
    if (!pages || !pages->table || !pages->free_pages || !pages->n_free || !states || !counts || !starts || !taken || n_tokens < 0 || (!slots && n_tokens > 0))
        return PK_ERR_INVALID_ARG;
    PagesArgs a;
    std::memset(&a, 0, sizeof(a));
    a.n_seq = cfg->n_seq;
    a.page_shift = log2_of(cfg->page_tokens);
    a.n_pages = cfg->n_pages;
    a.pages_per_seq = cfg->pages_per_seq;
    a.n_tokens = n_tokens;
    a.table = pages->table;
    a.free_pages = pages->free_pages;
    a.n_free = pages->n_free;
    a.n_free_out = pages->n_free_out ? pages->n_free_out : const_cast<int32_t *>(pages->n_free);
    a.states = states;
    a.states_out = states_out ? states_out : const_cast<int32_t *>(states);
    a.counts = counts;
    a.starts = starts;
    a.slots = slots;
    a.positions = positions;
    a.taken = taken;
    a.first = static_cast<int32_t *>(workspace);
    for (const void *p : {(const void *)a.table, (const void *)a.free_pages, (const void *)a.n_free, (const void *)a.n_free_out, (const void *)states,
                          (const void *)a.states_out, (const void *)counts, (const void *)starts, (const void *)slots, (const void *)positions,
                          (const void *)taken, (const void *)workspace})
        if (!aligned16(p)) return PK_ERR_ALIGNMENT;
    const uint64_t n = (uint64_t)cfg->n_seq * 4, need = pk_pages_workspace_bytes(cfg);
    if (!workspace || workspace_bytes < need) return PK_ERR_WORKSPACE;
    // what is written, then what is only read; the states and the number of free pages may be replaced where they are
    const struct {
        const void *p;
        uint64_t bytes;
    } out[] = {{a.table, n * cfg->pages_per_seq}, {a.free_pages, (uint64_t)cfg->n_pages * 4}, {a.n_free_out, 16}, {a.states_out, 4 * n}, {starts, n + 4},
               {slots, (uint64_t)n_tokens * 4}, {positions, (uint64_t)n_tokens * 4}, {taken, n}, {workspace, need},
               {a.n_free_out == a.n_free ? nullptr : a.n_free, 16}, {a.states_out == states ? nullptr : states, 4 * n}, {counts, n}};
    for (int i = 0; i < 9; ++i)
        for (int j = i + 1; j < 12; ++j)
            if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return PK_ERR_INVALID_ARG;
    return launch_pages(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_DEVICE;
}

uint64_t pk_kv16_cache_bytes(const pk_kv16_config *cfg)
{
    return check_kv16(cfg) == PK_OK ? (uint64_t)cfg->n_pages * cfg->n_kv_heads * cfg->page_tokens * cfg->head_dim * 2 : 0;
}

size_t pk_kv16_workspace_bytes(const pk_kv16_config *cfg, int64_t bound)
{
    if (check_kv16(cfg) != PK_OK || bound < 0 || bound > cfg->t_capacity) return 0;
    // Each form of the kernel needs more for a larger bound, but the one of small bounds, with fewer rows to a workgroup, may have more runs than the other.
    const int64_t turn = kOneTileTokens / ((int64_t)cfg->n_seq * cfg->n_kv_heads);
    const AttentionPlan p = plan_attention(cfg, bound), small = plan_attention(cfg, std::min(bound, turn));
    return std::max(p.o_bytes + p.ml_bytes, small.o_bytes + small.ml_bytes);
}

pk_status pk_kv16_append(const pk_kv16_config *cfg, const pk_kv16_cache *cache, const void *k_new, const void *v_new, const pk_strides *ks,
                         const pk_strides *vs, const int32_t *slots, int32_t n_tokens, void *stream)
{
    pk_status st = check_kv16(cfg);
    if (st != PK_OK || (st = check_cache(cache)) != PK_OK) return st;
    if (n_tokens < 0 || (n_tokens > 0 && (!k_new || !v_new || !slots))) return PK_ERR_INVALID_ARG;
    if ((st = check_strides(ks, &pk_strides::token, &pk_strides::head)) != PK_OK || (st = check_strides(vs, &pk_strides::token, &pk_strides::head)) != PK_OK) return st;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(slots)) return PK_ERR_ALIGNMENT;
    if (n_tokens == 0) return PK_OK;
    Kv16AppendArgs a;
    std::memset(&a, 0, sizeof(a));
    a.k = cache->k;
    a.v = cache->v;
    a.k_new = k_new;
    a.v_new = v_new;
    a.k_token = ks->token;
    a.k_head = ks->head;
    a.v_token = vs->token;
    a.v_head = vs->head;
    a.slots = slots;
    a.n_tokens = n_tokens;
    a.n_kv_heads = cfg->n_kv_heads;
    a.d = cfg->head_dim;
    a.page_shift = log2_of(cfg->page_tokens);
    a.n_slots = cfg->n_pages * cfg->page_tokens;
    return launch_kv16_append(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_DEVICE;
}

pk_status pk_kv16_attention(const pk_kv16_config *cfg, const pk_kv16_cache *cache, const int32_t *states, int32_t bound, const void *q,
                            const pk_strides *qs, const pk_fp8_scores *scores, void *out, const pk_strides *os, float *lse, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    pk_status st = check_kv16(cfg);
    if (st != PK_OK || (st = check_cache(cache)) != PK_OK) return st;
    if (!cache->page_table || !states || !q || !out || bound < 0) return PK_ERR_INVALID_ARG;
    if ((st = check_scores(scores)) != PK_OK) return st;
    if ((st = check_strides(qs, &pk_strides::seq, &pk_strides::head)) != PK_OK || (st = check_strides(os, &pk_strides::seq, &pk_strides::head)) != PK_OK) return st;
    if (within(cfg->n_seq, os->seq, cfg->head_dim) || within(cfg->n_q_heads, os->head, cfg->head_dim)) return PK_ERR_SHAPE;
    if (!aligned16(cache->page_table) || !aligned16(states) || !aligned16(q) || !aligned16(out) || !aligned16(lse) || !aligned16(workspace)) return PK_ERR_ALIGNMENT;
    if (bound > cfg->t_capacity) return PK_ERR_CAPACITY;
    const AttentionPlan p = plan_attention(cfg, bound);
    if (p.parts > 0 && (!workspace || workspace_bytes < p.o_bytes + p.ml_bytes)) return PK_ERR_WORKSPACE;
    Fp8AttentionArgs a;
    std::memset(&a, 0, sizeof(a));
    a.in.c.k_codes = static_cast<uint8_t *>(cache->k);
    a.in.c.v_codes = static_cast<uint8_t *>(cache->v);
    a.in.c.map.page_table = cache->page_table;
    a.in.c.map.page_shift = log2_of(cfg->page_tokens);
    a.in.c.map.pages_per_seq = cfg->t_capacity / cfg->page_tokens;
    a.in.c.map.n_pages = cfg->n_pages;
    a.in.c.map.n_kv_heads = cfg->n_kv_heads;
    a.in.c.map.t_capacity = cfg->t_capacity;
    a.in.c.t_capacity = cfg->t_capacity;
    a.in.c.n_kv_heads = cfg->n_kv_heads;
    a.in.states = states;
    a.in.q = q;
    a.in.qs = *qs;
    a.in.slopes = scores->slopes;
    a.in.scale = scores->softmax_scale;
    a.in.cap = scores->cap;
    a.in.window = scores->window;
    a.in.n_seq = cfg->n_seq;
    a.in.n_query = 1;
    a.in.r = cfg->n_q_heads / cfg->n_kv_heads;
    a.in.d = cfg->head_dim;
    a.in.bf16 = cfg->dtype == PK_DTYPE_BF16;
    a.out = out;
    a.os = *os;
    a.os.token = 0;
    a.lse = lse;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.o_bytes);
    a.parts = (int32_t)p.parts;
    a.bound = bound;
    return launch_kv16_attention(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_DEVICE;
}

pk_status pk_prompt_attention(const pk_prompt_config *cfg, const void *q, const void *k, const void *v, const pk_strides *qs, const pk_strides *ks,
                              const pk_strides *vs, const int32_t *starts, int32_t n_tokens, const pk_fp8_scores *scores, void *out,
                              const pk_strides *os, float *lse, void *stream)
{
    if (!cfg) return PK_ERR_INVALID_ARG;
    pk_status st = check_heads(cfg->n_seq, cfg->n_kv_heads, cfg->n_q_heads, cfg->head_dim, cfg->dtype);
    if (st != PK_OK) return st;
    if (cfg->n_seq > 4096) return PK_ERR_UNSUPPORTED;
    if (n_tokens < 0 || !starts || (n_tokens > 0 && (!q || !k || !v || !out))) return PK_ERR_INVALID_ARG;
    if ((st = check_scores(scores)) != PK_OK) return st;
    for (const pk_strides *s : {qs, ks, vs, os})
        if ((st = check_strides(s, &pk_strides::token, &pk_strides::head)) != PK_OK) return st;
    if (within(n_tokens, os->token, cfg->head_dim) || within(cfg->n_q_heads, os->head, cfg->head_dim)) return PK_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(starts) || !aligned16(out) || !aligned16(lse)) return PK_ERR_ALIGNMENT;
    if (n_tokens == 0) return PK_OK;
    const int64_t r = cfg->n_q_heads / cfg->n_kv_heads;
    if (n_tokens > kMostTokens || n_tokens * r > (1 << 28)) return PK_ERR_UNSUPPORTED;   // rows of a KV head, counted in 32 bits
    if (prompt_workgroups(cfg->n_seq, cfg->n_kv_heads, r, n_tokens) > kMostGroups) return PK_ERR_UNSUPPORTED;
    PromptArgs a;
    std::memset(&a, 0, sizeof(a));
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = out;
    a.lse = lse;
    a.starts = starts;
    a.slopes = scores->slopes;
    a.q_token = qs->token;
    a.q_head = qs->head;
    a.k_token = ks->token;
    a.k_head = ks->head;
    a.v_token = vs->token;
    a.v_head = vs->head;
    a.o_token = os->token;
    a.o_head = os->head;
    a.scale = scores->softmax_scale;
    a.cap = scores->cap;
    a.window = scores->window;
    a.n_seq = cfg->n_seq;
    a.n_kv_heads = cfg->n_kv_heads;
    a.r = (int32_t)r;
    a.d = cfg->head_dim;
    a.bf16 = cfg->dtype == PK_DTYPE_BF16;
    a.n_tokens = n_tokens;
    return launch_prompt(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_DEVICE;
}

}  // extern "C"
