// Host side of the paged 16-bit cache's entry points (pk_kv16_api.hip: checks, sizes, overlap of arrays) under AddressSanitizer /
// UndefinedBehaviorSanitizer, without a GPU: the launchers are the stubs below, so every pointer may be fake.  Prints "ok".
#include <cstdio>
#include <cstring>

#include "pk_kv16.h"

namespace pk {
static int g_launches = 0;
static PagesArgs g_pages;
static Kv16AppendArgs g_append;
static Fp8AttentionArgs g_attention;
static PromptArgs g_prompt;
hipError_t launch_pages(const PagesArgs &a, hipStream_t) { ++g_launches; g_pages = a; return hipSuccess; }
hipError_t launch_kv16_append(const Kv16AppendArgs &a, hipStream_t) { ++g_launches; g_append = a; return hipSuccess; }
int64_t kv16_attention_parts(int64_t n_seq, int64_t, int64_t, int, int64_t bound) { return bound > 512 ? 3 * n_seq : 0; }
hipError_t launch_kv16_attention(Fp8AttentionArgs &a, hipStream_t) { ++g_launches; g_attention = a; return hipErrorInvalidValue; }
hipError_t launch_prompt(const PromptArgs &a, hipStream_t) { ++g_launches; g_prompt = a; return hipSuccess; }
int64_t prompt_workgroups(int64_t n_seq, int64_t n_kv_heads, int64_t r, int64_t n_tokens) { return (n_tokens * r + n_seq * 127) / 128 * n_kv_heads; }
}  // namespace pk

#define CHECK(cond)                                                  \
    do {                                                             \
        if (!(cond)) {                                               \
            std::printf("failed at line %d: %s\n", __LINE__, #cond); \
            return 1;                                                \
        }                                                            \
    } while (0)

static int32_t *at(uintptr_t x) { return reinterpret_cast<int32_t *>(x); }

int main()
{
    // pages: the largest sizes, in place and not
    pk_pages_config g = {65535, 1, 0x7fffffff, 1 << 25};
    CHECK(pk_pages_workspace_bytes(&g) == 65535 * 4 + 4 && pk_pages_workspace_bytes(nullptr) == 0);
    const uintptr_t far = 1ull << 44;   // apart by more than the largest array
    pk_pages p = {at(far), at(2 * far), at(3 * far), nullptr};
    CHECK(pk_pages_update(&g, &p, at(4 * far), nullptr, at(5 * far), 0x7fffffff, at(6 * far), at(7 * far), nullptr, at(8 * far), at(9 * far), 1 << 20, nullptr) == PK_OK);
    CHECK(pk::g_launches == 1 && pk::g_pages.states_out == at(4 * far) && pk::g_pages.n_free_out == at(3 * far) && pk::g_pages.page_shift == 0);
    g.page_tokens = 64;
    g.n_pages = 1000;
    g.pages_per_seq = 5;
    p.n_free_out = at(10 * far);
    CHECK(pk_pages_update(&g, &p, at(4 * far), at(11 * far), at(5 * far), 0, at(6 * far), nullptr, nullptr, at(8 * far), at(9 * far), 1 << 20, nullptr) == PK_OK);
    CHECK(pk::g_launches == 2 && pk::g_pages.states_out == at(11 * far) && pk::g_pages.n_free_out == at(10 * far) && pk::g_pages.page_shift == 6);
    CHECK(pk_pages_update(&g, &p, at(4 * far), at(4 * far + 16), at(5 * far), 0, at(6 * far), nullptr, nullptr, at(8 * far), at(9 * far), 1 << 20, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_pages_update(&g, nullptr, at(4 * far), nullptr, at(5 * far), 0, at(6 * far), nullptr, nullptr, at(8 * far), at(9 * far), 1 << 20, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk::g_launches == 2);

    pk_kv16_config c = {2, 4, 16, 128, 1024, PK_DTYPE_BF16, 32, 100};
    CHECK(pk_kv16_cache_bytes(&c) == 100ull * 4 * 32 * 128 * 2 && pk_kv16_cache_bytes(nullptr) == 0);
    CHECK(pk_kv16_workspace_bytes(&c, 512) == 0 && pk_kv16_workspace_bytes(&c, 1024) > 0 && pk_kv16_workspace_bytes(nullptr, 1) == 0);
    pk_kv16_config big = {1, 65535, 65535, 256, 1 << 25, PK_DTYPE_FP16, 1 << 25, 63};
    CHECK(pk_kv16_cache_bytes(&big) == 63ull * 65535 * (1ull << 25) * 512);
    pk_kv16_cache k = {at(far), at(2 * far), at(3 * far)};
    const pk_strides s = {4096, 512, 128};
    CHECK(pk_kv16_append(&c, &k, at(far), at(far), &s, &s, at(far), 0x7fffffff, nullptr) == PK_OK && pk::g_launches == 3);
    CHECK(pk::g_append.n_slots == 3200 && pk::g_append.page_shift == 5 && pk::g_append.k_token == 512 && pk::g_append.v_head == 128);
    CHECK(pk_kv16_append(&c, &k, at(far), at(far), nullptr, &s, at(far), 1, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_kv16_append(nullptr, &k, at(far), at(far), &s, &s, at(far), 1, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_kv16_append(&c, nullptr, at(far), at(far), &s, &s, at(far), 1, nullptr) == PK_ERR_INVALID_ARG && pk::g_launches == 3);
    const pk_fp8_scores sc = {-0.5f, 30.f, 100, nullptr};
    CHECK(pk_kv16_attention(&c, &k, at(far), 512, at(far), &s, &sc, at(far), &s, nullptr, nullptr, 0, nullptr) == PK_ERR_DEVICE && pk::g_launches == 4);   // the stub's launch is refused
    CHECK(pk::g_attention.in.r == 4 && pk::g_attention.in.n_query == 1 && pk::g_attention.in.bf16 == 1 && pk::g_attention.in.c.map.pages_per_seq == 32 && pk::g_attention.parts == 0);
    CHECK(pk_kv16_attention(&c, &k, at(far), 1024, at(far), &s, &sc, at(far), &s, nullptr, nullptr, 0, nullptr) == PK_ERR_WORKSPACE);
    CHECK(pk_kv16_attention(&c, &k, at(far), 1024, at(far), &s, nullptr, at(far), &s, nullptr, at(far), 1 << 30, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_kv16_attention(&c, &k, at(far), 1024, at(far), nullptr, &sc, at(far), &s, nullptr, at(far), 1 << 30, nullptr) == PK_ERR_INVALID_ARG && pk::g_launches == 4);

    pk_prompt_config pc = {4096, 1, 1, 64, PK_DTYPE_FP16};
    CHECK(pk_prompt_attention(&pc, at(far), at(far), at(far), &s, &s, &s, at(far), 1 << 25, &sc, at(2 * far), &s, nullptr, nullptr) == PK_OK && pk::g_launches == 5);
    CHECK(pk::g_prompt.n_tokens == 1 << 25 && pk::g_prompt.q_token == 512 && pk::g_prompt.window == 100);
    CHECK(pk_prompt_attention(nullptr, at(far), at(far), at(far), &s, &s, &s, at(far), 5, &sc, at(2 * far), &s, nullptr, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_prompt_attention(&pc, at(far), at(far), at(far), &s, nullptr, &s, at(far), 5, &sc, at(2 * far), &s, nullptr, nullptr) == PK_ERR_INVALID_ARG);
    pc.n_kv_heads = pc.n_q_heads = 65535;
    CHECK(pk_prompt_attention(&pc, at(far), at(far), at(far), &s, &s, &s, at(far), 1 << 25, &sc, at(2 * far), &s, nullptr, nullptr) == PK_ERR_UNSUPPORTED && pk::g_launches == 5);
    std::printf("ok\n");
    return 0;
}
