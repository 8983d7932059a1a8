// Host side of the 8-bit cache's entry points (pk_fp8_api.hip: checks, sizes, overlap of caches) under AddressSanitizer /
// UndefinedBehaviorSanitizer, without a GPU: the launchers are the stubs below, so every pointer may be fake.  Prints "ok".
#include <cstdio>
#include <cstring>

#include "pk_fp8.h"

namespace pk {
static int g_launches = 0;
static Fp8AppendArgs g_append;
static Fp8AttentionArgs g_attention;
hipError_t launch_fp8_append(const Fp8AppendArgs &a, hipStream_t) { ++g_launches; g_append = a; return hipSuccess; }
int64_t fp8_attention_parts(int64_t n_seq, int64_t, int64_t, int64_t, int, int64_t bound) { return bound > 2048 ? 3 * n_seq : 0; }
hipError_t launch_fp8_attention(Fp8AttentionArgs &a, hipStream_t) { ++g_launches; g_attention = a; return hipSuccess; }
hipError_t launch_fp8_weights(Fp8WeightsArgs &, hipStream_t) { ++g_launches; return hipErrorInvalidValue; }
hipError_t launch_fp8_evict(const Fp8EvictArgs &, hipStream_t) { ++g_launches; return hipSuccess; }
}  // namespace pk

#define CHECK(cond)                                                  \
    do {                                                             \
        if (!(cond)) {                                               \
            std::printf("failed at line %d: %s\n", __LINE__, #cond); \
            return 1;                                                \
        }                                                            \
    } while (0)

static pk_fp8_cache cache_at(uintptr_t at, uint64_t step)
{
    pk_fp8_cache k;
    k.k_codes = reinterpret_cast<void *>(at);
    k.v_codes = reinterpret_cast<void *>(at + step);
    k.k_scale = reinterpret_cast<float *>(at + 2 * step);
    k.v_scale = reinterpret_cast<float *>(at + 3 * step);
    k.pos = reinterpret_cast<int32_t *>(at + 4 * step);
    k.weight = reinterpret_cast<float *>(at + 5 * step);
    k.page_table = nullptr;
    return k;
}

int main()
{
    pk_fp8_config c;
    std::memset(&c, 0, sizeof(c));
    c.n_seq = 2; c.n_kv_heads = 4; c.n_q_heads = 16; c.head_dim = 128; c.block = 64; c.t_capacity = 8192; c.dtype = PK_DTYPE_BF16;
    pk_fp8_layout lay;
    CHECK(pk_fp8_cache_layout(&c, &lay) == PK_OK && lay.k_codes == 8ull * 8192 * 128 && lay.k_scale == 8ull * 128 * 4);
    CHECK(pk_fp8_cache_layout(nullptr, &lay) == PK_ERR_INVALID_ARG && pk_fp8_cache_layout(&c, nullptr) == PK_ERR_INVALID_ARG);
    // the largest configurations: products stay in 64 bits
    pk_fp8_config big = c;
    big.n_seq = 65535; big.n_kv_heads = 1; big.n_q_heads = 64; big.head_dim = 256; big.t_capacity = 1 << 25;
    CHECK(pk_fp8_cache_layout(&big, &lay) == PK_OK && lay.k_codes == 65535ull * (1ull << 25) * 256);
    CHECK(pk_fp8_workspace_bytes(&big, PK_FP8_OP_ATTENTION, 1 << 25, 1 << 25) > 0);
    CHECK(pk_fp8_workspace_bytes(&big, PK_FP8_OP_EVICT, (1 << 25) - 1, 0) == 65535ull * ((1ull << 25) - 1) * 4 + (256 - 65535ull * ((1ull << 25) - 1) * 4 % 256) % 256);
    CHECK(pk_fp8_workspace_bytes(nullptr, PK_FP8_OP_EVICT, 1, 0) == 0);

    const uintptr_t at = 0x100000000ull;
    const pk_fp8_cache k = cache_at(at, 1ull << 32), other = cache_at(at + (1ull << 31), 1ull << 32);
    int32_t *states = reinterpret_cast<int32_t *>(0x1000), *after = reinterpret_cast<int32_t *>(0x2000);
    const void *x = reinterpret_cast<const void *>(0x30000);
    const pk_strides s = {4096, 512, 128};
    CHECK(pk_fp8_append(&c, &k, states, nullptr, x, x, &s, &s, 5, nullptr, nullptr) == PK_OK && pk::g_append.states_out == states && pk::g_append.c.log_block == 6);
    CHECK(pk_fp8_append(&c, &k, states, after, nullptr, nullptr, nullptr, nullptr, 0, nullptr, nullptr) == PK_OK && pk::g_append.n_new == 0);
    const int before = pk::g_launches;
    CHECK(pk_fp8_append(&c, &k, states, states + 4, x, x, &s, &s, 5, nullptr, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_fp8_append(&c, &k, states, nullptr, x, x, &s, nullptr, 5, nullptr, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_fp8_append(&c, nullptr, states, nullptr, x, x, &s, &s, 5, nullptr, nullptr) == PK_ERR_INVALID_ARG);
    const pk_fp8_scores sc = {0.1f, 0.f, 0, nullptr};
    float *out = reinterpret_cast<float *>(0x40000), *ws = reinterpret_cast<float *>(0x50000);
    const size_t need = pk_fp8_workspace_bytes(&c, PK_FP8_OP_ATTENTION, 3, 8192);
    CHECK(need > 0 && pk_fp8_workspace_bytes(&c, PK_FP8_OP_ATTENTION, 3, 100) == 0);
    CHECK(pk_fp8_attention(&c, &k, states, 8192, x, &s, 3, nullptr, nullptr, out, &s, nullptr, ws, need, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_fp8_attention(&c, &k, states, 8192, x, &s, 3, nullptr, &sc, out, &s, nullptr, ws, need - 1, nullptr) == PK_ERR_WORKSPACE);
    CHECK(pk::g_launches == before);
    CHECK(pk_fp8_attention(&c, &k, states, 8192, x, &s, 3, nullptr, &sc, out, &s, nullptr, ws, need, nullptr) == PK_OK);
    CHECK(pk::g_attention.parts == 6 && reinterpret_cast<char *>(pk::g_attention.part_ml) + 2 * 8 * 4 * 4 * 3 * 4 <= reinterpret_cast<char *>(ws) + need);
    CHECK(pk_fp8_attention(&c, &k, states, 100, x, &s, 3, nullptr, &sc, out, &s, nullptr, nullptr, 0, nullptr) == PK_OK && pk::g_attention.parts == 0);
    CHECK(pk_fp8_weights(&c, &k, states, 8192, x, &s, 3, nullptr, &sc, out, 1, nullptr) == PK_ERR_DEVICE);   // what the runtime refuses
    CHECK(pk_fp8_evict(&c, &k, states, &c, &other, after, 100, 4, 4, ws, 1 << 20, nullptr) == PK_OK);
    CHECK(pk_fp8_evict(&c, &k, states, &c, &k, after, 100, 4, 4, ws, 1 << 20, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_fp8_evict(&c, &k, states, &c, &other, states, 100, 4, 4, ws, 1 << 20, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_fp8_evict(&c, &k, states, &c, &other, after, 8192, 4, 4, nullptr, 0, nullptr) == PK_OK);   // everything is kept: no indices
    CHECK(pk_fp8_evict(&c, &k, states, nullptr, &other, after, 100, 4, 4, ws, 1 << 20, nullptr) == PK_ERR_INVALID_ARG);
    CHECK(pk_fp8_evict(&c, &k, states, &c, &other, after, 2147483647, 2147483647, 2147483647, ws, 1 << 20, nullptr) == PK_ERR_SHAPE);
    std::printf("ok\n");
    return 0;
}
