// The paged 16-bit cache, its pages and the attention of prompts (pk_pages_*, pk_kv16_*, pk_prompt_attention of include/patternkv.h): what the
// translation units share.
#pragma once

#include "pk_fp8.h"

namespace pk {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));   // 16-bit operands of a matrix instruction, of either type
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

struct PagesArgs {
    int32_t n_seq, page_shift, n_pages, pages_per_seq, n_tokens;
    int32_t *table, *free_pages;
    const int32_t *n_free;
    int32_t *n_free_out;      // may be n_free
    const int32_t *states;
    int32_t *states_out;      // may be states
    const int32_t *counts;
    int32_t *starts, *slots, *positions, *taken;   // positions may be null
    int32_t *first;           // workspace [n_seq]: where on the stack the pages of a sequence come from
};
hipError_t launch_pages(const PagesArgs &a, hipStream_t s);

struct Kv16AppendArgs {
    void *k, *v;
    const void *k_new, *v_new;
    int64_t k_token, k_head, v_token, v_head;      // strides in elements
    const int32_t *slots;
    int32_t n_tokens, n_kv_heads, d, page_shift, n_slots;
};
hipError_t launch_kv16_append(const Kv16AppendArgs &a, hipStream_t s);

// The 8-bit cache's arguments with 16-bit vectors in the places of the codes; n_query is 1.
// With 256 channels and more than 16 heads per KV head calls of more tokens (sequences * KV heads * bound) than this take two row tiles per wave.
constexpr int64_t kOneTileTokens = 1 << 18;
int64_t kv16_attention_parts(int64_t n_seq, int64_t n_kv_heads, int64_t r, int d, int64_t bound);
hipError_t launch_kv16_attention(Fp8AttentionArgs &a, hipStream_t s);

struct PromptArgs {
    const void *q, *k, *v;
    void *out;
    float *lse;               // or null
    const int32_t *starts;
    const float *slopes;      // or null
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;   // strides in elements
    float scale, cap;
    int32_t window;
    int32_t n_seq, n_kv_heads, r, d, bf16, n_tokens;
};
hipError_t launch_prompt(const PromptArgs &a, hipStream_t s);
// Workgroups of the launch at most: row tiles of all sequences and KV heads
int64_t prompt_workgroups(int64_t n_seq, int64_t n_kv_heads, int64_t r, int64_t n_tokens);

// ---- device helpers ---------------------------------------------------------------------------------------------------

template <bool BF16>
__device__ __forceinline__ float4v mfma16(short8v a, short8v b, float4v c)   // 16 x 16 x 32
{
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, a), __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}
template <bool BF16>
__device__ __forceinline__ float16v mfma32(short8v a, short8v b, float16v c)   // 32 x 32 x 16
{
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8v, a), __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// Softmax numerators are 2^(score - reference).  The reference for a largest score `top` serves scores up to kRoom above it, so that it moves a few times in a
// row, not with every larger score.  fp16's smallest step is 2^-24, so that its numerators go up to 2^11, 2^15 with the room (a token counts down to 2^-36 of the
// largest one); scores of 2^20 and more, whose own steps are large, are the reference themselves.  bf16 has the exponents of binary32: numerators
// of up to 2^-25 with the room, so that values up to the type's largest times 2^25 tokens stay finite; from 2^29 on, where half a step is more than that and the
// reference comes out as the score itself, numerators are taken kUnder below it (under_of).
constexpr float kRoom = 4.f, kUnder = 25.f + kRoom;
template <bool BF16>
__device__ __forceinline__ float reference_of(float top)
{
    if constexpr (BF16) return top + kUnder;
    else return fabsf(top) < 0x1p20f ? top - 11.f : top;
}
// How far below the reference a row's numerators are taken, as a power of two.  most: the largest score that the reference serves, which from 2^20 on is the largest
// score itself; -inf where nothing has been seen.
template <bool BF16>
__device__ __forceinline__ float under_of(float most)
{
    return BF16 && most + kUnder == most ? kUnder : 0.f;
}
// 2^(m - to), what numerators of the reference m are in those of `to`.  A row that comes to another side of 2^29 is seen to in a branch for the whole wave, which
// only large references take (a prompt of 32k tokens 7.36 -> 7.41 ms; in line 7.40 -> 7.50).  Where `to` is less than 2^28 and m was 2^29 or more, the factor is 0 anyhow.
template <bool BF16>
__device__ __forceinline__ float change_of(float m, float to, float was, float most)
{
    float by = __builtin_amdgcn_exp2f(m - to);
    if (BF16 && __any(fabsf(to) >= 0x1p28f)) by = __builtin_amdgcn_exp2f((m - to) + (under_of<BF16>(was) - under_of<BF16>(most)));
    return by;
}
// From here on scores are rounded before the reference is taken off, as their largest is: the multiply-add would take the factor in unrounded, and the numerator
// of a row's only token would be no power of two, which the 16-bit type holds exactly.
constexpr float kLarge = 0x1p12f;
// A mean of values of the type is none beyond its largest, but the numerators' rounding may bring it there.
template <bool BF16>
__device__ __forceinline__ float mean_of(float x)
{
    constexpr float most = BF16 ? 0x1.fep127f : 65504.f;
    return fabsf(x) < INFINITY ? fminf(fmaxf(x, -most), most) : x;
}

}  // namespace pk
