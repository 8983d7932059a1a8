// The 8-bit cache (pk_fp8_* of include/patternkv.h): what its translation units share.
#pragma once

#include "pk_internal.h"
#include "pk_lanes.h"

namespace pk {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

struct Fp8View {
    uint8_t *k_codes, *v_codes;
    float *k_scale, *v_scale;
    int32_t *pos;
    float *weight;            // or null
    PackedMap map;            // rows of the code arrays; a row's scale is entry row >> log_block of the scale arrays
    int32_t log_block;
    int32_t t_capacity, n_kv_heads;
};

struct Fp8AppendArgs {
    Fp8View c;
    const int32_t *states;
    int32_t *states_out;      // may be states
    const void *k_new, *v_new;
    pk_strides ks, vs;
    const int32_t *counts;    // or null
    int32_t n_seq, n_new, d, bf16;
};
hipError_t launch_fp8_append(const Fp8AppendArgs &a, hipStream_t s);

struct Fp8Queries {           // what attention and weights share
    Fp8View c;
    const int32_t *states;
    const void *q;
    pk_strides qs;
    const int32_t *counts;    // or null
    const float *slopes;      // or null
    float scale, cap;
    int32_t window;
    int32_t n_seq, n_query, r, d, bf16;   // r: query heads per KV head
};
struct Fp8AttentionArgs {
    Fp8Queries in;
    void *out;
    pk_strides os;
    float *lse;               // or null
    float *part_o, *part_ml;  // parts > 0: results of the slots, [slots][kv heads][rows][d] normalised, [slots][kv heads][rows][2] reference and sum
    int32_t parts;            // work items that the keys of a KV head and a group of rows are dealt out in, 0: one per sequence
    int32_t groups;           // of rows (set by the launch)
    int32_t bound;            // the caller's, of the tokens held
};
// Both from host values alone.
int64_t fp8_attention_parts(int64_t n_seq, int64_t n_kv_heads, int64_t r, int64_t n_query, int d, int64_t bound);
inline int64_t fp8_attention_slots(int64_t n_seq, int64_t parts) { return n_seq + parts; }
hipError_t launch_fp8_attention(Fp8AttentionArgs &a, hipStream_t s);
// The pieces of every row together; the pieces are as pk_attention.h deals them out.
hipError_t launch_attention_merge(const Fp8AttentionArgs &a, hipStream_t s);

struct Fp8WeightsArgs {
    Fp8Queries in;
    const float *lse;
    int32_t accumulate, bound;
    int32_t parts;            // as for the attention (set by the launch)
};
hipError_t launch_fp8_weights(Fp8WeightsArgs &a, hipStream_t s);

struct Fp8EvictArgs {
    Fp8View from, to;
    const int32_t *states;
    int32_t *to_states;
    int32_t n_seq, d, budget, keep_first, keep_last;
    int32_t *kept;            // [N][budget] workspace: the old index of every kept token
};
hipError_t launch_fp8_evict(const Fp8EvictArgs &a, hipStream_t s);

// ---- device helpers ---------------------------------------------------------------------------------------------------

// Exponent field of the scale of a block whose largest magnitude is amax (bits of a finite float >= 0): the smallest 2^e with
// amax <= 448 * 2^e.  448 = 1.75 * 2^8, so e is amax's exponent - 8, one more where its mantissa exceeds 0.75.
__device__ __forceinline__ int scale_field(uint32_t amax)
{
    const int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, 1);
}
__device__ __forceinline__ float scale_of_field(int field) { return __builtin_bit_cast(float, (uint32_t)field << 23); }
__device__ __forceinline__ int field_of_scale(float s) { return max((int)((__builtin_bit_cast(uint32_t, s) >> 23) & 255u), 1); }
// 2^-e of the scale with that field (1 <= field <= 253 here: the largest 16-bit values give 247)
__device__ __forceinline__ float inverse_of_field(int field) { return __builtin_bit_cast(float, (uint32_t)(254 - field) << 23); }

// four e4m3 codes of x * inv, |x * inv| <= 448 or NaN, nearest with ties to even (the conversion keeps NaN)
__device__ __forceinline__ uint32_t codes4(const float *x, float inv)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
    return (uint32_t)w;
}
__device__ __forceinline__ half2v codes_lo(uint32_t w) { return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false); }
__device__ __forceinline__ half2v codes_hi(uint32_t w) { return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true); }
// bit 7 of every byte that is a NaN code
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// two 16-bit values as binary32
__device__ __forceinline__ void widen(uint32_t w, int bf16, float &lo, float &hi)
{
    if (bf16) {
        lo = __builtin_bit_cast(float, w << 16);
        hi = __builtin_bit_cast(float, w & 0xffff0000u);
    } else {
        const half2v h = __builtin_bit_cast(half2v, w);
        lo = (float)h[0];
        hi = (float)h[1];
    }
}
// two binary32 values in the 16-bit type, nearest, ties to even
__device__ __forceinline__ uint32_t narrow(float lo, float hi, int bf16)
{
    if (bf16) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        const bf2 b = {(__bf16)lo, (__bf16)hi};
        return __builtin_bit_cast(uint32_t, b);
    }
    const half2v h = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, h);
}

// tokens held by a sequence, clamped to the cache, and the position of its next one
__device__ __forceinline__ int2 fp8_state(const int32_t *states, int seq, int t_capacity)
{
    const int2 v = *reinterpret_cast<const int2 *>(states + 4 * (int64_t)seq);
    return make_int2(min(max(v.x, 0), t_capacity), v.y);
}
__device__ __forceinline__ int fp8_count(const int32_t *counts, int seq, int n)
{
    return counts ? min(max(counts[seq], 0), n) : n;
}

}  // namespace pk
