// Appends to the 8-bit cache: one workgroup per (block of tokens, stream, K or V).
//
// For block b of a stream, x the new vectors that fall into it: field(b) = max(field that the block has, if it is partly
// filled, scale_field(max |x|)); code = nearest e4m3 of x * 2^-e.  A pass reads 2 d bytes and writes d per vector (K and V each):
// HBM bounds it for prompts, the chain state -> vectors -> reduction -> store for single tokens.
#include "pk_fp8.h"

namespace pk {

namespace {

constexpr int kThreads = 256;

// largest magnitude (bits) of 8 values of 16 bits, non-finite ones left out; those are replaced by NaN
template <bool BF16>
__device__ __forceinline__ void widen8(const uint4 &v, float (&x)[8], uint32_t &amax, bool &bad)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) widen(w[i], BF16, x[2 * i], x[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t m = __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu;
        const bool fin = m < 0x7f800000u;
        amax = max(amax, fin ? m : 0u);
        bad |= !fin;
        x[i] = fin ? x[i] : __builtin_nanf("");
    }
}

// NV: pieces of 8 values per thread
template <int D, int B, bool BF16>
__global__ __launch_bounds__(kThreads) void fp8_append_kernel(Fp8AppendArgs a)
{
    constexpr int kPieces = B * D / 8, NV = (kPieces + kThreads - 1) / kThreads, kPerRow = D / 8;
    __shared__ uint32_t sm_max[kThreads / 64];
    __shared__ int sm_bad[kThreads / 64];
    const int tid = threadIdx.x, seq = blockIdx.y;
    const int hkv = a.c.n_kv_heads;
    const int head = blockIdx.x % hkv, rest = blockIdx.x / hkv;
    const bool is_v = rest & 1;
    const int blk = rest >> 1;
    int2 st = fp8_state(a.states, seq, a.c.t_capacity);
    // the state may be replaced by this very launch once every workgroup of the sequence has read it: no second load
    asm volatile("" : "+v"(st.x), "+v"(st.y));
    const int len = __builtin_amdgcn_readfirstlane(st.x), next = __builtin_amdgcn_readfirstlane(st.y);
    const int count = min(fp8_count(a.counts, seq, a.n_new), a.c.t_capacity - len);
    const int t0 = (len / B + blk) * B, end = len + count;
    if (count > 0 && t0 < end) {
        const int stream = seq * hkv + head;
        const int64_t row0 = a.c.map.of(stream).pos(t0);
        const pk_strides &st3 = is_v ? a.vs : a.ks;
        const char *src = static_cast<const char *>(is_v ? a.v_new : a.k_new) + 2 * (seq * st3.seq + head * st3.head);
        uint8_t *codes = (is_v ? a.c.v_codes : a.c.k_codes) + row0 * D;
        float *scale = (is_v ? a.c.v_scale : a.c.k_scale) + (row0 >> a.c.log_block);
        const int held = max(len - t0, 0);   // tokens that the block has already
        float x[NV][8];
        uint32_t amax = 0;
        bool bad = false;
        uint4 raw[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = tid + i * kThreads, t = t0 + p / kPerRow;
            raw[i] = make_uint4(0, 0, 0, 0);
            if (p < kPieces && t >= len && t < end)
                raw[i] = *reinterpret_cast<const uint4 *>(src + 2 * ((int64_t)(t - len) * st3.token + (p % kPerRow) * 8));
        }
        const float was = held > 0 ? *scale : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) widen8<BF16>(raw[i], x[i], amax, bad);
        for (int o = 1; o < 64; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o));
        const bool any_bad = __any(bad);
        if ((tid & 63) == 0) {
            sm_max[tid >> 6] = amax;
            sm_bad[tid >> 6] = any_bad;
        }
        __syncthreads();
        amax = max(max(sm_max[0], sm_max[1]), max(sm_max[2], sm_max[3]));
        const int flagged = sm_bad[0] | sm_bad[1] | sm_bad[2] | sm_bad[3] | (was < 0.f ? 1 : 0);
        const int old = held > 0 ? field_of_scale(was) : 1;
        const int field = max(scale_field(amax), old);
        const float inv = inverse_of_field(field);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = tid + i * kThreads, t = t0 + p / kPerRow;
            if (p < kPieces && t >= len && t < end) {
                const uint2 w = make_uint2(codes4(x[i], inv), codes4(x[i] + 4, inv));
                *reinterpret_cast<uint2 *>(codes + (int64_t)p * 8) = w;
            }
        }
        if (held > 0 && field > old) {   // the codes that are there, at the larger scale
            const float shift = field - old > 126 ? 0.f : inverse_of_field(field - old + 127);
            for (int p = tid; p < held * kPerRow; p += kThreads) {
                uint2 *at = reinterpret_cast<uint2 *>(codes + (int64_t)p * 8);
                const uint2 w = *at;
                float y[8];
                const half2v h[4] = {codes_lo(w.x), codes_hi(w.x), codes_lo(w.y), codes_hi(w.y)};
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = (float)h[i >> 1][i & 1];
                *at = make_uint2(codes4(y, shift), codes4(y + 4, shift));
            }
        }
        if (tid == 0) *scale = __builtin_bit_cast(float, ((uint32_t)field << 23) | ((uint32_t)flagged << 31));
        if (!is_v && tid < B && t0 + tid >= len && t0 + tid < end) {
            const int64_t at = (int64_t)stream * a.c.t_capacity + t0 + tid;
            a.c.pos[at] = next + (t0 + tid - len);
            if (a.c.weight) a.c.weight[at] = 0.f;
        }
    }
    if (tid != 0) return;
    // The state afterwards: from one workgroup where it has a place of its own, else from the sequence's last one to come here, as
    // the others have read the old one by then (what a workgroup adds to the counter depends on what it read).
    int32_t *out = a.states_out + 4 * (int64_t)seq;
    if (a.states_out != a.states) {
        if (blockIdx.x == 0) *reinterpret_cast<int4 *>(out) = make_int4(len + count, next + count, 0, 0);
    } else {
        const int arrived = atomicAdd(out + 2, 1);
        if (arrived == (int)gridDim.x - 1) *reinterpret_cast<int4 *>(out) = make_int4(len + count, next + count, 0, 0);
    }
}

template <int D, int B>
hipError_t launch(const Fp8AppendArgs &a, hipStream_t s)
{
    // blocks that n_new vectors can touch, wherever the first of them falls
    const int64_t blocks = ((int64_t)a.n_new + B - 2) / B + 1;
    const dim3 grid((uint32_t)(blocks * 2 * a.c.n_kv_heads), a.n_seq);
    if (a.bf16) fp8_append_kernel<D, B, true><<<grid, kThreads, 0, s>>>(a);
    else fp8_append_kernel<D, B, false><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const Fp8AppendArgs &a, hipStream_t s)
{
    return a.c.log_block == 5 ? launch<D, 32>(a, s) : a.c.log_block == 6 ? launch<D, 64>(a, s) : launch<D, 128>(a, s);
}

}  // namespace

hipError_t launch_fp8_append(const Fp8AppendArgs &a, hipStream_t s)
{
    return a.d == 64 ? launch_d<64>(a, s) : a.d == 96 ? launch_d<96>(a, s) : a.d == 128 ? launch_d<128>(a, s) : launch_d<256>(a, s);
}

}  // namespace pk
