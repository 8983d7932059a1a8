// Appends to the 8-bit cache: one workgroup per block of tokens of a stream, for K and V or (blocks of many values) for one of them.
//
// For block b of a stream, x the new vectors that fall into it: field(b) = max(field that the block has, if it is partly
// filled, scale_field(max |x|)); code = nearest e4m3 of x * 2^-e.  A pass reads 2 d bytes and writes d per vector (K and V each):
// HBM bounds it for prompts, the chain state -> vectors -> reduction -> store for single tokens.
#include "pk_fp8.h"

namespace pk {

namespace {

// 8 values of 16 bits as binary32, non-finite ones as NaN
template <bool BF16>
__device__ __forceinline__ void widen8(const uint4 &v, float (&x)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) widen(w[i], BF16, x[2 * i], x[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__builtin_bit_cast(uint32_t, x[i]) & 0x7f800000u) == 0x7f800000u ? __builtin_nanf("") : x[i];
}
// largest magnitude among 8 values of 16 bits, in the type's own bits, non-finite ones left out
template <bool BF16>
__device__ __forceinline__ uint32_t largest8(const uint4 &v, bool &bad)
{
    constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
        bad |= lo >= kInf || hi >= kInf;
        most = max(most, max(lo < kInf ? lo : 0u, hi < kInf ? hi : 0u));
    }
    return most;
}

// Pieces of 8 values that a block of one of K and V has; threads so that a thread has three or four of them (what is on its way on a CU
// is what its resident threads have asked for: 16 ragged appends of 96 channels in 32-token blocks 29 us with 256 threads, 20 with 128 and K
// and V in one workgroup); K and V in one workgroup up to there (64 prompts of 8k tokens, 128 channels, 64-token blocks: 599 us in
// workgroups of their own, 618 in one).
template <int D, int B>
struct AppendShape {
    static constexpr int kPieces = B * D / 8;
    static constexpr int kThreads = kPieces <= 256 ? 64 : kPieces <= 512 ? 128 : 256;
    static constexpr int kPer = (kPieces + kThreads - 1) / kThreads;
    static constexpr int kSides = kPieces <= 512 ? 2 : 1;
};

template <int D, int B, bool BF16>
__global__ __launch_bounds__((AppendShape<D, B>::kThreads)) void fp8_append_kernel(Fp8AppendArgs a)
{
    using S = AppendShape<D, B>;
    constexpr int kPerRow = D / 8, kWaves = S::kThreads / 64, NS = S::kSides, NV = S::kPer;
    __shared__ uint32_t sm_max[NS][kWaves];
    __shared__ int sm_bad[NS][kWaves];
    const int tid = threadIdx.x, seq = blockIdx.y;
    const int hkv = a.c.n_kv_heads;
    const int head = blockIdx.x % hkv, rest = blockIdx.x / hkv;
    const int side = NS == 2 ? 0 : rest & 1, blk = NS == 2 ? rest : rest >> 1;   // the first side of the workgroup: 0 K, 1 V
    int2 st = fp8_state(a.states, seq, a.c.t_capacity);
    // the state may be replaced by this very launch once every wave of the sequence's workgroups has read it: no second load
    asm volatile("" : "+v"(st.x), "+v"(st.y));
    // nor a late one: one wave reports for its workgroup below, and a workgroup without a block has no other barrier before that.  (A wave that read
    // the grown state could take itself for one with a block, and write vectors behind the sequence's last into whatever page is named there.)
    __syncthreads();
    const int len = __builtin_amdgcn_readfirstlane(st.x), next = __builtin_amdgcn_readfirstlane(st.y);
    const int count = min(fp8_count(a.counts, seq, a.n_new), a.c.t_capacity - len);
    const int t0 = (len / B + blk) * B, end = len + count;
    if (count > 0 && t0 < end) {
        const int stream = seq * hkv + head;
        const int64_t row0 = a.c.map.of(stream).pos(t0);
        const int held = max(len - t0, 0);   // tokens that the block has already
        uint4 raw[NS][NV];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const bool v = NS == 2 ? s == 1 : side == 1;
            const int64_t seq_stride = v ? a.vs.seq : a.ks.seq, token = v ? a.vs.token : a.ks.token, head_stride = v ? a.vs.head : a.ks.head;
            const char *src = static_cast<const char *>(v ? a.v_new : a.k_new) + 2 * (seq * seq_stride + head * head_stride);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = tid + i * S::kThreads, t = t0 + p / kPerRow;
                raw[s][i] = make_uint4(0, 0, 0, 0);
                if (p < S::kPieces && t >= len && t < end) raw[s][i] = *reinterpret_cast<const uint4 *>(src + 2 * ((int64_t)(t - len) * token + (p % kPerRow) * 8));
            }
        }
        float *scale[NS];
        float was[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            scale[s] = ((NS == 2 ? s == 1 : side == 1) ? a.c.v_scale : a.c.k_scale) + (row0 >> a.c.log_block);
            was[s] = held > 0 ? *scale[s] : 0.f;
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            uint32_t most = 0;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < NV; ++i) most = max(most, largest8<BF16>(raw[s][i], bad));
            for (int o = 1; o < 64; o <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
            const bool any = __any(bad);
            if ((tid & 63) == 0) {
                sm_max[s][tid >> 6] = most;
                sm_bad[s][tid >> 6] = any;
            }
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            uint32_t most = 0;
            int flagged = was[s] < 0.f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                most = max(most, sm_max[s][i]);
                flagged |= sm_bad[s][i];
            }
            float amax, unused;
            widen(most, BF16, amax, unused);
            const int old = held > 0 ? field_of_scale(was[s]) : 1;
            const int field = max(scale_field(__builtin_bit_cast(uint32_t, amax)), old);
            const float inv = inverse_of_field(field);
            uint8_t *codes = ((NS == 2 ? s == 1 : side == 1) ? a.c.v_codes : a.c.k_codes) + row0 * D;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = tid + i * S::kThreads, t = t0 + p / kPerRow;
                if (p < S::kPieces && t >= len && t < end) {
                    float x[8];
                    widen8<BF16>(raw[s][i], x);
                    *reinterpret_cast<uint2 *>(codes + (int64_t)p * 8) = make_uint2(codes4(x, inv), codes4(x + 4, inv));
                }
            }
            if (held > 0 && field > old) {   // the codes that are there, at the larger scale
                const float shift = field - old > 126 ? 0.f : inverse_of_field(field - old + 127);
                for (int p = tid; p < held * kPerRow; p += S::kThreads) {
                    uint2 *at = reinterpret_cast<uint2 *>(codes + (int64_t)p * 8);
                    const uint2 w = *at;
                    float y[8];
                    const half2v h[4] = {codes_lo(w.x), codes_hi(w.x), codes_lo(w.y), codes_hi(w.y)};
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = (float)h[i >> 1][i & 1];
                    *at = make_uint2(codes4(y, shift), codes4(y + 4, shift));
                }
            }
            if (tid == 0) *scale[s] = __builtin_bit_cast(float, ((uint32_t)field << 23) | ((uint32_t)flagged << 31));
        }
        if (side == 0)
            for (int i = tid; i < B; i += S::kThreads) {
                if (t0 + i < len || t0 + i >= end) continue;
                const int64_t at = (int64_t)stream * a.c.t_capacity + t0 + i;
                a.c.pos[at] = next + (t0 + i - len);
                if (a.c.weight) a.c.weight[at] = 0.f;
            }
    }
    if (tid != 0) return;
    // The state afterwards: from one workgroup where it has a place of its own, else from the sequence's last one to come here, as
    // the others have read the old one by then, every wave of them (the barrier behind the load).
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
    using S = AppendShape<D, B>;
    // blocks that n_new vectors can touch, wherever the first of them falls
    const int64_t blocks = ((int64_t)a.n_new + B - 2) / B + 1;
    const dim3 grid((uint32_t)(blocks * (2 / S::kSides) * a.c.n_kv_heads), a.n_seq);
    if (a.bf16) fp8_append_kernel<D, B, true><<<grid, S::kThreads, 0, s>>>(a);
    else fp8_append_kernel<D, B, false><<<grid, S::kThreads, 0, s>>>(a);
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
