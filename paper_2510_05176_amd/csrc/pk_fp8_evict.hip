// Eviction from the 8-bit cache, in two launches: which tokens stay (one workgroup per stream, into the workspace), and their
// move into the other cache (one workgroup per new block of a stream, K and V).
//
// The choice is a radix selection over the weights as ordered integers: three histograms of 11, 11 and 10 bits find the weight of
// the last token that stays, then every wave counts and writes its own run of tokens, so that ties go to the earlier ones and
// the order is kept.  It reads the weights five times, from the caches but for the first.
#include "pk_fp8.h"

namespace pk {

namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64, kBins = 2048;

// Weights as integers in their order: NaN lowest, -0 as +0
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (w != w) return 0;
    const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ __launch_bounds__(kSelThreads) void fp8_select_kernel(Fp8EvictArgs a)
{
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t sm_prefix, sm_need, sm_wave[kSelWaves][2];
    const int stream = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int len = fp8_state(a.states, stream / a.from.n_kv_heads, a.from.t_capacity).x;
    int32_t *kept = a.kept + (int64_t)stream * a.budget;
    if (len <= a.budget) return;   // the move takes such a sequence whole
    const int lo = a.keep_first, hi = len - a.keep_last;   // candidates; more of them than the budget has room for
    const float *w = a.from.weight + (int64_t)stream * a.from.t_capacity;
    uint32_t need = (uint32_t)(a.budget - a.keep_first - a.keep_last);   // of those with the prefix found so far
    uint32_t prefix = 0;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
        for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
        __syncthreads();
        for (int t = lo + tid; t < hi; t += kSelThreads) {
            const uint32_t u = order_of(w[t]);
            if (pass == 0 || (u >> (shift + width)) == prefix) atomicAdd(&hist[(u >> shift) & ((1u << width) - 1)], 1u);
        }
        __syncthreads();
        // the bin, from the top, in which the need-th token lies: wave 0, 32 bins per lane
        if (wave == 0) {
            constexpr int per = kBins / 64;
            uint32_t sum = 0;
            for (int i = 0; i < per; ++i) sum += hist[kBins - 1 - (lane * per + i)];
            uint32_t before = sum;
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t v = __shfl_up(before, o);
                if (lane >= o) before += v;
            }
            before -= sum;
            if (need > 0 && before < need && need <= before + sum) {
                int bin = kBins - 1 - lane * per;
                while (before + hist[bin] < need) before += hist[bin--];
                sm_prefix = (prefix << width) | (uint32_t)bin;
                sm_need = need - before;
            }
        }
        __syncthreads();
        if (need > 0) {
            prefix = sm_prefix;
            need = sm_need;
        }
        __syncthreads();
    }
    const bool none = a.budget == a.keep_first + a.keep_last;
    // kept: larger than prefix, or equal and among the first `need` of those
    const int per_wave = ((hi - lo + kSelWaves - 1) / kSelWaves + 63) & ~63;
    const int from = lo + wave * per_wave, to = min(from + per_wave, hi);
    uint32_t above = 0, equal = 0;
    if (!none) {
        for (int t = from + lane; t < to; t += 64) {
            const uint32_t u = order_of(w[t]);
            above += u > prefix;
            equal += u == prefix;
        }
        for (int o = 1; o < 64; o <<= 1) {
            above += __shfl_xor(above, o);
            equal += __shfl_xor(equal, o);
        }
    }
    if (lane == 0) {
        sm_wave[wave][0] = above;
        sm_wave[wave][1] = equal;
    }
    __syncthreads();
    uint32_t above_before = 0, equal_before = 0;
    for (int i = 0; i < wave; ++i) {
        above_before += sm_wave[i][0];
        equal_before += sm_wave[i][1];
    }
    if (!none) {
        const uint64_t below = (1ull << lane) - 1;
        for (int t0 = from; t0 < to; t0 += 64) {
            const int t = t0 + lane;
            const uint32_t u = t < to ? order_of(w[t]) : 0;
            const bool gt = t < to && u > prefix, eq = t < to && u == prefix;
            const uint64_t m_gt = __ballot(gt), m_eq = __ballot(eq);
            const uint32_t n_gt = above_before + __popcll(m_gt & below), n_eq = equal_before + __popcll(m_eq & below);
            if (gt || (eq && n_eq < need)) kept[a.keep_first + n_gt + min(n_eq, need)] = t;
            above_before += __popcll(m_gt);
            equal_before += __popcll(m_eq);
        }
    }
    for (int i = tid; i < a.keep_first; i += kSelThreads) kept[i] = i;
    for (int i = tid; i < a.keep_last; i += kSelThreads) kept[a.budget - a.keep_last + i] = hi + i;
}

constexpr int kMoveThreads = 256;

template <int D>
__global__ __launch_bounds__(kMoveThreads) void fp8_move_kernel(Fp8EvictArgs a)
{
    constexpr int kPerRow = D / 16;
    constexpr int kMost = (128 * kPerRow + kMoveThreads - 1) / kMoveThreads;   // pieces of 16 codes per thread, largest block
    __shared__ int sm_max[kMoveThreads / 64], sm_bad[kMoveThreads / 64], sm_row[128], sm_field[128];
    const int tid = threadIdx.x, hkv = a.from.n_kv_heads;
    const int stream = blockIdx.y, seq = stream / hkv;
    const int B = 1 << a.from.log_block;
    const int2 st = fp8_state(a.states, seq, a.from.t_capacity);
    const int held = min(st.x, a.budget);
    const bool whole = st.x <= a.budget;
    const bool is_v = blockIdx.x & 1;
    const int t0 = (int)(blockIdx.x >> 1) * B, n = min(held - t0, B);
    if (tid == 0 && stream % hkv == 0 && blockIdx.x == 0) *reinterpret_cast<int4 *>(a.to_states + 4 * (int64_t)seq) = make_int4(held, st.y, 0, 0);
    if (n <= 0) return;
    const StreamMap from = a.from.map.of(stream);
    if (tid < n) {
        // an index from the workspace is one that the selection wrote, below the sequence's length
        const int t = whole ? t0 + tid : a.kept[(int64_t)stream * a.budget + t0 + tid];
        int64_t row;
        if (from.pages) {
            const int page = min(max(from.pages[t >> from.shift], 0), from.n_pages - 1);
            row = from.pos_in(page, t);
        } else {
            row = from.base + t;
        }
        sm_row[tid] = t;
        sm_field[tid] = field_of_scale((is_v ? a.from.v_scale : a.from.k_scale)[row >> a.from.log_block]);
        if (!is_v) {
            const int64_t x = (int64_t)stream * a.from.t_capacity + t, y = (int64_t)stream * a.to.t_capacity + t0 + tid;
            a.to.pos[y] = a.from.pos[x];
            if (a.to.weight) a.to.weight[y] = a.from.weight[x];
        }
    }
    __syncthreads();
    const uint8_t *src = is_v ? a.from.v_codes : a.from.k_codes;
    uint4 raw[kMost];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int p = tid + i * kMoveThreads;
        raw[i] = make_uint4(0, 0, 0, 0);
        if (p < n * kPerRow) {
            const int t = sm_row[p / kPerRow];
            const int64_t row = from.pages ? from.pos_in(min(max(from.pages[t >> from.shift], 0), from.n_pages - 1), t) : from.base + t;
            raw[i] = *reinterpret_cast<const uint4 *>(src + row * D + (p % kPerRow) * 16);
        }
    }
    // Magnitudes as binary32 bits with the scale's exponent added to theirs, which no exponent is too large or small for (a code may
    // stand for up to 2^128); the most negative integer stands for zero.
    int amax = INT32_MIN;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int p = tid + i * kMoveThreads;
        if (p >= n * kPerRow) continue;
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
        // e4m3 codes without their sign are ordered like what they stand for: the largest byte that is no NaN
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t b = (w[j] >> (8 * k)) & 0x7fu;
                bad |= b == 0x7fu;
                most = max(most, b == 0x7fu ? 0u : b);
            }
        if (most) amax = max(amax, __builtin_bit_cast(int, (float)codes_lo(most)[0]) + ((sm_field[p / kPerRow] - 127) << 23));
    }
    for (int o = 1; o < 64; o <<= 1) amax = max(amax, __shfl_xor(amax, o));
    const bool any_bad = __any(bad);
    if ((tid & 63) == 0) {
        sm_max[tid >> 6] = amax;
        sm_bad[tid >> 6] = any_bad;
    }
    __syncthreads();
    amax = max(max(sm_max[0], sm_max[1]), max(sm_max[2], sm_max[3]));
    const int flagged = sm_bad[0] | sm_bad[1] | sm_bad[2] | sm_bad[3];
    const int field = max((amax >> 23) - 8 + ((amax & 0x7fffff) > 0x600000 ? 1 : 0), 1);
    const int64_t row0 = a.to.map.of(stream).pos(t0);
    uint8_t *dst = (is_v ? a.to.v_codes : a.to.k_codes) + row0 * D;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int p = tid + i * kMoveThreads;
        if (p >= n * kPerRow) continue;
        const int shift = sm_field[p / kPerRow] - field;
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const half2v lo = codes_lo(w[j]), hi = codes_hi(w[j]);
            const float y[4] = {ldexpf((float)lo[0], shift), ldexpf((float)lo[1], shift), ldexpf((float)hi[0], shift), ldexpf((float)hi[1], shift)};
            o[j] = codes4(y, 1.f);
        }
        *reinterpret_cast<uint4 *>(dst + (int64_t)p * 16) = make_uint4(o[0], o[1], o[2], o[3]);
    }
    if (tid == 0)
        (is_v ? a.to.v_scale : a.to.k_scale)[row0 >> a.to.log_block] = __builtin_bit_cast(float, ((uint32_t)field << 23) | ((uint32_t)flagged << 31));
}

}  // namespace

hipError_t launch_fp8_evict(const Fp8EvictArgs &a, hipStream_t s)
{
    const int N = a.n_seq * a.from.n_kv_heads, B = 1 << a.from.log_block;
    fp8_select_kernel<<<N, kSelThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid(2 * (uint32_t)(((int64_t)a.budget + B - 1) / B), N);
    switch (a.d) {
    case 64: fp8_move_kernel<64><<<grid, kMoveThreads, 0, s>>>(a); break;
    case 96: fp8_move_kernel<96><<<grid, kMoveThreads, 0, s>>>(a); break;
    case 128: fp8_move_kernel<128><<<grid, kMoveThreads, 0, s>>>(a); break;
    default: fp8_move_kernel<256><<<grid, kMoveThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace pk
