// Eviction from the 8-bit cache, in two launches: which tokens stay (one workgroup per stream, into the workspace), and their
// move into the other cache (one workgroup per new block of a stream, K and V).
//
// Weights are chosen among as integers in the same order: the weight of the last token that stays, then which tokens are above it, and of
// the equal ones the first, so that the order is kept and ties go to the earlier ones.
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

// What both selections write besides: the tokens that are kept whatever their weight
__device__ __forceinline__ void keep_ends(const Fp8EvictArgs &a, int32_t *kept, int hi)
{
    for (int i = threadIdx.x; i < a.keep_first; i += blockDim.x) kept[i] = i;
    for (int i = threadIdx.x; i < a.keep_last; i += blockDim.x) kept[a.budget - a.keep_last + i] = hi + i;
}

// Up to 4 K tokens per thread, their weights in registers (four neighbours at a time: token 4 (threads i + thread) + j): the largest integer that
// at least `need` of them reach, bit by bit from the top; a pass is 4 K comparisons, a sum over the workgroup and one barrier.  Once at most
// kRanked are left between what is kept for certain and what is not, they go to LDS and are ranked against each other; it ends earlier where
// exactly `need` reach a bound.  (256 streams of 16k tokens to 1024: 33 us with the histograms below, 18.6 with this; 19.8 with eight waves, 27 with
// four, which do not cover each other's latencies.)
constexpr int kRegThreads = 1024, kRegWaves = kRegThreads / 64, kRanked = 64;

// set bits of the mask below the lane
__device__ __forceinline__ uint32_t below_lane(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

template <int K>
__global__ __launch_bounds__(kRegThreads) void fp8_select_kernel(Fp8EvictArgs a)
{
    __shared__ float sm_count[2][kRegWaves];
    __shared__ uint32_t sm_above[K * kRegWaves], sm_equal[K * kRegWaves];   // of four neighbours of a wave
    __shared__ uint32_t sm_left[kRanked], sm_n_left, sm_floor, sm_ties, sm_all_above;
    const int stream = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int len = __builtin_amdgcn_readfirstlane(fp8_state(a.states, stream / a.from.n_kv_heads, a.from.t_capacity).x);
    if (len <= a.budget) return;   // the move takes such a sequence whole
    int32_t *kept = a.kept + (int64_t)stream * a.budget;
    const int lo = a.keep_first, hi = len - a.keep_last;   // candidates; more of them than the budget has room for
    const float *w = a.from.weight + (int64_t)stream * a.from.t_capacity;
    uint32_t need = (uint32_t)(a.budget - a.keep_first - a.keep_last);
    // All loads on their way before the first is looked at (left to itself the compiler puts each into a branch with a wait of its own).
    // 0: no candidate, or a NaN; the capacity is a multiple of 64.
    uint32_t u[4 * K];
    {
        float4 x[K];
#pragma unroll
        for (int i = 0; i < K; ++i) x[i] = *reinterpret_cast<const float4 *>(w + min(4 * (i * kRegThreads + tid), a.from.t_capacity - 4));
#pragma unroll
        for (int i = 0; i < K; ++i) asm volatile("" : "+v"(x[i].x), "+v"(x[i].y), "+v"(x[i].z), "+v"(x[i].w));
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const float y[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = 4 * (i * kRegThreads + tid) + j;
                u[4 * i + j] = t >= lo && t < hi ? order_of(y[j]) : 0;
            }
        }
    }
    if (tid == 0) sm_n_left = 0;
    keep_ends(a, kept, hi);
    if (need == 0) return;
    uint32_t floor = 0;   // kept: above it, and the first of those equal to it
    uint32_t n_floor = hi - lo, n_certain = 0;   // that reach the floor; that reach the lowest bound found too high
    bool exact = false, ranked = false;   // exact: all that reach the floor are kept
    for (int bit = 31; bit >= 0 && !exact && !ranked; --bit) {
        const uint32_t to = floor | (1u << bit);
        uint32_t some[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4 * K; ++i) some[i & 3] += u[i] >= to;
        const float of_row[1] = {row_sum((float)(some[0] + some[1] + some[2] + some[3]))};   // (whole numbers below 2^24)
        const float of_wave = fold_rows(of_row, AddF());
        if (lane == 0) sm_count[bit & 1][wave] = of_wave;
        __syncthreads();   // (the other half is free: every wave is past the pass that read it)
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kRegWaves; ++i) sum += sm_count[bit & 1][i];
        const uint32_t all = __builtin_amdgcn_readfirstlane((uint32_t)sum);
        if (all >= need) {
            floor = to;
            n_floor = all;
        } else {
            n_certain = all;
        }
        exact = all == need;
        ranked = !exact && floor > 0 && bit > 0 && n_floor - n_certain <= kRanked;
        if (ranked) {
            // those in [floor, floor + 2^bit)
            const uint32_t span = 1u << bit;
#pragma unroll
            for (int i = 0; i < 4 * K; ++i)
                if (u[i] - floor < span) sm_left[atomicAdd(&sm_n_left, 1u)] = u[i];
            __syncthreads();
            const int n_left = n_floor - n_certain;
            const uint32_t wanted = need - n_certain;
            if (wave == 0) {
                const uint32_t v = sm_left[lane];
                uint32_t over = 0, same = 0;
                for (int i = 0; i < n_left; ++i) {   // (lanes past them have whatever is there)
                    const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)v, i);
                    over += other > v;
                    same += other == v;
                }
                if (lane < n_left && over < wanted && wanted <= over + same) {   // whoever has this value writes the same
                    sm_floor = v;
                    sm_ties = over + same != wanted;
                }
            }
            __syncthreads();
            floor = __builtin_amdgcn_readfirstlane(sm_floor);
            exact = __builtin_amdgcn_readfirstlane(sm_ties) == 0;
        }
    }
    // Places in the order of the tokens: how many of every four neighbours of a wave are above (with `exact`: reach the floor) or equal, sums of
    // these, then the lanes' own.
    const uint32_t above_at = exact ? floor : floor + 1;   // (a floor of 0xffffffff would be a NaN's, which is 0)
    const auto is_equal = [&](int i) {
        const int t = 4 * ((i >> 2) * kRegThreads + tid) + (i & 3);
        return u[i] == floor && t >= lo && t < hi;
    };
#pragma unroll
    for (int i = 0; i < K; ++i) {
        uint32_t n = 0, m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) n += __popcll(__ballot(u[4 * i + j] >= above_at));
        if (!exact)
#pragma unroll
            for (int j = 0; j < 4; ++j) m += __popcll(__ballot(is_equal(4 * i + j)));
        if (lane == 0) {
            sm_above[i * kRegWaves + wave] = n;
            sm_equal[i * kRegWaves + wave] = m;
        }
    }
    __syncthreads();
    if (wave == 0) {   // exclusive sums; K * kRegWaves are 16, 64 or 128 of them
        constexpr int kAll = K * kRegWaves, kPer = (kAll + 63) / 64;
        uint32_t x[kPer], y[kPer], sx = 0, sy = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            x[i] = sx;
            y[i] = sy;
            if (lane * kPer + i < kAll) {
                sx += sm_above[lane * kPer + i];
                sy += sm_equal[lane * kPer + i];
            }
        }
        uint32_t ex = sx, ey = sy;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t vx = __shfl_up(ex, o), vy = __shfl_up(ey, o);
            if (lane >= o) {
                ex += vx;
                ey += vy;
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (lane * kPer + i < kAll) {
                sm_above[lane * kPer + i] = ex - sx + x[i];
                sm_equal[lane * kPer + i] = ey - sy + y[i];
            }
        if (lane == 63) sm_all_above = ex;
    }
    __syncthreads();
    need -= sm_all_above;   // of the equal ones
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const int t = 4 * (i * kRegThreads + tid);
        uint32_t n = sm_above[i * kRegWaves + wave];
#pragma unroll
        for (int j = 0; j < 4; ++j) n += below_lane(__ballot(u[4 * i + j] >= above_at));
        if (exact) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (u[4 * i + j] >= above_at) kept[lo + n++] = t + j;
        } else {
            uint32_t m = sm_equal[i * kRegWaves + wave];
#pragma unroll
            for (int j = 0; j < 4; ++j) m += below_lane(__ballot(is_equal(4 * i + j)));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool gt = u[4 * i + j] >= above_at, eq = is_equal(4 * i + j);
                if (gt || (eq && m < need)) kept[lo + n + min(m, need)] = t + j;
                n += gt;
                m += eq;
            }
        }
    }
}

// Any number of candidates: three histograms of 11, 11 and 10 bits over the memory (or its caches), then every wave's own run of tokens.
__global__ __launch_bounds__(kSelThreads) void fp8_select_long_kernel(Fp8EvictArgs a)
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
    keep_ends(a, kept, hi);
}

constexpr int kMoveThreads = 256;

// Magnitudes as binary32 bits with the scale's exponent added to theirs, which no exponent is too large or small for (a code may
// stand for up to 2^128); the most negative integer stands for zero.
__device__ __forceinline__ int size_of_codes(const uint4 &v, int field, bool &bad)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
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
    return most ? __builtin_bit_cast(int, (float)codes_lo(most)[0]) + ((field - 127) << 23) : INT32_MIN;
}
__device__ __forceinline__ uint4 rescaled(const uint4 &v, int shift)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const half2v lo = codes_lo(w[j]), hi = codes_hi(w[j]);
        const float y[4] = {ldexpf((float)lo[0], shift), ldexpf((float)lo[1], shift), ldexpf((float)hi[0], shift), ldexpf((float)hi[1], shift)};
        o[j] = codes4(y, 1.f);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// K and V of a block together: where their tokens are is looked up once, and twice as much is on its way (of 256 streams of 1024 tokens
// kept 38.5 us with a workgroup each, 33 with this).
template <int D, int B>
__global__ __launch_bounds__(kMoveThreads) void fp8_move_kernel(Fp8EvictArgs a)
{
    constexpr int kPerRow = D / 16;                                              // pieces of 16 codes
    constexpr int kMost = (B * kPerRow + kMoveThreads - 1) / kMoveThreads;       // per thread
    __shared__ int sm_max[2][kMoveThreads / 64], sm_bad[2][kMoveThreads / 64], sm_field[2][B];
    __shared__ int64_t sm_row[B];
    const int tid = threadIdx.x, hkv = a.from.n_kv_heads;
    const int stream = blockIdx.y, seq = stream / hkv;
    const int2 st = fp8_state(a.states, seq, a.from.t_capacity);
    const int held = min(st.x, a.budget), t0 = (int)blockIdx.x * B, n = min(held - t0, B);
    if (tid == 0 && stream % hkv == 0 && blockIdx.x == 0) *reinterpret_cast<int4 *>(a.to_states + 4 * (int64_t)seq) = make_int4(held, st.y, 0, 0);
    if (n <= 0) return;
    const StreamMap from = a.from.map.of(stream);
    if (tid < n) {
        // an index is one that the selection wrote, below the sequence's length; whatever the workspace holds, it leads nowhere else
        const int t = st.x <= a.budget ? t0 + tid : min(max(a.kept[(int64_t)stream * a.budget + t0 + tid], 0), a.from.t_capacity - 1);
        const int page = from.pages ? min(max(from.pages[t >> from.shift], 0), from.n_pages - 1) : 0;
        const int64_t row = from.pos_in(page, t);
        sm_row[tid] = row;
        sm_field[0][tid] = field_of_scale(a.from.k_scale[row >> a.from.log_block]);
        sm_field[1][tid] = field_of_scale(a.from.v_scale[row >> a.from.log_block]);
        const int64_t x = (int64_t)stream * a.from.t_capacity + t, y = (int64_t)stream * a.to.t_capacity + t0 + tid;
        a.to.pos[y] = a.from.pos[x];
        if (a.to.weight) a.to.weight[y] = a.from.weight[x];
    }
    __syncthreads();
    uint4 raw[2][kMost];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int p = tid + i * kMoveThreads;
        raw[0][i] = raw[1][i] = make_uint4(0, 0, 0, 0);
        if (p < n * kPerRow) {
            const int64_t at = sm_row[p / kPerRow] * D + (p % kPerRow) * 16;
            raw[0][i] = *reinterpret_cast<const uint4 *>(a.from.k_codes + at);
            raw[1][i] = *reinterpret_cast<const uint4 *>(a.from.v_codes + at);
        }
    }
    int most[2] = {INT32_MIN, INT32_MIN};
    bool bad[2] = {false, false};
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int token = min((tid + i * kMoveThreads) / kPerRow, n - 1);   // (past the block: zeros, which do not count)
#pragma unroll
        for (int s = 0; s < 2; ++s) most[s] = max(most[s], size_of_codes(raw[s][i], sm_field[s][token], bad[s]));
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        for (int o = 1; o < 64; o <<= 1) most[s] = max(most[s], __shfl_xor(most[s], o));
        const bool any = __any(bad[s]);
        if ((tid & 63) == 0) {
            sm_max[s][tid >> 6] = most[s];
            sm_bad[s][tid >> 6] = any;
        }
    }
    __syncthreads();
    const int64_t row0 = a.to.map.of(stream).pos(t0);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int size = max(max(sm_max[s][0], sm_max[s][1]), max(sm_max[s][2], sm_max[s][3]));
        const int flagged = sm_bad[s][0] | sm_bad[s][1] | sm_bad[s][2] | sm_bad[s][3];
        const int field = max((size >> 23) - 8 + ((size & 0x7fffff) > 0x600000 ? 1 : 0), 1);
        uint8_t *dst = (s ? a.to.v_codes : a.to.k_codes) + row0 * D;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const int p = tid + i * kMoveThreads;
            if (p < n * kPerRow) *reinterpret_cast<uint4 *>(dst + (int64_t)p * 16) = rescaled(raw[s][i], sm_field[s][p / kPerRow] - field);
        }
        if (tid == 0)
            (s ? a.to.v_scale : a.to.k_scale)[row0 >> a.to.log_block] = __builtin_bit_cast(float, ((uint32_t)field << 23) | ((uint32_t)flagged << 31));
    }
}

template <int D>
void launch_move(const Fp8EvictArgs &a, const dim3 &grid, hipStream_t s)
{
    if (a.from.log_block == 5) fp8_move_kernel<D, 32><<<grid, kMoveThreads, 0, s>>>(a);
    else if (a.from.log_block == 6) fp8_move_kernel<D, 64><<<grid, kMoveThreads, 0, s>>>(a);
    else fp8_move_kernel<D, 128><<<grid, kMoveThreads, 0, s>>>(a);
}

}  // namespace

hipError_t launch_fp8_evict(const Fp8EvictArgs &a, hipStream_t s)
{
    const int N = a.n_seq * a.from.n_kv_heads, B = 1 << a.from.log_block;
    // what a sequence can have to choose from, by the cache's capacity
    const int64_t most = (int64_t)a.from.t_capacity - a.keep_last;
    if (a.budget < a.from.t_capacity) {
        if (most <= 4096) fp8_select_kernel<1024 / kRegThreads><<<N, kRegThreads, 0, s>>>(a);
        else if (most <= 16384) fp8_select_kernel<4096 / kRegThreads><<<N, kRegThreads, 0, s>>>(a);
        else if (most <= 32768) fp8_select_kernel<8192 / kRegThreads><<<N, kRegThreads, 0, s>>>(a);
        else fp8_select_long_kernel<<<N, kSelThreads, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // no sequence holds more than the capacity: blocks beyond it have nothing
    const int64_t kept = a.budget < a.from.t_capacity ? a.budget : a.from.t_capacity;
    const dim3 grid((uint32_t)((kept + B - 1) / B), N);
    switch (a.d) {
    case 64: launch_move<64>(a, grid, s); break;
    case 96: launch_move<96>(a, grid, s); break;
    case 128: launch_move<128>(a, grid, s); break;
    default: launch_move<256>(a, grid, s);
    }
    return hipGetLastError();
}

}  // namespace pk
