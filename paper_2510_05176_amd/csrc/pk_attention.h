// What the attention kernels share: the exponential and the scores' cap, a sequence's place, how a call's keys are dealt out to workgroups, rows of
// the result.
#pragma once

#include "pk_fp8.h"

namespace pk {

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// x[i] = m * tanh(x[i] * c[i / 8]) in binary32.  Below 0.55 the odd Taylor series, above it 1 - 2 / (e^{2y} + 1), whose rounding is no longer
// magnified there; how far the series goes, and whether the other form is computed at all, is the wave's largest argument's to say (the first term
// left out is 2e-10 of the result at 0.25 and 4e-8 at 0.55).  tanh y = y + y^3 s(y^2), s from 2^(2k) (2^(2k) - 1) B_2k / (2k)!.
// APART: the two forms in loops of their own, without a branch per score, where registers allow (prompts of 8k tokens with cap and distance bias 933 -> 886 us).
template <int N, bool APART = false>
__device__ __forceinline__ void capped(float (&x)[N], const float (&c)[N / 8], float m)
{
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(x[i]) * c[i >> 3]);   // (a NaN does not count and comes out of the series as one)
    if (!__any(most >= 0.25f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = x[i] * c[i >> 3], y2 = y * y;
            float s = fmaf(-1382.f / 155925.f, y2, 62.f / 2835.f);
            s = fmaf(s, y2, -17.f / 315.f);
            s = fmaf(s, y2, 2.f / 15.f);
            s = fmaf(s, y2, -1.f / 3.f);
            const float ym = y * m;
            x[i] = fmaf(s * y2, ym, ym);
        }
        return;
    }
    const bool far = __any(most >= 0.55f);
    const auto one = [&](int i, bool both) {
        const float y = x[i] * c[i >> 3], y2 = y * y;
        float s = fmaf(-929569.f / 638512875.f, y2, 21844.f / 6081075.f);
        s = fmaf(s, y2, -1382.f / 155925.f);
        s = fmaf(s, y2, 62.f / 2835.f);
        s = fmaf(s, y2, -17.f / 315.f);
        s = fmaf(s, y2, 2.f / 15.f);
        s = fmaf(s, y2, -1.f / 3.f);
        float t = fmaf(s * y2, y, y);
        if (both) {
            const float a = fabsf(y), e = exp2_(fminf(a, 16.f) * (2.f * kLog2e));
            const float big = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), y);
            t = a >= 0.55f ? big : t;
        }
        x[i] = t * m;
    };
    if (APART && far) {
#pragma unroll
        for (int i = 0; i < N; ++i) one(i, true);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) one(i, APART ? false : far);
    }
}

// The same value for all lanes, through the scalar path; nothing writes it while the kernel runs
__device__ __forceinline__ float scalar_load(const float *p) { return *(const __attribute__((address_space(4))) float *)(uintptr_t)p; }

// Where a workgroup's rows and keys are
struct Place {
    int stream, seq, kvh, len, next, count;
};
// ONE: all lanes of the wave ask for the same stream
template <bool ONE>
__device__ __forceinline__ Place place_of(const Fp8Queries &a, int stream)
{
    Place p;
    p.stream = stream;
    p.seq = stream / a.c.n_kv_heads;
    p.kvh = stream - p.seq * a.c.n_kv_heads;
    const int2 st = fp8_state(a.states, p.seq, a.c.t_capacity);
    const int count = fp8_count(a.counts, p.seq, a.n_query);
    p.len = ONE ? __builtin_amdgcn_readfirstlane(st.x) : st.x;
    p.next = ONE ? __builtin_amdgcn_readfirstlane(st.y) : st.y;
    p.count = ONE ? __builtin_amdgcn_readfirstlane(count) : count;
    return p;
}

// How the keys of a call are dealt out: the units of 64 visible tokens of all sequences (one at least of each), laid end to end, in
// `parts` runs of equal length (at least kLeastUnits), whatever the lengths of the sequences.  A run is one workgroup's; where it crosses
// from one sequence into the next it goes on with that.  The piece of sequence b in run i has slot i + b: they grow from piece to
// piece, so no two are alike and n_seq + parts are enough.  parts == 0: a workgroup per sequence.
constexpr int kMostSeqs = 256, kLeastUnits = 4;
__device__ __forceinline__ int first_visible(const Fp8Queries &a, int len, int count)   // a multiple of 64
{
    return a.window > 0 ? (int)min(max((int64_t)len - count + 1 - a.window, (int64_t)0), (int64_t)len) & ~63 : 0;
}
// Ends of the sequences' units (of the visible tokens, or of all), lane's sequences 64 i + lane; returns all of them.
template <bool VISIBLE>
__device__ __forceinline__ int ends_of(const Fp8Queries &a, int (&end)[kMostSeqs / 64])
{
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int i = 0; i < kMostSeqs / 64; ++i) {
        end[i] = 0;
        if (64 * i >= a.n_seq) continue;
        const int seq = 64 * i + lane;
        int units = 0;
        if (seq < a.n_seq) {
            const int len = fp8_state(a.states, seq, a.c.t_capacity).x;
            if constexpr (VISIBLE) {
                const int count = fp8_count(a.counts, seq, a.n_query);
                units = count > 0 ? max((len - first_visible(a, len, count) + 63) >> 6, 1) : 1;
            } else {
                units = max((len + 63) >> 6, 1);
            }
        }
        for (int o = 1; o < min(a.n_seq, 64); o <<= 1) {
            const int v = __shfl_up(units, o);
            if (lane >= o) units += v;
        }
        end[i] = units + before;
        before = __shfl(end[i], min(a.n_seq - 1 - 64 * i, 63));
    }
    return before;
}
__device__ __forceinline__ int run_length(int all, int parts) { return max((all + parts - 1) / parts, kLeastUnits); }

struct Run {
    int seq, seq_from;   // the sequence that the run begins in, and where its units begin
    int at, stop;        // the run's units
    int per;
};
// All waves of the workgroup; false: the run has nothing.  sm_end: kMostSeqs ends for the workgroup.
template <bool VISIBLE>
__device__ __forceinline__ bool find_run(const Fp8Queries &a, int parts, int run, int *sm_end, Run &r)
{
    const int lane = threadIdx.x & 63;
    int end[kMostSeqs / 64];
    const int all = __builtin_amdgcn_readfirstlane(ends_of<VISIBLE>(a, end));
    r.per = run_length(all, parts);
    r.at = run * r.per;
    r.stop = min(r.at + r.per, all);
    if (r.at >= r.stop) return false;
#pragma unroll
    for (int i = kMostSeqs / 64 - 1; i >= 0; --i) {
        if (64 * i + lane < a.n_seq && threadIdx.x < 64) sm_end[64 * i + lane] = end[i];
        const uint64_t behind = __ballot(64 * i + lane < a.n_seq && end[i] > r.at);
        if (behind) r.seq = 64 * i + __ffsll((unsigned long long)behind) - 1;
    }
    __syncthreads();
    r.seq_from = r.seq > 0 ? __builtin_amdgcn_readfirstlane(sm_end[r.seq - 1]) : 0;
    return true;
}

template <int D>
__device__ __forceinline__ void store_row(const Fp8AttentionArgs &a, const Place &p, int row, int c, const float *x, int n)
{
    const int i = row / a.in.r, h = row - i * a.in.r;
    uint32_t *o = reinterpret_cast<uint32_t *>(static_cast<char *>(a.out) + 2 * (p.seq * a.os.seq + i * a.os.token + (int64_t)(p.kvh * a.in.r + h) * a.os.head + c));
    for (int e = 0; e < n; e += 2) o[e / 2] = narrow(x[e], x[e + 1], a.in.bf16);
}
__device__ __forceinline__ void store_lse(const Fp8AttentionArgs &a, const Place &p, int row, float m, float l)
{
    if (!a.lse) return;
    const int i = row / a.in.r, h = row - i * a.in.r;
    // l's power of two joins the reference first: their sum is small where the log-sum-exp is, and takes no rounding of l's whole logarithm
    int e;
    const float part = frexpf(l, &e);
    a.lse[((int64_t)p.seq * a.in.c.n_kv_heads * a.in.r + p.kvh * a.in.r + h) * a.in.n_query + i] = l == 0.f ? -INFINITY : (m + (float)e + log2f(part)) * kLn2;
}

}  // namespace

}  // namespace pk
