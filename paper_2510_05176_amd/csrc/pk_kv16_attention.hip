// Attention of one token per sequence over the paged 16-bit cache.
//
// A wave takes 32 cached tokens of a sequence at a time against RT tiles of 16 query heads of the KV head.  S^T = K Q^T on the matrix cores: lane
// 16 g + n gets, for head n, tokens 4g .. 4g+3 of each tile of 16, which are the operand positions of the second product O^T = V^T P^T as
// they stand, so numerators go from one to the other in registers.  Rows of K and V are read as they lie; V's channels are dealt to the 16 rows of an
// operand tile so that a lane's bytes of a token are adjacent, and pairs of tokens are interleaved by byte permutes.  A tile of 16 tokens lies in one page
// (pages hold 16 or more).  All heads of the call see the same tokens of a sequence, so that what is masked for one of them is so for all, and
// V is cleared there before it reaches the product.
//
// HBM bounds it, 4 d bytes per token and KV head: 16 sequences x 32k tokens of 8 heads of 128 channels 354 us, 6.1 TB/s.  (The next tile asked for before this one is
// taken, with two workgroups per CU: 359 -> 357, and 15.0 -> 16.0 for one sequence of 1.1k tokens.)  Groups of rows over the same keys in one XCD's cache: 20 heads of 256 channels 52 -> 41 us.
#include <cfloat>

#include "pk_attention.h"
#include "pk_kv16.h"

namespace pk {

namespace {

constexpr int kTokens = 32;   // that a wave takes at a time

template <int D>
struct Part {
    static constexpr int kSteps = D / 32;   // of the contraction over channels
    static constexpr int kTiles = D / 16;   // of channels of the result
    static constexpr int kWords = D / 32;   // 32-bit words of a token's V per lane: a sixteenth of the row
};

template <int D>
__device__ __forceinline__ void load_values(uint32_t (&v)[Part<D>::kWords], const char *row, uint32_t off)
{
    if constexpr (D == 64) {
        const uint2 w = *reinterpret_cast<const uint2 *>(row + off);
        v[0] = w.x;
        v[1] = w.y;
    } else if constexpr (D == 96) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(row + off);
        v[0] = w[0];
        v[1] = w[1];
        v[2] = w[2];
    } else {
#pragma unroll
        for (int i = 0; i < D / 128; ++i) {
            const uint4 w = *reinterpret_cast<const uint4 *>(row + off + 16 * i);
            v[4 * i] = w.x;
            v[4 * i + 1] = w.y;
            v[4 * i + 2] = w.z;
            v[4 * i + 3] = w.w;
        }
    }
}

// Numerators as an operand.  (For bf16 a second term of what the first leaves would take its rounding out of the result, 2.1e-3 -> 1.7e-3 of it in the root mean
// square beside the 1.7e-3 of the result's own, but makes NaN of an infinite value that is seen.)
template <bool BF16>
__device__ __forceinline__ short8v numerators(const float (&p)[8])
{
    uint4 w;
    w.x = narrow(p[0], p[1], BF16);
    w.y = narrow(p[2], p[3], BF16);
    w.z = narrow(p[4], p[5], BF16);
    w.w = narrow(p[6], p[7], BF16);
    return __builtin_bit_cast(short8v, w);
}

template <int D, int RT, int NW, bool BF16, bool OPT>
__global__ __launch_bounds__(64 * NW, D == 256 && RT == 2 ? 1 : 2) void kv16_attention_kernel(Fp8AttentionArgs a)
{
    using S = Part<D>;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hkv = a.in.c.n_kv_heads, r = a.in.r;
    // Workgroups go to the eight XCDs in turn: heads next to each other, so that with eight of them every XCD has one head's keys in its cache, and the groups of
    // rows over the same keys eight apart.
    const int unit = blockIdx.x / (8 * a.groups) * 8 + (blockIdx.x & 7), group = (blockIdx.x >> 3) % a.groups;
    const int kvh = unit % hkv, run = unit / hkv, row0 = group * 16 * RT;
    if (run >= (a.parts > 0 ? a.parts : a.in.n_seq)) return;
    __shared__ int sm_end[kMostSeqs];
    Run deal = {run, 0, 0, 0, 0};
    if (a.parts > 0 && !find_run<true>(a.in, a.parts, run, sm_end, deal)) return;
    int seq = deal.seq, seq_from = deal.seq_from, seq_to = 0;
    for (;; seq_from = seq_to, ++seq) {   // the pieces of the run
        if (a.parts > 0) seq_to = __builtin_amdgcn_readfirstlane(sm_end[seq]);
        const bool whole = a.parts == 0 || (deal.at <= seq_from && seq_to <= deal.stop);   // the sequence is this piece
        const Place p = place_of<true>(a.in, seq * hkv + kvh);
        const int64_t part0 = ((int64_t)(run + seq) * hkv + kvh) * r;   // where partial results of the rows go
        // the tokens that are seen, and of them this piece's
        const int seen = a.in.window > 0 ? max(p.len - a.in.window, 0) : 0;
        int lo = seen & ~63, hi = p.len;
        if (!whole) {
            const int from = lo;
            lo = (int)min(from + (int64_t)(max(deal.at, seq_from) - seq_from) * 64, (int64_t)hi);
            hi = (int)min(from + (int64_t)(min(deal.stop, seq_to) - seq_from) * 64, (int64_t)hi);
        }

        short8v q[RT][S::kSteps];
        float slope[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int at = row0 + 16 * rt + n, head = kvh * r + min(at, r - 1);
            const char *from = static_cast<const char *>(a.in.q) + 2 * (seq * a.in.qs.seq + head * a.in.qs.head + 8 * g);
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                uint4 w = make_uint4(0, 0, 0, 0);
                if (at < r) w = *reinterpret_cast<const uint4 *>(from + 64 * s);
                if (a.in.scale < 0.f) w = make_uint4(w.x ^ 0x80008000u, w.y ^ 0x80008000u, w.z ^ 0x80008000u, w.w ^ 0x80008000u);
                q[rt][s] = __builtin_bit_cast(short8v, w);
            }
            slope[rt] = OPT && a.in.slopes && at < r ? a.in.slopes[head] * kLog2e : 0.f;
        }
        // the products' factor; never 0, so that a masked -inf stays one
        const float c = fmaxf(fabsf(a.in.scale) * kLog2e, 0x1p-126f);

        float m[RT], l[RT];   // the numerators' reference, their sum
        float4v o[RT][S::kTiles];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY;
            l[rt] = 0.f;
#pragma unroll
            for (int ct = 0; ct < S::kTiles; ++ct) o[rt][ct] = float4v{0.f, 0.f, 0.f, 0.f};
        }
        float most[RT];   // the largest score that the reference serves
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) most[rt] = -INFINITY;

        const StreamMap map = a.in.c.map.of(p.stream);
        const uint32_t k_off = 2 * (n * D + 8 * g), v_off = 2 * (4 * g * D + n * (D / 16));
        for (int t0 = lo + kTokens * wave; t0 < hi; t0 += kTokens * NW) {
            short8v k[2][S::kSteps];
            uint32_t v[8][S::kWords];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t at = map.pos(t0 + 16 * j) * (2 * D);
                const char *kp = reinterpret_cast<const char *>(a.in.c.k_codes) + at, *vp = reinterpret_cast<const char *>(a.in.c.v_codes) + at;
#pragma unroll
                for (int s = 0; s < S::kSteps; ++s) k[j][s] = *reinterpret_cast<const short8v *>(kp + k_off + 64 * s);
#pragma unroll
                for (int i = 0; i < 4; ++i) load_values<D>(v[4 * j + i], vp + 2 * i * D, v_off);
            }
            const bool edge = t0 < seen || t0 + kTokens > hi;
            float4v s[RT][2];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s[rt][j] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < S::kSteps; ++i) s[rt][j] = mfma16<BF16>(k[j][i], q[rt][i], s[rt][j]);
                }
            short8v pf[RT];
            float by[RT];
            bool moved = false;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float x[8], f = c;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = s[rt][i >> 2][i & 3];
                if constexpr (OPT) {
                    if (a.in.cap > 0.f) {
                        const float inv[1] = {fminf(fabsf(a.in.scale) / a.in.cap, FLT_MAX)};
                        capped(x, inv, a.in.cap * kLog2e);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] *= c;
                    }
                    if (a.in.slopes) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = fmaf(-slope[rt], (float)(p.len - 1 - (t0 + 16 * (i >> 2) + 4 * g + (i & 3))), x[i]);
                    }
                    f = 1.f;
                }
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int t = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
                        x[i] = t >= seen && t < hi ? x[i] : -INFINITY;
                    }
                }
                float top = x[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
                const float one[1] = {top * f};
                top = fold_rows(one, MaxF());
                by[rt] = 1.f;
                if (top > most[rt]) {
                    const float was = most[rt];
                    most[rt] = fabsf(top) < 0x1p20f ? top + kRoom : top;
                    const float to = reference_of<BF16>(top);
                    by[rt] = change_of<BF16>(m[rt], to, was, most[rt]);
                    m[rt] = to;
                    l[rt] *= by[rt];
                }
                moved |= by[rt] != 1.f;
                const float ref = m[rt] == -INFINITY ? 0.f : m[rt];
                float e[8], sum = 0.f;
                if (__any(fabsf(ref) >= kLarge)) {
                    // (see kLarge)
                    const float under = under_of<BF16>(most[rt]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] *= f;
                        asm volatile("" : "+v"(x[i]));   // (not contracted)
                        e[i] = exp2_((x[i] - ref) - under);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = exp2_(fmaf(x[i], f, -ref));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += e[i];
                l[rt] += sum;
                pf[rt] = numerators<BF16>(e);
            }
            if (__any(moved)) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int ct = 0; ct < S::kTiles; ++ct) o[rt][ct] *= by[rt];
            }
            if (edge) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int t = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
                    if (t < seen || t >= hi)
#pragma unroll
                        for (int w = 0; w < S::kWords; ++w) v[i][w] = 0;
                }
            }
#pragma unroll
            for (int w = 0; w < S::kWords; ++w)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint4 f;   // channel 2w + e of the lane's 8 tokens
                    const uint32_t pick = e ? 0x07060302u : 0x05040100u;
                    f.x = __builtin_amdgcn_perm(v[1][w], v[0][w], pick);
                    f.y = __builtin_amdgcn_perm(v[3][w], v[2][w], pick);
                    f.z = __builtin_amdgcn_perm(v[5][w], v[4][w], pick);
                    f.w = __builtin_amdgcn_perm(v[7][w], v[6][w], pick);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) o[rt][2 * w + e] = mfma16<BF16>(__builtin_bit_cast(short8v, f), pf[rt], o[rt][2 * w + e]);
                }
        }

        // results of the wave, normalised, then the waves' together
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float one[1] = {l[rt]};
            l[rt] = fold_rows(one, AddF());
            const float inv = l[rt] == 0.f ? 0.f : 1.f / l[rt];
#pragma unroll
            for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rt][ct][i] = mean_of<BF16>(o[rt][ct][i] * inv);
            l[rt] *= exp2_(under_of<BF16>(most[rt]));   // in units of 2^m, for the other waves and pieces
        }
        constexpr int kAtOnce = (D == 256 ? 8 : 16) * 4 / NW, kPad = 4;   // rows at a time: 32 to 34 KB of LDS
        __shared__ float sm_o[NW][kAtOnce][D + kPad];
        __shared__ float sm_m[NW][kAtOnce], sm_l[NW][kAtOnce];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int part = 0; part < 16 / kAtOnce; ++part) {
                const int from = row0 + 16 * rt + part * kAtOnce, here = min(r - from, kAtOnce);
                if (here <= 0) break;
                __syncthreads();   // the last rows' places are free
                if (n / kAtOnce == part) {
                    const int q_at = n % kAtOnce;
                    if (g == 0) {
                        sm_m[wave][q_at] = m[rt];
                        sm_l[wave][q_at] = l[rt];
                    }
#pragma unroll
                    for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sm_o[wave][q_at][(4 * g + i) * (D / 16) + ct] = o[rt][ct][i];
                }
                __syncthreads();
                for (int e = threadIdx.x; e < here * (D / 4); e += 64 * NW) {
                    const int q_at = e / (D / 4), ch = (e % (D / 4)) * 4, at = from + q_at;
                    float top = -INFINITY;
                    for (int w = 0; w < NW; ++w) top = fmaxf(top, sm_m[w][q_at]);
                    const float ref = top == -INFINITY ? 0.f : top;
                    float sum = 0.f, share[NW], y[4] = {0.f, 0.f, 0.f, 0.f};
                    for (int w = 0; w < NW; ++w) {
                        share[w] = sm_l[w][q_at] * exp2_(sm_m[w][q_at] - ref);
                        sum += share[w];
                    }
                    // shares of 1: a sum of many results near a binary32's largest need not be one, though their mean is
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    for (int w = 0; w < NW; ++w)
                        if (sm_l[w][q_at] != 0.f)
                            for (int i = 0; i < 4; ++i) y[i] = fmaf(share[w] * inv, sm_o[w][q_at][ch + i], y[i]);
                    if (whole) {
                        store_row<D>(a, p, at, ch, y, 4);
                        if (ch == 0) store_lse(a, p, at, top, sum);
                    } else {
                        const int64_t slot = part0 + at;
                        *reinterpret_cast<float4 *>(a.part_o + slot * D + ch) = make_float4(y[0], y[1], y[2], y[3]);
                        if (ch == 0) {
                            a.part_ml[2 * slot] = top;
                            a.part_ml[2 * slot + 1] = sum;
                        }
                    }
                }
            }
        if (a.parts == 0 || seq_to >= deal.stop) break;
    }
}

// 16 query heads per tile, two tiles share what is read.  With 256 channels they take a SIMD's registers for one wave, which pays over many tokens (16 sequences of
// 16k tokens, two KV heads of 32 heads each, 131 -> 114 us; of 10k tokens and 33 heads 152 -> 102; 32 of up to 20k, 20 heads, 113 -> 90; 256k tokens of all KV heads
// 61.5 and 59.7, one sequence of 128k and two KV heads 64.4 and 66.1; but 160k with a window 39.9 -> 44.7, 4000 tokens 18 -> 24).  The tokens are the bound's, the window or not: two KV heads of 24 over
// 4000 tokens in a cache of 2^18 take 21.7 us with the capacity as the bound, 17.8 with 4000.
int tiles_of(int64_t r, int d, int64_t tokens) { return r <= 16 || (d == 256 && tokens <= kOneTileTokens) ? 1 : 2; }

template <int D, int RT, bool BF16>
void launch_rt(const Fp8AttentionArgs &a, uint32_t grid, bool opt, hipStream_t s)
{
    if (opt) kv16_attention_kernel<D, RT, 4, BF16, true><<<grid, 256, 0, s>>>(a);
    else kv16_attention_kernel<D, RT, 4, BF16, false><<<grid, 256, 0, s>>>(a);
}

template <int D>
hipError_t launch_d(Fp8AttentionArgs &a, hipStream_t s)
{
    const int tiles = tiles_of(a.in.r, D, (int64_t)a.in.n_seq * a.in.c.n_kv_heads * a.bound);
    a.groups = (a.in.r + 16 * tiles - 1) / (16 * tiles);
    const uint32_t units = (uint32_t)((a.parts > 0 ? a.parts : a.in.n_seq) * a.in.c.n_kv_heads), grid = (units + 7) / 8 * 8 * a.groups;
    const bool opt = a.in.cap > 0.f || a.in.slopes;
    if (tiles == 1) {
        if (a.in.bf16) launch_rt<D, 1, true>(a, grid, opt, s);
        else launch_rt<D, 1, false>(a, grid, opt, s);
    } else {
        if (a.in.bf16) launch_rt<D, 2, true>(a, grid, opt, s);
        else launch_rt<D, 2, false>(a, grid, opt, s);
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.parts == 0 ? e : launch_attention_merge(a, s);
}

}  // namespace

// Runs for one workgroup per CU where a run stays in one or two sequences (16 sequences x 32k tokens 354 us, 361 with two workgroups per CU; one of 32k 31 and 35, of
// 128k 103 and 107), for two where it goes through more, each with its end (64 sequences of up to 6000 tokens 130 and 121; of up to 2000 56 and 53).  Three and four
// per CU: 364 and 362, 122 and 126.  (Short caches whole by eight waves, with nothing to merge: 22.5 us for 2k tokens of 8 heads where runs of 256 take 14.7.)
// From four sequences to a run on, and beyond kMostSeqs, a workgroup has a sequence of a KV head whatever its length (256 sequences of 8 KV heads, 128 of 16, 64 of 32): lengths of 1 to
// 6000 make little of it (300 sequences of 8 KV heads 657 us, their bytes 630), but one of 32k tokens among 255 of 500 takes 515 us, among 199, which are dealt, 111.
int64_t kv16_attention_parts(int64_t n_seq, int64_t n_kv_heads, int64_t r, int d, int64_t bound)
{
    const int64_t rows = 16 * tiles_of(r, d, n_seq * n_kv_heads * bound), across = n_kv_heads * ((r + rows - 1) / rows);   // workgroups per run
    int64_t parts = (256 / across >= n_seq ? 256 : 512) / across;
    if (parts < 1) parts = 1;
    if (n_seq > kMostSeqs || n_seq >= 4 * parts) return 0;
    const int64_t most = n_seq * ((bound + 64 * kLeastUnits - 1) / (64 * kLeastUnits));
    if (parts > most) parts = most;
    return parts <= 1 && n_seq == 1 ? 0 : parts;
}

hipError_t launch_kv16_attention(Fp8AttentionArgs &a, hipStream_t s)
{
    return a.in.d == 64 ? launch_d<64>(a, s) : a.in.d == 96 ? launch_d<96>(a, s) : a.in.d == 128 ? launch_d<128>(a, s) : launch_d<256>(a, s);
}

}  // namespace pk
