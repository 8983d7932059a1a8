// Causal attention of whole prompts, packed one after the other.
//
// The rows of a KV head are its query heads' tokens, row = token * r + head of the group, so that what a workgroup loads of K and V serves all heads,
// and a tile of rows spans few tokens.  A wave has 32 rows.  S^T = K Q^T, 32 keys at a time, on v_mfma_f32_32x32x16: lane 32 h + n gets, for row n, keys 8i + 4h .. + 3, which are
// the operand positions of the second product O^T = V^T P^T as they stand (a contraction runs over the keys in whatever order both operands agree on),
// so softmax numerators go from one product to the other in registers.  K and V lie in LDS, row major, in tiles of 64 keys that all waves
// walk together; V's operands are read transposed.  Rows are padded so that neither read has bank conflicts.
#include <cfloat>

#include "pk_attention.h"
#include "pk_kv16.h"

namespace pk {

namespace {

constexpr int kKeys = 64;   // of a tile

template <int D>
struct PromptShape {
    static constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 32 * kWaves;   // of a workgroup
    static constexpr int kSteps = D / 16;    // of the contraction over channels
    static constexpr int kTiles = D / 32;    // of channels of the result
    static constexpr int kPieces = kKeys * D / 8, kPer = (kPieces + kThreads - 1) / kThreads;   // 16-byte pieces of a tile, per thread
    static constexpr int kKRow = 2 * D + 16;   // bytes between rows in LDS: 16 rows from any 16-byte column on lie in 64 different banks,
    static constexpr int kVRow = 2 * D + (D == 96 ? 0 : 64);   // and four rows of 64 bytes do
};

// Sum of an int over the wave, in every lane
__device__ __forceinline__ int wave_sum(int x)
{
    uint32_t v = (uint32_t)x;
    v += dpp<0xb1>(v);
    v += dpp<0x4e>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    const rows2 a = swap16(v, v);
    v = a[0] + a[1];
    const rows2 b = swap32(v, v);
    return (int)(b[0] + b[1]);
}

struct Prompt {
    int start, len;
};
__device__ __forceinline__ Prompt prompt_of(const PromptArgs &a, int seq)
{
    const int from = min(max(a.starts[seq], 0), a.n_tokens), to = min(max(a.starts[seq + 1], 0), a.n_tokens);
    return {from, max(to - from, 0)};
}

// Row tiles are taken in order of their number within their sequence, the last ones, which see most keys, first.  Item w is the one of level L (tile
// L of its sequence) for the largest L with more than w tiles on levels >= L, and there one of the sequences that have such a tile, in their order.
// sm: n_seq + kThreads / 64 numbers.
template <int ROWS, int THREADS>
__device__ __forceinline__ bool find_tile(const PromptArgs &a, int w, int *sm, int &seq, int &tile)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const auto tiles_of = [&](int i) { return i < a.n_seq ? (prompt_of(a, i).len * a.r + ROWS - 1) / ROWS : 0; };
    if (a.n_seq == 1) {
        seq = 0;
        tile = __builtin_amdgcn_readfirstlane(tiles_of(0)) - 1 - w;
        return tile >= 0;
    }
    if (a.n_seq <= 64) {   // every wave for itself
        const int tiles = tiles_of(lane);
        if (__builtin_amdgcn_readfirstlane(wave_sum(tiles)) <= w) return false;
        int lo = 0, hi = 1;   // G(lo) > w >= G(hi), G(L) = sum of max(tiles - L, 0)
        const auto at_least = [&](int level) { return __builtin_amdgcn_readfirstlane(wave_sum(max(tiles - level, 0))); };
        while (at_least(hi) > w) {
            lo = hi;
            hi *= 2;
        }
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (at_least(mid) > w) lo = mid;
            else hi = mid;
        }
        uint64_t those = __ballot(tiles > lo);
        for (int skip = w - at_least(lo + 1); skip > 0; --skip) those &= those - 1;
        seq = __ffsll((unsigned long long)those) - 1;
        tile = lo;
        return true;
    }
    int *sm_sum = sm + a.n_seq;
    for (int i = threadIdx.x; i < a.n_seq; i += THREADS) sm[i] = tiles_of(i);
    const auto at_least = [&](int level) {
        int sum = 0;
        for (int i = threadIdx.x; i < a.n_seq; i += THREADS) sum += max(sm[i] - level, 0);
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) sm_sum[wave] = sum;
        __syncthreads();
        int all = 0;
        for (int i = 0; i < THREADS / 64; ++i) all += sm_sum[i];
        return __builtin_amdgcn_readfirstlane(all);
    };
    if (at_least(0) <= w) return false;
    int lo = 0, hi = 1;
    while (at_least(hi) > w) {
        lo = hi;
        hi *= 2;
    }
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at_least(mid) > w) lo = mid;
        else hi = mid;
    }
    int skip = w - at_least(lo + 1);
    tile = lo;
    for (int i0 = 0;; i0 += 64) {   // every wave for itself
        uint64_t those = __ballot(i0 + lane < a.n_seq && sm[min(i0 + lane, a.n_seq - 1)] > lo);
        const int here = __popcll(those);
        if (skip >= here) {
            skip -= here;
            continue;
        }
        for (; skip > 0; --skip) those &= those - 1;
        seq = i0 + __ffsll((unsigned long long)those) - 1;
        break;
    }
    __syncthreads();   // sm's place is needed for something else
    return true;
}

// Whether a 32-bit word has a 16-bit value that is infinite or NaN
template <bool BF16>
__device__ __forceinline__ bool not_finite(uint32_t w)
{
    constexpr uint32_t e = BF16 ? 0x7f80u : 0x7c00u;
    return (w & e) == e || ((w >> 16) & e) == e;
}

template <int D, bool BF16, bool OPT>
__global__ __launch_bounds__(PromptShape<D>::kThreads, D == 256 ? 1 : 2) void prompt_kernel(PromptArgs a)
{
    using S = PromptShape<D>;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    __shared__ __attribute__((aligned(16))) char sm_k[2][kKeys * S::kKRow];
    __shared__ __attribute__((aligned(16))) char sm_v[2][kKeys * S::kVRow];
    __shared__ int sm_bad[2][S::kWaves];   // whether V of the tile has infinities or NaN, looked at where some row does not see all of the tile
    // heads next to each other: with eight of them every XCD has one head's keys in its cache
    const int kvh = blockIdx.x % a.n_kv_heads;
    int seq, tile;
    static_assert(sizeof(sm_k) >= (4096 + S::kWaves) * 4, "numbers of find_tile");
    if (!find_tile<S::kRows, S::kThreads>(a, blockIdx.x / a.n_kv_heads, reinterpret_cast<int *>(sm_k), seq, tile)) return;
    seq = __builtin_amdgcn_readfirstlane(seq);
    const Prompt p = prompt_of(a, seq);
    const int start = __builtin_amdgcn_readfirstlane(p.start), len = __builtin_amdgcn_readfirstlane(p.len);
    const int rows = len * a.r, row0 = tile * S::kRows, wave_row = row0 + 32 * wave;
    const bool has_rows = wave_row < rows;

    // the row (those behind the last one stand in for it, and are not stored)
    const int row = min(wave_row + n, rows - 1), tok = row / a.r, head = kvh * a.r + row - tok * a.r;
    const auto token_of = [&](int at) { return min(at, rows - 1) / a.r; };
    const int first_tok = token_of(row0), last_tok = token_of(row0 + S::kRows - 1), wave_first = token_of(wave_row), wave_last = token_of(wave_row + 31);
    const auto first_key = [&](int token) { return a.window > 0 ? max(token - a.window + 1, 0) : 0; };
    const int lo = first_key(first_tok) & ~(kKeys - 1), hi = last_tok + 1;

    short8v q[S::kSteps];
    {
        const char *from = static_cast<const char *>(a.q) + 2 * ((start + tok) * a.q_token + head * a.q_head + 8 * h);
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {
            uint4 w = *reinterpret_cast<const uint4 *>(from + 32 * s);
            // the products take the scale's sign, so that what multiplies them later is positive
            if (a.scale < 0.f) w = make_uint4(w.x ^ 0x80008000u, w.y ^ 0x80008000u, w.z ^ 0x80008000u, w.w ^ 0x80008000u);
            q[s] = __builtin_bit_cast(short8v, w);
        }
    }
    // the products' factor; never 0, so that a masked -inf stays one
    const float c = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);
    const float slope = OPT && a.slopes ? a.slopes[head] * kLog2e : 0.f;

    float m = -INFINITY, most = -INFINITY, l = 0.f;   // the numerators' reference, the largest score that it serves, their sum in this lane
    float16v o[S::kTiles];
#pragma unroll
    for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[ct][i] = 0.f;

    const char *k_from = static_cast<const char *>(a.k) + 2 * (start * a.k_token + kvh * a.k_head);
    const char *v_from = static_cast<const char *>(a.v) + 2 * (start * a.v_token + kvh * a.v_head);
    // pieces of a tile that are on their way: of K, of V
    uint4 k_new[S::kPer], v_new[S::kPer];
    const auto fetch = [&](int t0) {
#pragma unroll
        for (int j = 0; j < S::kPer; ++j) {
            const int piece = tid + j * S::kThreads;
            if (S::kPieces % S::kThreads != 0 && piece >= S::kPieces) break;
            const int64_t t = min(t0 + piece / (D / 8), len - 1);   // (behind the last token: it again; those keys are masked)
            const int at = piece % (D / 8) * 16;
            k_new[j] = *reinterpret_cast<const uint4 *>(k_from + 2 * t * a.k_token + at);
            v_new[j] = *reinterpret_cast<const uint4 *>(v_from + 2 * t * a.v_token + at);
        }
    };
    const auto lay_down = [&](int t0, int buf) {
        bool bad = false;
        const bool look = t0 + kKeys - 1 > first_tok || t0 < first_key(last_tok);
#pragma unroll
        for (int j = 0; j < S::kPer; ++j) {
            const int piece = tid + j * S::kThreads;
            if (S::kPieces % S::kThreads != 0 && piece >= S::kPieces) break;
            const int key = piece / (D / 8), at = piece % (D / 8) * 16;
            *reinterpret_cast<uint4 *>(sm_k[buf] + key * S::kKRow + at) = k_new[j];
            *reinterpret_cast<uint4 *>(sm_v[buf] + key * S::kVRow + at) = v_new[j];
            if (look) bad |= not_finite<BF16>(v_new[j].x) || not_finite<BF16>(v_new[j].y) || not_finite<BF16>(v_new[j].z) || not_finite<BF16>(v_new[j].w);
        }
        if (look) {
            const bool any = __any(bad);
            if (lane == 0) sm_bad[buf][wave] = any;
        }
    };

    const int k_at = n * S::kKRow + 16 * h, v_at = (4 * h + ((lane & 15) >> 2)) * S::kVRow + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    const auto v_operand = [&](int buf, int t, int ct) {   // of keys 16 t + 8 (j / 4) + 4 h + j % 4, channels 32 ct + n
        typedef __attribute__((address_space(3))) short4v *lds4;
        const char *at = sm_v[buf] + v_at + 16 * t * S::kVRow + 64 * ct;
        const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at));
        const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 8 * S::kVRow));
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    fetch(lo);
    lay_down(lo, 0);
    int buf = 0;
    for (int t0 = lo; t0 < hi; t0 += kKeys, buf ^= 1) {
        __syncthreads();
        const bool more = t0 + kKeys < hi;
        if (more) fetch(t0 + kKeys);
        if (has_rows && t0 <= wave_last && t0 + kKeys > first_key(wave_first)) {
            float16v s[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[j][i] = 0.f;
#pragma unroll
            for (int i = 0; i < S::kSteps; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    s[j] = mfma32<BF16>(*reinterpret_cast<const short8v *>(sm_k[buf] + k_at + 32 * j * S::kKRow + 32 * i), q[i], s[j]);

            const bool edge = t0 + kKeys - 1 > wave_first || t0 < first_key(wave_last);
            const auto sees = [&](int t) { return t <= tok && (a.window <= 0 || tok - t < a.window); };
            float x[2][16], f = c;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[j][i] = s[j][i];
            if constexpr (OPT) {
                const float inv = a.cap > 0.f ? fminf(fabsf(a.scale) / a.cap, FLT_MAX) : 0.f, both[2] = {inv, inv};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (a.cap > 0.f) {
                        capped(x[j], both, a.cap * kLog2e);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[j][i] *= c;
                    }
                    if (a.slopes) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[j][i] = fmaf(-slope, (float)(tok - (t0 + 32 * j + 8 * (i >> 2) + 4 * h + (i & 3))), x[j][i]);
                    }
                }
                f = 1.f;
            }
            if (edge) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[j][i] = sees(t0 + 32 * j + 8 * (i >> 2) + 4 * h + (i & 3)) ? x[j][i] : -INFINITY;
            }
            float top = x[0][0];
#pragma unroll
            for (int i = 1; i < 32; ++i) top = fmaxf(top, x[i >> 4][i & 15]);
            top = op_rows(swap32(bits_of(top), bits_of(top)), MaxF()) * f;
            float by = 1.f;
            if (top > most) {
                most = top;
                const float to = reference_of<BF16>(top);
                by = exp2_(m - to);
                m = to;
                l *= by;
            }
            if (__any(by != 1.f)) {
#pragma unroll
                for (int ct = 0; ct < S::kTiles; ++ct) o[ct] *= by;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            float sum = 0.f;
            if (__any(fabsf(ref) >= 0x1p20f)) {
                // scores of large steps as their largest is, rounded; the multiply-add would take their factor in unrounded
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    float y = x[i >> 4][i & 15] * f;
                    asm volatile("" : "+v"(y));   // (not contracted)
                    x[i >> 4][i & 15] = exp2_(y - ref);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i >> 4][i & 15] = exp2_(fmaf(x[i >> 4][i & 15], f, -ref));
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) sum += x[i >> 4][i & 15];
            l += sum;
            short8v pf[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const float *y = &x[t >> 1][8 * (t & 1)];
                const uint4 w = make_uint4(narrow(y[0], y[1], BF16), narrow(y[2], y[3], BF16), narrow(y[4], y[5], BF16), narrow(y[6], y[7], BF16));
                pf[t] = __builtin_bit_cast(short8v, w);
            }

            bool bad = false;
            if (edge) {
                int any = 0;
#pragma unroll
                for (int w = 0; w < S::kWaves; ++w) any |= sm_bad[buf][w];
                bad = __builtin_amdgcn_readfirstlane(any) != 0;
            }
            if (!bad) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int ct = 0; ct < S::kTiles; ++ct) o[ct] = mfma32<BF16>(v_operand(buf, t, ct), pf[t], o[ct]);
            } else {
                // Values that are not finite reach only the rows that see them: they are taken out, and products of marks (1.0 for +inf or NaN, for -inf
                // or NaN) and of who sees whom say which results have one.
                constexpr short kOne = BF16 ? 0x3f80 : 0x3c00;
                constexpr int kExp = BF16 ? 0x7f80 : 0x7c00, kMant = BF16 ? 0x007f : 0x03ff;
#pragma unroll 1
                for (int t = 0; t < 4; ++t) {
                    short8v see, pt;
#pragma unroll
                    for (int i = 0; i < 8; ++i) see[i] = sees(t0 + 16 * t + 8 * (i >> 2) + 4 * h + (i & 3)) ? kOne : (short)0;
                    pt = t == 0 ? pf[0] : t == 1 ? pf[1] : t == 2 ? pf[2] : pf[3];
#pragma unroll
                    for (int ct = 0; ct < S::kTiles; ++ct) {
                        short8v v = v_operand(buf, t, ct), up, down;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const bool odd = (v[i] & kExp) == kExp, nan = odd && (v[i] & kMant) != 0;
                            up[i] = odd && (nan || v[i] >= 0) ? kOne : (short)0;
                            down[i] = odd && (nan || v[i] < 0) ? kOne : (short)0;
                            v[i] = odd ? (short)0 : v[i];
                        }
                        float16v none;
#pragma unroll
                        for (int i = 0; i < 16; ++i) none[i] = 0.f;
                        const float16v ups = mfma32<BF16>(up, see, none), downs = mfma32<BF16>(down, see, none);
                        o[ct] = mfma32<BF16>(v, pt, o[ct]);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (ups[i] > 0.f) o[ct][i] += INFINITY;
                            if (downs[i] > 0.f) o[ct][i] -= INFINITY;
                        }
                    }
                }
            }
        }
        if (more) lay_down(t0 + kKeys, buf ^ 1);
    }

    if (!has_rows || wave_row + n >= rows) return;
    l = op_rows(swap32(bits_of(l), bits_of(l)), AddF());
    const float inv = l == 0.f ? 0.f : 1.f / l;
    char *to = static_cast<char *>(a.out) + 2 * ((start + tok) * a.o_token + head * a.o_head + 4 * h);
#pragma unroll
    for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = mean_of<BF16>(o[ct][4 * i + e] * inv);
            *reinterpret_cast<uint2 *>(to + 2 * (32 * ct + 8 * i)) = make_uint2(narrow(y[0], y[1], BF16), narrow(y[2], y[3], BF16));
        }
    if (a.lse && h == 0) {
        // l's power of two joins the reference first: their sum is small where the log-sum-exp is, and takes no rounding of l's whole logarithm
        int e;
        const float part = frexpf(l, &e);
        a.lse[(int64_t)head * a.n_tokens + start + tok] = l == 0.f ? -INFINITY : (m + (float)e + log2f(part)) * kLn2;
    }
}

template <int D>
hipError_t launch_d(const PromptArgs &a, uint32_t grid, hipStream_t s)
{
    constexpr int threads = PromptShape<D>::kThreads;
    const bool opt = a.cap > 0.f || a.slopes;
    if (a.bf16) {
        if (opt) prompt_kernel<D, true, true><<<grid, threads, 0, s>>>(a);
        else prompt_kernel<D, true, false><<<grid, threads, 0, s>>>(a);
    } else {
        if (opt) prompt_kernel<D, false, true><<<grid, threads, 0, s>>>(a);
        else prompt_kernel<D, false, false><<<grid, threads, 0, s>>>(a);
    }
    return hipGetLastError();
}

int rows_of(int d) { return d == 64 ? PromptShape<64>::kRows : d == 96 ? PromptShape<96>::kRows : d == 128 ? PromptShape<128>::kRows : PromptShape<256>::kRows; }

}  // namespace

int64_t prompt_workgroups(int64_t n_seq, int64_t n_kv_heads, int64_t r, int64_t n_tokens, int d)
{
    const int64_t rows = rows_of(d);
    return (n_tokens * r + n_seq * (rows - 1)) / rows * n_kv_heads;
}

hipError_t launch_prompt(const PromptArgs &a, hipStream_t s)
{
    const uint32_t grid = (uint32_t)prompt_workgroups(a.n_seq, a.n_kv_heads, a.r, a.n_tokens, a.d);
    return a.d == 64    ? launch_d<64>(a, grid, s)
           : a.d == 96  ? launch_d<96>(a, grid, s)
           : a.d == 128 ? launch_d<128>(a, grid, s)
                        : launch_d<256>(a, grid, s);
}

}  // namespace pk
