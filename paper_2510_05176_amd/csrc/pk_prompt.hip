// Causal attention of whole prompts, packed one after the other.
//
// The rows of a KV head are its query heads' tokens, row = token * r + head of the group, so that what a workgroup loads of K and V serves all heads,
// and a tile of rows spans few tokens.  A wave has 32 rows.  S^T = K Q^T, 32 keys at a time, on v_mfma_f32_32x32x16: lane 32 h + n gets, for row n, keys 8i + 4h .. + 3, which are
// the operand positions of the second product O^T = V^T P^T as they stand (a contraction runs over the keys in whatever order both operands agree on),
// so softmax numerators go from one product to the other in registers.  K and V lie in LDS, row major, in tiles of 64 keys that all waves
// walk together, two of each; V's operands are read transposed.  Tiles go to LDS without registers in between, 16-byte pieces swapped within their rows so that
// neither read has bank conflicts (none counted), and are asked for a phase before they are needed.
//
// The matrix instructions bound it, and beside them the numerators, 4.5 vector instructions per score of their own (5.2 with all others counted, 6.0 at 64 channels), of which
// a SIMD starts one in four to ten cycles: at 128 channels both take the same time, and two groups of waves that change places hide one behind the other; at 64 the numerators take twice the products' time.
// One prompt of 32k tokens, 32 heads of 128 channels, 8.9 TFLOP: 7.4 ms (7.3 to 8.1 from card to card), 1.2 PFLOP/s, where a library product of 16384 cubed reaches 1.31 to 1.35 (one group 8.2 ms,
// tiles through registers 8.4).  The card's power is the last bound of it: the same launch over zeros, which take less, runs a quarter to a third faster.
#include <cfloat>
#include <type_traits>
#include <utility>

#include "pk_attention.h"
#include "pk_kv16.h"

namespace pk {

namespace {

constexpr int kKeys = 64;   // of a tile

typedef uint32_t word4 __attribute__((ext_vector_type(4)));

template <int D, int GROUPS>
struct PromptShape {
    static constexpr int kGroups = GROUPS;   // of four waves
    static constexpr int kWaves = 4 * kGroups, kThreads = 64 * kWaves, kRows = 32 * kWaves;   // of a workgroup
    static constexpr int kSteps = D / 16;    // of the contraction over channels
    static constexpr int kTiles = D / 32;    // of channels of the result
    static constexpr int kRow = D == 96 ? 256 : 2 * D;   // bytes of a key in LDS
    static constexpr int kSlots = kRow / 16, kTileBytes = kKeys * kRow;
    static constexpr int kLoaders = 256, kPer = kKeys * kSlots / kLoaders;   // threads that bring the tiles in: the first group's; 16-byte pieces of a tile for each
    // Which piece of a key's vector lies in which slot of its row: piece ^ swizzle, so that 16 keys' pieces of the same number (K's operands) and 64
    // bytes of four keys (V's) lie in 64 different banks.
    static __device__ __forceinline__ int k_swizzle(int key) { return D == 64 ? (key >> 1) & 7 : key & 15; }
    static __device__ __forceinline__ int v_swizzle(int key) { return D == 64 ? ((key >> 1) & 1) << 2 : (key & 3) << 2; }
};

// f(0), f(1), ..: unrolled whatever its size
template <typename F, int... I>
__device__ __forceinline__ void for_each(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>()), ...);
}

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
    seq = -1;
    for (int i0 = 0; i0 < a.n_seq; i0 += 64) {   // every wave for itself
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
    return seq >= 0;   // (starts that do not grow may have sums beyond 32 bits, which find none)
}

// A word's 16-bit values that are infinite or NaN
template <bool BF16>
__device__ __forceinline__ uint32_t not_finite(uint32_t w)
{
    constexpr uint32_t e = BF16 ? 0x7f80u : 0x7c00u;
    return ((w & e) == e ? 0xffffu : 0u) | (((w >> 16) & e) == e ? 0xffff0000u : 0u);
}

// Groups of four waves, one wave of each on every SIMD.  With two of them a step of the loop has two phases, barriers between them: one group is at its
// matrix instructions (the products with V of the last tile and with K of the next) while the other one computes softmax numerators, then they change places.
// With one, what overlaps is left to the workgroups of a CU (two; three at 64 channels, one at 256).
template <int D, int GROUPS, bool BF16, bool OPT>
__global__ __launch_bounds__((PromptShape<D, GROUPS>::kThreads), D == 256 ? 1 : 2) void prompt_kernel(PromptArgs a)
{
    using S = PromptShape<D, GROUPS>;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    __shared__ __attribute__((aligned(16))) char sm[4][S::kTileBytes];   // K of two tiles, V of two
    __shared__ int sm_special;   // V has infinities or NaN in a tile that some row does not see all of
    // heads next to each other: with eight of them every XCD has one head's keys in its cache
    const int kvh = blockIdx.x % a.n_kv_heads;
    int seq, tile;
    static_assert(sizeof(sm) >= (4096 + S::kWaves) * 4, "numbers of find_tile");
    if (!find_tile<S::kRows, S::kThreads>(a, blockIdx.x / a.n_kv_heads, reinterpret_cast<int *>(sm), seq, tile)) return;
    seq = __builtin_amdgcn_readfirstlane(seq);
    const Prompt p = prompt_of(a, seq);
    const int start = __builtin_amdgcn_readfirstlane(p.start), len = __builtin_amdgcn_readfirstlane(p.len);
    const int rows = len * a.r, row0 = tile * S::kRows, wave_row = row0 + 32 * wave;

    // the row (those behind the last one stand in for it, and are not stored)
    const int row = min(wave_row + n, rows - 1), tok = row / a.r, head = kvh * a.r + row - tok * a.r;
    const auto token_of = [&](int at) { return __builtin_amdgcn_readfirstlane(min(at, rows - 1) / a.r); };
    const int first_tok = token_of(row0), last_tok = token_of(row0 + S::kRows - 1), wave_first = token_of(wave_row), wave_last = token_of(wave_row + 31);
    const auto first_key = [&](int token) { return a.window > 0 ? max(token - a.window + 1, 0) : 0; };
    const int lo = first_key(first_tok) & ~(kKeys - 1), hi = last_tok + 1, tiles = (hi - lo + kKeys - 1) / kKeys;

    const char *k_from = static_cast<const char *>(a.k) + 2 * (start * a.k_token + kvh * a.k_head);
    const char *v_from = static_cast<const char *>(a.v) + 2 * (start * a.v_token + kvh * a.v_head);
    // A tile's way into LDS, without registers in between.  Lane l of a wave's request writes 16 l bytes behind the request's place; what it reads is its to choose.
    // (The compiler would wait for it before every read from LDS that follows, whatever tile that is of; it has no registers to wait for, and arrive() waits for it.  m0, where the place goes, is an operand, so that the compiler writes it.)
    // A lane's part of the addresses is the same for every whole tile, where strides let it fit 32 bits.
    uint32_t k_lane[S::kPer], v_lane[S::kPer];
#pragma unroll
    for (int j = 0; j < S::kPer; ++j) {
        const int slot = tid + j * S::kLoaders, key = slot / S::kSlots;
        k_lane[j] = 2 * key * (uint32_t)a.k_token + 16 * ((slot % S::kSlots) ^ S::k_swizzle(key));
        v_lane[j] = 2 * key * (uint32_t)a.v_token + 16 * ((slot % S::kSlots) ^ S::v_swizzle(key));
    }
    const bool k_fits = a.k_token >= 0 && a.k_token <= 1 << 24, v_fits = a.v_token >= 0 && a.v_token <= 1 << 24;
    const auto place_of_piece = [&](const char *tile_at, int j) {
        return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)tile_at) + 1024 * (wave + 4 * j);
    };
    const auto has_piece = [&](int j, bool v) {   // (96 channels leave four of sixteen slots empty)
        const int slot = tid + j * S::kLoaders, key = slot / S::kSlots;
        return D != 96 || ((slot % S::kSlots) ^ (v ? S::v_swizzle(key) : S::k_swizzle(key))) < D / 8;
    };
    const auto request_whole = [&](int j, const char *tile_from, const uint32_t (&lane_at)[S::kPer], const char *to, bool v) {
        if (has_piece(j, v)) asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "{m0}"(place_of_piece(to, j)), "v"(lane_at[j]), "s"(tile_from) : "memory");
    };
    // a tile that the sequence ends in, or with strides that do not fit: all of it
    const auto request_slowly = [&](const char *from, int64_t token, int t0, const char *to, bool v) {
#pragma unroll 1
        for (int j = 0; j < S::kPer; ++j) {
            const int slot = tid + j * S::kLoaders, key = slot / S::kSlots, piece = (slot % S::kSlots) ^ (v ? S::v_swizzle(key) : S::k_swizzle(key));
            const int64_t t = min(t0 + key, len - 1);   // (behind the last token: it again; those keys are masked)
            if (has_piece(j, v)) asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(place_of_piece(to, j)), "v"(from + 2 * t * token + 16 * piece) : "memory");
        }
    };
    const bool loads = S::kGroups == 1 || wave < 4;
    if (loads) request_slowly(k_from, a.k_token, lo, sm[0], false);

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
    if (loads) request_slowly(v_from, a.v_token, lo, sm[2], true);
    // the products' factor; never 0, so that a masked -inf stays one
    const float c = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);
    const float slope = OPT && a.slopes ? a.slopes[head] * kLog2e : 0.f;

    float m = -INFINITY, most = -INFINITY, l = 0.f;   // the numerators' reference, the largest score that it serves, their sum in this lane
    float16v o[S::kTiles], s[2];
    short8v pf[4];
#pragma unroll
    for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[ct][i] = 0.f;

    const int k_at = n * S::kRow, k_piece = 16 * (S::k_swizzle(n) ^ h);
    const int v_key = 4 * h + ((lane & 15) >> 2), v_at = v_key * S::kRow + 32 * ((lane >> 4) & 1) + 8 * (lane & 3), v_piece = 16 * S::v_swizzle(v_key);
    const auto k_operand = [&](int buf, int i, int j) -> short8v {
        return *reinterpret_cast<const short8v *>(sm[buf] + k_at + 32 * j * S::kRow + (k_piece ^ (32 * i)));
    };
    const auto v_operand = [&](int buf, int t, int ct) -> short8v {   // of keys 16 t + 8 (j / 4) + 4 h + j % 4, channels 32 ct + n
        typedef __attribute__((address_space(3))) short4v *lds4;
        const char *at = sm[2 + buf] + v_at + 16 * t * S::kRow + (v_piece ^ (64 * ct));
        const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at));
        const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 8 * S::kRow));
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const uint32_t reach = a.window > 0 ? (uint32_t)a.window : 0x80000000u;   // a token sees those less than this before it, and none behind (a difference below 0 is larger)
    const auto sees = [&](int t) { return (uint32_t)(tok - t) < reach; };

    // K of tile i + 1 and V of tile i: asked for piece by piece between the first group's matrix instructions (requests at once stand in line for their addresses,
    // and beside the numerators each costs some 140 cycles), and a phase later there, where tile i - 1's and i - 2's were
    constexpr int kRequests = 2 * S::kPer;
    const auto asking = [&](int i) {
        const int k_t0 = lo + (i + 1) * kKeys, v_t0 = lo + i * kKeys;
        const char *k_to = sm[(i + 1) & 1], *v_to = sm[2 + (i & 1)];
        const bool k_whole = k_fits && k_t0 + kKeys <= len, v_whole = v_fits && v_t0 + kKeys <= len;
        if (!k_whole) request_slowly(k_from, a.k_token, k_t0, k_to, false);
        if (!v_whole && i > 0) request_slowly(v_from, a.v_token, v_t0, v_to, true);   // (the first tile's is on its way)
        return [=, &k_lane, &v_lane, &request_whole, k_at = k_from + 2 * k_t0 * a.k_token, v_at = v_from + 2 * v_t0 * a.v_token](int from, int to) {
#pragma unroll
            for (int j = 0; j < kRequests; ++j) {
                if ((2 * j + 1) * 32 / kRequests < from || (2 * j + 1) * 32 / kRequests >= to) continue;
                if (j < S::kPer) {
                    if (k_whole) request_whole(j, k_at, k_lane, k_to, false);
                } else {
                    if (v_whole && i > 0) request_whole(j - S::kPer, v_at, v_lane, v_to, true);
                }
            }
        };
    };
    const auto nothing = [](int, int) {};

    // Products with V of tile i - 1 (WITH_V) and with K of tile i (WITH_K).  Operands are read from LDS kAhead products ahead.
    const auto multiply = [&](int i, auto with_v, auto with_k, auto &&between) {   // between(x, y): from the x-th to the y-th 64th of it
        constexpr bool kV = decltype(with_v)::value, kK = decltype(with_k)::value;
        constexpr int kOfV = kV ? 4 * S::kTiles : 0, kAll = kOfV + (kK ? 2 * S::kSteps : 0), kAhead = 4;
        const int k_buf = i & 1, v_buf = k_buf ^ 1;
        const auto operand = [&](int u) -> short8v {
            if (u < kOfV) return v_operand(v_buf, u / S::kTiles, u % S::kTiles);
            return k_operand(k_buf, (u - kOfV) / 2, (u - kOfV) % 2);
        };
        short8v ahead[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) ahead[u] = operand(u);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kK)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[j][e] = 0.f;
        for_each([&](auto at) {
            constexpr int u = decltype(at)::value;
            if constexpr (u < kOfV) o[u % S::kTiles] = mfma32<BF16>(ahead[u % kAhead], pf[u / S::kTiles], o[u % S::kTiles]);
            else s[(u - kOfV) % 2] = mfma32<BF16>(ahead[u % kAhead], q[(u - kOfV) / 2], s[(u - kOfV) % 2]);
            if constexpr (u + kAhead < kAll) ahead[u % kAhead] = operand(u + kAhead);
            between(u * 64 / kAll, (u + 1) * 64 / kAll);
            __builtin_amdgcn_sched_barrier(0x6);   // (arithmetic may be moved across)
        }, std::make_integer_sequence<int, kAll>());
    };

    // From the products with K of tile i to its numerators
    const auto soften = [&](int i) {
        const int t0 = lo + i * kKeys;
        const bool edge = t0 + kKeys - 1 > wave_first || t0 < first_key(wave_last);
        float f = c;
        if constexpr (OPT) {
            const float inv = a.cap > 0.f ? fminf(fabsf(a.scale) / a.cap, FLT_MAX) : 0.f, both[2] = {inv, inv};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = s[j][e];
                if (a.cap > 0.f) {
                    capped<16, true>(x, both, a.cap * kLog2e);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] *= c;
                }
                if (a.slopes) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = fmaf(-slope, (float)(tok - (t0 + 32 * j + 8 * (e >> 2) + 4 * h + (e & 3))), x[e]);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) s[j][e] = x[e];
            }
            f = 1.f;
        }
        if (edge) {
            const int back = tok - t0 - 4 * h;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[j][e] = (uint32_t)(back - (32 * j + 8 * (e >> 2) + (e & 3))) < reach ? s[j][e] : -INFINITY;
        }
        float top = s[0][0], other = s[1][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) {
            top = fmaxf(top, s[0][e]);
            other = fmaxf(other, s[1][e]);
        }
        top = fmaxf(top, other);
        top = op_rows(swap32(bits_of(top), bits_of(top)), MaxF()) * f;
        float by = 1.f;
        if (top > most) {
            const float was = most;
            most = fabsf(top) < 0x1p20f ? top + kRoom : top;
            const float to = reference_of<BF16>(top);
            by = change_of<BF16>(m, to, was, most);
            m = to;
            l *= by;
        }
        if (__any(by != 1.f)) {
#pragma unroll
            for (int ct = 0; ct < S::kTiles; ++ct) o[ct] *= by;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float sum[2] = {0.f, 0.f};
        if (__any(fabsf(ref) >= kLarge)) {
            // (see kLarge)
            const float under = under_of<BF16>(most);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                float y = s[e >> 4][e & 15] * f;
                asm volatile("" : "+v"(y));   // (not contracted)
                s[e >> 4][e & 15] = (y - ref) - under;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) s[e >> 4][e & 15] = fmaf(s[e >> 4][e & 15], f, -ref);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            float16v &y = s[t >> 1];
#pragma unroll
            for (int x = 8 * (t & 1); x < 8 * (t & 1) + 8; ++x) {
                y[x] = exp2_(y[x]);
                sum[x & 1] += y[x];
            }
            const int e = 8 * (t & 1);
            const uint4 w = make_uint4(narrow(y[e], y[e + 1], BF16), narrow(y[e + 2], y[e + 3], BF16), narrow(y[e + 4], y[e + 5], BF16), narrow(y[e + 6], y[e + 7], BF16));
            pf[t] = __builtin_bit_cast(short8v, w);
        }
        l += sum[0] + sum[1];
        // here, not behind the barrier, where the compiler would put what is not needed before
        asm volatile("" : "+v"(l), "+v"(pf[0]), "+v"(pf[1]), "+v"(pf[2]), "+v"(pf[3]));
    };
    // whether a tile is seen in part by some row of the workgroup
    const auto in_part = [&](int t0) { return t0 + kKeys - 1 > first_tok || t0 < first_key(last_tok); };
    const auto arrive = [&](int i) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (in_part(lo + i * kKeys)) {
            // Values that are not finite would make NaN of a masked key's numerator of 0: they are taken out, and rows that see them get them afterwards.
            uint32_t bad = 0;
#pragma unroll
            for (int j = 0; j < S::kPer; ++j) {
                const int slot = tid + j * S::kLoaders;   // (this thread's own)
                if (D == 96 && ((slot % S::kSlots) ^ S::v_swizzle(slot / S::kSlots)) >= D / 8) continue;
                word4 *at = reinterpret_cast<word4 *>(sm[2 + (i & 1)] + 16 * slot);
                word4 w = *at;
                uint32_t here = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t out = not_finite<BF16>(w[e]);
                    w[e] &= ~out;
                    here |= out;
                }
                if (here) *at = w;
                bad |= here;
            }
            if (bad) sm_special = 1;
        }
    };
    constexpr auto yes = std::integral_constant<bool, true>();
    constexpr auto no = std::integral_constant<bool, false>();
    const auto change = [&] {
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };

    if (tid == 0) sm_special = 0;
    if (loads) {
        asm volatile("s_waitcnt vmcnt(%0)" : : "n"(S::kPer) : "memory");   // all but V's
        change();
        multiply(0, no, yes, asking(0));
        if constexpr (S::kGroups == 2) change();
        soften(0);
        arrive(0);
        change();
        for (int i = 1; i < tiles; ++i) {
            multiply(i, yes, yes, asking(i));
            if constexpr (S::kGroups == 2) change();
            soften(i);
            arrive(i);
            change();
        }
        multiply(tiles, yes, no, nothing);
    } else {
        change();
        change();
        multiply(0, no, yes, nothing);
        change();
        for (int i = 1; i < tiles; ++i) {
            soften(i - 1);
            change();
            multiply(i, yes, yes, nothing);
            change();
        }
        soften(tiles - 1);
        multiply(tiles, yes, no, nothing);
    }

    l = op_rows(swap32(bits_of(l), bits_of(l)), AddF());
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[ct][i] = mean_of<BF16>(o[ct][i] * inv);
    if (sm_special) {   // (written before a barrier that all have passed)
        for (int t = lo; t < hi; ++t) {
            if (!in_part(t & ~(kKeys - 1)) || !sees(t)) continue;
            const char *at = v_from + 2 * ((int64_t)t * a.v_token + 4 * h);
#pragma unroll
            for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(at + 2 * (32 * ct + 8 * i));
                    const uint32_t x = not_finite<BF16>(w.x), y = not_finite<BF16>(w.y);
                    if ((x | y) == 0) continue;
                    float v[4];
                    widen(w.x & x, BF16, v[0], v[1]);
                    widen(w.y & y, BF16, v[2], v[3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[ct][4 * i + e] += v[e];
                }
        }
    }
    if (wave_row + n >= rows) return;
    char *to = static_cast<char *>(a.out) + 2 * ((start + tok) * a.o_token + head * a.o_head + 4 * h);
#pragma unroll
    for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint2 *>(to + 2 * (32 * ct + 8 * i)) = make_uint2(narrow(o[ct][4 * i], o[ct][4 * i + 1], BF16), narrow(o[ct][4 * i + 2], o[ct][4 * i + 3], BF16));
    if (a.lse && h == 0) {
        // l's power of two joins the reference first: their sum is small where the log-sum-exp is, and takes no rounding of l's whole logarithm
        l *= exp2_(under_of<BF16>(most));
        int e;
        const float part = frexpf(l, &e);
        a.lse[(int64_t)head * a.n_tokens + start + tok] = l == 0.f ? -INFINITY : (m + (float)e + log2f(part)) * kLn2;
    }
}

// Two groups where the matrix instructions are as long as the numerators (96 and 128 channels) and there are enough rows for two workgroups of 256 per CU: one
// prompt of 32k tokens, 32 heads of 128 channels 7.69 ms, one group 8.24; 16 of 512 tokens 79 and 81 us; but one of 1000 tokens 32 and 29, 2048 tokens of
// one KV head 52 and 46.  With 64 channels (a packed batch 779 and 713 us) or a cap and distance bias (8k tokens 1146 and 907) the numerators are longer, and
// two groups that wait for each other waste the matrix unit's time; 256 channels leave registers for one wave per SIMD.
// Rows are those of the whole call, whatever a sequence has of them: 64 prompts of 128 tokens 58 and 60 us, but 70 of 64 tokens 45 and 42, and 300 of 20 tokens (80
// rows in each workgroup of 256 or 128) 92 and 56.
int groups_of(int64_t rows, int d, bool opt) { return (d == 96 || d == 128) && !opt && rows >= 512 * 256 ? 2 : 1; }

template <int D, int GROUPS>
void launch_groups(const PromptArgs &a, uint32_t grid, bool opt, hipStream_t s)
{
    constexpr int threads = PromptShape<D, GROUPS>::kThreads;
    if constexpr (GROUPS == 1) {
        if (opt) {
            if (a.bf16) prompt_kernel<D, GROUPS, true, true><<<grid, threads, 0, s>>>(a);
            else prompt_kernel<D, GROUPS, false, true><<<grid, threads, 0, s>>>(a);
            return;
        }
    }
    if (a.bf16) prompt_kernel<D, GROUPS, true, false><<<grid, threads, 0, s>>>(a);
    else prompt_kernel<D, GROUPS, false, false><<<grid, threads, 0, s>>>(a);
}

template <int D>
hipError_t launch_d(const PromptArgs &a, hipStream_t s)
{
    const bool opt = a.cap > 0.f || a.slopes;
    const int groups = groups_of((int64_t)a.n_tokens * a.r * a.n_kv_heads, D, opt), rows = 128 * groups;
    const uint32_t grid = (uint32_t)(((int64_t)a.n_tokens * a.r + (int64_t)a.n_seq * (rows - 1)) / rows * a.n_kv_heads);
    if constexpr (D == 96 || D == 128) {
        if (groups == 2) {
            launch_groups<D, 2>(a, grid, opt, s);
            return hipGetLastError();
        }
    }
    launch_groups<D, 1>(a, grid, opt, s);
    return hipGetLastError();
}

}  // namespace

int64_t prompt_workgroups(int64_t n_seq, int64_t n_kv_heads, int64_t r, int64_t n_tokens) { return (n_tokens * r + n_seq * 127) / 128 * n_kv_heads; }

hipError_t launch_prompt(const PromptArgs &a, hipStream_t s)
{
    return a.d == 64 ? launch_d<64>(a, s) : a.d == 96 ? launch_d<96>(a, s) : a.d == 128 ? launch_d<128>(a, s) : launch_d<256>(a, s);
}

}  // namespace pk
