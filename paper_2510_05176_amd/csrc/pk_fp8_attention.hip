// Attention over the 8-bit cache, and the attention weight of its tokens.
//
// A wave takes 64 cached tokens of one stream at a time against RT tiles of 16 query rows (row = query token * r + query head of the
// group).  S^T = K Q^T with K's codes as fp16 (exact) on the matrix cores: lane 16 g + n gets, for row n, tokens 4g .. 4g+3 of
// each tile of 16.  Those are the operand positions of the second product O^T = V^T P^T as they stand (the contraction runs over the
// tokens in whatever order both operands agree on), so softmax numerators go from one product to the other in registers.  Rows of
// K and V are read as they lie in memory: the contraction over channels takes the quarter row that a lane holds, and V's channels are
// dealt to the 16 rows of an operand tile so that a lane's bytes of a token are adjacent; pairs of tokens are interleaved by byte
// permutes before the conversion to fp16.  Block scales are powers of two and stay outside both products.  (e4m3 operands as they are, with the
// queries in two or three e4m3 terms, would save K's conversion but not V's, which needs the numerators in as many terms.)
//
// One token over long caches is bound by HBM (16 sequences x 32k tokens, 8 KV heads of 128 channels: 189 us, 5.7 TB/s, where a plain
// read reaches 5.5).  Many rows are far from the matrix cores' rate (1024 queries of 32 heads over 16k tokens: 332 to 338 us, 0.80 PFLOP/s; 256 channels
// 651 us, 0.82): per 64 tokens and 32 rows 64 matrix instructions beside about 290 vector ones, 32 of them exponentials, and of a SIMD's time 35 % are
// matrix and some 52 % vector instructions, which hardly overlap (nothing sets its two waves against each other).
// There the operands of a tile are converted once for four waves and lie in LDS (each wave converting for itself: 385 us, and 1121 with 256 channels).
// With two row tiles and at 256 channels a few registers are spilled (22 at 128 channels, 28 at 96, 6 at 256, with options 28, 42, 14), before and
// behind the loop over the keys.
#include "pk_attention.h"

namespace pk {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

template <int D>
struct Shape {
    static constexpr int kSteps = D / 32;          // products over channels per tile of tokens
    static constexpr int kTiles = D / 16;          // channel tiles of the output
    static constexpr int kKWords = D / 16;         // 32-bit words of K per lane and token: a quarter row
    static constexpr int kVWords = (D + 63) / 64;  // of V: a sixteenth row (96 channels: one word of the first 64, half a word of the rest)
};

// A lane's part of a row: `tile` points to a tile's first row and is the same for all lanes, `off` is the lane's own offset, so that an
// address takes no vector registers beyond that.
template <int D>
__device__ __forceinline__ void load_k(uint32_t (&k)[D / 16], const uint8_t *tile, uint32_t off)
{
    if constexpr (D == 96) {
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const uint2 v = *reinterpret_cast<const uint2 *>(tile + off + 8 * i);
            k[2 * i] = v.x;
            k[2 * i + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const uint4 v = *reinterpret_cast<const uint4 *>(tile + off + 16 * i);
            k[4 * i] = v.x;
            k[4 * i + 1] = v.y;
            k[4 * i + 2] = v.z;
            k[4 * i + 3] = v.w;
        }
    }
}
// n: which sixteenth of the row, off: its offset
template <int D>
__device__ __forceinline__ void load_v(uint32_t (&v)[Shape<D>::kVWords], const uint8_t *row, uint32_t off, uint32_t n)
{
    if constexpr (D == 64) {
        v[0] = *reinterpret_cast<const uint32_t *>(row + off);
    } else if constexpr (D == 96) {
        v[0] = *reinterpret_cast<const uint32_t *>(row + off);
        v[1] = *reinterpret_cast<const uint16_t *>(row + (off + 64 - 2 * n));
    } else if constexpr (D == 128) {
        const uint2 w = *reinterpret_cast<const uint2 *>(row + off);
        v[0] = w.x;
        v[1] = w.y;
    } else {
        const uint4 w = *reinterpret_cast<const uint4 *>(row + off);
        v[0] = w.x;
        v[1] = w.y;
        v[2] = w.z;
        v[3] = w.w;
    }
}
// Channel of output tile ct and operand row m: the inverse of how load_v deals them.
template <int D>
__device__ __forceinline__ int channel_of(int m, int ct)
{
    if constexpr (D == 96) return ct < 4 ? 4 * m + ct : 64 + 2 * m + (ct - 4);
    return m * (D / 16) + ct;
}

// 8 channels of a query (16-bit) as fp16: as they are, or from bfloat16 times a power of two
__device__ __forceinline__ half8v query8(const uint4 &v, int bf16, float mul)
{
    if (!bf16) return __builtin_bit_cast(half8v, v);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    half8v h;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        widen(w[i], 1, lo, hi);
        h[2 * i] = (_Float16)(lo * mul);
        h[2 * i + 1] = (_Float16)(hi * mul);
    }
    return h;
}

// The query of a row as operands of the products over channels, and the factor that belongs to the products (a power of two).
template <int D>
__device__ __forceinline__ void load_query(half8v (&qf)[D / 32], float &factor, const Fp8Queries &a, int seq, int kvh, int row, bool live, int g)
{
    uint4 raw[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; ++s) raw[s] = make_uint4(0, 0, 0, 0);
    if (live) {
        const int i = row / a.r, h = row - i * a.r;
        const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const char *>(a.q) + 2 * (seq * a.qs.seq + i * a.qs.token + (int64_t)(kvh * a.r + h) * a.qs.head)) +
                         g * (D / 32);
#pragma unroll
        for (int s = 0; s < D / 32; ++s) raw[s] = p[s];
    }
    // the products take the scale's sign, so that what multiplies them later is positive
    const bool negative = a.scale < 0.f;
    float mul = 1.f;
    factor = 1.f;
    if (a.bf16) {
        uint32_t most = 0;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const uint32_t w[4] = {raw[s].x, raw[s].y, raw[s].z, raw[s].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
                most = max(most, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
            }
        }
        const float x[1] = {__builtin_bit_cast(float, most << 16)};
        const uint32_t all = __builtin_bit_cast(uint32_t, fold_rows(x, MaxF()));
        // the largest element to [2^14, 2^15), within what a binary32 holds on both sides
        const int shift = min(max((int)(all >> 23) - 127 - 14, -126), 126);
        factor = __builtin_bit_cast(float, (uint32_t)(127 + shift) << 23);
        mul = __builtin_bit_cast(float, ((uint32_t)(127 - shift) << 23) | (negative ? 0x80000000u : 0u));
    } else if (negative) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) raw[s] = make_uint4(raw[s].x ^ 0x80008000u, raw[s].y ^ 0x80008000u, raw[s].z ^ 0x80008000u, raw[s].w ^ 0x80008000u);
    }
#pragma unroll
    for (int s = 0; s < D / 32; ++s) qf[s] = query8(raw[s], a.bf16, mul);
}

// Per lane: what its query row sees
struct Row {
    int last;       // index of the last token it sees, -1: none
    int pos;        // its position
    float slope;    // of its head
    float factor;   // of its products
};

template <int D>
__device__ __forceinline__ half8v k_operand(const uint32_t (&k)[D / 16], int s)
{
    const half2v a = codes_lo(k[2 * s]), b = codes_hi(k[2 * s]), c = codes_lo(k[2 * s + 1]), d = codes_hi(k[2 * s + 1]);
    return half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// From the products of 16 tokens of a row (4 each of the tiles at t, t + 16, t + 32, t + 48) to its scores times `post`: score = x * f of the
// token's half.  Without options x stays the product and f takes scale and units in, so that the factor costs nothing where the caller
// subtracts something anyway; f is never 0, so that a masked x = -inf stays one.
template <bool OPT>
__device__ __forceinline__ void to_scores(float (&x)[16], float (&f)[2], const float (&ks)[2], const Fp8Queries &a, float post, const Row &row, int t,
                                          const int32_t *pos, bool edge, bool windowed)
{
    const float c = row.factor * fabsf(a.scale);
#pragma unroll
    for (int h = 0; h < 2; ++h) f[h] = ks[h] * c;
    if constexpr (OPT) {
        if (a.cap > 0.f) {
            const float inv = 1.f / a.cap;
            f[0] *= inv;
            f[1] *= inv;
            capped(x, f, a.cap * post);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] *= f[i >> 3] * post;
        }
        if (pos) {
            const float slope = row.slope * post;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int4 p = *reinterpret_cast<const int4 *>(pos + t + 16 * j);
                const int back[4] = {row.pos - p.x, row.pos - p.y, row.pos - p.z, row.pos - p.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[4 * j + i] = fmaf(-slope, (float)back[i], x[4 * j + i]);
                    if (windowed && back[i] >= a.window) x[4 * j + i] = -INFINITY;
                }
            }
        }
        f[0] = f[1] = 1.f;
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) f[h] = fmaxf(f[h] * post, 0x1p-126f);
    }
    if (edge) {
        const int more = row.last - t;   // tokens after t that the row sees
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 16 * (i >> 2) + (i & 3) <= more ? x[i] : -INFINITY;
    }
}

__device__ __forceinline__ Row row_of(const Fp8Queries &a, const Place &p, int row)
{
    const int i = row / a.r;
    Row x;
    x.last = i < p.count ? p.len - p.count + i : -1;
    x.pos = p.next - p.count + i;
    x.slope = a.slopes ? a.slopes[p.kvh * a.r + row - i * a.r] : 0.f;
    x.factor = 1.f;
    return x;
}
// Tokens [lo, hi) that rows first .. last (clamped to the live ones) can see: positions are distinct and grow, so a token that is at most
// window - 1 positions back is at most as many tokens back.
__device__ __forceinline__ void key_range(const Fp8Queries &a, const Place &p, int first_row, int last_row, int &lo, int &hi)
{
    const int i0 = first_row / a.r, i1 = min(last_row / a.r, p.count - 1);
    hi = i0 <= i1 ? max(p.len - p.count + i1 + 1, 0) : 0;
    lo = 0;
    if (a.window > 0) lo = (int)min(max((int64_t)p.len - p.count + i0 + 1 - a.window, (int64_t)0), (int64_t)hi) & ~63;
}

// 64 tokens as operands of both products, for the four waves of a workgroup that walk the same keys: two read and convert K, two V, half of
// the tokens each.  (All four with a part of both takes 10 loads each instead of 4 or 8, and the four issue theirs together behind a barrier:
// 16 cycles of address work per load.)
template <int D>
struct Tile {
    half8v k[Shape<D>::kSteps][4][64];   // of 16 tokens each
    half8v v[2][Shape<D>::kTiles][64];   // of 32 tokens each
};
// What a wave reads of them: eight times a piece of a row, at strides that depend on whether it is K or V, so that no branch stands between
// the loads and a use an iteration later (registers that two branches load into are copied behind them, which waits).
template <int D>
struct Share {
    static constexpr int kV = Shape<D>::kVWords, kK = D / 16;   // words of a row that a lane takes of V, K
    uint32_t words[8 * kV];   // V [8][kV]; K [2][kK] (96 channels: [2][4] of its words 0 .. 3 and then [2][2] of the rest, V [8] and then [8])
    float scales;             // of K's and V's halves, in lanes 0 .. 3
    const uint8_t *from;
    uint32_t off, step;

    __device__ __forceinline__ Share(const Fp8View &c, int wave, int n, int g)
    {
        const bool v = wave >= 2;
        from = v ? c.v_codes : c.k_codes;
        off = v ? 4 * g * D + n * (D == 96 ? 4 : D / 16) : n * D + g * (D / 4);
        step = v ? D : D == 96 ? 4 : 4 * kV;
    }
    __device__ __forceinline__ void fetch_scales(const Fp8View &c, int64_t at, int lane)
    {
        const int64_t block = (at + 32 * (lane & 1)) >> c.log_block;
        scales = (lane & 2 ? c.v_scale : c.k_scale)[block];
    }
    // piece j of 8; p: place()
    __device__ __forceinline__ const uint8_t *place(int64_t at, int wave) const { return from + (at + 32 * (wave & 1)) * D; }
    __device__ __forceinline__ void fetch(const uint8_t *p, int wave, int lane, int j)
    {
        const uint8_t *row = p + (16 * (j >> 2) * D + (j & 3) * step);
        if constexpr (D == 96) {
            words[j] = *reinterpret_cast<const uint32_t *>(row + off);
            // V: the aligned word with channels 64 + 2n and 65 + 2n; K: words 4 and 5 of its tiles, twice
            const uint8_t *rest = wave >= 2 ? row : p + (16 * ((j >> 1) & 1) * D + 16 + 4 * (j & 1));
            words[8 + j] = *reinterpret_cast<const uint32_t *>(rest + (wave >= 2 ? off + 64 - 4 * (lane & 15) + 4 * ((lane & 15) >> 1) : off));
        } else if constexpr (D == 64) {
            words[j] = *reinterpret_cast<const uint32_t *>(row + off);
        } else if constexpr (D == 128) {
            const uint2 w = *reinterpret_cast<const uint2 *>(row + off);
            words[2 * j] = w.x;
            words[2 * j + 1] = w.y;
        } else {
            const uint4 w = *reinterpret_cast<const uint4 *>(row + off);
            words[4 * j] = w.x;
            words[4 * j + 1] = w.y;
            words[4 * j + 2] = w.z;
            words[4 * j + 3] = w.w;
        }
    }
    __device__ __forceinline__ void fetch_all(const Fp8View &c, int64_t at, int wave, int lane)
    {
        fetch_scales(c, at, lane);
        const uint8_t *p = place(at, wave);
#pragma unroll
        for (int j = 0; j < 8; ++j) fetch(p, wave, lane, j);
    }
    __device__ __forceinline__ void k(int tile, uint32_t (&w)[kK]) const
    {
#pragma unroll
        for (int i = 0; i < kK; ++i) w[i] = D == 96 ? words[i < 4 ? 4 * tile + i : 8 + 2 * tile + i - 4] : words[kK * tile + i];
    }
    __device__ __forceinline__ uint32_t v(int j, int w, int lane) const { return D == 96 ? (w ? words[8 + j] >> (16 * (lane & 1)) : words[j]) : words[kV * j + w]; }
    __device__ __forceinline__ float scale(int i) const { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scales), i)); }
};
// The operands of one word of V of 8 tokens: 4 channels, the first `n` of them
template <typename STORE>
__device__ __forceinline__ void v_operands(const uint32_t (&w)[8], int n, const STORE &store)
{
#pragma unroll
    for (int c = 0; c < n; c += 2) {
        uint32_t pair[4];   // of tokens
#pragma unroll
        for (int q = 0; q < 4; ++q) pair[q] = __builtin_amdgcn_perm(w[2 * q + 1], w[2 * q], c ? 0x07030602u : 0x05010400u);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            half8v f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const half2v h = e ? codes_hi(pair[q]) : codes_lo(pair[q]);
                f[2 * q] = h[0];
                f[2 * q + 1] = h[1];
            }
            store(c + e, f);
        }
    }
}
// left: tokens from the tile's first that exist; codes behind them may be anything, and are not to reach the product
template <int D>
__device__ __forceinline__ void lay_down(Tile<D> &to, const Share<D> &x, int wave, int lane, int left)
{
    const int half = wave & 1;
    if (wave < 2) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t w[D / 16];
            x.k(j, w);
#pragma unroll
            for (int s = 0; s < Shape<D>::kSteps; ++s) to.k[s][2 * half + j][lane] = k_operand<D>(w, s);
        }
        return;
    }
    const bool clean = left < 64 || x.scale(2 + half) < 0.f;
    int g = lane >> 4;
    if (clean) asm volatile("" : "+v"(g));   // what follows from it is computed here, not kept for the whole loop
#pragma unroll
    for (int w = 0; w < Shape<D>::kVWords; ++w) {
        uint32_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x.v(j, w, lane);
        if (clean)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // (NaN codes have a product of their own)
                const bool none = 32 * half + 16 * (j >> 2) + 4 * g + (j & 3) >= left;
                v[j] = none ? 0u : v[j] & ~((nan_codes(v[j]) >> 7) * 0xffu);
            }
        v_operands(v, min(Shape<D>::kTiles - 4 * w, 4), [&](int c, const half8v &f) { to.v[half][4 * w + c][lane] = f; });
    }
}

// Operands of products that follow each other, read from LDS four ahead: left to itself, the compiler reads each one just before its product
// and waits.
constexpr int kAhead = 4;
constexpr int kArithmetic = 0x6;   // what may be moved across a step
template <int N, int STRIDE, typename PRODUCT>
__device__ __forceinline__ void products(half8v (&ahead)[kAhead], const half8v *operands, const PRODUCT &product)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        product(i, ahead[i % kAhead]);
        if (i + kAhead < N) ahead[i % kAhead] = operands[(i + kAhead) * STRIDE];
        __builtin_amdgcn_sched_barrier(kArithmetic);
    }
}
template <int STRIDE>
__device__ __forceinline__ void read_first(half8v (&ahead)[kAhead], const half8v *operands)
{
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i] = operands[i * STRIDE];
    __builtin_amdgcn_sched_barrier(0);
}

// Rows of a workgroup: BY_ROWS, every wave has RT tiles of its own and walks all keys, which lie in LDS as operands; else the waves share RT
// tiles and deal the keys out among them, 64 at a time, each converting what it takes in registers.
template <int D, int RT, int NW, bool BY_ROWS, bool OPT>
__global__ __launch_bounds__(64 * NW, 2) void fp8_attention_kernel(Fp8AttentionArgs a)
{
    using S = Shape<D>;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = a.in.r * a.in.n_query, hkv = a.in.c.n_kv_heads;
    // heads next to each other: with eight of them every XCD has one head's keys in its cache
    const int kvh = blockIdx.x % hkv, rest = blockIdx.x / hkv;
    const int group = rest % a.groups, run = rest / a.groups;
    __shared__ int sm_end[kMostSeqs];
    Run deal = {run, 0, 0, 0, 0};
    if (a.parts > 0 && !find_run<true>(a.in, a.parts, run, sm_end, deal)) return;
    constexpr int kTilesInLds = D == 256 ? 1 : 2;   // (of 64 and 32 KB)
    __shared__ Tile<BY_ROWS ? D : 64> sm_tile[BY_ROWS ? kTilesInLds : 1];
    int turn = 0;   // of the tiles
    int seq = deal.seq, seq_from = deal.seq_from, seq_to = 0;
    const int at_unit = deal.at, stop = deal.stop;
    for (;; seq_from = seq_to, ++seq) {   // the pieces of the run
    if (a.parts > 0) seq_to = __builtin_amdgcn_readfirstlane(sm_end[seq]);
    const bool whole = a.parts == 0 || (at_unit <= seq_from && seq_to <= stop);   // the sequence is this piece
    const Place p = place_of<true>(a.in, seq * hkv + kvh);
    const int64_t part0 = ((int64_t)(run + seq) * hkv + kvh) * rows;   // where partial results of the rows go
    const int row0 = BY_ROWS ? (group * NW + wave) * 16 * RT : group * 16 * RT;

    // queries: in registers for one tile of up to 128 channels, else in LDS (the registers then hold two tiles' results or 256 channels' of one)
    constexpr bool kQueriesInLds = !BY_ROWS && (RT > 1 || D == 256);
    __shared__ half8v sm_q[kQueriesInLds ? RT : 1][kQueriesInLds ? S::kSteps : 1][64];
    Row row[RT];
    half8v q_reg[kQueriesInLds ? 1 : RT][S::kSteps];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int at = row0 + 16 * rt + n;
        row[rt] = row_of(a.in, p, at);
        half8v (&qf)[S::kSteps] = q_reg[kQueriesInLds ? 0 : rt];
        load_query<D>(qf, row[rt].factor, a.in, p.seq, p.kvh, at, at < p.count * a.in.r, g);
        if constexpr (kQueriesInLds) {
            if (wave == 0)
#pragma unroll
                for (int s = 0; s < S::kSteps; ++s) sm_q[rt][s][lane] = qf[s];
        }
    }
    if constexpr (kQueriesInLds) __syncthreads();
    int q_lane = lane;
    const auto query = [&](int rt, int s) -> half8v {
        if constexpr (kQueriesInLds) return sm_q[rt][s][q_lane];
        else return q_reg[rt][s];
    };
    const auto keys_of = [&](int first_row, int end_row, int &lo, int &hi) {   // of the run's
        key_range(a.in, p, first_row, min(end_row, rows) - 1, lo, hi);
        if (whole) return;
        const int64_t from = first_visible(a.in, p.len, p.count);
        lo = (int)max(from + (int64_t)(max(at_unit, seq_from) - seq_from) * 64, (int64_t)lo);
        hi = (int)min(from + (int64_t)(min(stop, seq_to) - seq_from) * 64, (int64_t)hi);
    };
    int lo, hi;
    keys_of(row0, row0 + 16 * RT, lo, hi);
    // the first token that some live row does not see, and the largest position of a live row
    const int sees_all = p.len - p.count + min(row0 / a.in.r, max(p.count - 1, 0)) + 1;
    const int pos_most = p.next - p.count + min((row0 + 16 * RT - 1) / a.in.r, p.count - 1);
    const int32_t *pos = OPT && (a.in.slopes || a.in.window > 0) ? a.in.c.pos + (int64_t)p.stream * a.in.c.t_capacity : nullptr;

    float m[RT], m_most[RT], l[RT];   // the numerators' reference, the largest score that it serves, the numerators' sum
    float4v o[RT][S::kTiles];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = m_most[rt] = -INFINITY;
        l[rt] = 0.f;
#pragma unroll
        for (int ct = 0; ct < S::kTiles; ++ct) o[rt][ct] = float4v{0.f, 0.f, 0.f, 0.f};
    }
    bool large = false;   // a row of the wave has scores of 2^20 or more
    int unit = 0, unit_most = 0;   // exponent field of the V scale that o is in units of, and the largest one (0: none yet, o = 0)

    const uint32_t k_off = n * D + g * (D / 4), v_off = 4 * g * D + n * (D == 96 ? 4 : D / 16);
    const StreamMap map = a.in.c.map.of(p.stream);
    int first = lo + 64 * wave, last = hi;
    Share<D> share(a.in.c, wave, n, g);
    if constexpr (BY_ROWS) {
        keys_of(group * NW * 16 * RT, (group + 1) * NW * 16 * RT, first, last);
        if (first < last) share.fetch_all(a.in.c, map.pos(first), wave, lane);
    }
    for (int t0 = first; t0 < last; t0 += BY_ROWS ? 64 : 64 * NW) {
        uint32_t kw[4][S::kKWords], vw[16][S::kVWords];
        float ks[2], vs[2];
        int64_t next = 0;
        if constexpr (BY_ROWS) {
            // a tile may be overwritten when all waves are past it: with two of them, that is known from the barrier of the one after it
            if (kTilesInLds == 1) __syncthreads();
            else turn ^= 1;
            lay_down<D>(sm_tile[turn], share, wave, lane, last - t0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ks[h] = fabsf(share.scale(h));
                vs[h] = share.scale(2 + h);
            }
            __syncthreads();
            next = map.pos(min(t0 + 64, (last - 1) & ~63));   // (behind the last tile: it again)
            if (t0 < lo || t0 >= hi) {
                share.fetch_all(a.in.c, next, wave, lane);
                continue;
            }   // not this wave's rows'
        } else {
            const int64_t at = map.pos(t0);
#pragma unroll
            for (int j = 0; j < 4; ++j) load_k<D>(kw[j], a.in.c.k_codes + at * D + 16 * j * D, k_off);
#pragma unroll
            for (int j = 0; j < 16; ++j) load_v<D>(vw[j], a.in.c.v_codes + at * D + (16 * (j >> 2) + (j & 3)) * D, v_off, n);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t block = (at + 32 * h) >> a.in.c.log_block;
                ks[h] = fabsf(scalar_load(a.in.c.k_scale + block));
                vs[h] = scalar_load(a.in.c.v_scale + block);
            }
        }
        const bool edge = t0 + 64 > sees_all;
        const bool windowed = OPT && a.in.window > 0 && (int64_t)pos_most - t0 >= a.in.window;

        half8v ahead[BY_ROWS ? kAhead : 1];
        if constexpr (kQueriesInLds) asm volatile("" : "+v"(q_lane));   // read again every time, not kept in registers
        float4v s[RT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][j] = float4v{0.f, 0.f, 0.f, 0.f};
        }
        if constexpr (BY_ROWS) {
            // the next tile is requested between the products: 8 loads of four waves at once stand 500 cycles in line for their addresses
            share.fetch_scales(a.in.c, next, lane);
            const uint8_t *p_next = share.place(next, wave);
            read_first<64>(ahead, &sm_tile[turn].k[0][0][lane]);
            constexpr int kProducts = 4 * S::kSteps;
            products<kProducts, 64>(ahead, &sm_tile[turn].k[0][0][lane], [&](int i, const half8v &k) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][i % 4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, query(rt, i / 4), s[rt][i % 4], 0, 0, 0);
                if ((i + 1) * 8 / kProducts > i * 8 / kProducts) share.fetch(p_next, wave, lane, i * 8 / kProducts);
            });
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int q = 0; q < S::kSteps; ++q) {
                    const half8v k = k_operand<D>(kw[j], q);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) s[rt][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, query(rt, q), s[rt][j], 0, 0, 0);
                }
        }
        float x[RT][16], f[RT][2], by[RT];
        bool moved = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[rt][i] = s[rt][i >> 2][i & 3];
            to_scores<OPT>(x[rt], f[rt], ks, a.in, kLog2e, row[rt], t0 + 4 * g, pos, edge, windowed);
            float most = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float top = x[rt][8 * h];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, x[rt][8 * h + i]);
                most = fmaxf(most, top * f[rt][h]);
            }
            const float one[1] = {most};
            most = fold_rows(one, MaxF());
            // The reference moves when a score is far above the last ones: to 2^11 below it, so that numerators stay below 2^15 and fp16's smallest step is
            // 2^-35 of the largest or less (2^-24 of it, with the reference at the score, leaves nothing of many tokens of 2^-26 each).
            // Scores of 2^20 and more, whose own steps are large, are the reference themselves.
            by[rt] = 1.f;
            if (most > m_most[rt]) {
                m_most[rt] = most + 4.f;
                const float to = fabsf(most) < 0x1p20f ? most - 11.f : most;
                by[rt] = exp2_(m[rt] - to);
                m[rt] = to;
                l[rt] *= by[rt];
            }
            moved |= by[rt] != 1.f;
        }
        const bool some_moved = __any(moved);
        if constexpr (!OPT) {
            // Of scores whose steps are large, rounded ones, as their largest is: the exponent's multiply-add takes their factor in unrounded, and half a
            // step above the reference is beyond fp16 from scores of 2^28 on.
            if (some_moved) {
                bool now = false;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) now |= fabsf(m[rt]) >= 0x1p20f && m[rt] != -INFINITY;
                large |= __any(now);
            }
            if (large) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        x[rt][i] *= f[rt][i >> 3];
                        asm volatile("" : "+v"(x[rt][i]));   // (not contracted, and not computed without the branch)
                    }
                    f[rt][0] = f[rt][1] = 1.f;
                }
            }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (t0 + 32 * half >= hi) break;
            if constexpr (BY_ROWS) read_first<64>(ahead, &sm_tile[turn].v[half][0][lane]);
            // o is in units of a block's scale.  Blocks of a scale up to 2^6 smaller enter with numerators that are smaller by as much (a power of two,
            // which costs bits only below 2^-19 of the largest numerator); others bring o to their unit, up or down, but no further down from the
            // largest scale so far than a binary32 has room for (2^68, beside 2^49 for the sum itself).
            const int field = field_of_scale(vs[half]);
            int shift = 0;
            if (field > unit || field < unit - 6) {
                unit_most = max(unit_most, field);
                const int to = max(field, unit_most - 68);
                shift = unit - to;
                unit = to;
            }
            const int fold = min(unit - field, 60);   // from 40 on fp16 leaves nothing of the numerators
            if (half == 0 ? shift != 0 || some_moved : shift != 0) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float f = ldexpf(half == 0 ? by[rt] : 1.f, shift);
#pragma unroll
                    for (int ct = 0; ct < S::kTiles; ++ct) {
                        asm volatile("" : "+v"(o[rt][ct]));   // a branch, not a multiplication by 1 for the many blocks that leave o as it is
                        o[rt][ct] *= f;
                    }
                }
            }
            half8v pf[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float ref = (m[rt] == -INFINITY ? 0.f : m[rt]) + (float)fold;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e = exp2_(fmaf(x[rt][8 * half + i], f[rt][half], -ref));
                    sum += e;
                    pf[rt][i] = (_Float16)e;
                }
                l[rt] += ldexpf(sum, fold);
            }
            const bool flagged = vs[half] < 0.f;
            if (edge || windowed || flagged) {
                // what no row of the wave sees must not reach the product, whatever its codes
                const bool cut = !BY_ROWS && t0 + 32 * half + 32 > hi;
                if (cut) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (t0 + 32 * half + 16 * (j >> 2) + 4 * g + (j & 3) >= hi)
#pragma unroll
                            for (int w = 0; w < S::kVWords; ++w) vw[8 * half + j][w] = 0;
                }
                if (flagged) {
                    // NaN codes reach only the rows that see them: a product of their own of marks (1.0 for a NaN) and of who sees whom
                    half8v see[RT];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int t = t0 + 32 * half + 16 * (j >> 2) + 4 * g + (j & 3);
                            bool yes = t <= row[rt].last;
                            if (OPT && a.in.window > 0) yes = yes && (int64_t)row[rt].pos - pos[t] < a.in.window;
                            see[rt][j] = yes ? (_Float16)1.f : (_Float16)0.f;
                        }
                    if constexpr (BY_ROWS) {
                        const uint8_t *v = a.in.c.v_codes + (map.pos(t0) + 32 * half) * D;
#pragma unroll
                        for (int j = 0; j < 8; ++j) load_v<D>(vw[8 * half + j], v + (16 * (j >> 2) + (j & 3)) * D, v_off, n);
                    }
#pragma unroll
                    for (int w = 0; w < S::kVWords; ++w) {
                        uint32_t mark[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const uint32_t nan = nan_codes(vw[8 * half + j][w]) >> 7;
                            mark[j] = nan * 0x38u;                      // 0x38: 1.0
                            vw[8 * half + j][w] &= ~(nan * 0xffu);
                        }
                        constexpr int kPer = 4;
#pragma unroll
                        for (int c = 0; c < kPer; ++c) {
                            const int ct = 4 * w + c;
                            if (ct >= S::kTiles) break;
                            half8v f;
#pragma unroll
                            for (int j = 0; j < 8; ++j) f[j] = (mark[j] >> (8 * c)) & 0xffu ? (_Float16)1.f : (_Float16)0.f;
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt) {
                                const float4v seen = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, see[rt], float4v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                                for (int i = 0; i < 4; ++i) o[rt][ct][i] = seen[i] > 0.f ? __builtin_nanf("") : o[rt][ct][i];
                            }
                        }
                    }
                }
            }
            if constexpr (BY_ROWS) {
                products<S::kTiles, 64>(ahead, &sm_tile[turn].v[half][0][lane], [&](int ct, const half8v &f) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) o[rt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, pf[rt], o[rt][ct], 0, 0, 0);
                });
                continue;
            }
#pragma unroll
            for (int w = 0; w < S::kVWords; ++w) {
                uint32_t v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = vw[8 * half + j][w];
                v_operands(v, min(S::kTiles - 4 * w, 4), [&](int c, const half8v &f) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) o[rt][4 * w + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, pf[rt], o[rt][4 * w + c], 0, 0, 0);
                });
            }
        }
    }

    // results of the wave, normalised: o / l * 2^unit
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float one[1] = {l[rt]};
        l[rt] = fold_rows(one, AddF());
        const float inv = l[rt] == 0.f ? 0.f : 1.f / l[rt];
#pragma unroll
        for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[rt][ct][i] = ldexpf(o[rt][ct][i] * inv, max(unit, 1) - 127);
    }
    if constexpr (BY_ROWS) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int at = row0 + 16 * rt + n;
            if (at >= p.count * a.in.r) continue;
            if (whole) {
                if (g == 0) store_lse(a, p, at, m[rt], l[rt]);
            } else if (g == 0) {
                float *ml = a.part_ml + (part0 + at) * 2;
                ml[0] = m[rt];
                ml[1] = l[rt];
            }
            // a lane has the channels of operand rows 4g .. 4g+3: runs of neighbours
            constexpr int kMain = D == 96 ? 4 : S::kTiles;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y[S::kTiles];
#pragma unroll
                for (int ct = 0; ct < S::kTiles; ++ct) y[ct] = o[rt][ct][i];
                if (whole) {
                    store_row<D>(a, p, at, channel_of<D>(4 * g + i, 0), y, kMain);
                    if constexpr (D == 96) store_row<D>(a, p, at, channel_of<D>(4 * g + i, 4), y + 4, 2);
                } else {
                    float *to = a.part_o + (part0 + at) * D;
#pragma unroll
                    for (int ct = 0; ct < S::kTiles; ++ct) to[channel_of<D>(4 * g + i, ct)] = y[ct];
                }
            }
        }
    } else {
        // rows that the waves bring together at a time: 32 to 34 KB of LDS
        constexpr int kAtOnce = (D == 256 ? 8 : 16) * 4 / NW, kPad = 4;
        __shared__ float sm_o[NW][kAtOnce][D + kPad];
        __shared__ float sm_m[NW][kAtOnce], sm_l[NW][kAtOnce];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int part = 0; part < 16 / kAtOnce; ++part) {
                const int from = row0 + 16 * rt + part * kAtOnce, here = min(rows - from, kAtOnce);
                if (here <= 0) break;
                if (rt + part > 0) __syncthreads();
                if (n / kAtOnce == part) {
                    const int q = n % kAtOnce;
                    if (g == 0) {
                        sm_m[wave][q] = m[rt];
                        sm_l[wave][q] = l[rt];
                    }
#pragma unroll
                    for (int ct = 0; ct < S::kTiles; ++ct)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sm_o[wave][q][channel_of<D>(4 * g + i, ct)] = o[rt][ct][i];
                }
                __syncthreads();
                for (int e = threadIdx.x; e < here * (D / 4); e += 64 * NW) {
                    const int q = e / (D / 4), c = (e % (D / 4)) * 4, at = from + q;
                    if (at >= p.count * a.in.r) continue;
                    float top = -INFINITY;
                    for (int w = 0; w < NW; ++w) top = fmaxf(top, sm_m[w][q]);
                    const float ref = top == -INFINITY ? 0.f : top;
                    float sum = 0.f, share[NW], y[4] = {0.f, 0.f, 0.f, 0.f};
                    for (int w = 0; w < NW; ++w) {
                        share[w] = sm_l[w][q] * exp2_(sm_m[w][q] - ref);
                        sum += share[w];
                    }
                    // parts of 1: a sum of many results near a binary32's largest need not be one, though their mean is
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    for (int w = 0; w < NW; ++w)
                        for (int i = 0; i < 4; ++i) y[i] = fmaf(share[w] * inv, sm_o[w][q][c + i], y[i]);
                    if (whole) {
                        store_row<D>(a, p, at, c, y, 4);
                        if (c == 0) store_lse(a, p, at, top, sum);
                    } else {
                        const int64_t slot = part0 + at;
                        *reinterpret_cast<float4 *>(a.part_o + slot * D + c) = make_float4(y[0], y[1], y[2], y[3]);
                        if (c == 0) {
                            a.part_ml[2 * slot] = top;
                            a.part_ml[2 * slot + 1] = sum;
                        }
                    }
                }
            }
    }
    if (a.parts == 0 || seq_to >= stop) break;
    if constexpr (!BY_ROWS) __syncthreads();   // before the next piece's results take these places
    }
}

// The pieces of a row together: sum_s l_s 2^(m_s - m) o_s / sum_s l_s 2^(m_s - m).  A wave takes a row of a (sequence, KV head) that was
// cut: the factors of 64 pieces in its lanes, then the pieces' results one after the other, a lane D / 64 channels (two of 48 lanes at
// 96), with TOGETHER loads in flight: eight over the 16-bit cache where there are many pieces (of eight sequences, 16 each, 256 channels, 5.6 us, four 6.7; of one of
// 32k tokens the call 29.4 and 30.7; but of 64 sequences, two or so each, 6.7 and 6.0; over the 8-bit cache 55.9 and 55.4 for the call of drafts).  (A thread that read every piece's factors itself took 20 us for the 64 pieces of one sequence of 32k.)
constexpr int kMergeRows = 4;
template <int D, int TOGETHER = 4>
__global__ __launch_bounds__(64 * kMergeRows) void fp8_merge_kernel(Fp8AttentionArgs a)
{
    constexpr int kPer = D <= 128 ? 2 : 4, kTogether = TOGETHER;   // channels per lane, pieces whose loads are on their way together
    const int rows = a.in.r * a.in.n_query, hkv = a.in.c.n_kv_heads, groups = (rows + kMergeRows - 1) / kMergeRows;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kvh = blockIdx.x % hkv, rest = blockIdx.x / hkv, row = rest % groups * kMergeRows + wave, seq = rest / groups;
    const Place p = place_of<false>(a.in, seq * hkv + kvh);   // (requested before the rest)
    int end[kMostSeqs / 64], from = 0, to = 0;
    const int all = __builtin_amdgcn_readfirstlane(ends_of<true>(a.in, end)), per = run_length(all, a.parts);
#pragma unroll
    for (int i = 0; i < kMostSeqs / 64; ++i) {
        const int before = __shfl(end[i], (seq - 1) & 63), here = __shfl(end[i], seq & 63);
        if (seq > 0 && (seq - 1) / 64 == i) from = before;
        if (seq / 64 == i) to = here;
    }
    from = __builtin_amdgcn_readfirstlane(from);
    to = __builtin_amdgcn_readfirstlane(to);
    const int first_run = from / per, pieces = (to - 1) / per - first_run + 1;
    if (pieces == 1) return;   // written already
    if (row >= p.count * a.in.r) return;
    const int64_t first = ((int64_t)(first_run + seq) * hkv + kvh) * rows + row, step = (int64_t)hkv * rows;
    const int c = min(lane * kPer, D - kPer);
    float top = -INFINITY, sum = 0.f, y[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) y[i] = 0.f;
    float2 ml;   // of the lane's piece
    const auto load_ml = [&](int s0) {
        ml = make_float2(-INFINITY, 0.f);
        if (s0 + lane < pieces) ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (first + (s0 + lane) * step));
    };
    for (int s0 = 0; s0 < pieces; s0 += 64) {
        load_ml(s0);
        const float most_of_row[1] = {row_max(ml.x)};
        const float most = fold_rows(most_of_row, MaxF());
        if (most > top) {
            sum *= exp2_(top - most);
            top = most;
        }
        const float sum_of_row[1] = {row_sum(ml.y * exp2_(ml.x - (top == -INFINITY ? 0.f : top)))};
        sum += fold_rows(sum_of_row, AddF());
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    for (int s0 = 0; s0 < pieces; s0 += 64) {
        if (pieces > 64) load_ml(s0);
        const float share = ml.y * exp2_(ml.x - (top == -INFINITY ? 0.f : top)) * inv;   // parts of 1, as above
        const int here = min(pieces - s0, 64);
        for (int s = 0; s < here; s += kTogether) {
            float v[kTogether][kPer];
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {   // (past the last piece: it again, with no weight)
                const float *o = a.part_o + (first + (s0 + min(s + k, here - 1)) * step) * D + c;
                if constexpr (kPer == 2) {
                    const float2 x = *reinterpret_cast<const float2 *>(o);
                    v[k][0] = x.x;
                    v[k][1] = x.y;
                } else {
                    const float4 x = *reinterpret_cast<const float4 *>(o);
                    v[k][0] = x.x;
                    v[k][1] = x.y;
                    v[k][2] = x.z;
                    v[k][3] = x.w;
                }
            }
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                const float w = s + k < here ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, share), min(s + k, 63))) : 0.f;
                if (s + k < here)
#pragma unroll
                    for (int i = 0; i < kPer; ++i) y[i] = fmaf(w, v[k][i], y[i]);
            }
        }
    }
    if (lane * kPer < D) store_row<D>(a, p, row, c, y, kPer);
    if (lane == 0) store_lse(a, p, row, top, sum);
}

// ---- the weight of every token -------------------------------------------------------------------------------------------

// Query operands of up to this many tiles of 16 rows in LDS at a time: 32 KB at 128 channels, 64 at 256
constexpr int kWeightTiles = 8;

// exp(s - lse) as 2^(x f - l) where no option changes the score x f: f takes |scale| * log2 e in, rounded once, and l is lse times the very
// factor that this makes of log2 e, so that the rounding costs only where s and lse differ.
__device__ __forceinline__ float scale2_of(float scale) { return fabsf(scale) * kLog2e; }
__device__ __forceinline__ double log2e_of(float scale)
{
    const double s = fabs((double)scale), s2 = (double)scale2_of(scale);
    return s > 0.0 && s2 > 0.0 && s2 < 3e38 ? s2 / s : 1.4426950408889634;
}

// A wave takes 64 tokens at a time, their K operands in registers, against the rows in LDS; the sums over rows stay in registers
// until all tiles are done.  More rows than fit go in rounds that add to what the first wrote, each token in the same lane.
// One query over 16 x 32k tokens: 104 us, 5.3 TB/s of K.  32 queries of four heads over 8k: 95 us, 0.73 PFLOP/s; per pair a multiply-add, an
// exponential and an addition beside the products, and vector and matrix instructions of the two waves of a SIMD hide each other only in part.
template <int D, bool OPT>
__global__ __launch_bounds__(kThreads, 2) void fp8_weights_kernel(Fp8WeightsArgs a)
{
    using S = Shape<D>;
    __shared__ half8v sm_q[kWeightTiles][S::kSteps][64];
    __shared__ Row sm_row[kWeightTiles * 16];
    __shared__ float sm_lse[kWeightTiles * 16];
    __shared__ int sm_last[kWeightTiles];   // the first row of a tile that sees least
    __shared__ int sm_end[kMostSeqs];
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hkv = a.in.c.n_kv_heads, run = blockIdx.x / hkv, kvh = blockIdx.x - run * hkv;
    const uint32_t k_off = n * D + g * (D / 4);
    const float scale2 = scale2_of(a.in.scale);
    const double to_log2 = log2e_of(a.in.scale);
    Run deal = {run, 0, 0, 0, 0};
    if (a.parts > 0 && !find_run<false>(a.in, a.parts, run, sm_end, deal)) return;
    int seq = deal.seq, seq_from = deal.seq_from, seq_to = 0;
    for (;; seq_from = seq_to, ++seq) {   // the pieces of the run
        const Place p = place_of<true>(a.in, seq * hkv + kvh);
        const int rows = p.count * a.in.r;
        int from = 0, to = p.len;
        if (a.parts > 0) {
            seq_to = __builtin_amdgcn_readfirstlane(sm_end[seq]);
            from = (max(deal.at, seq_from) - seq_from) * 64;
            to = (int)min((int64_t)(min(deal.stop, seq_to) - seq_from) * 64, (int64_t)to);
        }
        const int32_t *pos = OPT && (a.in.slopes || a.in.window > 0) ? a.in.c.pos + (int64_t)p.stream * a.in.c.t_capacity : nullptr;
        float *weight = a.in.c.weight + (int64_t)p.stream * a.in.c.t_capacity;
        const StreamMap map = a.in.c.map.of(p.stream);
        for (int first = 0; first < max(rows, 1); first += 16 * kWeightTiles) {
            const int tiles = (min(rows - first, 16 * kWeightTiles) + 15) / 16;
            __syncthreads();   // the last round's rows are not needed any more
            for (int tile = wave; tile < tiles; tile += kWaves) {
                const int at = first + 16 * tile + n;
                half8v qf[S::kSteps];
                Row row = row_of(a.in, p, at);
                load_query<D>(qf, row.factor, a.in, p.seq, p.kvh, at, at < rows, g);
                const int i = at / a.in.r, h = at - i * a.in.r;
                float lse = INFINITY;
                if (at < rows) lse = a.lse[((int64_t)p.seq * hkv * a.in.r + p.kvh * a.in.r + h) * a.in.n_query + i];
                // a NaN becomes the row's products', so that only tokens that it sees get it: -inf - NaN would be one for all of them
                const bool none = lse != lse;
                if (none) lse = 0.f;
#pragma unroll
                for (int s = 0; s < S::kSteps; ++s) {
                    if (none) qf[s][0] = (_Float16)__builtin_nanf("");
                    sm_q[tile][s][lane] = qf[s];
                }
                if (lse == -INFINITY) {   // a row that saw nothing adds nothing
                    lse = INFINITY;
                    row.last = -1;
                }
                if constexpr (!OPT) {
                    row.factor *= scale2;
                    lse = (float)((double)lse * to_log2);
                }
                int least = row.last;
                for (int o = 1; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o));
                if (g == 0) {
                    sm_lse[16 * tile + n] = lse;
                    sm_row[16 * tile + n] = row;
                }
                if (lane == 0) sm_last[tile] = least;
            }
            __syncthreads();
            int lo, hi;
            key_range(a.in, p, first, min(first + 16 * kWeightTiles, rows) - 1, lo, hi);
            for (int t0 = from + 64 * wave; t0 < to; t0 += 64 * kWaves) {
                float sum[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] = 0.f;
                if (rows > 0 && t0 < hi && t0 + 64 > lo) {
                    const int64_t at = map.pos(t0);
                    uint32_t kw[4][S::kKWords];
#pragma unroll
                    for (int j = 0; j < 4; ++j) load_k<D>(kw[j], a.in.c.k_codes + at * D + 16 * j * D, k_off);
                    const float ks[2] = {fabsf(scalar_load(a.in.c.k_scale + (at >> a.in.c.log_block))), fabsf(scalar_load(a.in.c.k_scale + ((at + 32) >> a.in.c.log_block)))};
                    half8v kf[4][S::kSteps];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int s = 0; s < S::kSteps; ++s) kf[j][s] = k_operand<D>(kw[j], s);
                    // a tile's operands and factors are read from LDS while the last one's exponentials run
                    half8v q[S::kSteps];
                    float next_lse, next_c;
                    int next_last;
                    const auto read_tile = [&](int tile) {
#pragma unroll
                        for (int s = 0; s < S::kSteps; ++s) q[s] = sm_q[tile][s][lane];
                        next_lse = sm_lse[16 * tile + n];
                        next_c = sm_row[16 * tile + n].factor;
                        next_last = sm_last[tile];
                    };
                    read_tile(0);
                    for (int tile = 0; tile < tiles; ++tile) {
                        float4v x[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[j] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int s = 0; s < S::kSteps; ++s)
#pragma unroll
                            for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[j][s], q[s], x[j], 0, 0, 0);
                        const float lse = next_lse, c = next_c;
                        const bool edge = t0 + 63 > __builtin_amdgcn_readfirstlane(next_last);
                        read_tile(min(tile + 1, tiles - 1));
                        float y[16], f[2];
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = x[i >> 2][i & 3];
                        if constexpr (OPT) {
                            const Row row = sm_row[16 * tile + n];
                            to_scores<true>(y, f, ks, a.in, 1.f, row, t0 + 4 * g, pos, edge, a.in.window > 0);
#pragma unroll
                            for (int i = 0; i < 16; ++i) sum[i] += exp2_((y[i] - lse) * kLog2e);
                        } else {
#pragma unroll
                            for (int h = 0; h < 2; ++h) f[h] = fmaxf(ks[h] * c, 0x1p-126f);
                            if (edge) {
                                const int more = sm_row[16 * tile + n].last - (t0 + 4 * g);   // tokens after the lane's first that the row sees
#pragma unroll
                                for (int i = 0; i < 16; ++i) y[i] = 16 * (i >> 2) + (i & 3) <= more ? y[i] : -INFINITY;
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i) sum[i] += exp2_(fmaf(y[i], f[i >> 3], -lse));
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] = row_sum(sum[i]);
                if (n < 4) {   // lane 16 g + n writes tokens 16 n + 4 g .. + 3
                    float4 v;
                    v.x = n == 0 ? sum[0] : n == 1 ? sum[4] : n == 2 ? sum[8] : sum[12];
                    v.y = n == 0 ? sum[1] : n == 1 ? sum[5] : n == 2 ? sum[9] : sum[13];
                    v.z = n == 0 ? sum[2] : n == 1 ? sum[6] : n == 2 ? sum[10] : sum[14];
                    v.w = n == 0 ? sum[3] : n == 1 ? sum[7] : n == 2 ? sum[11] : sum[15];
                    const int t = t0 + 16 * n + 4 * g;
                    float *w = weight + t;
                    const bool add = a.accumulate || first > 0;
                    if (t + 3 < to) {
                        float4 old = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (add) old = *reinterpret_cast<const float4 *>(w);
                        *reinterpret_cast<float4 *>(w) = make_float4(old.x + v.x, old.y + v.y, old.z + v.z, old.w + v.w);
                    } else {
                        const float y[4] = {v.x, v.y, v.z, v.w};
                        for (int i = 0; i < 4; ++i)
                            if (t + i < to) w[i] = (add ? w[i] : 0.f) + y[i];
                    }
                }
            }
        }
        if (a.parts == 0 || seq_to >= deal.stop) break;
    }
}

// How many rows a workgroup of the attention takes, and how.  Up to 128 channels: two tiles of 16 from 17 rows on, as K and V are converted once
// for both (32 sequences, 20 rows 67 us, in two groups of one tile 81).  Up to 256 rows the waves share them and deal out the keys, with more
// every wave has rows of its own and the keys lie in LDS (one sequence of 16k tokens: 128 rows 31 us against 41 with rows of their own, 256 rows 41
// and 47, 1024 rows 126 and 101; 32 sequences of 700 to 6000 tokens: 128 rows both 128, 256 rows 215 and 209; 64 channels, 256 rows 30 and 35).
// At 256 channels the registers hold one tile, and sharing the conversions counts from the second on (the same 32 sequences, 32 rows 166 and 122
// us, 256 rows 636 and 372; one sequence, 32 rows over 16k tokens 33 and 35, 20 rows over 2k 33 and 19).
struct Rows {
    int tiles;      // per wave (RT)
    bool by_rows;
    int per_group;
};
Rows rows_of(int64_t rows, int d)
{
    Rows x;
    x.by_rows = rows > (d == 256 ? 16 : 256);
    x.tiles = d == 256 || rows <= 16 ? 1 : 2;
    x.per_group = 16 * x.tiles * (x.by_rows ? kWaves : 1);
    return x;
}

// Workgroups of eight waves that share a sequence's rows, instead of four:
// few workgroups over short caches, where nothing is then left to merge (8 heads, 32 query heads of 128 channels, one token: 1.1k tokens 14.7 us
// against 18.7 with runs, merged; 2k 17.7 and 19.4; 3k 22.3 and 19.3), and
bool eight_waves(int64_t workgroups, int64_t bound) { return workgroups <= 256 && bound <= 2048; }
// long runs, which make half as many pieces then (16 sequences x 32k tokens 185.6 -> 181.4 us, 8 of them with 256 channels 201 -> 186); shorter
// ones change from sequence to sequence more often, where eight waves wait for each other (32 sequences of 700 to 6000 tokens, five
// queries: 72.5 -> 77.5).
bool long_runs(int64_t n_seq, int64_t across, int64_t bound) { return across <= 256 && n_seq * ((bound + 63) / 64) * across >= 128 * 256; }

template <int D, int RT, int NW, bool BY_ROWS>
void launch_rt(const Fp8AttentionArgs &a, uint32_t grid, bool opt, hipStream_t s)
{
    if (opt) fp8_attention_kernel<D, RT, NW, BY_ROWS, true><<<grid, 64 * NW, 0, s>>>(a);
    else fp8_attention_kernel<D, RT, NW, BY_ROWS, false><<<grid, 64 * NW, 0, s>>>(a);
}

template <int D, int TOGETHER = 4>
hipError_t launch_merge_d(const Fp8AttentionArgs &a, hipStream_t s)
{
    const int64_t rows = (int64_t)a.in.r * a.in.n_query;
    fp8_merge_kernel<D, TOGETHER><<<(uint32_t)((int64_t)a.in.n_seq * a.in.c.n_kv_heads * ((rows + kMergeRows - 1) / kMergeRows)), 64 * kMergeRows, 0, s>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(Fp8AttentionArgs &a, hipStream_t s)
{
    const int64_t rows = (int64_t)a.in.r * a.in.n_query;
    const Rows x = rows_of(rows, D);
    a.groups = (int)((rows + x.per_group - 1) / x.per_group);
    const uint32_t grid = (uint32_t)((a.parts > 0 ? a.parts : a.in.n_seq) * a.in.c.n_kv_heads * a.groups);
    const bool opt = a.in.cap > 0.f || a.in.slopes || a.in.window > 0;
    const bool wide = a.parts > 0 ? long_runs(a.in.n_seq, (int64_t)a.in.c.n_kv_heads * a.groups, a.bound) : eight_waves(grid, a.bound);
    if (x.tiles == 1) {
        if (x.by_rows) launch_rt<D, 1, 4, true>(a, grid, opt, s);
        else if (wide) launch_rt<D, 1, 8, false>(a, grid, opt, s);
        else launch_rt<D, 1, 4, false>(a, grid, opt, s);
    } else if constexpr (D < 256) {
        if (x.by_rows) launch_rt<D, 2, 4, true>(a, grid, opt, s);
        else if (wide) launch_rt<D, 2, 8, false>(a, grid, opt, s);
        else launch_rt<D, 2, 4, false>(a, grid, opt, s);
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.parts == 0 ? e : launch_merge_d<D>(a, s);
}

// One round of workgroups, as above (16 sequences x 32k tokens: 104 us with 512 runs, 118 with 768, 115 with 1536).
template <int D>
hipError_t launch_weights_d(Fp8WeightsArgs &a, hipStream_t s)
{
    const int64_t units = (int64_t)a.in.n_seq * ((a.bound + 63) / 64), hkv = a.in.c.n_kv_heads;
    int64_t parts = 512 / hkv < 1 ? 1 : 512 / hkv;
    if (parts * kLeastUnits > units) parts = (units + kLeastUnits - 1) / kLeastUnits;
    a.parts = a.in.n_seq > kMostSeqs || a.in.n_seq >= 4 * parts || parts <= 1 ? 0 : (int)parts;
    const uint32_t grid = (uint32_t)((a.parts > 0 ? a.parts : a.in.n_seq) * hkv);
    if (a.in.cap > 0.f || a.in.slopes || a.in.window > 0) fp8_weights_kernel<D, true><<<grid, kThreads, 0, s>>>(a);
    else fp8_weights_kernel<D, false><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

// 512 workgroups are resident at once (two per CU; 256 of eight waves): as many runs as make one round of them (16 sequences x 32k tokens 185 us,
// in twice as many runs 200).  A batch of many more sequences than runs is left to the order in which workgroups finish.
int64_t fp8_attention_parts(int64_t n_seq, int64_t n_kv_heads, int64_t r, int64_t n_query, int d, int64_t bound)
{
    const Rows x = rows_of(r * n_query, d);
    const int64_t across = n_kv_heads * ((r * n_query + x.per_group - 1) / x.per_group);   // workgroups per run
    int64_t parts = (!x.by_rows && long_runs(n_seq, across, bound) ? 256 : 512) / across;
    if (parts < 1) parts = 1;
    if (n_seq > kMostSeqs || n_seq >= 4 * parts || (!x.by_rows && eight_waves(n_seq * across, bound))) return 0;
    const int64_t most = n_seq * ((bound + 64 * kLeastUnits - 1) / (64 * kLeastUnits));
    if (parts > most) parts = most;
    return parts <= 1 && n_seq == 1 ? 0 : parts;
}

hipError_t launch_fp8_attention(Fp8AttentionArgs &a, hipStream_t s)
{
    return a.in.d == 64 ? launch_d<64>(a, s) : a.in.d == 96 ? launch_d<96>(a, s) : a.in.d == 128 ? launch_d<128>(a, s) : launch_d<256>(a, s);
}

hipError_t launch_attention_merge(const Fp8AttentionArgs &a, hipStream_t s)
{
    // eight loads in flight where a sequence has eight pieces or more (see fp8_merge_kernel)
    const bool many = a.parts >= 8 * a.in.n_seq;
    if (a.in.d == 64) return many ? launch_merge_d<64, 8>(a, s) : launch_merge_d<64>(a, s);
    if (a.in.d == 96) return many ? launch_merge_d<96, 8>(a, s) : launch_merge_d<96>(a, s);
    if (a.in.d == 128) return many ? launch_merge_d<128, 8>(a, s) : launch_merge_d<128>(a, s);
    return many ? launch_merge_d<256, 8>(a, s) : launch_merge_d<256>(a, s);
}

hipError_t launch_fp8_weights(Fp8WeightsArgs &a, hipStream_t s)
{
    return a.in.d == 64    ? launch_weights_d<64>(a, s)
           : a.in.d == 96  ? launch_weights_d<96>(a, s)
           : a.in.d == 128 ? launch_weights_d<128>(a, s)
                           : launch_weights_d<256>(a, s);
}

}  // namespace pk
