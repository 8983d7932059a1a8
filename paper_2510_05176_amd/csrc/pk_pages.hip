// Page tables and slot maps of a step (pk_pages_update), and the append by slot (pk_kv16_append).
//
// A step's plan is three prefix sums over the sequences (new tokens, pages that come back, pages that are needed) and a lookup per new token:
// all of it together is a few bytes per sequence and token, so launches and the chain state -> sum -> page -> slot bound it: a step of 200 sequences 14 us in
// one launch (20 in two), 96 sequences with up to 8192 new tokens each, 315k rows, 17.  The append moves every vector once: 72k tokens of 8 heads of 128 channels,
// 590 MB read and written, in 115 us, 5.1 TB/s, which is what a copy reaches.
#include "pk_kv16.h"

namespace pk {

namespace {

constexpr int kPlanThreads = 1024;
// Up to so many tokens the plan's workgroup looks them up itself, and the call is one launch; and up to so many sequences with a thread each.
constexpr int kFewTokens = 4096, kFewSeqs = 1024;

// a + b, at most `most`: an associative operation on numbers in [0, most], most < 2^31
__device__ __forceinline__ uint32_t add_up_to(uint32_t a, uint32_t b, uint32_t most) { return min(a + b, most); }

// Exclusive sums over the workgroup, all of them at most `most`; before: what came before the workgroup's, and the total with it afterwards.
template <int THREADS>
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t most, uint32_t &before, uint32_t *sm)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t to = x;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = (uint32_t)__shfl_up((int)to, o);
        if (lane >= o) to = add_up_to(to, v, most);
    }
    uint32_t mine = (uint32_t)__shfl_up((int)to, 1);
    if (lane == 0) mine = 0;
    __syncthreads();   // the last call's sums are not needed any more
    if (lane == 63) sm[wave] = to;
    __syncthreads();
    uint32_t first = before;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w == wave) mine = add_up_to(mine, first, most);
        first = add_up_to(first, sm[w], most);
    }
    before = first;
    return mine;
}

struct Held {
    int tokens, next, count;
};
__device__ __forceinline__ Held held_by(const PagesArgs &a, int seq, int capacity)
{
    Held h = {0, 0, 0};
    if (seq < a.n_seq) {
        const int2 st = fp8_state(a.states, seq, capacity);
        h = {st.x, st.y, a.counts[seq]};
    }
    return h;
}
__device__ __forceinline__ int pages_of(const PagesArgs &a, int tokens) { return (tokens + (1 << a.page_shift) - 1) >> a.page_shift; }
__device__ __forceinline__ int page_at(const PagesArgs &a, int32_t entry) { return min(max(entry, 0), a.n_pages - 1); }

// What a token's place follows from, of its sequence
struct Place {
    int start, held, next, taken, first;   // first: where on the stack its first new page is; held and next before the step
};
__device__ __forceinline__ void place_token(const PagesArgs &a, int j, int seq, const Place &p)
{
    int slot = -1;
    const int k = j - p.start, t = p.held + k, logical = t >> a.page_shift, have = pages_of(a, p.held);
    if (k < p.taken) {
        int32_t *entry = a.table + (int64_t)seq * a.pages_per_seq + logical;
        int page;
        if (logical < have) {
            page = page_at(a, *entry);
        } else {
            page = page_at(a, a.free_pages[min(max(p.first - (logical - have), 0), a.n_pages - 1)]);
            if ((t & ((1 << a.page_shift) - 1)) == 0) *entry = page;
        }
        slot = (page << a.page_shift) + (t & ((1 << a.page_shift) - 1));
    }
    a.slots[j] = slot;
    if (a.positions) a.positions[j] = p.next + k;
}
__device__ __forceinline__ void no_token(const PagesArgs &a, int j)
{
    a.slots[j] = -1;
    if (a.positions) a.positions[j] = 0;
}
// The first sequence that ends behind j; starts[n_seq] > j
template <typename STARTS>
__device__ __forceinline__ int sequence_of(const STARTS &starts, int n_seq, int j)
{
    int seq = 0, end = n_seq - 1;
    while (seq < end) {
        const int mid = (seq + end) >> 1;
        if (starts[mid + 1] > j) end = mid;
        else seq = mid + 1;
    }
    return seq;
}

// The sequences' part: what comes back, states, where everything begins.  FEW: at most THREADS sequences, and the tokens' part as well.
template <int THREADS, bool FEW>
__global__ __launch_bounds__(THREADS) void pages_plan_kernel(PagesArgs a)
{
    __shared__ uint32_t sm[THREADS / 64];
    __shared__ Place sm_place[FEW ? THREADS : 1];
    __shared__ int sm_start[FEW ? THREADS + 1 : 1];
    const int capacity = a.pages_per_seq << a.page_shift, lane = threadIdx.x & 63;
    const uint32_t most_pages = (uint32_t)a.n_pages, most_tokens = (uint32_t)a.n_tokens;
    Held h = held_by(a, threadIdx.x, capacity);   // (requested before the rest)
    const uint32_t n_free = (uint32_t)min(max(*a.n_free, 0), a.n_pages);
    uint32_t back = 0;
    for (int s0 = 0; s0 < a.n_seq; s0 += THREADS) {
        if (s0 > 0) h = held_by(a, s0 + threadIdx.x, capacity);
        const int need = pages_of(a, max(h.tokens + min(h.count, 0), 0)), have = pages_of(a, h.tokens);
        if (__syncthreads_or(have > need) == 0) continue;
        const uint32_t at = sum_before<THREADS>((uint32_t)(have - need), most_pages, back, sm);
        // a wave puts the pages of its sequences on the stack, one sequence after the other
        uint64_t some = __ballot(have > need);
        while (some) {
            const int from = __ffsll((unsigned long long)some) - 1;
            some &= some - 1;
            const int first = __shfl(need, from), end = __shfl(have, from);
            const uint32_t to = n_free + (uint32_t)__shfl((int)at, from);
            const int32_t *row = a.table + (int64_t)(s0 + (threadIdx.x & ~63) + from) * a.pages_per_seq;
            for (int l = first + lane; l < end; l += 64)
                if (to + (uint32_t)(l - first) < most_pages) a.free_pages[to + (l - first)] = page_at(a, row[l]);
        }
    }
    const uint32_t there = add_up_to(n_free, back, most_pages);
    uint32_t tokens = 0, pages = 0;
    for (int s0 = 0; s0 < a.n_seq; s0 += THREADS) {
        const int seq = s0 + threadIdx.x;
        if (a.n_seq > THREADS) h = held_by(a, seq, capacity);
        const uint32_t asked = min((uint32_t)max(h.count, 0), most_tokens);
        const uint32_t start = sum_before<THREADS>(asked, most_tokens, tokens, sm);
        const int fresh = (int)(add_up_to(start, asked, most_tokens) - start);   // as many as there are rows
        const int want = h.count < 0 ? max(h.tokens + h.count, 0) : h.tokens + min(fresh, capacity - h.tokens);
        const int have = pages_of(a, h.tokens), more = max(pages_of(a, want) - have, 0);
        const uint32_t first = sum_before<THREADS>((uint32_t)min(more, a.n_pages), most_pages, pages, sm);
        if (seq >= a.n_seq) continue;
        const int got = (int)min((uint32_t)more, there > first ? there - first : 0u);
        const int taken = h.count > 0 ? (int)min((int64_t)want, (int64_t)(have + got) << a.page_shift) - h.tokens : 0;
        const int change = h.count < 0 ? want - h.tokens : taken;
        a.starts[seq] = (int)start;
        a.taken[seq] = taken;
        if constexpr (FEW) {
            sm_place[seq] = {(int)start, h.tokens, h.next, taken, (int)there - 1 - (int)first};
            sm_start[seq] = (int)start;
        } else {
            a.first[seq] = (int)there - 1 - (int)first;
        }
        *reinterpret_cast<int4 *>(a.states_out + 4 * (int64_t)seq) = make_int4(h.tokens + change, h.next + change, 0, 0);
    }
    if (threadIdx.x == 0) {
        a.starts[a.n_seq] = (int)tokens;
        *reinterpret_cast<int4 *>(a.n_free_out) = make_int4((int)(there - min(there, pages)), 0, 0, 0);
    }
    if constexpr (FEW) {
        if (threadIdx.x == 0) sm_start[a.n_seq] = (int)tokens;
        __syncthreads();   // (the stack, too, is as this workgroup left it)
        for (int j = threadIdx.x; j < a.n_tokens; j += THREADS) {
            if (j >= (int)tokens) {
                no_token(a, j);
            } else {
                const int seq = sequence_of(sm_start, a.n_seq, j);
                place_token(a, j, seq, sm_place[seq]);
            }
        }
    }
}

// The tokens' part
__global__ __launch_bounds__(256) void pages_slots_kernel(PagesArgs a)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= a.n_tokens) return;
    if (j >= a.starts[a.n_seq]) {
        no_token(a, j);
        return;
    }
    const int seq = sequence_of(a.starts, a.n_seq, j), taken = a.taken[seq];
    const int2 st = *reinterpret_cast<const int2 *>(a.states_out + 4 * (int64_t)seq);
    place_token(a, j, seq, {a.starts[seq], st.x - taken, st.y - taken, taken, a.first[seq]});
}

__global__ __launch_bounds__(256) void kv16_append_kernel(Kv16AppendArgs a)
{
    const int per_row = a.d / 8, per = a.n_kv_heads * per_row;   // pieces of 8 values of a head's vector, of a token
    const int64_t all = (int64_t)a.n_tokens * per;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (int64_t)gridDim.x * 256) {
        const int token = (int)(e / per), p = (int)(e - (int64_t)token * per), head = p / per_row, c = (p - head * per_row) * 8;
        const int slot = a.slots[token];
        if (slot < 0 || slot >= a.n_slots) continue;
        const int64_t page = slot >> a.page_shift, row = ((page * a.n_kv_heads + head) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
        const uint4 k = *reinterpret_cast<const uint4 *>(static_cast<const char *>(a.k_new) + 2 * (token * a.k_token + head * a.k_head + c));
        const uint4 v = *reinterpret_cast<const uint4 *>(static_cast<const char *>(a.v_new) + 2 * (token * a.v_token + head * a.v_head + c));
        *reinterpret_cast<uint4 *>(static_cast<char *>(a.k) + 2 * (row * a.d + c)) = k;
        *reinterpret_cast<uint4 *>(static_cast<char *>(a.v) + 2 * (row * a.d + c)) = v;
    }
}

}  // namespace

hipError_t launch_pages(const PagesArgs &a, hipStream_t s)
{
    const bool few = a.n_tokens <= kFewTokens && a.n_seq <= kFewSeqs;
    if (few && a.n_seq <= 256) pages_plan_kernel<256, true><<<1, 256, 0, s>>>(a);
    else if (few) pages_plan_kernel<kFewSeqs, true><<<1, kFewSeqs, 0, s>>>(a);
    else if (a.n_seq <= 256) pages_plan_kernel<256, false><<<1, 256, 0, s>>>(a);
    else pages_plan_kernel<kPlanThreads, false><<<1, kPlanThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || few || a.n_tokens == 0) return e;
    pages_slots_kernel<<<(a.n_tokens + 255u) / 256u, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv16_append(const Kv16AppendArgs &a, hipStream_t s)
{
    const int64_t pieces = (int64_t)a.n_tokens * a.n_kv_heads * (a.d / 8), groups = (pieces + 255) / 256;
    kv16_append_kernel<<<(uint32_t)(groups < (1 << 20) ? groups : 1 << 20), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace pk
