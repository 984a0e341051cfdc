// The order of the pairs of tokens and chosen experts by slot, on gfx950: a
// stable counting sort.
//
// A layer's pairs are cut into chunks of 4096, 8 a thread: a chunk's pairs are
// counted by slot (k_order_count), a slot's counts are summed over the chunks
// before (k_order_scan, a wave each), and each chunk places its pairs behind
// those (k_order_place).  Pairs without a choice count for a slot of their own
// behind the last.  Within a chunk each wave has counters of its own; 64 pairs
// at a time find their rank among those of the same slot by ballots over the
// slot's bits, so rows do not depend on the order of atomics.  The chunk is put
// in order in LDS first: a slot's rows then leave as a run (written from where
// they are found they were 4 bytes each, and 46 us where now 23).  One chunk
// needs the last kernel alone.
//
// 131072 x 4 x 8 byte ids, 256 slots, placed: 34 us (9 to count, 5 to scan,
// 23 to place, each by itself).
#include "rp_experts.h"

namespace rp {

constexpr int kOrderThreads = 512, kOrderWaves = kOrderThreads / kWave, kEach = 8;
constexpr int32_t kChunk = kOrderThreads * kEach;

struct OrderArgs {
    const void *ids;
    int64_t ts, ls;
    int32_t P, L, E, k;     // pairs of a layer
    uint32_t k_inv;         // p / k = p k_inv >> k_shift for p < 2^31
    int32_t k_shift;
    const int32_t *slots;
    int32_t n_chunks;
    int32_t bits;           // of a slot, 0 .. E
    int32_t *counts;        // [L][E + 1][n_chunks], then sums over the chunks before
    int32_t *totals;        // [L][E + 1]
    int32_t *rows;
    int64_t *offsets;
    int32_t *places;
};

__device__ inline int32_t token_of(const OrderArgs &a, int32_t p) {
    return (int32_t)((uint64_t)(uint32_t)p * a.k_inv >> a.k_shift);
}

// A workgroup's layer and chunk: workgroups go to the eight XCDs in turn, and the
// layers of a chunk, whose ids and places share lines, to the same one.
__device__ inline bool order_item(const OrderArgs &a, int32_t &l, int32_t &c) {
    const uint32_t i = blockIdx.x >> 3, q = i / (uint32_t)a.L;
    l = (int32_t)(i - q * a.L);
    c = (int32_t)(q * 8 + (blockIdx.x & 7));
    return c < a.n_chunks;
}

// The slots of pairs p, p + step, .. (E for none and from `end` on): 8 loads at a
// time, without branches that would part them.  NEAR: a layer's ids and places lie
// within 2^31 elements of their first.
template <class I, bool NEAR>
__device__ inline void slots_of_pairs(const OrderArgs &a, int32_t l, int32_t p, int32_t step, int32_t end,
                                      int32_t (&slot)[kEach]) {
    I id[kEach];
    const I *ids = static_cast<const I *>(a.ids) + l * a.ls;
#pragma unroll
    for (int i = 0; i < kEach; ++i) slot[i] = a.E;
    if (end == 0) return;  // (no pair at all)
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int32_t x = p + i * step < end ? p + i * step : end - 1, t = token_of(a, x), j = x - t * a.k;
        id[i] = NEAR ? ids[(uint32_t)(t * (int32_t)a.ts + j)] : ids[t * a.ts + j];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t v = (int64_t)id[i];
        slot[i] = p + i * step < end && v >= 0 && v < a.E ? (int32_t)v : a.E;
    }
    if (!a.slots) return;
    int32_t s[kEach];
    const int32_t *slots = a.slots + (int64_t)l * a.E;
#pragma unroll
    for (int i = 0; i < kEach; ++i) s[i] = slots[(uint32_t)(slot[i] < a.E ? slot[i] : 0)];
#pragma unroll
    for (int i = 0; i < kEach; ++i) slot[i] = slot[i] < a.E && s[i] >= 0 && s[i] < a.E ? s[i] : a.E;
}

template <class I, bool NEAR>
__global__ void __launch_bounds__(kOrderThreads) k_order_count(OrderArgs a) {
    extern __shared__ int32_t n[];
    int32_t l, c;
    if (!order_item(a, l, c)) return;
    const int32_t b = c * kChunk, e = a.P - b < kChunk ? a.P : b + kChunk;
    int32_t slot[kEach];
    slots_of_pairs<I, NEAR>(a, l, b + (int32_t)threadIdx.x, kOrderThreads, e, slot);
    for (int32_t s = threadIdx.x; s <= a.E; s += kOrderThreads) n[s] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (b + (int32_t)threadIdx.x + i * kOrderThreads < e) atomicAdd(&n[slot[i]], 1);
    __syncthreads();
    int32_t *out = a.counts + (int64_t)l * (a.E + 1) * a.n_chunks + c;
    for (int32_t s = threadIdx.x; s <= a.E; s += kOrderThreads) out[(int64_t)s * a.n_chunks] = n[s];
}

// A wave a slot: its counts become sums over the chunks before.
__global__ void __launch_bounds__(256) k_order_scan(OrderArgs a) {
    const int64_t s = group_index() * 4 + (threadIdx.x >> 6);
    if (s >= (int64_t)a.L * (a.E + 1)) return;
    const int lane = threadIdx.x & 63;
    int32_t *row = a.counts + s * a.n_chunks;
    int32_t before = 0;
    for (int32_t c0 = 0; c0 < a.n_chunks; c0 += kWave * 4) {
        int32_t v[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t c = c0 + lane * 4 + i;
            v[i] = c < a.n_chunks ? row[c] : 0;
            sum += v[i];
        }
        int32_t upto = sum;
        for (int d = 1; d < kWave; d <<= 1) {
            const int32_t x = __shfl_up(upto, d, kWave);
            upto += lane >= d ? x : 0;
        }
        int32_t at = before + upto - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t c = c0 + lane * 4 + i;
            if (c < a.n_chunks) row[c] = at;
            at += v[i];
        }
        before += __shfl(upto, kWave - 1, kWave);
    }
    if (lane == 0) a.totals[s] = before;
}

template <class I, bool NEAR>
__global__ void __launch_bounds__(kOrderThreads) k_order_place(OrderArgs a) {
    extern __shared__ int32_t lds[];
    const int32_t S = a.E + 1;
    __shared__ uint64_t wave_sum[kOrderWaves];
    int32_t *sorted = lds;                               // [kChunk]: slot, and pair within the chunk
    int32_t *from = sorted + kChunk;                     // [S]: a slot's first row less its first place in `sorted`
    int32_t *next = from + S + (threadIdx.x >> 6) * S;   // [waves][S]: this wave's counts, then its next places
    int32_t l, c;
    if (!order_item(a, l, c)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t b = c * kChunk, e = a.P - b < kChunk ? a.P : b + kChunk, first = b + wave * (kWave * kEach) + lane;
    int32_t slot[kEach];
    // (the sums of the first of a thread's slots, which is its only one up to 511)
    const bool one = a.n_chunks == 1;
    const int32_t each = (S + kOrderThreads - 1) / kOrderThreads, s0 = threadIdx.x * each;
    const int32_t s1 = s0 + each < S ? s0 + each : S;
    auto total_of = [&](int32_t s) { return a.totals[(int64_t)l * S + s]; };
    auto before_of = [&](int32_t s) { return a.counts[((int64_t)l * S + s) * a.n_chunks + c]; };
    const bool early = !one && s0 < S;
    const int32_t total0 = early ? total_of(s0) : 0, before0 = early ? before_of(s0) : 0;
    slots_of_pairs<I, NEAR>(a, l, first, kWave, e, slot);
    for (int32_t s = threadIdx.x; s < kOrderWaves * S; s += kOrderThreads) from[S + s] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (first + i * kWave < e) atomicAdd(&next[slot[i]], 1);
    __syncthreads();
    // A thread's slots: their rows (of all chunks) and their places in this one.
    uint64_t sum = 0;  // rows << 32 | places
    for (int32_t s = s0; s < s1; ++s) {
        uint32_t here = 0;
        for (int w = 0; w < kOrderWaves; ++w) here += (uint32_t)from[S + w * S + s];
        sum += (uint64_t)(one ? here : (uint32_t)(s == s0 ? total0 : total_of(s))) << 32 | here;
    }
    uint64_t upto = sum;
    for (int d = 1; d < kWave; d <<= 1) {
        const uint64_t v = (uint64_t)__shfl_up((unsigned long long)upto, d, kWave);
        upto += lane >= d ? v : 0;
    }
    if (lane == kWave - 1) wave_sum[wave] = upto;
    __syncthreads();
    uint64_t at = upto - sum;
    for (int w = 0; w < wave; ++w) at += wave_sum[w];
    int32_t row = (int32_t)(at >> 32), place = (int32_t)(uint32_t)at;
    for (int32_t s = s0; s < s1; ++s) {
        if (c == 0) a.offsets[(int64_t)l * S + s] = row;  // (S = E + 1: the last is the end of slot E - 1)
        const int32_t before = one ? 0 : s == s0 ? before0 : before_of(s);
        from[s] = row + before - place;
        if (!one) row += s == s0 ? total0 : total_of(s);
        for (int w = 0; w < kOrderWaves; ++w) {
            const int32_t v = from[S + w * S + s];
            from[S + w * S + s] = place;
            place += v;
            if (one) row += v;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int32_t p = first + i * kWave;
        const bool live = p < e;
        // lanes with the same slot, bit by bit, in 32-bit halves
        const uint64_t all_live = __ballot(live);
        uint32_t lo = (uint32_t)all_live, hi = (uint32_t)(all_live >> 32);
        for (int k = 0; k < a.bits; ++k) {
            const uint32_t mine = 0u - ((uint32_t)slot[i] >> k & 1u);
            const uint64_t ones = __ballot(mine != 0);
            lo &= ~((uint32_t)ones ^ mine);
            hi &= ~((uint32_t)(ones >> 32) ^ mine);
        }
        const int32_t rank = (int32_t)__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
        const int32_t all = __popc(lo) + __popc(hi);
        const int32_t base = next[slot[i]];
        __builtin_amdgcn_wave_barrier();  // (all reads of a wave's counters before the writes)
        if (live && rank == 0) next[slot[i]] = base + all;
        __builtin_amdgcn_wave_barrier();
        if (live) {
            sorted[base + rank] = slot[i] << 12 | (p - b);
            const int32_t place = slot[i] < a.E ? from[slot[i]] + base + rank : -1;
            const int32_t t = token_of(a, p), j = p - t * a.k;
            int32_t *places = a.places + (int64_t)l * a.k;
            if (NEAR) places[(uint32_t)(t * (a.L * a.k) + j)] = place;
            else places[(int64_t)t * a.L * a.k + j] = place;
        }
    }
    __syncthreads();
    int32_t *rows = a.rows + (int64_t)l * a.P;
    for (int32_t i = threadIdx.x; i < e - b; i += kOrderThreads) {
        const int32_t v = sorted[i], s = v >> 12;
        rows[from[s] + i] = s < a.E ? b + (v & (kChunk - 1)) : -1;
    }
}

inline int32_t order_chunks(int64_t P) { return (int32_t)((P + kChunk - 1) / kChunk); }

inline int check_order(const routepack_problem *p, int64_t n_tokens) {
    if (!p || n_tokens < 0 || p->n_layers < 0 || p->n_experts < 1 || p->top_k < 1) return ROUTEPACK_E_INVALID;
    if (p->n_experts > kMaxSlots || p->top_k > 256 || n_tokens > INT32_MAX / p->top_k) return ROUTEPACK_E_UNSUPPORTED;
    // (2^31 / kChunk + 1 chunks at most)
    if ((int64_t)p->n_layers * (p->n_experts + 1) > kMaxBytes >> 24) return ROUTEPACK_E_UNSUPPORTED;
    return ROUTEPACK_OK;
}

inline int64_t order_bytes(const routepack_problem *p, int64_t n_tokens) {
    const int64_t n = order_chunks(n_tokens * p->top_k);
    return n <= 1 ? 0 : (int64_t)p->n_layers * (n + 1) * (p->n_experts + 1) * 4;
}

}  // namespace rp

using namespace rp;

extern "C" int64_t routepack_order_workspace(const routepack_problem *prob, int64_t n_tokens) {
    const int rc = check_order(prob, n_tokens);
    return rc != ROUTEPACK_OK ? rc : order_bytes(prob, n_tokens);
}

extern "C" int routepack_order_tokens(const routepack_problem *prob, const routepack_ids *ids, const int32_t *slots,
                                      int32_t *rows, int64_t *offsets, int32_t *places, void *workspace,
                                      int64_t workspace_bytes, hipStream_t stream) {
    if (!ids) return ROUTEPACK_E_INVALID;
    RP_TRY(check_order(prob, ids->n_tokens));
    RP_TRY(check_ids(prob, ids, ids->n_tokens));
    if (prob->n_layers == 0) return ROUTEPACK_OK;
    const int64_t bytes = order_bytes(prob, ids->n_tokens);
    if (!offsets || workspace_bytes < bytes || (bytes > 0 && (!workspace || ((uintptr_t)workspace & 15))))
        return ROUTEPACK_E_INVALID;
    if (ids->n_tokens > 0 && (!rows || !places)) return ROUTEPACK_E_INVALID;
    OrderArgs a = {};
    a.ids = ids->data;
    a.ts = ids->token_stride;
    a.ls = ids->layer_stride;
    a.P = (int32_t)(ids->n_tokens * prob->top_k);
    a.L = prob->n_layers;
    a.E = prob->n_experts;
    a.k = prob->top_k;
    a.slots = slots;
    a.n_chunks = order_chunks(a.P) > 1 ? order_chunks(a.P) : 1;
    a.k_shift = 31;  // k_inv = ceil(2^k_shift / k), below 2^32: exact for p < 2^31
    while ((int64_t)1 << (a.k_shift - 31) < a.k) ++a.k_shift;
    a.k_inv = (uint32_t)((((uint64_t)1 << a.k_shift) + a.k - 1) / a.k);
    a.bits = 32 - __builtin_clz((unsigned)a.E);
    a.counts = static_cast<int32_t *>(workspace);
    a.totals = a.counts + (int64_t)a.L * a.n_chunks * (a.E + 1);
    a.rows = rows;
    a.offsets = offsets;
    a.places = places;
    if ((int64_t)a.L * (a.n_chunks + 7) > INT32_MAX / kOrderThreads) return ROUTEPACK_E_UNSUPPORTED;
    const unsigned n = (unsigned)((a.n_chunks + 7) / 8 * 8 * (int64_t)a.L);
    const size_t one = 4 * (size_t)(a.E + 1), all = 4 * kChunk + one * (1 + kOrderWaves);
    const int64_t last = ids->n_tokens > 0 ? ids->n_tokens - 1 : 0;
    const bool near = a.ts <= INT32_MAX && last * a.ts + a.k <= INT32_MAX && (last + 1) * a.L * a.k <= INT32_MAX;
    auto launch = [&](auto tag, auto near_) -> int {
        using I = decltype(tag);
        constexpr bool NEAR = decltype(near_)::value != 0;
        if (a.n_chunks > 1) {
            hipLaunchKernelGGL((k_order_count<I, NEAR>), dim3(n), dim3(kOrderThreads), one, stream, a);
            hipLaunchKernelGGL(k_order_scan, grid_of(((int64_t)a.L * (a.E + 1) + 3) / 4), dim3(256), 0, stream, a);
        }
        const auto place = k_order_place<I, NEAR>;
        if (all > 64 * 1024 - 256 && hipFuncSetAttribute(reinterpret_cast<const void *>(place),
                                                         hipFuncAttributeMaxDynamicSharedMemorySize, (int)all) != hipSuccess)
            return ROUTEPACK_E_DEVICE;
        hipLaunchKernelGGL(place, dim3(n), dim3(kOrderThreads), all, stream, a);
        return launched();
    };
    auto go = [&](auto tag) { return near ? launch(tag, Int<1>()) : launch(tag, Int<0>()); };
    switch (ids->type) {
        case ROUTEPACK_U8: return go(uint8_t());
        case ROUTEPACK_I16: return go(int16_t());
        case ROUTEPACK_I32: return go(int32_t());
        default: return go(int64_t());
    }
}
