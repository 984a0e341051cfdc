// The order of the pairs of tokens and chosen experts by slot, on gfx950: a
// stable counting sort.
//
// A layer's pairs are cut into chunks; a chunk's pairs are counted by slot
// (k_order_count), the counts of a slot are summed over the chunks before
// (k_order_scan), and each chunk places its pairs behind those (k_order_place).
// Pairs without a choice count for a slot of their own behind the last.  Within
// a chunk each wave holds a part in order and counters of its own; 64 pairs at a
// time find their rank among those with the same slot by ballots over the
// slot's bits, so rows do not depend on the order of atomics.  One chunk needs
// the last kernel alone.
#include "rp_experts.h"

namespace rp {

struct OrderArgs {
    const void *ids;
    int32_t type;
    int64_t ts, ls;
    int32_t P, L, E, k;     // pairs of a layer
    const int32_t *slots;
    int32_t chunk, n_chunks;
    int32_t bits;           // of a slot, 0 .. E
    int32_t *counts;        // [L][n_chunks][E + 1], then sums over the chunks before
    int32_t *totals;        // [L][E + 1]
    int32_t *rows;
    int64_t *offsets;
    int32_t *places;
};

constexpr int kOrderThreads = 512, kOrderWaves = kOrderThreads / kWave;

// Pair p's slot; E for none.
template <class I>
__device__ inline int32_t slot_of_pair(const OrderArgs &a, int32_t l, int32_t p) {
    const int32_t t = (int32_t)((uint32_t)p / (uint32_t)a.k), j = p - t * a.k;
    const int64_t v = (int64_t) static_cast<const I *>(a.ids)[t * a.ts + l * a.ls + j];
    if (v < 0 || v >= a.E) return a.E;
    if (!a.slots) return (int32_t)v;
    const int32_t s = a.slots[(int64_t)l * a.E + v];
    return s >= 0 && s < a.E ? s : a.E;
}

template <class I>
__global__ void __launch_bounds__(kOrderThreads) k_order_count(OrderArgs a) {
    extern __shared__ int32_t n[];
    const int32_t l = (int32_t)(blockIdx.x / a.n_chunks), c = (int32_t)(blockIdx.x - (uint32_t)l * a.n_chunks);
    for (int32_t s = threadIdx.x; s <= a.E; s += kOrderThreads) n[s] = 0;
    __syncthreads();
    const int32_t b = c * a.chunk, e = a.P - b < a.chunk ? a.P : b + a.chunk;
    for (int32_t p = b + (int32_t)threadIdx.x; p < e; p += kOrderThreads) atomicAdd(&n[slot_of_pair<I>(a, l, p)], 1);
    __syncthreads();
    int32_t *out = a.counts + ((int64_t)l * a.n_chunks + c) * (a.E + 1);
    for (int32_t s = threadIdx.x; s <= a.E; s += kOrderThreads) out[s] = n[s];
}

// A wave sums 16 slots over the chunks, a quarter of a round's chunks each lane.
__global__ void __launch_bounds__(256) k_order_scan(OrderArgs a) {
    const int32_t per = (a.E + 1 + 63) / 64, l = (int32_t)(blockIdx.x / per);
    const int32_t s = (int32_t)(blockIdx.x - (uint32_t)l * per) * 64 + (int32_t)(threadIdx.x >> 2), q = threadIdx.x & 3;
    if (s > a.E) return;  // (all four lanes of a slot)
    int32_t *col = a.counts + (int64_t)l * a.n_chunks * (a.E + 1) + s;
    const int32_t part = (a.n_chunks + 3) / 4, b = q * part, e = b + part < a.n_chunks ? b + part : a.n_chunks;
    int32_t sum = 0;
    for (int32_t c = b; c < e; ++c) sum += col[(int64_t)c * (a.E + 1)];
    const int32_t s0 = __shfl(sum, 0, 4), s1 = __shfl(sum, 1, 4), s2 = __shfl(sum, 2, 4), s3 = __shfl(sum, 3, 4);
    int32_t before = (q > 0 ? s0 : 0) + (q > 1 ? s1 : 0) + (q > 2 ? s2 : 0);
    if (q == 0) a.totals[(int64_t)l * (a.E + 1) + s] = s0 + s1 + s2 + s3;
    for (int32_t c = b; c < e; ++c) {
        const int32_t v = col[(int64_t)c * (a.E + 1)];
        col[(int64_t)c * (a.E + 1)] = before;
        before += v;
    }
}

template <class I>
__global__ void __launch_bounds__(kOrderThreads) k_order_place(OrderArgs a) {
    extern __shared__ int32_t lds[];
    const int32_t S = a.E + 1;
    __shared__ int32_t wave_sum[kOrderWaves];
    int32_t *mine = lds + (threadIdx.x >> 6) * S;  // this wave's counters, then its next rows
    const int32_t l = (int32_t)(blockIdx.x / a.n_chunks), c = (int32_t)(blockIdx.x - (uint32_t)l * a.n_chunks);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int32_t s = threadIdx.x; s < kOrderWaves * S; s += kOrderThreads) lds[s] = 0;
    __syncthreads();
    const int32_t b = c * a.chunk, e = a.P - b < a.chunk ? a.P : b + a.chunk;
    const int32_t part = ((e - b + kOrderWaves - 1) / kOrderWaves + 63) / 64 * 64;
    const int32_t pb = e - b < wave * part ? e : b + wave * part, pe = e - pb < part ? e : pb + part;
    for (int32_t p = pb + lane; p < pe; p += kWave) atomicAdd(&mine[slot_of_pair<I>(a, l, p)], 1);
    __syncthreads();
    // the first row of every slot, and of this chunk's and wave's part of it
    const int32_t each = (S + kOrderThreads - 1) / kOrderThreads, s0 = threadIdx.x * each;
    const int32_t s1 = s0 + each < S ? s0 + each : S;
    const int64_t at = ((int64_t)l * a.n_chunks + c) * S;
    int32_t sum = 0;
    for (int32_t s = s0; s < s1; ++s) {
        if (a.n_chunks > 1) {
            sum += a.totals[(int64_t)l * S + s];
        } else {
            for (int w = 0; w < kOrderWaves; ++w) sum += lds[w * S + s];
        }
    }
    int32_t upto = sum;
    for (int d = 1; d < kWave; d <<= 1) {
        const int32_t v = __shfl_up(upto, d, kWave);
        upto += lane >= d ? v : 0;
    }
    if (lane == kWave - 1) wave_sum[wave] = upto;
    __syncthreads();
    int32_t row = upto - sum;
    for (int w = 0; w < wave; ++w) row += wave_sum[w];
    for (int32_t s = s0; s < s1; ++s) {
        if (c == 0) a.offsets[(int64_t)l * S + s] = row;  // (S = E + 1: the last is the end of slot E - 1)
        int32_t next = row, total = 0;
        if (a.n_chunks > 1) {
            total = a.totals[(int64_t)l * S + s];
            next += a.counts[at + s];
        }
        for (int w = 0; w < kOrderWaves; ++w) {
            const int32_t v = lds[w * S + s];
            lds[w * S + s] = next;
            next += v;
        }
        row = a.n_chunks > 1 ? row + total : next;
    }
    __syncthreads();
    int32_t *rows = a.rows + (int64_t)l * a.P;
    for (int32_t p0 = pb; p0 < pe; p0 += kWave) {
        const int32_t p = p0 + lane;
        const bool live = p < pe;
        const int32_t s = live ? slot_of_pair<I>(a, l, p) : a.E;
        uint64_t same = __ballot(live);
        for (int i = 0; i < a.bits; ++i) {
            const bool bit = s >> i & 1;
            const uint64_t ones = __ballot(bit);
            same &= bit ? ones : ~ones;
        }
        const int32_t rank = __popcll(same & (((uint64_t)1 << lane) - 1)), all = __popcll(same);
        const int32_t first = mine[s];
        __builtin_amdgcn_wave_barrier();  // (all reads of a wave's counters before the writes)
        if (live && rank == 0) mine[s] = first + all;
        __builtin_amdgcn_wave_barrier();
        if (live) {
            const int32_t r = first + rank;
            const bool made = s < a.E;
            rows[r] = made ? p : -1;
            const int32_t t = (int32_t)((uint32_t)p / (uint32_t)a.k), j = p - t * a.k;
            a.places[((int64_t)t * a.L + l) * a.k + j] = made ? r : -1;
        }
    }
}

// Chunks of a layer: of 4096 pairs, fewer than 512 of them.
inline int32_t order_chunk(int64_t P) {
    const int64_t c = (P / 512 + 4095) / 4096 * 4096;
    return (int32_t)(c < 4096 ? 4096 : c);
}

inline int check_order(const routepack_problem *p, int64_t n_tokens) {
    if (!p || n_tokens < 0 || p->n_layers < 0 || p->n_experts < 1 || p->top_k < 1) return ROUTEPACK_E_INVALID;
    if (p->n_experts > kMaxSlots || p->top_k > 256 || n_tokens > INT32_MAX / p->top_k) return ROUTEPACK_E_UNSUPPORTED;
    if (p->n_layers > 0 && (int64_t)p->n_layers * (p->n_experts + 1) > INT64_MAX / 16 / 1024) return ROUTEPACK_E_UNSUPPORTED;
    return ROUTEPACK_OK;
}

// (of one chunk: none, but a workspace of size 0 would be a special case)
inline int64_t order_bytes(const routepack_problem *p, int64_t n_tokens) {
    const int64_t P = n_tokens * p->top_k, chunk = order_chunk(P), n = (P + chunk - 1) / chunk;
    return n <= 1 ? 16 : (int64_t)p->n_layers * (n + 1) * (p->n_experts + 1) * 4;
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
    if (!offsets || !workspace || ((uintptr_t)workspace & 15) || workspace_bytes < order_bytes(prob, ids->n_tokens))
        return ROUTEPACK_E_INVALID;
    if (ids->n_tokens > 0 && (!rows || !places)) return ROUTEPACK_E_INVALID;
    OrderArgs a = {};
    a.ids = ids->data;
    a.type = ids->type;
    a.ts = ids->token_stride;
    a.ls = ids->layer_stride;
    a.P = (int32_t)(ids->n_tokens * prob->top_k);
    a.L = prob->n_layers;
    a.E = prob->n_experts;
    a.k = prob->top_k;
    a.slots = slots;
    a.chunk = order_chunk(a.P);
    a.n_chunks = a.P > a.chunk ? (int32_t)(((int64_t)a.P + a.chunk - 1) / a.chunk) : 1;
    a.bits = 32 - __builtin_clz((unsigned)a.E);
    a.counts = static_cast<int32_t *>(workspace);
    a.totals = a.counts + (int64_t)a.L * a.n_chunks * (a.E + 1);
    a.rows = rows;
    a.offsets = offsets;
    a.places = places;
    if ((int64_t)a.L * a.n_chunks > INT32_MAX / kOrderThreads) return ROUTEPACK_E_UNSUPPORTED;
    const unsigned n = (unsigned)(a.L * a.n_chunks);
    const size_t one = 4 * (size_t)(a.E + 1), all = one * kOrderWaves;
    auto go = [&](auto tag) -> int {
        using I = decltype(tag);
        if (a.n_chunks > 1) {
            hipLaunchKernelGGL(k_order_count<I>, dim3(n), dim3(kOrderThreads), one, stream, a);
            hipLaunchKernelGGL(k_order_scan, dim3((unsigned)a.L * (unsigned)((a.E + 1 + 63) / 64)), dim3(256), 0, stream, a);
        }
        if (all > 64 * 1024 - 256 &&
            hipFuncSetAttribute(reinterpret_cast<const void *>(k_order_place<I>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, (int)all) != hipSuccess)
            return ROUTEPACK_E_DEVICE;
        hipLaunchKernelGGL(k_order_place<I>, dim3(n), dim3(kOrderThreads), all, stream, a);
        return launched();
    };
    switch (ids->type) {
        case ROUTEPACK_U8: return go(uint8_t());
        case ROUTEPACK_I16: return go(int16_t());
        case ROUTEPACK_I32: return go(int32_t());
        default: return go(int64_t());
    }
}
