// The router's gates (chosen or replayed experts) and the gradient of gates
// and balance loss with respect to the logits, on gfx950.
#include <math.h>

#include "rp_internal.h"
#include "rp_route.h"

namespace rp {

// The choices of logits of one type (rp_route_choose.h, a translation unit
// for each type).
int choose_f32(const RouteArgs &a, hipStream_t stream);
int choose_bf16(const RouteArgs &a, hipStream_t stream);
int choose_f16(const RouteArgs &a, hipStream_t stream);

// Gates of recorded experts that need no more of a row than the experts'
// logits: a group of G >= k lanes a token, a choice a lane.
template <class T, int G>
__global__ void __launch_bounds__(256) k_replay_chosen(RouteArgs a) {
    const int c = threadIdx.x & (G - 1);
    const Item it = item_of<G>(a.T, a.L);
    const T *row = static_cast<const T *>(a.logits) + it.t * a.ts + it.l * a.ls;
    int32_t id = -1;
    if (c < a.k) id = load_id(a.rec, a.rec_type, it.t * a.rts + it.l * a.rls + c, a.E);
    const float zc[1] = {id >= 0 ? to_f32(row[id]) : 0.0f};
    const bool on[1] = {id >= 0};
    float w[1], less[1];
    choice_gates<G, 1>(zc, on, a.score, a.normalize, 0.0f, 0.0f, w, less);
    if (it.live && c < a.k) a.gates[it.at * a.k + c] = a.scale * w[0];
}

// Unnormalised softmax gates of recorded experts: the row's sum, then its k
// choices, S of them a lane.
template <class T, int G, int NV>
__global__ void __launch_bounds__(256) k_replay_row(RouteArgs a) {
    constexpr int V = NV * (16 / sizeof(T)), S = kMaxChoices / G > 0 ? kMaxChoices / G : 1;
    const int c = threadIdx.x & (G - 1);
    const Item it = item_of<G>(a.T, a.L);
    const T *row = static_cast<const T *>(a.logits) + it.t * a.ts + it.l * a.ls;
    float z[V], zc[S], w[S], less[S];
    bool on[S];
    load_row<T, G, V>(row, a.E, c, z);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int j = s * G + c;
        int32_t id = -1;
        if (j < a.k) id = load_id(a.rec, a.rec_type, it.t * a.rts + it.l * a.rls + j, a.E);
        on[s] = id >= 0;
        zc[s] = on[s] ? to_f32(row[id]) : 0.0f;
    }
    float m, inv;
    row_sum<G, V>(z, m, inv);
    choice_gates<G, S>(zc, on, ROUTEPACK_SOFTMAX, false, m, inv, w, less);
#pragma unroll
    for (int s = 0; s < S; ++s)
        if (it.live && s * G + c < a.k) a.gates[it.at * a.k + s * G + c] = a.scale * w[s];
}

struct BackArgs {
    const void *logits;
    int64_t ts, ls;
    int64_t T;
    int32_t L, E, k;
    const void *ids;  // null: no gates
    int32_t id_type;
    int64_t its, ils;
    const float *dgates;
    bool normalize;
    float scale;
    int32_t n_groups;
    const int64_t *offsets;
    const void *counts;
    int32_t counts_type;
    const float *dloss;  // null: no balance loss
    int32_t score;
    void *dlogits;
};

// The group that holds token t, or -1: the last one that begins at or before
// it.
__device__ inline int32_t group_of(const int64_t *offsets, int32_t n, int64_t t) {
    if (t < offsets[0] || t >= offsets[n]) return -1;
    int32_t lo = 0, hi = n;  // offsets[lo] <= t < offsets[hi]
    while (hi - lo > 1) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (offsets[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A wave per token and layer.  The gates' gradient D of the chosen experts
// goes through a row of LDS to the lanes that hold them.
template <class T, int V>
__global__ void __launch_bounds__(256) k_route_back(BackArgs a) {
    extern __shared__ float direct_rows[];  // [4][E]
    const int64_t item = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + wave_id();
    if (item >= a.T * a.L) return;  // (no barrier below)
    const int64_t t = item / a.L;
    const int32_t l = (int32_t)(item - t * a.L);
    const int c = lane_id();
    const T *row = static_cast<const T *>(a.logits) + t * a.ts + l * a.ls;
    float z[V], less[V], f[V];
    load_row<T, kWave, V>(row, a.E, c, z);
    float m = -kInf, inv = 0.0f;
    const bool softmax = a.score == ROUTEPACK_SOFTMAX;
    if (softmax) {
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) m = __builtin_fmaxf(m, z[v]);
        m = group_max<kWave>(m);
        m = m == -kInf ? 0.0f : m;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            z[v] = exp32(z[v] - m);
            sum += z[v];
        }
        sum = group_sum<kWave>(sum);
        inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] *= inv;
    } else {
        logistic_row<kWave, V>(z, less);
    }
    float drop = 0.0f;  // sum D, where the row's softmax takes part
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = 0.0f;
    if (a.dloss) {
        const int32_t g = group_of(a.offsets, a.n_groups, t);
        if (g >= 0) {
            const int64_t at = ((int64_t)g * a.L + l) * a.E;
            int64_t sum = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int e = elem_of<T, kWave>(v, c);
                int64_t n = 0;
                if (e < a.E)
                    n = a.counts_type == ROUTEPACK_I32 ? static_cast<const int32_t *>(a.counts)[at + e]
                                                       : static_cast<const int64_t *>(a.counts)[at + e];
                sum += n;
                f[v] = (float)n;
            }
            sum = group_sum64<kWave>(sum);
            const float len = (float)(a.offsets[g + 1] - a.offsets[g]);
            const float by = sum > 0 ? (float)a.E / (float)sum * (a.dloss[l] / ((float)a.n_groups * len)) : 0.0f;
            float dot = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[v] *= by;
                dot += z[v] * f[v];
            }
            dot = group_sum<kWave>(dot);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[v] = z[v] * (f[v] - dot);
                if (!softmax) f[v] *= less[v];
            }
        }
    }
    if (a.ids) {
        float *direct = direct_rows + wave_id() * a.E;
        for (int e = c; e < a.E; e += kWave) direct[e] = 0.0f;
        int32_t id = -1;
        float dg = 0.0f;
        if (c < a.k) id = load_id(a.ids, a.id_type, t * a.its + l * a.ils + c, a.E);
        if (id >= 0) dg = a.dgates[item * a.k + c];
        float zc[1] = {id >= 0 ? to_f32(row[id]) : 0.0f}, w[1], sl[1];
        const bool on[1] = {id >= 0};
        choice_gates<kWave, 1>(zc, on, a.score, a.normalize, m, inv, w, sl);
        float d = id >= 0 ? a.scale * w[0] * dg : 0.0f;
        if (a.normalize) {
            const float dot = group_sum<kWave>(id >= 0 ? w[0] * dg : 0.0f);
            d = id >= 0 ? a.scale * w[0] * (dg - dot) : 0.0f;
        }
        if (!softmax && id >= 0) d *= sl[0];
        if (softmax && !a.normalize) drop = group_sum<kWave>(d);
        wave_sync();
        // choices of one expert are added in their order
        for (int j = 0; j < a.k; ++j) {
            if (c == j && id >= 0) direct[id] += d;
            wave_sync();
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = elem_of<T, kWave>(v, c);
            if (e < a.E) f[v] += direct[e];
            f[v] -= z[v] * drop;
        }
    }
    store_row<T, kWave, V>(static_cast<T *>(a.dlogits) + item * a.E, a.E, c, f);
}

}  // namespace rp

using namespace rp;

extern "C" int routepack_route_tokens(const routepack_problem *prob, const routepack_logits *logits,
                                      const routepack_ids *replay, const float *bias, int32_t score,
                                      int32_t normalize, float scale, int32_t *ids, float *gates,
                                      hipStream_t stream) {
    RP_TRY(check_logits(prob, logits, score));
    if (prob->top_k < 1 || prob->top_k > prob->n_experts || !isfinite(scale)) return ROUTEPACK_E_INVALID;
    if (prob->top_k > kMaxChoices) return ROUTEPACK_E_UNSUPPORTED;
    if (replay) {
        RP_TRY(check_ids(prob, replay, logits->n_tokens));
        if (bias) return ROUTEPACK_E_INVALID;
    }
    const int64_t items = logits->n_tokens * prob->n_layers;
    if (items == 0) return ROUTEPACK_OK;
    if (!gates || (!replay && !ids)) return ROUTEPACK_E_INVALID;
    RouteArgs a = {logits->data, logits->token_stride, logits->layer_stride, logits->n_tokens, prob->n_layers,
                   prob->n_experts, prob->top_k, replay ? replay->data : nullptr, replay ? replay->type : 0,
                   replay ? replay->token_stride : 0, replay ? replay->layer_stride : 0, bias, score, normalize != 0,
                   scale, ids, gates};
    if (!replay) {
        switch (logits->type) {
            case ROUTEPACK_F32: return choose_f32(a, stream);
            case ROUTEPACK_BF16: return choose_bf16(a, stream);
            default: return choose_f16(a, stream);
        }
    }
    return by_type(logits->type, [&](auto tag) -> int {
        using T = decltype(tag);
        auto go = [&](auto kern, int g) {
            hipLaunchKernelGGL(kern, grid_of((items + 256 / g - 1) / (256 / g)), dim3(256), 0, stream, a);
            return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
        };
        if (score == ROUTEPACK_SOFTMAX && !normalize)
            return by_geometry<T, 2 * sizeof(T)>(a.E, [&](auto g, auto nv) {
                return go(k_replay_row<T, g.value, nv.value>, g.value);
            });
        if (a.k <= 4) return go(k_replay_chosen<T, 4>, 4);
        if (a.k <= 8) return go(k_replay_chosen<T, 8>, 8);
        if (a.k <= 16) return go(k_replay_chosen<T, 16>, 16);
        return go(k_replay_chosen<T, 32>, 32);
    });
}

extern "C" int routepack_route_backward(const routepack_problem *prob, const routepack_logits *logits,
                                        const routepack_ids *ids, const float *dgates, int32_t normalize,
                                        float scale, int32_t n_groups, const int64_t *offsets,
                                        const void *counts, int32_t counts_type, const float *dloss,
                                        int32_t score, void *dlogits, hipStream_t stream) {
    RP_TRY(check_logits(prob, logits, score));
    if (!ids && !dloss) return ROUTEPACK_E_INVALID;
    const int64_t items = logits->n_tokens * prob->n_layers;
    if (ids) {
        if (prob->top_k < 1 || prob->top_k > prob->n_experts || !isfinite(scale)) return ROUTEPACK_E_INVALID;
        if (prob->top_k > kMaxChoices) return ROUTEPACK_E_UNSUPPORTED;
        RP_TRY(check_ids(prob, ids, logits->n_tokens));
        if (!dgates && items > 0) return ROUTEPACK_E_INVALID;
    }
    if (dloss) {
        if (n_groups < 1 || !offsets || !counts) return ROUTEPACK_E_INVALID;
        if (counts_type != ROUTEPACK_I32 && counts_type != ROUTEPACK_I64) return ROUTEPACK_E_INVALID;
    }
    if (items == 0) return ROUTEPACK_OK;
    if (!dlogits) return ROUTEPACK_E_INVALID;
    BackArgs a = {logits->data, logits->token_stride, logits->layer_stride, logits->n_tokens, prob->n_layers,
                  prob->n_experts, prob->top_k, ids ? ids->data : nullptr, ids ? ids->type : 0,
                  ids ? ids->token_stride : 0, ids ? ids->layer_stride : 0, dgates, normalize != 0, scale, n_groups,
                  offsets, counts, counts_type, dloss, score, dlogits};
    return by_type(logits->type, [&](auto tag) -> int {
        using T = decltype(tag);
        const dim3 grid = grid_of((items + 3) / 4);
        const size_t lds = ids ? (size_t)16 * a.E : 0;
        if (a.E <= 512) hipLaunchKernelGGL((k_route_back<T, 8>), grid, dim3(256), lds, stream, a);
        else hipLaunchKernelGGL((k_route_back<T, 32>), grid, dim3(256), lds, stream, a);
        return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
    });
}
