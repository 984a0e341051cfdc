// The router's gates (chosen or replayed experts) and the gradient of gates
// and balance loss with respect to the logits, on gfx950.
#include <math.h>

#include "rp_internal.h"
#include "rp_route.h"

namespace rp {

// The choices and the gradient for logits of one type (rp_route_choose.h and
// rp_route_back.h, translation units for each type).
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
template <class T, int G, int NV, int K>
__global__ void __launch_bounds__(256) k_replay_row(RouteArgs a) {
    constexpr int V = NV * (16 / sizeof(T)), S = K > G ? K / G : 1;
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

int back_f32(const BackArgs &a, hipStream_t stream);
int back_bf16(const BackArgs &a, hipStream_t stream);
int back_f16(const BackArgs &a, hipStream_t stream);

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
                if (a.k <= 8) return go(k_replay_row<T, g.value, nv.value, 8>, g.value);
                return go(k_replay_row<T, g.value, nv.value, kMaxChoices>, g.value);
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
    switch (logits->type) {
        case ROUTEPACK_F32: return back_f32(a, stream);
        case ROUTEPACK_BF16: return back_bf16(a, stream);
        default: return back_f16(a, stream);
    }
}
