// Device-side building blocks of the router's operators: logits of three
// types, scores in 32 bits, reductions over the group of lanes that holds a
// token's row, and the gates of a token's choices.
//
// A token's row of E logits lies in G adjacent lanes of a wave (G a power of
// two), V values a lane, in vectors of 16 bytes: lane c holds the elements
// (i G + c) W + x, with i the vector, W its elements and x < W.
#pragma once

#include "rp_device.h"
#include "rp_internal.h"
#include "routepack/router.h"

namespace rp {

constexpr float kInf = __builtin_inff();
constexpr int kMaxExperts = 2048, kMaxChoices = 32;

template <class T>
__device__ inline float to_f32(T v) { return (float)v; }

template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Vec16 {
    T v[16 / sizeof(T)];
};

// The row's part of one lane; elements past the row are -inf (no score).
template <class T, int G, int V>
__device__ inline void load_row(const T *row, int E, int c, float (&z)[V]) {
    constexpr int W = 16 / sizeof(T);
    static_assert(V % W == 0, "whole vectors");
#pragma unroll
    for (int i = 0; i < V / W; ++i) {
        const int e0 = (i * G + c) * W;
        if (e0 + W <= E) {
            const Vec16<T> w = *reinterpret_cast<const Vec16<T> *>(row + e0);
#pragma unroll
            for (int x = 0; x < W; ++x) z[i * W + x] = to_f32(w.v[x]);
        } else {
#pragma unroll
            for (int x = 0; x < W; ++x) z[i * W + x] = e0 + x < E ? to_f32(row[e0 + x]) : -kInf;
        }
    }
}

template <class T, int G, int V>
__device__ inline void store_row(T *row, int E, int c, const float (&z)[V]) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < V / W; ++i) {
        const int e0 = (i * G + c) * W;
        if (e0 + W <= E) {
            Vec16<T> w;
#pragma unroll
            for (int x = 0; x < W; ++x) w.v[x] = (T)z[i * W + x];
            *reinterpret_cast<Vec16<T> *>(row + e0) = w;
        } else {
#pragma unroll
            for (int x = 0; x < W; ++x)
                if (e0 + x < E) row[e0 + x] = (T)z[i * W + x];
        }
    }
}

// Element of a lane's v-th value.
template <class T, int G>
__device__ inline int elem_of(int v, int c) {
    constexpr int W = 16 / sizeof(T);
    return ((v / W) * G + c) * W + v % W;
}

// e^x in 32 bits: 2^t for t = x log2(e) rounded, times 1 + the part of the
// product that the rounding lost, times ln 2 (a relative error of about one
// step whatever x is; the plain product alone loses |x| log2(e) / 2 steps).
// Results below the smallest normal number are 0.
__device__ inline float exp32(float x) {
    const float kHi = 1.44269502f, kLo = 1.92596299e-8f, kLn2 = 0.693147182f;
    const float t = x * kHi;
    const float lost = __builtin_fmaf(x, kLo, __builtin_fmaf(x, kHi, -t));
    const float p = __builtin_amdgcn_exp2f(t);
    return x < -87.0f ? 0.0f : __builtin_fmaf(p * kLn2, lost, p);
}

// s = 1 / (1 + e^-z) and 1 - s, without cancellation on either side.
__device__ inline void logistic(float z, float &s, float &one_less) {
    const float e = exp32(-__builtin_fabsf(z));
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    const float q = e * r;
    s = z >= 0.0f ? r : q;
    one_less = z >= 0.0f ? q : r;
    if (z != z) s = one_less = z;
}

// Reductions over the G lanes of a token; every lane ends with the result.
template <int G>
__device__ inline float group_sum(float v) {
#pragma unroll
    for (int d = 1; d < G; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}
template <int G>
__device__ inline float group_max(float v) {
#pragma unroll
    for (int d = 1; d < G; d <<= 1) v = __builtin_fmaxf(v, __shfl_xor(v, d, kWave));
    return v;
}
template <int G>
__device__ inline int64_t group_sum64(int64_t v) {
#pragma unroll
    for (int d = 1; d < G; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// Softmax of a row, in place: z becomes p.  A row without an available
// expert becomes 0; a NaN or +inf in it makes it NaN.
template <int G, int V>
__device__ inline void softmax_row(float (&z)[V]) {
    float m = z[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = __builtin_fmaxf(m, z[v]);
    m = group_max<G>(m);
    m = m == -kInf ? 0.0f : m;
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        z[v] = exp32(z[v] - m);
        sum += z[v];
    }
    sum = group_sum<G>(sum);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] *= inv;
}

// Logistic shares of a row, in place: z becomes s / sum s, and `less` 1 - s.
// Where every logit is below 0 the scores may leave the range of 32 bits, but
// their ratios do not: with a maximum m < 0 all are taken times e^-m.
template <int G, int V>
__device__ inline void logistic_row(float (&z)[V], float (&less)[V]) {
    float m = z[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = __builtin_fmaxf(m, z[v]);
    m = group_max<G>(m);
    const bool low = m < 0.0f && m > -kInf;
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float s;
        const float x = z[v];
        logistic(x, s, less[v]);
        if (low) s = exp32(x - m) * less[v];  // e^x / (1 + e^x) and 1 / (1 + e^x)
        z[v] = s;
        sum += s;
    }
    sum = group_sum<G>(sum);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] *= inv;
}

// The gates, divided by scale, of a token's choices, S of them a lane (slot s
// of lane c is choice s G + c): logits zc, `on` where a choice was made.
// softmax without normalising: `m` and `inv` are the row's maximum and the
// inverse of its sum.  less: 1 - s of logistic scores.
template <int G, int S>
__device__ inline void choice_gates(const float (&zc)[S], const bool (&on)[S], int score, bool normalize, float m,
                                    float inv, float (&w)[S], float (&less)[S]) {
    if (score == ROUTEPACK_SOFTMAX && !normalize) {
#pragma unroll
        for (int s = 0; s < S; ++s) w[s] = on[s] ? exp32(zc[s] - m) * inv : 0.0f;
        return;
    }
    if (score == ROUTEPACK_SIGMOID) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            logistic(zc[s], w[s], less[s]);
            w[s] = on[s] ? w[s] : 0.0f;
        }
        if (!normalize) return;
    }
    float top = -kInf;
#pragma unroll
    for (int s = 0; s < S; ++s) top = on[s] ? __builtin_fmaxf(top, zc[s]) : top;
    top = group_max<G>(top);
    if (score == ROUTEPACK_SOFTMAX || (top < 0.0f && top > -kInf)) {
        // (logistic scores as in logistic_row)
        const float base = top == -kInf ? 0.0f : top;
#pragma unroll
        for (int s = 0; s < S; ++s)
            w[s] = on[s] ? exp32(zc[s] - base) * (score == ROUTEPACK_SOFTMAX ? 1.0f : less[s]) : 0.0f;
    }
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) sum += w[s];
    sum = group_sum<G>(sum);
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int s = 0; s < S; ++s) w[s] *= by;
}

// One recorded id, as an expert or -1.
__device__ inline int32_t load_id(const void *data, int type, int64_t at, int32_t E) {
    int64_t v;
    switch (type) {
        case ROUTEPACK_U8: v = static_cast<const uint8_t *>(data)[at]; break;
        case ROUTEPACK_I16: v = static_cast<const int16_t *>(data)[at]; break;
        case ROUTEPACK_I32: v = static_cast<const int32_t *>(data)[at]; break;
        default: v = static_cast<const int64_t *>(data)[at]; break;
    }
    return v >= 0 && v < E ? (int32_t)v : -1;
}

// Argument checks that the entry points share.
inline int check_logits(const routepack_problem *p, const routepack_logits *z, int32_t score) {
    if (!p || !z) return ROUTEPACK_E_INVALID;
    if (p->n_layers < 0 || p->n_experts < 1) return ROUTEPACK_E_INVALID;
    if (z->type < ROUTEPACK_F32 || z->type > ROUTEPACK_F16) return ROUTEPACK_E_INVALID;
    if (z->n_tokens < 0 || z->token_stride < 0 || z->layer_stride < 0) return ROUTEPACK_E_INVALID;
    if (!z->data && z->n_tokens > 0 && p->n_layers > 0) return ROUTEPACK_E_INVALID;
    if (score != ROUTEPACK_SOFTMAX && score != ROUTEPACK_SIGMOID) return ROUTEPACK_E_INVALID;
    if (p->n_experts > kMaxExperts) return ROUTEPACK_E_UNSUPPORTED;
    return ROUTEPACK_OK;
}

inline int check_ids(const routepack_problem *p, const routepack_ids *r, int64_t n_tokens) {
    if (r->type < ROUTEPACK_U8 || r->type > ROUTEPACK_I64) return ROUTEPACK_E_INVALID;
    if (r->n_tokens != n_tokens || r->token_stride < 0 || r->layer_stride < 0) return ROUTEPACK_E_INVALID;
    if (!r->data && n_tokens > 0 && p->n_layers > 0) return ROUTEPACK_E_INVALID;
    return ROUTEPACK_OK;
}

// Calls f with a value of the logits' type.
template <class F>
int by_type(int32_t type, F &&f) {
    switch (type) {
        case ROUTEPACK_F32: return f(float());
        case ROUTEPACK_BF16: return f((__bf16)0.0f);
        default: return f((_Float16)0.0f);
    }
}

}  // namespace rp
