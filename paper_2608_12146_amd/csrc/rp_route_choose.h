// The router's choices: the k largest of each token's E logits, or of its
// scores and a bias, and their gates.  Included by one translation unit for
// each type of logits.
//
// The row lies in G lanes as vectors of 16 bytes, the vectors that a load
// brings.  The k elements sought lie in the k vectors of largest maximum (an
// element outside of them is preceded by k maxima; equal ones precede by their
// index, as the vectors' order is the elements').  So the first selection runs
// over the vectors' maxima, an eighth (16-bit logits) or a quarter of the
// elements; the k vectors are then taken again, one or a few to a lane, and a
// second selection runs over their elements.  Both sort a lane's keys into its
// K largest and merge lists of K across lanes, in registers (no LDS, no
// loop over the choices, no branch that depends on the values).
#pragma once

#include "rp_route.h"

namespace rp {

// The largest of a vector's elements; NaN where it holds a signalling NaN
// or NaN only.
__device__ inline float max3(float a, float b, float c) {
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}
__device__ inline float most_of(const float (&x)[4]) { return max3(max3(x[0], x[1], x[2]), x[3], x[3]); }
__device__ inline float most_of(const float (&x)[8]) {
    return max3(max3(max3(x[0], x[1], x[2]), x[3], x[4]), max3(x[5], x[6], x[7]), x[7]);
}

template <class T>
struct Row {
    static constexpr int W = 16 / sizeof(T);
    const T *data;
    int32_t E;
    // vector v of the row; elements past its end are -inf
    __device__ Vec16<T> vec(int v) const {
        const int e0 = v * W;
        if (e0 + W <= E) return *reinterpret_cast<const Vec16<T> *>(data + e0);
        Vec16<T> x;
#pragma unroll
        for (int i = 0; i < W; ++i) x.v[i] = e0 + i < E ? data[e0 + i] : (T)(-kInf);
        return x;
    }
};

template <class T, int G, int NV, int K>
__global__ void __launch_bounds__(256) k_route(RouteArgs a) {
    using Key = typename KeyOf<T>::type;
    using Word = typename Key::Word;
    constexpr int W = 16 / sizeof(T), M = G < K ? G : K, S = K / M;
    const int c = threadIdx.x & (G - 1);
    const Item it = item_of<G>(a.T, a.L);
    const Row<T> row = {static_cast<const T *>(a.logits) + it.t * a.ts + it.l * a.ls, a.E};
    Vec16<T> raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = row.vec(i * G + c);
    // the k vectors of largest maximum
    float mx[NV];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float x[W];
#pragma unroll
        for (int w = 0; w < W; ++w) x[w] = to_f32(raw[i].v[w]);
        mx[i] = most_of(x);
        odd = odd || mx[i] != mx[i];
    }
    if (__any(odd)) {  // NaN among the logits
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            mx[i] = -kInf;
#pragma unroll
            for (int w = 0; w < W; ++w) mx[i] = __builtin_fmaxf(mx[i], to_f32(raw[i].v[w]) + 0.0f);
        }
    }
    Word vk[NV], first[K];
#pragma unroll
    for (int i = 0; i < NV; ++i) vk[i] = Key::make(mx[i], kIndexMask ^ (uint32_t)c ^ (uint32_t)(i * G));
    lane_top<Key, K, NV>(vk, first);
    group_top<Key, K, G>(first);
    float m = 0.0f, inv = 0.0f;
    if (a.score == ROUTEPACK_SOFTMAX && !a.normalize) {
        m = Key::available(first[0]) ? Key::value(first[0]) : 0.0f;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int w = 0; w < W; ++w) sum += exp_plain(to_f32(raw[i].v[w]) - m);
        sum = group_sum<G>(sum);
        inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    }
    // their elements, vector s M + c in lane c
    Word x[S * W], top[K];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        Word mine = Word(0);
#pragma unroll
        for (int j = 0; j < M; ++j) mine = c == j ? first[s * M + j] : mine;
        const bool ok = s * M + c < a.k && Key::available(mine);
        const uint32_t v = Key::index(mine);
#pragma unroll
        for (int w = 0; w < W; ++w) x[s * W + w] = Word(0);
        if (ok) {
            const Vec16<T> y = row.vec((int)v);
            const uint32_t inv0 = kIndexMask ^ (v * W);
#pragma unroll
            for (int w = 0; w < W; ++w) x[s * W + w] = Key::make(to_f32(y.v[w]), inv0 ^ (uint32_t)w);
        }
    }
    lane_top<Key, K, S * W>(x, top);
    group_top<Key, K, M>(top);
    float zc[S], g[S], less[S];
    bool on[S];
    int32_t id[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        Word mine = Word(0);
#pragma unroll
        for (int j = 0; j < M; ++j) mine = c == j ? top[s * M + j] : mine;
        on[s] = s * M + c < a.k && Key::available(mine);
        zc[s] = Key::value(mine);
        id[s] = on[s] ? (int32_t)Key::index(mine) : -1;
    }
    choice_gates<M, S>(zc, on, a.score, a.normalize, m, inv, g, less);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int j = s * M + c;
        if (it.live && c < M && j < a.k) {
            a.ids[it.at * a.k + j] = id[s];
            a.gates[it.at * a.k + j] = a.scale * g[s];
        }
    }
}

// A double's order as an unsigned number (-0 equals +0); 0 stands for "not
// available".
__device__ inline uint64_t order64(double x) {
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | (uint64_t)1 << 63;
}

// One round of a maximum over (key, -index) across the G lanes.
template <int G, int D = 2>
__device__ inline void group_first(uint64_t &key, uint32_t &at) {
    if constexpr (D <= G) {
        const uint64_t ok = (uint64_t)across<D>((uint32_t)(key >> 32)) << 32 | across<D>((uint32_t)key);
        const uint32_t oa = across<D>(at);
        const bool take = ok > key || (ok == key && oa < at);
        key = take ? ok : key;
        at = take ? oa : at;
        group_first<G, 2 * D>(key, at);
    }
}

// The choices by score + bias.  The two selections run on keys in 32 bits,
// which are off by at most (64 + 2 |key|) 2^-24 (see below).  Where that
// leaves the order of the k choices, or the last of them against the rest,
// open (two keys within twice that), the wave repeats the selection on keys in
// 64 bits, by k rounds of a maximum over the row: about one wave in a hundred
// with random logits; exact ties always.
//
// A score's error in 32 bits, in steps u = 2^-24: logistic, 8 s u
// (exponential 4 u, the sum, the inverse and the product 4 u); softmax,
// p (|z - m| + 54) u with p |z - m| < 0.37, so at most 55 u.  The
// sum with the bias is rounded once: |key| u.
template <class T, int G, int NV, int K>
__global__ void __launch_bounds__(256) k_route_bias(RouteArgs a) {
    using Key = Key32;
    using Word = Key::Word;
    constexpr int W = 16 / sizeof(T), M = G < K ? G : K, S = K / M;
    const int c = threadIdx.x & (G - 1);
    const Item it = item_of<G>(a.T, a.L);
    const Row<T> row = {static_cast<const T *>(a.logits) + it.t * a.ts + it.l * a.ls, a.E};
    const float *bias = a.bias + (int64_t)it.l * a.E;
    const bool softmax = a.score == ROUTEPACK_SOFTMAX;
    Vec16<T> raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = row.vec(i * G + c);
    float m = 0.0f, inv = 0.0f;
    if (softmax) {
        float z[NV * W];
#pragma unroll
        for (int v = 0; v < NV * W; ++v) z[v] = to_f32(raw[v / W].v[v % W]);
        row_sum<G, NV * W>(z, m, inv);
    }
    // a vector's keys in 32 bits; -inf where the expert is not available
    auto keys_of = [&](const Vec16<T> &r, int v, float (&y)[W]) {
        float b[W];
        if (v * W + W <= a.E) {
#pragma unroll
            for (int w = 0; w < W; ++w) b[w] = bias[v * W + w];
        } else {
#pragma unroll
            for (int w = 0; w < W; ++w) b[w] = v * W + w < a.E ? bias[v * W + w] : -kInf;
        }
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float z = to_f32(r.v[w]);
            float s, less;
            if (softmax) s = exp32(z - m) * inv;
            else logistic(z, s, less);
            const float key = s + b[w];
            y[w] = z > -kInf && key > -kInf ? key : -kInf;
        }
    };
    float mx[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float y[W];
        keys_of(raw[i], i * G + c, y);
        mx[i] = y[0];
#pragma unroll
        for (int w = 1; w < W; ++w) mx[i] = __builtin_fmaxf(mx[i], y[w]);
    }
    Word vk[NV], first[K];
#pragma unroll
    for (int i = 0; i < NV; ++i) vk[i] = Key::make(mx[i], kIndexMask ^ (uint32_t)c ^ (uint32_t)(i * G));
    lane_top<Key, K, NV>(vk, first);
    group_top<Key, K, G>(first);
    Word x[S * W], top[K];
    float near_[S * W], most[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        Word mine = Word(0);
#pragma unroll
        for (int j = 0; j < M; ++j) mine = c == j ? first[s * M + j] : mine;
        const bool ok = c < M && s * M + c < a.k && Key::available(mine);
        const int v = (int)Key::index(mine);
        most[s] = ok ? Key::value(mine) : -kInf;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            x[s * W + w] = Word(0);
            near_[s * W + w] = -kInf;
        }
        if (ok) {
            float y[W];
            keys_of(row.vec(v), v, y);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                near_[s * W + w] = y[w];
                x[s * W + w] = Key::make(y[w], kIndexMask ^ (uint32_t)(v * W + w));
            }
        }
    }
    lane_top<Key, K, S * W>(x, top);
    group_top<Key, K, M>(top);
    // is the order beyond doubt?
    bool open = false;
    float last = 0.0f;
    bool full = false;  // k experts are available
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (j >= a.k || !Key::available(top[j])) continue;
        const float v = Key::value(top[j]);
        if (j > 0) {
            const float u = Key::value(top[j > 0 ? j - 1 : 0]);
            const float slack = (128.0f + 4.0f * __builtin_fmaxf(__builtin_fabsf(u), __builtin_fabsf(v))) * 0x1p-24f;
            open = open || !(u - v > slack);
        }
        if (j == a.k - 1) {
            last = v;
            full = true;
        }
    }
    if (full) {
        const float edge = last - (128.0f + 8.0f * __builtin_fabsf(last)) * 0x1p-24f;
        float over = 0.0f;  // elements at or over the edge, besides the choices, and vectors not taken
#pragma unroll
        for (int n = 0; n < S * W; ++n) over += near_[n] >= edge && near_[n] > -kInf ? 1.0f : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) over += mx[i] >= edge && mx[i] > -kInf ? 1.0f : 0.0f;
#pragma unroll
        for (int s = 0; s < S; ++s) over -= most[s] >= edge && most[s] > -kInf ? 1.0f : 0.0f;
        open = open || !(group_sum<G>(over) == (float)a.k) || !(edge == edge);
    }
    float zc[S], g[S], less[S];
    bool on[S];
    int32_t id[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        Word mine = Word(0);
#pragma unroll
        for (int j = 0; j < M; ++j) mine = c == j ? top[s * M + j] : mine;
        id[s] = s * M + c < a.k && Key::available(mine) ? (int32_t)Key::index(mine) : -1;
    }
    if (__any(open)) {
        uint64_t key[NV * W];
        double sum = 0.0;
        if (softmax) {
#pragma unroll
            for (int v = 0; v < NV * W; ++v) {
                const float z = to_f32(raw[v / W].v[v % W]);
                sum += z > -kInf ? exp((double)z - (double)m) : 0.0;
            }
#pragma unroll
            for (int d = 1; d < G; d <<= 1) sum += __shfl_xor(sum, d, kWave);
        }
#pragma unroll
        for (int v = 0; v < NV * W; ++v) {
            const float z = to_f32(raw[v / W].v[v % W]);
            const int e = elem_of<T, G>(v, c);
            key[v] = 0;
            if (z > -kInf && e < a.E) {
                double s = softmax ? exp((double)z - (double)m) / sum : 1.0 / (1.0 + exp(-(double)z));
                s += (double)bias[e];
                if (s > -__builtin_inf()) key[v] = order64(s);
            }
        }
#pragma unroll
        for (int s = 0; s < S; ++s) id[s] = -1;
        for (int j = 0; j < a.k; ++j) {
            uint64_t best = 0;
            uint32_t at = UINT32_MAX;
#pragma unroll
            for (int v = 0; v < NV * W; ++v) {  // (a lane's elements ascend)
                if (key[v] > best) {
                    best = key[v];
                    at = (uint32_t)elem_of<T, G>(v, c);
                }
            }
            group_first<G>(best, at);
#pragma unroll
            for (int v = 0; v < NV * W; ++v)
                if ((uint32_t)elem_of<T, G>(v, c) == at) key[v] = 0;
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (j == s * M + c && best) id[s] = (int32_t)at;
        }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
        on[s] = c < M && id[s] >= 0;
        zc[s] = on[s] ? to_f32(row.data[id[s]]) : 0.0f;
    }
    choice_gates<M, S>(zc, on, a.score, a.normalize, m, inv, g, less);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int j = s * M + c;
        if (it.live && c < M && j < a.k) {
            a.ids[it.at * a.k + j] = id[s];
            a.gates[it.at * a.k + j] = a.scale * g[s];
        }
    }
}

template <class T>
int choose(const RouteArgs &a, hipStream_t stream) {
    const int64_t items = a.T * a.L;
    auto go = [&](auto kern, int g) {
        hipLaunchKernelGGL(kern, grid_of((items + 256 / g - 1) / (256 / g)), dim3(256), 0, stream, a);
        return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
    };
    if (a.bias)
        return by_geometry<T, 2 * sizeof(T)>(a.E, [&](auto g, auto nv) {
            if (a.k <= 8) return go(k_route_bias<T, g.value, nv.value, 8>, g.value);
            return go(k_route_bias<T, g.value, nv.value, 32>, g.value);
        });
    return by_geometry<T, 8>(a.E, [&](auto g, auto nv) {
        if (a.k <= 4) return go(k_route<T, g.value, nv.value, 4>, g.value);
        if (a.k <= 8) return go(k_route<T, g.value, nv.value, 8>, g.value);
        if (a.k <= 16) return go(k_route<T, g.value, nv.value, 16>, g.value);
        return go(k_route<T, g.value, nv.value, 32>, g.value);
    });
}

}  // namespace rp
