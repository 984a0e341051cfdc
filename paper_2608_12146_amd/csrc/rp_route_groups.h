// The router's choices among a few groups of experts: each token keeps the
// `keep` of its n_groups groups (of E / n_groups adjacent experts) whose
// group_top largest keys have the largest sum, and chooses among their experts.
// Included by one translation unit for each type of logits.
//
// A group lies in Q adjacent lanes (a power of two) of up to V values, a token
// in the Q n_groups lanes of its groups, rounded up to a power of two: a
// group's best keys are reductions over its lanes, its rank is the number of
// groups that precede it, and the choice is the selection of rp_route.h over
// the lanes of the groups kept.
// Without a bias and with group_top = 1 the keys are the logits, whose order
// is the scores'.  Otherwise keys are compared in 64 bits, as two
// implementations in 32 bits would choose differently.
#pragma once

#include "rp_route.h"

namespace rp {

struct GroupArgs {
    RouteArgs r;
    int32_t groups, keep, top;  // top: 1 or 2 keys a group
    int32_t size;               // experts of a group
    int32_t q_shift, lane_shift;  // lanes of a group, of a token (powers of two)
};

__device__ inline double value64(uint64_t o) {
    return __longlong_as_double((long long)(o >> 63 ? o ^ (uint64_t)1 << 63 : ~o));
}

// Reductions over aligned groups of `lanes` lanes, a power of two that is
// uniform: the steps are those of rp_route.h, those beyond it are skipped.
template <int D = 2>
__device__ inline float lanes_max(float v, int lanes) {
    if (D > lanes) return v;
    v = __builtin_fmaxf(v, across<D>(v));
    if constexpr (D < kWave) return lanes_max<2 * D>(v, lanes);
    else return v;
}
template <int D = 2, class T>
__device__ inline T lanes_add(T v, int lanes) {
    if (D > lanes) return v;
    v += across<D>(v);
    if constexpr (D < kWave) return lanes_add<2 * D>(v, lanes);
    else return v;
}
__device__ inline uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ inline uint64_t min64(uint64_t a, uint64_t b) { return a < b ? a : b; }
template <int D>
__device__ inline uint64_t across64(uint64_t v) {
    return (uint64_t)across<D>((uint32_t)(v >> 32)) << 32 | across<D>((uint32_t)v);
}
// The two largest over the lanes.
template <int D = 2>
__device__ inline void lanes_two(uint64_t &first, uint64_t &second, int lanes) {
    if (D > lanes) return;
    const uint64_t f = across64<D>(first), s = across64<D>(second);
    second = max64(min64(first, f), max64(second, s));
    first = max64(first, f);
    if constexpr (D < kWave) lanes_two<2 * D>(first, second, lanes);
}
// The largest (key, -index) over the lanes.
template <int D = 2>
__device__ inline void lanes_first(uint64_t &key, uint32_t &at, int lanes) {
    if (D > lanes) return;
    const uint64_t ok = across64<D>(key);
    const uint32_t oa = across<D>(at);
    const bool take = ok > key || (ok == key && oa < at);
    key = take ? ok : key;
    at = take ? oa : at;
    if constexpr (D < kWave) lanes_first<2 * D>(key, at, lanes);
}
template <class Key, int K, int D = 2>
__device__ inline void lanes_top(typename Key::Word (&top)[K], int lanes) {
    if (D > lanes) return;
    typename Key::Word y[K];
#pragma unroll
    for (int i = 0; i < K; ++i) y[i] = across<D>(top[i]);
    merge_top<Key, K>(top, y);
    if constexpr (D < kWave) lanes_top<Key, K, 2 * D>(top, lanes);
}

// Whether group g's best (an order, 0 where none is available) is among the
// `keep` largest: the groups that precede it are counted.  Every lane of the
// token's group calls it with its own.
__device__ inline bool kept(const GroupArgs &a, uint64_t best, int g, int first_lane_of_token) {
    int before = 0;
    for (int o = 0; o < a.groups; ++o) {
        const int from = first_lane_of_token + (o << a.q_shift);
        const uint64_t b = (uint64_t)(uint32_t)__shfl((int)(best >> 32), from, kWave) << 32 |
                           (uint32_t)__shfl((int)(uint32_t)best, from, kWave);
        before += b > best || (b == best && o < g) ? 1 : 0;
    }
    return best != 0 && before < a.keep;
}

template <class T, int V, int K, bool SCORES>
__global__ void __launch_bounds__(256) k_route_groups(GroupArgs ga) {
    using Key = typename KeyOf<T>::type;
    using Word = typename Key::Word;
    constexpr int W = 16 / sizeof(T);
    const RouteArgs &a = ga.r;
    const int lanes = 1 << ga.lane_shift, Q = 1 << ga.q_shift;
    const int c = threadIdx.x & (lanes - 1), g = c >> ga.q_shift, q = c & (Q - 1);
    // (the token and layer, as item_of)
    const int64_t n = a.T * a.L;
    int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (256 >> ga.lane_shift) + (threadIdx.x >> ga.lane_shift);
    const bool live = at < n;
    at = live ? at : n - 1;
    const int64_t t = a.L == 1 ? at : n <= UINT32_MAX ? (uint32_t)at / (uint32_t)a.L : at / a.L;
    const int32_t l = (int32_t)(at - t * a.L);
    const T *data = static_cast<const T *>(a.logits) + t * a.ts + l * a.ls;
    const Row<T> row = {data + g * ga.size, g < ga.groups ? ga.size : 0};
    float z[V];
#pragma unroll
    for (int i = 0; i < V / W; ++i) {
        const Vec<T> x = row.vec(i * Q + q);
#pragma unroll
        for (int w = 0; w < W; ++w) z[i * W + w] = x.at(w);
    }
    // element v of this lane within its group
    auto elem = [&](int v) { return ((v / W) * Q + q) * W + v % W; };
    const int lane0 = (int)(threadIdx.x & 63) - c;
    const bool softmax = a.score == ROUTEPACK_SOFTMAX;
    float m = 0.0f, inv = 0.0f;
    if (softmax && !a.normalize) {
        m = -kInf;
#pragma unroll
        for (int v = 0; v < V; ++v) m = __builtin_fmaxf(m, z[v]);
        m = lanes_max(m, lanes);
        m = m == -kInf ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) sum += exp_plain(z[v] - m);
        sum = lanes_add(sum, lanes);
        inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    }
    constexpr int S = K >= 32 ? 8 : K / 4;  // choices of each of the first lanes
    constexpr int M = K / S;                // (4 lanes)
    int32_t id[K];
    if constexpr (!SCORES) {
        uint32_t best = 0;
        Word x[V], top[K];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t o = order32(z[v]);
            best = o > best ? o : best;
            x[v] = Key::make(z[v], kIndexMask ^ (uint32_t)(g * ga.size + elem(v)));
        }
        best = best > 0x007FFFFFu ? best : 0;
        uint64_t f = best, s = 0;
        lanes_two(f, s, Q);
        const bool on = kept(ga, f, g, lane0);
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = on ? x[v] : Word(0);
        lane_top<Key, K, V>(x, top);
        lanes_top<Key, K>(top, lanes);
#pragma unroll
        for (int j = 0; j < K; ++j) id[j] = j < a.k && Key::available(top[j]) ? (int32_t)Key::index(top[j]) : -1;
    } else {
        uint64_t key[V];
        double sum = 1.0, base = 0.0;
        if (softmax) {  // NaN takes no part; experts of +inf share the scores alone
            float b = -kInf;
#pragma unroll
            for (int v = 0; v < V; ++v) b = z[v] > b ? z[v] : b;
            b = lanes_max(b, lanes);
            base = b;
            sum = 0.0;
#pragma unroll
            for (int v = 0; v < V; ++v) sum += z[v] > -kInf ? exp(__builtin_fmin((double)z[v] - base, 0.0)) : 0.0;
            sum = lanes_add(sum, lanes);
        }
        uint64_t f = 0, s = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = elem(v);
            double k0 = softmax ? exp(__builtin_fmin((double)z[v] - base, 0.0)) / sum : 1.0 / (1.0 + exp(-(double)z[v]));
            if (a.bias && e < row.E) k0 += (double)a.bias[(int64_t)l * a.E + g * ga.size + e];
            key[v] = z[v] > -kInf && k0 > -__builtin_inf() ? order64(k0) : 0;
            s = max64(s, min64(f, key[v]));
            f = max64(f, key[v]);
        }
        lanes_two(f, s, Q);
        if (ga.top == 2 && s) f = order64(value64(f) + value64(s));
        const bool on = kept(ga, f, g, lane0);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = on ? key[v] : 0;
#pragma unroll
        for (int j = 0; j < K; ++j) id[j] = -1;
#pragma unroll 1
        for (int j = 0; j < a.k; ++j) {
            uint64_t k0 = 0;
            uint32_t e0 = UINT32_MAX;
#pragma unroll
            for (int v = 0; v < V; ++v) {  // (a lane's elements ascend)
                const bool more = key[v] > k0;
                k0 = more ? key[v] : k0;
                e0 = more ? (uint32_t)(g * ga.size + elem(v)) : e0;
            }
            lanes_first(k0, e0, lanes);
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = (uint32_t)(g * ga.size + elem(v)) == e0 ? 0 : key[v];
#pragma unroll
            for (int i = 0; i < K; ++i) id[i] = i == j && k0 ? (int32_t)e0 : id[i];
        }
    }
    // the gates: choice s M + c in lane c < M (of the token's 4 lanes and more)
    float zc[S], w[S], less[S];
    bool on[S];
    int32_t mine[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        mine[s] = -1;
#pragma unroll
        for (int j = 0; j < M; ++j) mine[s] = c == j ? id[s * M + j] : mine[s];
        on[s] = mine[s] >= 0;
        zc[s] = on[s] ? to_f32(data[mine[s]]) : 0.0f;
    }
    choice_gates<M, S>(zc, on, a.score, a.normalize, m, inv, w, less);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int j = s * M + c;
        if (live && c < M && j < a.k) {
            a.ids[at * a.k + j] = mine[s];
            a.gates[at * a.k + j] = a.scale * w[s];
        }
    }
}

// Lanes of a group and a token: as few as hold the group in V values a lane
// (at least 4 a token, for the gates).
template <class T>
int choose_groups(GroupArgs a, hipStream_t stream) {
    constexpr int W = 16 / sizeof(T);
    int groups = 1;  // rounded up to a power of two
    a.lane_shift = 0;
    while (groups < a.groups) {
        groups *= 2;
        ++a.lane_shift;
    }
    a.q_shift = 0;
    const int vecs = (a.size + W - 1) / W;
    while ((vecs + (1 << a.q_shift) - 1) / (1 << a.q_shift) * W > (sizeof(T) == 4 ? 16 : 32) && (groups << a.q_shift) < kWave)
        ++a.q_shift;
    while ((groups << a.q_shift) < 4) ++a.q_shift;
    a.lane_shift += a.q_shift;
    const int V = (vecs + (1 << a.q_shift) - 1) / (1 << a.q_shift) * W;
    const int64_t items = a.r.T * a.r.L, per = 256 >> a.lane_shift;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid_of((items + per - 1) / per), dim3(256), 0, stream, a);
        return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
    };
    auto by_k = [&](auto v) {
        constexpr int N = decltype(v)::value;
        const bool scores = a.r.bias || a.top > 1;
        if (a.r.k <= 8) return scores ? go(k_route_groups<T, N, 8, true>) : go(k_route_groups<T, N, 8, false>);
        return scores ? go(k_route_groups<T, N, 32, true>) : go(k_route_groups<T, N, 32, false>);
    };
    if (V <= 8) return by_k(Int<8>());
    if (V <= 16) return by_k(Int<16>());
    if (V <= 32) return by_k(Int<32>());
    return ROUTEPACK_E_UNSUPPORTED;
}

}  // namespace rp
