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
//
// Bound by the read of the logits at size: 131072 x 512 bf16, 8 choices, 27 us
// (5.3 TB/s; a large copy reaches 5.4), 131072 x 256 fp32 30 us (4.9 TB/s); k
// rounds of a maximum over the row took 297 us for the first.  4 lanes and more
// a token, with up to 8 vectors each: fewer lanes merge in fewer steps (each
// step costs K maxima and K log K / 2 exchanges), 4 keep a load's lines whole.
// One token: 3 us, a launch and two dependent reads.
#pragma once

#include "rp_route.h"

namespace rp {

template <class T, int G, int NV, int K>
__global__ void __launch_bounds__(256) k_route(RouteArgs a) {
    using Key = typename KeyOf<T>::type;
    using Word = typename Key::Word;
    constexpr int W = 16 / sizeof(T), M = G < K ? G : K, S = K / M;
    const int c = threadIdx.x & (G - 1);
    const Item it = item_of<G>(a.T, a.L);
    const Row<T> row = {static_cast<const T *>(a.logits) + it.t * a.ts + it.l * a.ls, a.E};
    Vec<T> raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = row.vec(i * G + c);
    // the k vectors of largest maximum
    float mx[NV];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float x[W];
#pragma unroll
        for (int w = 0; w < W; ++w) x[w] = raw[i].at(w);
        mx[i] = most_of(x);
        odd = odd || mx[i] != mx[i];
    }
    if (__any(odd)) {  // NaN among the logits
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            mx[i] = -kInf;
#pragma unroll
            for (int w = 0; w < W; ++w) mx[i] = __builtin_fmaxf(mx[i], raw[i].at(w) + 0.0f);
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
            for (int w = 0; w < W; ++w) sum += exp_plain(raw[i].at(w) - m);
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
            const Vec<T> y = row.vec((int)v);
            const uint32_t inv0 = kIndexMask ^ (v * W);
#pragma unroll
            for (int w = 0; w < W; ++w) x[s * W + w] = Key::make(y.at(w), inv0 ^ (uint32_t)w);
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

template <class T, int N>
__device__ inline void shift_down(T (&a)[N]) {
#pragma unroll
    for (int i = 0; i + 1 < N; ++i) a[i] = a[i + 1];
}

// The choices by score + bias.  The two selections run on keys in 32 bits.
// Where their error leaves the order of the k choices, or the last of them
// against the rest, open, the wave orders the elements of the vectors in
// question (the chosen ones and, in a second batch, the next K) by keys in 64
// bits, or the whole row where even the second batch does not hold every
// candidate.  With random logits about one token in 500 is open and none needs
// the whole row; tokens with equal keys always are.  That part is loops of
// little code: few waves run it, each would wait for all of its instructions.
//
// A score's error in 32 bits, in steps u = 2^-24 (the plain exponential e^x is
// off by (1.3 |x| + 2) u, and z - m is rounded once):
// - logistic: s (1 - s) (1.3 |z| + 2) u, at most 0.8 u as s (1 - s) |z| < 0.23,
//   and 4 u of the sum, the inverse and the product: below 8 u;
// - softmax: p (2.3 |z - m| + 2) u with p |z - m| < 0.37, and of p the row sum's
//   error: 38 additions, 2.3 times the mean of |z - m| (at most ln 2048) and 7
//   more: at most (1 + 66 p) u, and p is at most inv, the inverse of the sum.
// The sum with the bias is rounded once: |key| u.
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
    Vec<T> raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = row.vec(i * G + c);
    float m = 0.0f, inv = 0.0f;
    if (softmax) {
        float z[NV * W];
#pragma unroll
        for (int v = 0; v < NV * W; ++v) z[v] = raw[v / W].at(v % W);
        row_sum<G, NV * W>(z, m, inv);
    }
    // a vector's keys in 32 bits; -inf where the expert is not available
    const Row<float> bias_row = {bias, a.E};
    auto keys_of = [&](const Vec<T> &r, int v, float (&y)[W]) {
        Vec<float> b[W / 4];
#pragma unroll
        for (int n = 0; n < W / 4; ++n) b[n] = bias_row.vec(v * (W / 4) + n);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float z = r.at(w);
            float s, less;
            if (softmax) s = exp_plain(z - m) * inv;
            else logistic<false>(z, s, less);
            const float key = s + b[w / 4].at(w % 4);
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
    float cand[S * W], most[S];
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
            cand[s * W + w] = -kInf;
        }
        if (ok) {
            float y[W];
            keys_of(row.vec(v), v, y);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                cand[s * W + w] = y[w];
                x[s * W + w] = Key::make(y[w], kIndexMask ^ (uint32_t)(v * W + w));
            }
        }
    }
    lane_top<Key, K, S * W>(x, top);
    group_top<Key, K, M>(top);
    // is the order beyond doubt?  Two keys further apart than `slack` are in order.
    const float err = softmax ? 1.0f + 66.0f * inv : 8.0f;
    auto slack = [&](float key) { return (err + 2.0f * __builtin_fabsf(key)) * 0x1p-23f; };
    bool open = false;
    float edge = -kInf;  // a key below it is not among the k largest
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (j >= a.k || !Key::available(top[j])) continue;
        const float v = Key::value(top[j]);
        if (j > 0) {
            const float u = Key::value(top[j > 0 ? j - 1 : 0]);
            open = open || !(u - v > slack(u) && u - v > slack(v));
        }
        if (j == a.k - 1) edge = v - slack(v);
    }
    edge = group_max<G>(edge);  // (lanes from M on hold no list)
    // from the edge on: elements of the chosen vectors, and other vectors
    float over = 0.0f, more = 0.0f;
#pragma unroll
    for (int n = 0; n < S * W; ++n) over += cand[n] >= edge && cand[n] > -kInf ? 1.0f : 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) more += mx[i] >= edge && mx[i] > -kInf ? 1.0f : 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) more -= most[s] >= edge && most[s] > -kInf ? 1.0f : 0.0f;
    over = group_sum<G>(over);
    more = group_sum<G>(more);
    open = open || (edge > -kInf && (over != (float)a.k || more != 0.0f)) || edge != edge;
    // a softmax row with NaN or +inf has no keys in 32 bits
    const bool odd = inv != inv;
    open = open || odd;
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
        const bool any_odd = __any(odd);
        float base = m;  // the largest logit that is no NaN
        if (any_odd) {
            base = -kInf;
#pragma unroll 1
            for (int i = 0; i < NV; ++i) {
                const Vec<T> y = row.vec(i * G + c);
#pragma unroll
                for (int w = 0; w < W; ++w) base = y.at(w) > base ? y.at(w) : base;
            }
            base = group_max<G>(base);
        }
        // e^(z - base) in 64 bits; the minimum makes inf - inf a 0
        auto part = [&](float z) { return exp(__builtin_fmin((double)z - (double)base, 0.0)); };
        double sum = 0.0;
        if (softmax) {
#pragma unroll 1
            for (int i = 0; i < NV; ++i) {
                float z[W];
                const Vec<T> y = row.vec(i * G + c);
#pragma unroll
                for (int w = 0; w < W; ++w) z[w] = y.at(w);
#pragma unroll 1
                for (int w = 0; w < W; ++w) {
                    sum += z[0] > -kInf ? part(z[0]) : 0.0;
                    shift_down(z);
                }
            }
#pragma unroll
            for (int d = 1; d < G; d <<= 1) sum += __shfl_xor(sum, d, kWave);
        }
        Word next[K];
#pragma unroll
        for (int j = 0; j < K; ++j) next[j] = Word(0);
        const bool second = __any(more > 0.0f);
        bool deep = any_odd;
        if (second) {  // the vectors after the first k
            Word kth = Word(0);
#pragma unroll
            for (int j = 0; j < K; ++j) kth = j == a.k - 1 ? first[j] : kth;
#pragma unroll
            for (int i = 0; i < NV; ++i) vk[i] = Key::available(kth) && vk[i] < kth ? vk[i] : Word(0);
            lane_top<Key, K, NV>(vk, next);
            group_top<Key, K, G>(next);
            deep = deep || __any(Key::available(next[K - 1]) && Key::value(next[K - 1]) >= edge);
        }
        int at[2 * S];  // this lane's vectors of both batches
#pragma unroll
        for (int s = 0; s < 2 * S; ++s) {
            Word mine = Word(0);
#pragma unroll
            for (int j = 0; j < M; ++j) {
                const Word w = s < S ? first[s % S * M + j] : next[s % S * M + j];
                mine = c == j ? w : mine;
            }
            const bool ok = c < M && (s >= S || s * M + c < a.k) && Key::available(mine);
            at[s] = ok ? (int)Key::index(mine) : kMaxExperts;
        }
        // a lane's K largest candidates, sorted by insertion
        uint64_t best[K];
        uint32_t who[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            best[j] = 0;
            who[j] = UINT32_MAX;
        }
#pragma unroll 1
        for (int i = 0; i < (deep ? NV : second ? 2 * S : S); ++i) {
            int v = i * G + c;
            if (!deep) {
                v = at[0];
                shift_down(at);
            }
            if (v * W >= a.E) continue;
            float z[W], b[W];
            const Vec<T> y = row.vec(v);
            Vec<float> bv[W / 4];
#pragma unroll
            for (int n = 0; n < W / 4; ++n) bv[n] = bias_row.vec(v * (W / 4) + n);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                z[w] = y.at(w);
                b[w] = bv[w / 4].at(w % 4);
            }
#pragma unroll 1
            for (int w = 0; w < W; ++w) {
                double key = softmax ? part(z[0]) / sum : 1.0 / (1.0 + exp(-(double)z[0]));
                key += (double)b[0];
                uint64_t k0 = z[0] > -kInf && key > -__builtin_inf() ? order64(key) : 0;
                uint32_t e0 = (uint32_t)(v * W + w);
                shift_down(z);
                shift_down(b);
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    const bool before = k0 > best[j] || (k0 == best[j] && e0 < who[j]);
                    const uint64_t k1 = best[j];
                    const uint32_t e1 = who[j];
                    best[j] = before ? k0 : k1;
                    who[j] = before ? e0 : e1;
                    k0 = before ? k1 : k0;
                    e0 = before ? e1 : e0;
                }
            }
        }
#pragma unroll
        for (int s = 0; s < S; ++s) id[s] = -1;
#pragma unroll 1
        for (int j = 0; j < a.k; ++j) {
            uint64_t k0 = best[0];
            uint32_t e0 = who[0];
            group_first<G>(k0, e0);
            if (who[0] == e0) {
                shift_down(best);
                shift_down(who);
                best[K - 1] = 0;
                who[K - 1] = UINT32_MAX;
            }
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (j == s * M + c && k0) id[s] = (int32_t)e0;
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
            if (a.k <= 16) return go(k_route_bias<T, g.value, nv.value, 16>, g.value);
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
