// The gradient of gates and balance loss with respect to the logits.  Included
// by one translation unit for each type of logits.
//
// A token's row is read once and its gradient written once:
//   dz = D + p (f - sum p f - sum D)           softmax
//   dz = D + s' (1 - s) (f - sum s' f)         logistic, s' = s / sum s
// with D the chosen experts' part (sum D enters where the gates are not
// normalised) and f the loss's weight of every expert, which a group of lanes
// keeps in registers as long as its tokens belong to one group of the loss.
// D goes through a row of LDS, zero but for the choices, to the lanes that hold
// their experts: that costs an eighth of the LDS reads that comparing every
// element with every choice would cost in instructions.
//
// 131072 x 512 bf16, both parts: 58 us, 4.7 TB/s read and written, where a
// large copy reaches 4.9 to 5.4; its 16 vector instructions an element, one of
// them an exponential, would take 32 us alone.  Logistic rows take 86 us, about
// 73 of them the issue of 37 vector instructions an element, two of a quarter of
// the others' rate.
#pragma once

#include "rp_route.h"

namespace rp {

// The group of the loss that holds token t (the last one that begins at or
// before it), or -1, and where it begins and ends; the G lanes of a token
// probe together.  The whole wave takes part.
template <int G>
__device__ inline int32_t find_group(const int64_t *offsets, int32_t n, int64_t t, int64_t &begin, int64_t &end) {
    const int c = threadIdx.x & (G - 1);
    const int base = lane_id() & ~(G - 1);
    int32_t lo = 0, hi = n;
    while (__any(hi - lo > 1)) {
        const int32_t step = (hi - lo - 1) / (G + 1) + 1;  // (of any n up to 2^31 - 1)
        const int64_t p = lo + (int64_t)(c + 1) * step;
        const uint64_t yes = __ballot(p < hi && offsets[p < hi ? p : lo] <= t);
        const int cnt = __popcll(yes >> base & low_lanes(G));
        const int64_t to = lo + (int64_t)(cnt + 1) * step;
        lo += cnt * step;
        hi = to < hi ? (int32_t)to : hi;
    }
    begin = offsets[lo];
    end = offsets[lo + 1];
    return t >= begin && t < end ? lo : -1;
}

// f of one group: E counts / sum counts, times dloss / (groups tokens).
template <class T, int G, int V, bool WHOLE>
__device__ inline void load_weights(const BackArgs &a, int32_t g, int32_t l, int64_t len, int c, float (&f)[V]) {
    const int64_t at = ((int64_t)g * a.L + l) * a.E;
    int64_t sum = 0;
    if (a.counts_type == ROUTEPACK_I32) {
        const Row<float, WHOLE> row = {static_cast<const float *>(a.counts) + at, a.E};  // (words of 32 bits)
#pragma unroll
        for (int v = 0; v < V; v += 4) {
            const int e0 = elem_of<T, G>(v, c);
            const Vec<float> x = row.vec(e0 / 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t n = WHOLE || e0 + i < a.E ? (int32_t)x.w[i] : 0;
                sum += n;
                f[v + i] = (float)n;
            }
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = elem_of<T, G>(v, c);
            const int64_t n = WHOLE || e < a.E ? static_cast<const int64_t *>(a.counts)[at + e] : 0;
            sum += n;
            f[v] = __builtin_fmaf((float)(int32_t)(n >> 32), 0x1p32f, (float)(uint32_t)n);
        }
    }
    sum = group_sum64<G>(sum);
    const float by = sum > 0 ? (float)a.E / (float)sum * (a.dloss[l] / ((float)a.n_groups * (float)len)) : 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] *= by;
}

template <class T, int G, int NV, int K, bool SOFTMAX, bool WHOLE>
__global__ void __launch_bounds__(256) k_route_back(BackArgs a, int32_t iters) {
    constexpr int W = 16 / sizeof(T), V = NV * W, S = K > G ? K / G : 1, SLOTS = 256 / G;
    constexpr bool FINE = sizeof(T) == 4;  // (else the result's rounding hides the plain exponential's error)
    __shared__ __align__(16) float direct_rows[SLOTS][G * V];
    const int c = threadIdx.x & (G - 1), slot = threadIdx.x / G;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t ch = a.L == 1 ? block : block / a.L;
    const int32_t l = a.L == 1 ? 0 : (int32_t)(block - ch * a.L);
    const bool gates = a.ids != nullptr, loss = a.dloss != nullptr;
    const bool whole = loss || (SOFTMAX && !a.normalize);  // the row's scores take part
    float *direct = direct_rows[slot];
    if (gates) {
#pragma unroll
        for (int v = 0; v < V; v += 4)
            *reinterpret_cast<float4 *>(direct + elem_of<T, G>(v, c)) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        wave_sync();
    }
    float f[V];
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = 0.0f;
    int64_t begin = 0, end = 0;  // the tokens that f stands for
    bool known = false;
    for (int32_t r = 0; r < iters; ++r) {
        int64_t t = (ch * iters + r) * SLOTS + slot;
        const bool live = t < a.T;
        t = live ? t : a.T - 1;
        const T *row = static_cast<const T *>(a.logits) + t * a.ts + l * a.ls;
        float z[V], less[SOFTMAX ? 1 : V];
        int32_t id[S];
        float zc[S], dg[S];
        bool on[S];
        if (whole) load_row<T, G, V, WHOLE>(row, a.E, c, z);
        if (gates) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int j = s * G + c;
                id[s] = -1;
                zc[s] = dg[s] = 0.0f;
                if (j < a.k) id[s] = load_id(a.ids, a.id_type, t * a.its + l * a.ils + j, a.E);
                on[s] = id[s] >= 0;
                if (on[s]) {
                    zc[s] = to_f32(row[id[s]]);
                    dg[s] = a.dgates[(t * a.L + l) * a.k + j];
                }
            }
        }
        if (loss && __any(!known || t < begin || t >= end)) {
            const int32_t g = find_group<G>(a.offsets, a.n_groups, t, begin, end);
            known = g >= 0;
            if (g >= 0) {
                load_weights<T, G, V, WHOLE>(a, g, l, end - begin, c, f);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) f[v] = 0.0f;
            }
        }
        float m = 0.0f, inv = 0.0f, drop = 0.0f;
        if (whole) {
            if constexpr (SOFTMAX) softmax_row<FINE, G, V>(z, m, inv);
            else logistic_row<FINE, G, V>(z, less, inv);
        }
        if (gates) {
            float w[S], sl[S], d[S];
            choice_gates<G, S>(zc, on, SOFTMAX ? ROUTEPACK_SOFTMAX : ROUTEPACK_SIGMOID, a.normalize, m, inv, w, sl);
            float dot = 0.0f;
            if (a.normalize) {
#pragma unroll
                for (int s = 0; s < S; ++s) dot += on[s] ? w[s] * dg[s] : 0.0f;
                dot = group_sum<G>(dot);
            }
#pragma unroll
            for (int s = 0; s < S; ++s) {
                d[s] = on[s] ? a.scale * w[s] * (dg[s] - dot) : 0.0f;
                if (!SOFTMAX && on[s]) d[s] *= sl[s];
            }
            if (SOFTMAX && !a.normalize) {
#pragma unroll
                for (int s = 0; s < S; ++s) drop += d[s];
                drop = group_sum<G>(drop);
            }
            // Does an expert occur twice?  Every choice leaves its mark.
            bool twice = false;
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (on[s]) direct[id[s]] = (float)(s * G + c);
            wave_sync();
#pragma unroll
            for (int s = 0; s < S; ++s) twice = twice || (on[s] && direct[id[s]] != (float)(s * G + c));
            if (__any(twice)) {  // its parts are added in the order of the choices
                wave_sync();
#pragma unroll
                for (int s = 0; s < S; ++s)
                    if (on[s]) direct[id[s]] = 0.0f;
                wave_sync();
#pragma unroll
                for (int s = 0; s < S; ++s)
                    for (int j = 0; j < G; ++j) {
                        if (c == j && on[s]) direct[id[s]] += d[s];
                        wave_sync();
                    }
            } else {
                wave_sync();
#pragma unroll
                for (int s = 0; s < S; ++s)
                    if (on[s]) direct[id[s]] = d[s];
                wave_sync();
            }
        }
        float mean = 0.0f;
        if (whole) {
            // (z holds the scores before the factor inv)
            float dot = 0.0f;
            if (loss) {
#pragma unroll
                for (int v = 0; v < V; ++v) dot = __builtin_fmaf(z[v], f[v], dot);
                dot = group_sum<G>(dot) * inv;
            }
            mean = -(dot + drop) * inv;
        }
        // padding may hold anything, NaN among it: where the gates do not need the
        // row, nothing of it reaches the gradient
        const bool part = whole && (known || !loss || (gates && SOFTMAX && !a.normalize));
        T *to = static_cast<T *>(a.dlogits) + (t * a.L + l) * a.E;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float y[W];
            const int e0 = (i * G + c) * W;
#pragma unroll
            for (int w = 0; w < W; ++w) y[w] = 0.0f;
            if (gates) {
#pragma unroll
                for (int w = 0; w < W; w += 4) {
                    const float4 x = *reinterpret_cast<const float4 *>(direct + e0 + w);
                    y[w] = x.x;
                    y[w + 1] = x.y;
                    y[w + 2] = x.z;
                    y[w + 3] = x.w;
                }
            }
            if (part) {
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const int v = i * W + w;
                    const float rel = __builtin_fmaf(f[v], inv, mean);
                    if constexpr (SOFTMAX) y[w] = __builtin_fmaf(z[v], rel, y[w]);
                    else y[w] = __builtin_fmaf(z[v] * less[v], rel, y[w]);
                }
            }
            if (live) store_vec<T, WHOLE>(to, a.E, e0, y);
        }
        if (gates) {
            wave_sync();
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (on[s]) direct[id[s]] = 0.0f;
            wave_sync();
        }
    }
}

template <class T, bool SOFTMAX, int G, int NV>
int launch_back(const BackArgs &a, hipStream_t stream) {
    const int64_t slots = 256 / G, n = (a.T + slots - 1) / slots;
    // Several tokens a group of lanes, which loads the weights of a group of the
    // loss once for them, where that leaves 1024 workgroups (131072 x 512 bf16
    // takes 1.03 times as long at 4 tokens as at 8, and 1.6 times at 1; 1797 x 23
    // x 432 1.2 times at 1 as at 2).
    int64_t iters = n * a.L / 1024;
    iters = iters < 1 ? 1 : (iters > 8 ? 8 : iters);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid_of((n + iters - 1) / iters * a.L), dim3(256), 0, stream, a, (int32_t)iters);
        return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
    };
    // Up to 8 choices, and rows that fill the lanes exactly (E a power of two,
    // mostly), take kernels without the further slots and the checks of every
    // vector (131072 x 512 bf16 takes 1.13 times as long with the checks, 9 choices
    // of 110325 x 5 x 28 fp32 1.3 times with 32 slots as with 16).
    const bool few = !a.ids || a.k <= 8, fills = a.E == G * NV * (16 / (int)sizeof(T));
    if (few && fills) return go(k_route_back<T, G, NV, 8, SOFTMAX, true>);
    if (few) return go(k_route_back<T, G, NV, 8, SOFTMAX, false>);
    if (a.k <= 16) return go(k_route_back<T, G, NV, 16, SOFTMAX, false>);
    return go(k_route_back<T, G, NV, 32, SOFTMAX, false>);
}

template <class T>
int route_back(const BackArgs &a, hipStream_t stream) {
    constexpr int kMost = 2 * sizeof(T);  // 32 values a lane
    if (a.score == ROUTEPACK_SOFTMAX)
        return by_geometry<T, kMost>(a.E, [&](auto g, auto nv) {
            return launch_back<T, true, g.value, nv.value>(a, stream);
        });
    // logistic rows keep 1 - s too: 16 values a lane while the wave holds the row
    if (a.E > 1024) return launch_back<T, false, kWave, kMost>(a, stream);
    return by_geometry<T, kMost / 2>(a.E, [&](auto g, auto nv) {
        return launch_back<T, false, g.value, nv.value>(a, stream);
    });
}

}  // namespace rp
