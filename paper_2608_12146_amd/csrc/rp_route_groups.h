// The router's choices among a few groups of experts: each token keeps the
// `keep` of its n_groups groups (of E / n_groups adjacent experts) whose
// group_top largest keys have the largest sum, and chooses among their experts.
// Included by one translation unit for each type of logits.
//
// A group lies in Q adjacent lanes (a power of two) of up to 8 vectors of 16
// bytes, a token in the Q n_groups lanes of its groups, rounded up to a power of
// two and 8: a group's best keys are reductions over its lanes, its rank is the
// number of groups that precede it, and the choice runs as without groups
// (rp_route_choose.h) over the vectors of the groups kept: their maxima, then the
// elements of the k vectors that lead.  Few lanes, as each doubling costs a merge
// of lists: 8 lanes of 8 vectors a token.
//
// Without a bias the keys' order is the logits', and only sums of two scores
// rank groups.  Scores are compared in 64 bits, as two implementations in 32
// bits would choose differently: they are formed in 32 bits, and where their
// error leaves the groups kept, the choices or their order open, the wave forms
// them in 64.  With a bias that is one token in 200 at most, and ties.  Without one
// the error is absolute while the scores of wide logits crowd at 0 (or 1), and it
// grows with the logits' deviation: of 256 experts in 8 groups, 8 choices, at 1.5, 5
// and 8 softmax leaves 0.3, 8 and 37% of the tokens open (65536 fp32: 44, 72, 145 us)
// and logistic scores 0.1, 56 and 100% (34, 143, 176 us).
//
// Bound by HBM and vector instructions: 131072 x 512 bf16, 8 groups: 40 us
// (a copy of the logits takes 26); 65536 x 256 fp32, logistic, two keys a group
// and a bias: 39 us (78 with all keys in 64 bits); 48255 x 352 bf16 in 16 groups,
// softmax, two keys a group: 53 us (105 with scores as the experts' keys, where
// equal logits left a third of the tokens in doubt).
#pragma once

#include "rp_route.h"

namespace rp {

struct GroupArgs {
    RouteArgs r;
    int32_t groups, keep, top;  // top: 1 or 2 keys a group
    int32_t size;               // experts of a group
    int32_t q_shift, lane_shift;  // lanes of a group, of a token (powers of two)
};

template <bool B, class X, class Y> struct Choose { using type = X; };
template <class X, class Y> struct Choose<false, X, Y> { using type = Y; };

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
template <int D = 2>
__device__ inline void lanes_two(float &first, float &second, int lanes) {
    if (D > lanes) return;
    const float f = across<D>(first), s = across<D>(second);
    second = __builtin_fmaxf(__builtin_fminf(first, f), __builtin_fmaxf(second, s));
    first = __builtin_fmaxf(first, f);
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
// The K largest of the lanes' lists, in every lane, in no order: the upper half of
// the lanes has them the other way round.  (A loop over the steps: one network for
// all of them, where a network for each took twice the registers.)
template <int D, class T, int K>
__device__ inline void all_across(const T (&x)[K], T (&y)[K]) {
#pragma unroll
    for (int i = 0; i < K; ++i) y[i] = across<D>(x[i]);
}
template <class Key, int K>
__device__ inline void lanes_top(typename Key::Word (&top)[K], int lanes) {
#pragma unroll 1
    for (int d = 2;; d *= 2) {
        typename Key::Word y[K];
        switch (d) {
            case 2: all_across<2>(top, y); break;
            case 4: all_across<4>(top, y); break;
            case 8: all_across<8>(top, y); break;
            case 16: all_across<16>(top, y); break;
            case 32: all_across<32>(top, y); break;
            default: all_across<64>(top, y);
        }
#pragma unroll
        for (int i = 0; i < K; ++i) top[i] = Key::max(top[i], y[K - 1 - i]);
        if (d >= lanes) break;  // (the last step need not sort)
        bitonic_sort<Key, 0, K>(top);
    }
}

// The groups that precede group g of the token whose lanes begin at lane0: with
// a larger `best`, or an equal one and a lower index.  Every lane of a group
// calls it with its group's.
__device__ inline int groups_before(int groups, int q_shift, float best, int g, int lane0) {
    int n = 0;
    for (int o = 0; o < groups; ++o) {
        const float b = __shfl(best, lane0 + (o << q_shift), kWave);
        n += b > best || (b == best && o < g) ? 1 : 0;
    }
    return n;
}
__device__ inline int groups_before(int groups, int q_shift, uint64_t best, int g, int lane0) {
    int n = 0;
    for (int o = 0; o < groups; ++o) {
        const int from = lane0 + (o << q_shift);
        const uint64_t b = (uint64_t)(uint32_t)__shfl((int)(best >> 32), from, kWave) << 32 |
                           (uint32_t)__shfl((int)(uint32_t)best, from, kWave);
        n += b > best || (b == best && o < g) ? 1 : 0;
    }
    return n;
}

// What the keys are: the logits, whose order is the scores' (kLogits); the same for
// the experts, while groups go by the sum of two scores (kSums); scores with a bias
// (kBiased).  WHOLE: every lane's vectors are whole.
enum { kLogits, kSums, kBiased };
template <class T, int NV, int K, int KEYS, bool WHOLE>
__global__ void __launch_bounds__(256, K == 8 ? 4 : 1) k_route_groups(GroupArgs ga) {
    constexpr bool BIASED = KEYS == kBiased, SCORES = KEYS != kLogits;
    using Key = typename KeyOf<typename Choose<BIASED, float, T>::type>::type;
    using Word = typename Key::Word;
    constexpr int W = 16 / sizeof(T), M = 8, S = K / M;
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
    const float *bias = BIASED ? a.bias + (int64_t)l * a.E : nullptr;
    const Row<T, WHOLE> row = {data + g * ga.size, g < ga.groups ? ga.size : 0};
    Vec<T> raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = row.vec(i * Q + q);
    // a vector's number among the token's: group by group, in the order of its
    // elements (so that ties go to the lowest)
    const int per_group = NV * Q;
    const int lane0 = (int)(threadIdx.x & 63) - c;
    const bool softmax = a.score == ROUTEPACK_SOFTMAX;
    float m = 0.0f, inv = 0.0f;
    float mx[NV], f1 = -kInf, f2 = -kInf;  // the vectors' largest logits, then keys
    if (!BIASED || softmax) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[W];
#pragma unroll
            for (int w = 0; w < W; ++w) x[w] = raw[i].at(w);
            mx[i] = most_of(x);
            odd = odd || mx[i] != mx[i];
        }
        if (__any(odd)) {  // NaN takes no part (the sum quiets it, the maximum drops it)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                mx[i] = -kInf;
#pragma unroll
                for (int w = 0; w < W; ++w) mx[i] = __builtin_fmaxf(mx[i], raw[i].at(w) + 0.0f);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) f1 = __builtin_fmaxf(f1, mx[i]);
    }
    if (softmax && (SCORES || !a.normalize)) {
        m = lanes_max(f1, lanes);
        m = m == -kInf ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV * W; ++v) sum += exp_plain(raw[v / W].at(v % W) - m);
        sum = lanes_add(sum, lanes);
        inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    }
    // (a logistic score this way keeps the absolute error below, not 1 - s)
    auto score = [&](float z) { return softmax ? exp_plain(z - m) * inv : __builtin_amdgcn_rcpf(1.0f + exp_plain(-z)); };
    // a vector's keys in 32 bits, -inf where the expert is not available
    auto keys_of = [&](const Vec<T> &r, int group, int vec, float (&y)[W]) {
        if constexpr (BIASED) {
            float b[W];
            const Row<float, WHOLE> bias_row = {bias + group * ga.size, group < ga.groups ? ga.size : 0};
#pragma unroll
            for (int k = 0; k < W / 4; ++k) {
                const Vec<float> x = bias_row.vec(vec * (W / 4) + k);
#pragma unroll
                for (int w = 0; w < 4; ++w) b[k * 4 + w] = x.at(w);
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float z = r.at(w);
                const float key = score(z) + b[w];
                y[w] = z > -kInf && key > -kInf ? key : -kInf;
            }
        } else {
#pragma unroll
            for (int w = 0; w < W; ++w) y[w] = r.at(w);
        }
    };
    // the vectors' largest keys, and the group's two
    if constexpr (KEYS == kSums) {
        f1 = -kInf;
#pragma unroll
        for (int v = 0; v < NV * W; ++v) {
            const float x = raw[v / W].at(v % W), z = x > -kInf ? x : -kInf;  // (NaN too)
            f2 = __builtin_fmaxf(f2, __builtin_fminf(f1, z));
            f1 = __builtin_fmaxf(f1, z);
        }
    }
    if constexpr (BIASED) {
        f1 = -kInf;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float y[W];
            keys_of(raw[i], g, i * Q + q, y);
            mx[i] = -kInf;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                f2 = __builtin_fmaxf(f2, __builtin_fminf(f1, y[w]));
                f1 = __builtin_fmaxf(f1, y[w]);
                mx[i] = __builtin_fmaxf(mx[i], y[w]);
            }
        }
    }
    // A key's error in 32 bits is (err + |key|) u, u = 2^-24, as for the choices
    // without groups: logistic scores 8 u, softmax scores (1 + 98 p) u with up to
    // 64 additions in a lane and 6 across lanes, and p <= inv.
    const float err = softmax ? 1.0f + 98.0f * inv : 8.0f;
    bool open = false, on;
    {
        lanes_two(f1, f2, Q);
        const bool two = SCORES && ga.top == 2 && f2 > -kInf;
        const float k1 = KEYS == kSums && f1 > -kInf ? score(f1) : f1, k2 = KEYS == kSums && two ? score(f2) : f2;
        const float best = two ? k1 + k2 : k1;
        // (twice the errors of the keys and of their sum)
        const float slack = (2.0f * err + __builtin_fabsf(k1) + (f2 > -kInf ? __builtin_fabsf(k2) : 0.0f) + __builtin_fabsf(best)) * 0x1p-23f;
        on = groups_before(ga.groups, ga.q_shift, best, g, lane0) < ga.keep && f1 > -kInf;
        if constexpr (KEYS == kSums) {
            // Groups of the same two logits as the last one kept are equal, whatever the
            // error: others must be clearly above those left out and those equal ones, and
            // the equal ones clearly above the others left out.
            const float last = -lanes_max(on ? -best : -kInf, lanes);
            const float l1 = lanes_max(on && best == last ? f1 : -kInf, lanes);
            const float l2 = lanes_max(on && best == last && f1 == l1 ? f2 : -kInf, lanes);
            const bool same = f1 == l1 && f2 == l2;
            const float low = -lanes_max(on && !same ? slack - best : -kInf, lanes);
            const float low_same = -lanes_max(on && same ? slack - best : -kInf, lanes);
            const float high = lanes_max(!on && !same && f1 > -kInf ? best + slack : -kInf, lanes);
            const float high_same = lanes_max(!on && same && f1 > -kInf ? best + slack : -kInf, lanes);
            open = (high > -kInf && !(low > high && low_same > high)) || (high_same > -kInf && !(low > high_same));
            open = open || inv != inv || best != best;
        }
        if constexpr (BIASED) {
            const float low = -lanes_max(on ? slack - best : -kInf, lanes);
            const float high = lanes_max(!on && f1 > -kInf ? best + slack : -kInf, lanes);
            open = high > -kInf && !(low > high);
            open = open || inv != inv || low != low || high != high;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) mx[i] = on ? mx[i] : -kInf;
    Word vk[NV], first[K];
#pragma unroll
    for (int i = 0; i < NV; ++i) vk[i] = Key::make(mx[i], kIndexMask ^ (uint32_t)(g * per_group + i * Q + q));
    lane_top<Key, K, NV>(vk, first);
    lanes_top<Key, K>(first, lanes);
    // the elements of the K vectors that lead, one or a few in each lane c < M
    Word x[S * W], top[K];
    float cand[BIASED ? S * W : 1], most[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        Word mine = Word(0);
#pragma unroll
        for (int j = 0; j < M; ++j) {
            const int up = s * M + j;
            mine = c == j ? (j >= M / 2 && lanes == M ? first[K - 1 - up] : first[up]) : mine;
        }
        const bool ok = c < M && Key::available(mine);
        const int id = (int)Key::index(mine), vg = id / per_group, v = id - vg * per_group;
        most[s] = ok ? Key::value(mine) : -kInf;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            x[s * W + w] = Word(0);
            if constexpr (BIASED) cand[s * W + w] = -kInf;
        }
        if (ok) {
            float y[W];
            const Row<T, WHOLE> r = {data + vg * ga.size, ga.size};
            keys_of(r.vec(v), vg, v, y);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if constexpr (BIASED) cand[s * W + w] = y[w];
                x[s * W + w] = Key::make(y[w], kIndexMask ^ (uint32_t)(vg * ga.size + v * W + w));
            }
        }
    }
    lane_top<Key, K, S * W>(x, top);
    group_top<Key, K, M>(top);
    int32_t id[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        Word mine = Word(0);
#pragma unroll
        for (int j = 0; j < M; ++j) mine = c == j ? top[s * M + j] : mine;
        id[s] = c < M && s * M + c < a.k && Key::available(mine) ? (int32_t)Key::index(mine) : -1;
    }
    // is the order beyond doubt?  Two keys further apart than `slack` are in order.
    auto slack = [&](float key) { return (err + 2.0f * __builtin_fabsf(key)) * 0x1p-23f; };
    if constexpr (KEYS == kSums) {
        // Equal logits have equal scores.  Different ones that are next to each other
        // among the chosen, and the largest one below them, must differ clearly.
        float before = 0.0f, s_before = 0.0f, edge = 0.0f, z_last = -kInf;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (j >= a.k || !Key::available(top[j])) continue;
            const float z = Key::value(top[j]), s = score(z);
            open = open || (j > 0 && z != before && !(s_before - s > slack(s_before) && s_before - s > slack(s)));
            before = z;
            s_before = s;
            if (j == a.k - 1) {
                edge = s - slack(s);
                z_last = z;
            }
        }
        const float z_k = lanes_max(c < M ? z_last : -kInf, lanes);
        edge = lanes_max(c < M && z_last > -kInf ? edge : -kInf, lanes);
        float below = -kInf;
#pragma unroll
        for (int v = 0; v < NV * W; ++v) {
            const float x = raw[v / W].at(v % W);
            below = on && x < z_k ? __builtin_fmaxf(below, x) : below;
        }
        below = lanes_max(below, lanes);
        open = open || (below > -kInf && !(score(below) < edge));
    }
    if constexpr (BIASED) {
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
        edge = lanes_max(c < M ? edge : -kInf, lanes);
        // from the edge on: elements of the chosen vectors, and other vectors
        float over = 0.0f, more = 0.0f;
#pragma unroll
        for (int i = 0; i < S * W; ++i) over += cand[i] >= edge && cand[i] > -kInf ? 1.0f : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) more += mx[i] >= edge && mx[i] > -kInf ? 1.0f : 0.0f;
#pragma unroll
        for (int s = 0; s < S; ++s) more -= most[s] >= edge && most[s] > -kInf ? 1.0f : 0.0f;
        over = lanes_add(over, lanes);
        more = lanes_add(more, lanes);
        open = open || (edge > -kInf && (over != (float)a.k || more != 0.0f)) || edge != edge;
    }
    if constexpr (SCORES) {
        // The tokens in doubt, one at a time by the whole wave, in 64 bits: loops of
        // little code, an element at a time from memory, a group in as many lanes as
        // fit 64 (a wave that took them by their own lanes took 15 us, and kept the
        // rest waiting).  A lane's keys stand in LDS, where it alone reads them: they
        // cost the calls without doubt no registers.  NaN takes no part; experts of +inf share the scores alone.
        extern __shared__ uint64_t keys_of_waves[];
        uint64_t *const keys = keys_of_waves + (threadIdx.x >> 6) * a.E;
        int q_shift = 0;
        while ((ga.groups << (q_shift + 1)) <= kWave) ++q_shift;
        for (uint64_t todo = __ballot(open); todo;) {
            const int from = __builtin_amdgcn_readfirstlane(__builtin_ctzll(todo) & ~(lanes - 1));
            const uint64_t its = (lanes == kWave ? ~(uint64_t)0 : ((uint64_t)1 << lanes) - 1) << from;
            todo &= ~its;
            const int lane = threadIdx.x & 63, group = lane >> q_shift, step = 1 << q_shift;
            const int64_t where = (int64_t)readlane64((uint64_t)(uintptr_t)data, from);
            const int64_t what = (int64_t)readlane64((uint64_t)(uintptr_t)bias, from);
            const int count = group < ga.groups ? ga.size : 0;
            const T *z_of = reinterpret_cast<const T *>(where) + group * ga.size;
            const float *b_of = reinterpret_cast<const float *>(what) + group * ga.size;
            double base = 0.0, sum = 1.0;
            auto part = [&](float z) { return exp(__builtin_fmin((double)z - base, 0.0)); };
            if (softmax) {
                float b = -kInf;
#pragma unroll 1
                for (int e = lane & (step - 1); e < count; e += step) {
                    const float z = to_f32(z_of[e]);
                    b = z > b ? z : b;
                }
                base = lanes_max(b, kWave);
                double mine = 0.0;
#pragma unroll 1
                for (int e = lane & (step - 1); e < count; e += step) {
                    const float z = to_f32(z_of[e]);
                    mine += z > -kInf ? part(z) : 0.0;
                }
                sum = lanes_add(mine, kWave);
            }
            auto key_at = [&](int e) -> uint64_t {
                const float z = to_f32(z_of[e]);
                double key = softmax ? part(z) / sum : 1.0 / (1.0 + exp(-(double)z));
                if (what) key += (double)b_of[e];
                return z > -kInf && key > -__builtin_inf() ? order64(key) : 0;
            };
            uint64_t g1 = 0, g2 = 0;
#pragma unroll 1
            for (int e = lane & (step - 1); e < count; e += step) {
                const uint64_t key = key_at(e);
                keys[group * ga.size + e] = key;
                g2 = max64(g2, min64(g1, key));
                g1 = max64(g1, key);
            }
            lanes_two(g1, g2, step);
            if (ga.top == 2 && g2) g1 = order64(value64(g1) + value64(g2));
            const bool keep = g1 != 0 && groups_before(ga.groups, q_shift, g1, group, 0) < ga.keep;
            uint64_t best;  // of what this lane still has
            uint32_t who;
            auto look = [&] {
                best = 0;
                who = UINT32_MAX;
#pragma unroll 1
                for (int e = lane & (step - 1); e < (keep ? count : 0); e += step) {
                    const uint64_t key = keys[group * ga.size + e];
                    who = key > best ? (uint32_t)(group * ga.size + e) : who;
                    best = key > best ? key : best;
                }
            };
            look();
            const bool its_lane = its >> lane & 1;
#pragma unroll 1
            for (int j = 0; j < a.k; ++j) {
                uint64_t k0 = best;
                uint32_t e0 = who;
                lanes_first(k0, e0, kWave);
                if (k0 && who == e0) {
                    keys[e0] = 0;
                    look();
                }
#pragma unroll
                for (int s = 0; s < S; ++s)
                    if (its_lane && j == s * M + c) id[s] = k0 ? (int32_t)e0 : -1;
            }
        }
    }
    float zc[S], w[S], less[S];
    bool made[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        made[s] = c < M && id[s] >= 0;
        zc[s] = made[s] ? to_f32(data[id[s]]) : 0.0f;
    }
    choice_gates<M, S>(zc, made, a.score, a.normalize, m, inv, w, less);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int j = s * M + c;
        if (live && c < M && j < a.k) {
            a.ids[at * a.k + j] = id[s];
            a.gates[at * a.k + j] = a.scale * w[s];
        }
    }
}

// Lanes of a group and a token: as few as hold a group in 8 vectors a lane, where
// scores are keys in 32 elements (at least 8 a token, for the second selection).
constexpr int kScoresALane = 32;
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
    const int keys = a.r.bias ? kBiased : a.top > 1 ? kSums : kLogits;
    const int most = keys != kLogits ? kScoresALane / W : 8;  // (E <= 1024: 64 lanes never need more)
    auto each = [&] { return (vecs + (1 << a.q_shift) - 1) >> a.q_shift; };
    while ((each() > most && (groups << a.q_shift) < kWave) || (groups << a.q_shift) < 8) ++a.q_shift;
    a.lane_shift += a.q_shift;
    const int64_t items = a.r.T * a.r.L, per = 256 >> a.lane_shift;
    const size_t lds = keys != kLogits ? 4 * (size_t)a.r.E * sizeof(uint64_t) : 0;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid_of((items + per - 1) / per), dim3(256), lds, stream, a);
        return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
    };
    auto by_k = [&](auto v) {
        constexpr int N = decltype(v)::value;
        // (8 choices at most, whole vectors and no idle lanes: without the checks of
        // every vector)
        const bool whole = a.r.k <= 8 && a.size == (N * W) << a.q_shift && a.groups == groups;
        auto by_keys = [&](auto keys_) {
            constexpr int KEYS = decltype(keys_)::value;
            if (whole) return go(k_route_groups<T, N, 8, KEYS, true>);
            if (a.r.k <= 8) return go(k_route_groups<T, N, 8, KEYS, false>);
            if (a.r.k <= 16) return go(k_route_groups<T, N, 16, KEYS, false>);
            return go(k_route_groups<T, N, 32, KEYS, false>);
        };
        if constexpr (N * W <= kScoresALane) {
            if (keys == kBiased) return by_keys(Int<kBiased>());
            if (keys == kSums) return by_keys(Int<kSums>());
        }
        return by_keys(Int<kLogits>());
    };
    if (each() <= 1) return by_k(Int<1>());
    if (each() <= 2) return by_k(Int<2>());
    if (each() <= 4) return by_k(Int<4>());
    if (each() <= 8) return by_k(Int<8>());
    return ROUTEPACK_E_UNSUPPORTED;  // (never: E <= 1024)
}

}  // namespace rp
