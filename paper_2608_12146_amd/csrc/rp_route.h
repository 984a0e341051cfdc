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

struct RouteArgs {
    const void *logits;
    int64_t ts, ls;      // strides of the logits
    int64_t T;
    int32_t L, E, k;
    const void *rec;     // replayed ids, or null
    int32_t rec_type;
    int64_t rts, rls;    // their strides
    const float *bias;
    int32_t score;
    bool normalize;
    float scale;
    int32_t *ids;
    float *gates;
};

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


template <class T>
__device__ inline float to_f32(T v) { return (float)v; }

// A vector of 16 bytes of logits, as four words; it may start at any element
// (global memory takes unaligned accesses of any width).
template <class T>
struct Vec {
    static constexpr int W = 16 / sizeof(T);
    uint32_t w[4];
    __device__ float at(int i) const;
    __device__ void set(const float (&x)[W]);
};
struct __attribute__((packed, aligned(2))) Words16 {
    uint32_t w[4];
};
// 16 bytes at any address; ONCE: that nothing reads again (a hint that keeps
// them from displacing others in the caches: it took counting 300007 x 24 x 8
// ids from 55 to 50 us).
template <bool ONCE>
__device__ inline void load16(const void *p, uint32_t (&w)[4]) {
    typedef uint32_t four __attribute__((ext_vector_type(4), aligned(1)));
    const four *q = static_cast<const four *>(p);
    const four x = ONCE ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
}
template <> __device__ inline float Vec<float>::at(int i) const { return __uint_as_float(w[i]); }
template <> __device__ inline float Vec<__bf16>::at(int i) const {
    return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}
template <> __device__ inline float Vec<_Float16>::at(int i) const {
    typedef _Float16 half2_ __attribute__((ext_vector_type(2)));
    return (float)__builtin_bit_cast(half2_, w[i / 2])[i & 1];
}
template <> __device__ inline void Vec<float>::set(const float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
}
template <> __device__ inline void Vec<__bf16>::set(const float (&x)[8]) {
    typedef __bf16 two __attribute__((ext_vector_type(2)));
    typedef float two32 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const two32 y = {x[2 * i], x[2 * i + 1]};
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, two));
    }
}
template <> __device__ inline void Vec<_Float16>::set(const float (&x)[8]) {
    typedef _Float16 two __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const two y = {(_Float16)x[2 * i], (_Float16)x[2 * i + 1]};
        w[i] = __builtin_bit_cast(uint32_t, y);
    }
}

template <class T>
__device__ inline uint32_t bits_of(const T *p) {
    if constexpr (sizeof(T) == 4) return *reinterpret_cast<const uint32_t *>(p);
    else return *reinterpret_cast<const uint16_t *>(p);
}

// A row of E elements by vectors; those past its end are -inf.  WHOLE: the
// caller asks for none that reaches past it.
template <class T, bool WHOLE = false>
struct Row {
    static constexpr int W = Vec<T>::W;
    const T *data;
    int32_t E;
    __device__ Vec<T> vec(int v) const {
        constexpr uint32_t kLow = sizeof(T) == 4 ? 0xFF800000u : (__is_same(T, __bf16) ? 0xFF80u : 0xFC00u);
        const int e0 = v * W;
        Vec<T> x;
        if (WHOLE || e0 + W <= E) {
            load16<false>(data + e0, x.w);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x.w[i] = sizeof(T) == 4 ? kLow : kLow << 16 | kLow;
            // (one vector of the row at most is cut: a loop, not W branches)
            for (int i = 0; e0 + i < E; ++i) {
                const uint32_t b = bits_of(data + e0 + i);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    if constexpr (sizeof(T) == 4) {
                        x.w[n] = n == i ? b : x.w[n];
                    } else {
                        x.w[n] = 2 * n == i ? (x.w[n] & 0xFFFF0000u) | b : x.w[n];
                        x.w[n] = 2 * n + 1 == i ? (x.w[n] & 0xFFFFu) | b << 16 : x.w[n];
                    }
                }
            }
        }
        return x;
    }
};

// The row's part of one lane.
template <class T, int G, int V, bool WHOLE = false>
__device__ inline void load_row(const T *row, int E, int c, float (&z)[V]) {
    constexpr int W = Vec<T>::W;
    static_assert(V % W == 0, "whole vectors");
    const Row<T, WHOLE> r = {row, E};
    Vec<T> x[V / W];
#pragma unroll
    for (int i = 0; i < V / W; ++i) x[i] = r.vec(i * G + c);
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] = x[v / W].at(v % W);
}

// Elements e0 .. e0 + W of a row of E.
template <class T, bool WHOLE>
__device__ inline void store_vec(T *row, int E, int e0, const float (&y)[Vec<T>::W]) {
    constexpr int W = Vec<T>::W;
    if (WHOLE || e0 + W <= E) {
        Vec<T> w;
        w.set(y);
        Words16 b;
#pragma unroll
        for (int n = 0; n < 4; ++n) b.w[n] = w.w[n];
        *reinterpret_cast<Words16 *>(row + e0) = b;
    } else {
#pragma unroll
        for (int x = 0; x < W; ++x)
            if (e0 + x < E) row[e0 + x] = (T)y[x];
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

// 2^(x log2 e) without that correction: a relative error of up to 1.3 |x| + 2
// steps, in two instructions instead of eight.  It serves where it is lost in
// a sum or a mean of scores (the terms with large |x| are the small ones), or
// in the rounding of the result to 16 bits.  -inf gives 0, NaN gives NaN.
__device__ inline float exp_plain(float x) { return __builtin_amdgcn_exp2f(x * 1.44269502f); }

template <bool FINE>
__device__ inline float exp_of(float x) { return FINE ? exp32(x) : exp_plain(x); }

// s = 1 / (1 + e^-z) and 1 - s, without cancellation on either side.
template <bool FINE>
__device__ inline void logistic(float z, float &s, float &one_less) {
    const float e = exp_of<FINE>(-__builtin_fabsf(z));
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    const float q = e * r;
    s = z >= 0.0f ? r : q;
    one_less = z >= 0.0f ? q : r;
}

// The value of the lane at the other side of a group of D lanes' middle (D a
// power of two in 2..64): lane i of an aligned group sees lane i ^ 1, i ^ 2,
// 7 - i, 15 - i, i ^ 16 or i ^ 32.  Taken for D = 2, 4, .. G in turn, a
// symmetric function of both sides reduces a group of G lanes.
template <int D>
__device__ inline uint32_t across(uint32_t v) {
    if constexpr (D == 2) return (uint32_t)dpp32<kDppXor1>((int32_t)v, (int32_t)v);
    else if constexpr (D == 4) return (uint32_t)dpp32<kDppXor2>((int32_t)v, (int32_t)v);
    else if constexpr (D == 8) return (uint32_t)dpp32<kDppHalfMirror>((int32_t)v, (int32_t)v);
    else if constexpr (D == 16) return (uint32_t)dpp32<kDppMirror>((int32_t)v, (int32_t)v);
    else return (uint32_t)__shfl_xor((int32_t)v, D / 2, kWave);
}
template <int D>
__device__ inline float across(float v) {
    return __uint_as_float(across<D>(__float_as_uint(v)));
}
template <int D>
__device__ inline double across(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint64_t lo = across<D>((uint32_t)u), hi = across<D>((uint32_t)(u >> 32));
    return __longlong_as_double((long long)(hi << 32 | lo));
}

// Reductions over the G lanes of a token; every lane ends with the result.
template <int G, int D = 2>
__device__ inline float group_sum(float v) {
    if constexpr (D > G) return v;
    else return group_sum<G, 2 * D>(v + across<D>(v));
}
template <int G, int D = 2>
__device__ inline float group_max(float v) {
    if constexpr (D > G) return v;
    else return group_max<G, 2 * D>(__builtin_fmaxf(v, across<D>(v)));
}
template <int G>
__device__ inline int64_t group_sum64(int64_t v) {
#pragma unroll
    for (int d = 1; d < G; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

template <int G, int V>
__device__ inline float row_max(const float (&z)[V]) {
    float m = z[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = __builtin_fmaxf(m, z[v]);
    return group_max<G>(m);
}

// Softmax of a row in place, but for the factor `inv`, the inverse of the sum:
// z becomes e^(z - m), m the row's maximum.  A row without an available expert
// becomes 0 (m and inv too); a NaN or +inf in it makes inv NaN.
template <bool FINE, int G, int V>
__device__ inline void softmax_row(float (&z)[V], float &m, float &inv) {
    m = row_max<G, V>(z);
    m = m == -kInf ? 0.0f : m;
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        z[v] = exp_of<FINE>(z[v] - m);
        sum += z[v];
    }
    sum = group_sum<G>(sum);
    inv = sum == 0.0f ? 0.0f : 1.0f / sum;
}

// A row's m and inv alone.
template <int G, int V>
__device__ inline void row_sum(const float (&z)[V], float &m, float &inv) {
    float e[V];
#pragma unroll
    for (int v = 0; v < V; ++v) e[v] = z[v];
    softmax_row<false, G, V>(e, m, inv);
}

// Logistic scores of a row in place, but for the factor `inv`, the inverse of
// their sum, and 1 - s in `less`.  Where every logit is below 0 the scores may
// leave the range of 32 bits, but their ratios do not: with a maximum m < 0
// all are taken times e^-m.
template <bool FINE, int G, int V>
__device__ inline void logistic_row(float (&z)[V], float (&less)[V], float &inv) {
    const float m = row_max<G, V>(z);
    const bool low = m < 0.0f && m > -kInf;
    float sum = 0.0f;
    if (__any(low)) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float x = z[v];
            logistic<FINE>(x, z[v], less[v]);
            // e^x / (1 + e^x), and less is 1 / (1 + e^x)
            z[v] = low ? exp_of<FINE>(x - m) * less[v] : z[v];
            sum += z[v];
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            logistic<FINE>(z[v], z[v], less[v]);
            sum += z[v];
        }
    }
    sum = group_sum<G>(sum);
    inv = sum == 0.0f ? 0.0f : 1.0f / sum;
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
            logistic<true>(zc[s], w[s], less[s]);
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

// The largest of a vector's elements; NaN where it holds one (the instruction
// that drops a quiet NaN returns a signalling one, and the next would drop that
// with the elements before it).
__device__ inline float max3(float a, float b, float c) {
    float d;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}
__device__ inline float most_of(const float (&x)[4]) { return max3(max3(x[0], x[1], x[2]), x[3], x[3]); }
__device__ inline float most_of(const float (&x)[8]) {
    return max3(max3(max3(x[0], x[1], x[2]), x[3], x[4]), max3(x[5], x[6], x[7]), x[7]);
}

// ---------------------------------------------------------------------------
// Selection of the largest of many values, lowest index first among equals,
// on keys that hold a value's order and the complement of its index: then a
// larger key precedes, no two keys are equal, and a compare and exchange is
// one maximum and one minimum.  The key 0 (and any below `least`) stands for
// an unavailable expert: -inf, NaN, or none.  -0 equals +0.

constexpr uint32_t kIndexMask = 2047;  // an index below 2048 (kMaxExperts)

// A float's order as an unsigned number; -inf is 0x007FFFFF, NaN too.
__device__ inline uint32_t order32(float z) {
    const uint32_t u = __float_as_uint(__builtin_fmaxf(z + 0.0f, -kInf));
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float value32(uint32_t o) {
    return __uint_as_float(o >> 31 ? o ^ 0x80000000u : ~o);
}

// A double's order as an unsigned number (-0 equals +0); 0 stands for "not
// available".
__device__ inline uint64_t order64(double x) {
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | (uint64_t)1 << 63;
}

// 16-bit logits: their 32-bit form has at most 19 significant leading bits
// (bf16 16, fp16 1 + 8 + 10), so 21 bits of order and 11 of index are one
// 32-bit word.
struct Key16 {
    using Word = uint32_t;
    static constexpr Word least = 0x00800000u;
    static __device__ Word make(float z, uint32_t inv) { return (order32(z) & ~kIndexMask) | inv; }
    static __device__ bool available(Word k) { return k >= least; }
    // (a negative number's order ends in ones, which the index took)
    static __device__ float value(Word k) { return value32(k >> 31 ? k & ~kIndexMask : k | kIndexMask); }
    static __device__ uint32_t index(Word k) { return ~k & kIndexMask; }
    static __device__ Word max(Word a, Word b) { return a > b ? a : b; }
    static __device__ Word min(Word a, Word b) { return a < b ? a : b; }
};

// 32-bit logits: the 32 bits of order and the index as the bits of a normal
// positive double (its order is that of its bits), which has a maximum and a
// minimum instruction where 64-bit integers have none.  The instructions are
// written out: the compiler would first quiet each operand.
struct Key32 {
    using Word = double;
    static __device__ Word make(float z, uint32_t inv) {
        const uint32_t o = order32(z);
        return __hiloint2double((int)((o >> 2) + 0x00100000u), (int)(o << 30 | inv));
    }
    static __device__ uint32_t order(Word k) {
        return ((uint32_t)__double2hiint(k) - 0x00100000u) << 2 | (uint32_t)__double2loint(k) >> 30;
    }
    static __device__ bool available(Word k) {
        return (uint32_t)__double2hiint(k) >= (0x00800000u >> 2) + 0x00100000u;
    }
    static __device__ float value(Word k) { return value32(order(k)); }
    static __device__ uint32_t index(Word k) { return ~(uint32_t)__double2loint(k) & kIndexMask; }
    static __device__ Word max(Word a, Word b) {
        Word d;
        asm("v_max_f64 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
        return d;
    }
    static __device__ Word min(Word a, Word b) {
        Word d;
        asm("v_min_f64 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
        return d;
    }
};

template <class T> struct KeyOf { using type = Key16; };
template <> struct KeyOf<float> { using type = Key32; };

template <class Key, int A, int B, int N>
__device__ inline void order_pair(typename Key::Word (&a)[N]) {
    const typename Key::Word x = a[A], y = a[B];
    a[A] = Key::max(x, y);
    a[B] = Key::min(x, y);
}

// Batcher's odd-even merge sort of a[LO .. LO + M), largest first.
template <class Key, int LO, int M, int R, int I, int N>
__device__ inline void odd_even_pairs(typename Key::Word (&a)[N]) {
    if constexpr (I + R < LO + M) {
        order_pair<Key, I, I + R>(a);
        odd_even_pairs<Key, LO, M, R, I + 2 * R>(a);
    }
}
template <class Key, int LO, int M, int R, int N>
__device__ inline void odd_even_merge(typename Key::Word (&a)[N]) {
    if constexpr (2 * R < M) {
        odd_even_merge<Key, LO, M, 2 * R>(a);
        odd_even_merge<Key, LO + R, M, 2 * R>(a);
        odd_even_pairs<Key, LO, M, R, LO + R>(a);
    } else {
        order_pair<Key, LO, LO + R>(a);
    }
}
template <class Key, int LO, int M, int N>
__device__ inline void sort_keys(typename Key::Word (&a)[N]) {
    if constexpr (M > 1) {
        sort_keys<Key, LO, M / 2>(a);
        sort_keys<Key, LO + M / 2, M / 2>(a);
        odd_even_merge<Key, LO, M, 1>(a);
    }
}

// Sorts a bitonic sequence a[LO .. LO + M), largest first.
template <class Key, int LO, int M, int I, int N>
__device__ inline void bitonic_pairs(typename Key::Word (&a)[N]) {
    if constexpr (I < M / 2) {
        order_pair<Key, LO + I, LO + I + M / 2>(a);
        bitonic_pairs<Key, LO, M, I + 1>(a);
    }
}
template <class Key, int LO, int M, int N>
__device__ inline void bitonic_sort(typename Key::Word (&a)[N]) {
    if constexpr (M > 1) {
        bitonic_pairs<Key, LO, M, 0>(a);
        bitonic_sort<Key, LO, M / 2>(a);
        bitonic_sort<Key, LO + M / 2, M / 2>(a);
    }
}

// The K largest of two sorted lists of K: the larger of each a[i], b[K-1-i]
// is among them, and these form a bitonic sequence.
template <class Key, int K>
__device__ inline void merge_top(typename Key::Word (&a)[K], const typename Key::Word (&b)[K]) {
#pragma unroll
    for (int i = 0; i < K; ++i) a[i] = Key::max(a[i], b[K - 1 - i]);
    bitonic_sort<Key, 0, K>(a);
}

// The K largest of a lane's M keys (powers of two), sorted.
template <class Key, int K, int M>
__device__ inline void lane_top(const typename Key::Word (&x)[M], typename Key::Word (&top)[K]) {
    constexpr int B = M < K ? M : K;
#pragma unroll
    for (int i = 0; i < K; ++i) top[i] = i < B ? x[i] : typename Key::Word(0);
    sort_keys<Key, 0, B>(top);
    if constexpr (M > K) {
#pragma unroll
        for (int b = 1; b < M / K; ++b) {
            typename Key::Word y[K];
#pragma unroll
            for (int i = 0; i < K; ++i) y[i] = x[b * K + i];
            sort_keys<Key, 0, K>(y);
            merge_top<Key, K>(top, y);
        }
    }
}

// The K largest of G lanes' lists, in every one of them.
template <class Key, int K, int G, int D = 2>
__device__ inline void group_top(typename Key::Word (&top)[K]) {
    if constexpr (D <= G) {
        typename Key::Word y[K];
#pragma unroll
        for (int i = 0; i < K; ++i) y[i] = across<D>(top[i]);
        merge_top<Key, K>(top, y);
        group_top<Key, K, G, 2 * D>(top);
    }
}

// The token and layer of a group of G lanes in a workgroup of 256 threads;
// groups past the last item repeat it and are not live.
struct Item {
    int64_t at, t;
    int32_t l;
    bool live;
};
template <int G>
__device__ inline Item item_of(int64_t T, int32_t L) {
    Item it;
    const int64_t n = T * L;
    it.at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (256 / G) + threadIdx.x / G;
    it.live = it.at < n;
    it.at = it.live ? it.at : n - 1;
    if (L == 1) {
        it.t = it.at;
        it.l = 0;
    } else if (n <= UINT32_MAX) {
        const uint32_t t = (uint32_t)it.at / (uint32_t)L;
        it.t = t;
        it.l = (int32_t)((uint32_t)it.at - t * (uint32_t)L);
    } else {
        it.t = it.at / L;
        it.l = (int32_t)(it.at - it.t * L);
    }
    return it;
}

// The first of n places where `yes` holds, which holds for all after it (n if
// for none): the lanes of a wave probe 64 places a round.  In 32 bits and with
// a minimum, not with uniform 64-bit selects behind the ballot: a build of such
// a search counted some of 1000 samples of 9 tokens as empty, and its assembly
// had a select on the condition of the compare before its own.  (No build of
// the other forms that were looked at does; the tests count 63 to 5000 samples.)
template <class F>
__device__ inline int32_t first_where(int32_t n, F &&yes) {
    int32_t lo = 0;
    while (n > 0) {  // the answer is in [lo, lo + n]
        const int32_t step = (n - 1) / kWave + 1, at = lane_id() * step;
        const uint64_t mask = __ballot(at < n ? (bool)yes(lo + at) : true);
        const int32_t f = mask ? first_lane(mask) : kWave;
        if (f == 0) break;
        // behind probe f - 1, up to probe f or the end (64 steps may be 2^31)
        const int32_t past = (f - 1) * step + 1;
        n = (int32_t)__builtin_elementwise_min((uint32_t)n, (uint32_t)f * (uint32_t)step) - past;
        lo += past;
    }
    return lo;
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
    // (all products of tokens, layers and experts, in bytes, fit 64 bits)
    if (p->n_layers > 0 && z->n_tokens > INT64_MAX / 16 / ((int64_t)p->n_layers * p->n_experts))
        return ROUTEPACK_E_UNSUPPORTED;
    return ROUTEPACK_OK;
}

inline int check_ids(const routepack_problem *p, const routepack_ids *r, int64_t n_tokens) {
    if (r->type < ROUTEPACK_U8 || r->type > ROUTEPACK_I64) return ROUTEPACK_E_INVALID;
    if (r->n_tokens != n_tokens || r->token_stride < 0 || r->layer_stride < 0) return ROUTEPACK_E_INVALID;
    if (!r->data && n_tokens > 0 && p->n_layers > 0) return ROUTEPACK_E_INVALID;
    return ROUTEPACK_OK;
}

template <int N>
struct Int {
    static constexpr int value = N;
};

// Calls f with the lanes of a token and the vectors of a lane for rows of E
// logits: 4 lanes of 1, 2 .. MOST vectors, or more lanes of MOST.
template <class T, int MOST, class F>
int by_geometry(int32_t E, F &&f) {
    const int32_t n = (E * (int32_t)sizeof(T) + 15) / 16;
    if (n <= 4) return f(Int<4>(), Int<1>());
    if constexpr (MOST >= 4)
        if (n <= 8) return f(Int<4>(), Int<2>());
    if constexpr (MOST >= 8)
        if (n <= 16) return f(Int<4>(), Int<4>());
    if (n <= 4 * MOST) return f(Int<4>(), Int<MOST>());
    if (n <= 8 * MOST) return f(Int<8>(), Int<MOST>());
    if (n <= 16 * MOST) return f(Int<16>(), Int<MOST>());
    if (n <= 32 * MOST) return f(Int<32>(), Int<MOST>());
    if constexpr (32 * MOST * 16 / (int)sizeof(T) < kMaxExperts)
        if (n <= 64 * MOST) return f(Int<64>(), Int<MOST>());
    return ROUTEPACK_E_UNSUPPORTED;
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
