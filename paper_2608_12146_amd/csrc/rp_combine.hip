// The sum of a token's rows under its gates and its gradients, on gfx950.
//
// Both are streams: out reads every row once; the gradients read it once more
// for the gates' part and write it once, with dout read once a token.  A token
// lies in LT lanes (a power of two, up to a wave), 16 bytes a lane.
#include "rp_experts.h"

namespace rp {

struct CombineArgs {
    const void *y;
    int64_t stride, n_rows;
    int32_t cols, vecs;        // vectors of 16 bytes a row
    int32_t lt, chunks;        // lanes of a token, vectors / lanes
    const int32_t *places;
    int64_t place_stride;
    int32_t k;
    const float *gates;
    int64_t gate_stride;
    int64_t T;
    void *out;
    // gradients
    const void *dout;
    int64_t dout_stride;
    const int32_t *rows;
    void *dy;
    float *dgates;
    int64_t token_groups;      // workgroups of tokens; those behind look for rows of no pair
};

// One vector of a row, zeros past its end.
template <class T>
__device__ inline Vec<T> row_vec(const T *row, int32_t cols, int32_t c) {
    constexpr int W = Vec<T>::W;
    Vec<T> x;
    if (c + W <= cols) {
        load16<false>(row + c, x.w);
    } else {
        float v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = c + i < cols ? to_f32(row[c + i]) : 0.0f;
        x.set(v);
    }
    return x;
}

template <class T, int N>
__device__ inline void add_rows(const CombineArgs &a, const int32_t *places, const float *gates, int32_t c,
                                float (&sum)[Vec<T>::W]) {
    constexpr int W = Vec<T>::W;
    Vec<T> x[N];
    float g[N];
    bool on[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int64_t r = places[j];
        on[j] = r >= 0 && r < a.n_rows;
        g[j] = gates ? gates[j] : 1.0f;
        x[j] = row_vec<T>(static_cast<const T *>(a.y) + (on[j] ? r : 0) * a.stride, a.cols, c);
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int w = 0; w < W; ++w) sum[w] = on[j] ? __builtin_fmaf(g[j], x[j].at(w), sum[w]) : sum[w];
}

// ONE: a wave has one token, whose places and gates are read by scalar loads.
template <class T, bool ONE>
__global__ void __launch_bounds__(256) k_combine(CombineArgs a) {
    constexpr int W = Vec<T>::W;
    const int lt = ONE ? kWave : a.lt, lane = threadIdx.x & (lt - 1);
    int64_t item = group_index() * (256 / lt) + threadIdx.x / lt;
    if (ONE) item = ((int64_t)__builtin_amdgcn_readfirstlane((int)(item >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)item);
    int64_t t = item;
    int32_t v = lane;
    if (ONE) {
        t = item <= UINT32_MAX ? (uint32_t)item / (uint32_t)a.chunks : item / a.chunks;
        v += (int32_t)(item - t * a.chunks) * kWave;
    }
    if (t >= a.T || v >= a.vecs) return;
    const int32_t *places = a.places + t * a.place_stride;
    const float *gates = a.gates ? a.gates + t * a.gate_stride : nullptr;
    float sum[W] = {};
    int j = 0;
    if (a.n_rows > 0) {
        for (; j + 4 <= a.k; j += 4) add_rows<T, 4>(a, places + j, gates ? gates + j : nullptr, v * W, sum);
        if (j + 2 <= a.k) {
            add_rows<T, 2>(a, places + j, gates ? gates + j : nullptr, v * W, sum);
            j += 2;
        }
        if (j < a.k) add_rows<T, 1>(a, places + j, gates ? gates + j : nullptr, v * W, sum);
    }
    store_vec<T, false>(static_cast<T *>(a.out) + t * a.cols, a.cols, v * W, sum);
}

// The pair that stands in row r, if its place is r; else -1.
__device__ inline int64_t pair_of_row(const CombineArgs &a, int64_t r) {
    const int32_t p = a.rows[r];
    if (p < 0) return -1;
    const uint32_t t = (uint32_t)p / (uint32_t)a.k;
    if (t >= a.T) return -1;
    return a.places[t * a.place_stride + (p - t * (uint32_t)a.k)] == r ? p : -1;
}

// The sum over aligned groups of lt lanes.
__device__ inline float lanes_sum(float v, int lt) {
    for (int d = 1; d < lt; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// Gradients of a token: each chunk's dout is held while its k rows are read
// (for the gates) and written.  NW waves share a token's columns (lt < 64: a
// wave has several tokens).
template <class T, int K, int NW>
__global__ void __launch_bounds__(256) k_spread(CombineArgs a) {
    constexpr int W = Vec<T>::W;
    __shared__ float part[4][K];
    if (group_index() >= a.token_groups) {  // rows of no pair: zeros
        const int lane = threadIdx.x & 63;
        const int64_t r0 = (group_index() - a.token_groups) * 256 + (threadIdx.x & ~63);
        const bool mine = r0 + lane < a.n_rows && pair_of_row(a, r0 + lane) < 0;
        for (uint64_t m = __ballot(mine); m; m &= m - 1) {
            T *row = static_cast<T *>(a.dy) + (r0 + __builtin_ctzll(m)) * a.cols;
            const float zero[W] = {};
            for (int32_t v = lane; v < a.vecs; v += kWave) store_vec<T, false>(row, a.cols, v * W, zero);
        }
        return;
    }
    const int lt = NW > 1 ? kWave : a.lt, lane = threadIdx.x & (lt - 1), wave = threadIdx.x >> 6;
    const int64_t t = NW > 1 ? group_index() * (4 / NW) + wave / NW : group_index() * (256 / lt) + threadIdx.x / lt;
    const bool live = t < a.T;
    float dots[K] = {};
    if (live) {
        const int32_t *places = a.places + t * a.place_stride;
        const float *gates = a.gates ? a.gates + t * a.gate_stride : nullptr;
        const T *dout = static_cast<const T *>(a.dout) + t * a.dout_stride;
        for (int32_t v = lane + wave % NW * kWave; v < a.vecs; v += lt * NW) {
            const Vec<T> d = row_vec<T>(dout, a.cols, v * W);
#pragma unroll
            for (int j0 = 0; j0 < K; j0 += 4) {
                if (j0 >= a.k) continue;
                int64_t r[4];
                bool on[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    r[j] = j0 + j < a.k ? places[j0 + j] : -1;
                    on[j] = r[j] >= 0 && r[j] < a.n_rows;
                }
                if (a.dgates && a.n_rows > 0) {
                    Vec<T> y[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        y[j] = row_vec<T>(static_cast<const T *>(a.y) + (on[j] ? r[j] : 0) * a.stride, a.cols, v * W);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int w = 0; w < W; ++w)
                            dots[j0 + j] = on[j] ? __builtin_fmaf(y[j].at(w), d.at(w), dots[j0 + j]) : dots[j0 + j];
                }
                if (a.dy) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (!on[j] || a.rows[r[j]] != t * a.k + j0 + j) continue;
                        const float g = gates ? gates[j0 + j] : 1.0f;
                        float x[W];
#pragma unroll
                        for (int w = 0; w < W; ++w) x[w] = g * d.at(w);
                        store_vec<T, false>(static_cast<T *>(a.dy) + r[j] * a.cols, a.cols, v * W, x);
                    }
                }
            }
        }
    }
    if (!a.dgates) return;
#pragma unroll
    for (int j = 0; j < K; ++j)
        if (j < a.k) dots[j] = lanes_sum(dots[j], lt);
    if (NW > 1) {
        if (lane == 0)
#pragma unroll
            for (int j = 0; j < K; ++j) part[wave][j] = dots[j];
        __syncthreads();
        if (wave % NW == 0 && live && lane < a.k) {
            float s = 0.0f;
            for (int w = 0; w < NW; ++w) s += part[wave + w][lane];
            a.dgates[t * a.k + lane] = s;
        }
    } else if (live && lane == 0) {
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < a.k) a.dgates[t * a.k + j] = dots[j];
    }
}

inline int check_places(const routepack_ids *p, int32_t k, int64_t gate_stride) {
    if (!p || p->type != ROUTEPACK_I32 || p->n_tokens < 0 || p->token_stride < 0 || k < 1 || gate_stride < 0)
        return ROUTEPACK_E_INVALID;
    if (k > kMaxChoices || p->n_tokens > INT32_MAX / k || !sizes_fit(p->n_tokens, p->token_stride) ||
        !sizes_fit(p->n_tokens, gate_stride))
        return ROUTEPACK_E_UNSUPPORTED;
    return ROUTEPACK_OK;
}

inline void geometry(CombineArgs &a, int W) {
    a.vecs = (a.cols + W - 1) / W;
    a.lt = 1;
    while (a.lt < kWave && a.lt < a.vecs) a.lt *= 2;
    a.chunks = (a.vecs + a.lt - 1) / a.lt;
}

}  // namespace rp

using namespace rp;

extern "C" int routepack_combine_tokens(const routepack_matrix *y, const routepack_ids *places, int32_t top_k,
                                        const float *gates, int64_t gate_stride, const routepack_matrix *out,
                                        hipStream_t stream) {
    RP_TRY(check_matrix(y));
    RP_TRY(check_places(places, top_k, gate_stride));
    RP_TRY(check_output(out, places->n_tokens, y->n_cols));
    if (out->type != y->type) return ROUTEPACK_E_INVALID;
    if (places->n_tokens == 0 || y->n_cols == 0) return ROUTEPACK_OK;
    if (!places->data || !out->data || (!y->data && y->n_rows > 0)) return ROUTEPACK_E_INVALID;
    CombineArgs a = {};
    a.y = y->data;
    a.stride = y->row_stride;
    a.n_rows = y->n_rows;
    a.cols = (int32_t)y->n_cols;
    a.places = static_cast<const int32_t *>(places->data);
    a.place_stride = places->token_stride;
    a.k = top_k;
    a.gates = gates;
    a.gate_stride = gate_stride;
    a.T = places->n_tokens;
    a.out = out->data;
    return by_type(y->type, [&](auto tag) -> int {
        using T = decltype(tag);
        geometry(a, Vec<T>::W);
        const int64_t items = a.T * a.chunks, per = 256 / a.lt;
        auto kern = a.lt == kWave ? k_combine<T, true> : k_combine<T, false>;
        hipLaunchKernelGGL(kern, grid_of((items + per - 1) / per), dim3(256), 0, stream, a);
        return launched();
    });
}

extern "C" int routepack_combine_backward(const routepack_matrix *dout, const routepack_matrix *y, const int32_t *rows,
                                          const routepack_ids *places, int32_t top_k, const float *gates,
                                          int64_t gate_stride, const routepack_matrix *dy, float *dgates,
                                          hipStream_t stream) {
    RP_TRY(check_matrix(dout));
    RP_TRY(check_matrix(y));
    RP_TRY(check_places(places, top_k, gate_stride));
    if (!dy && !dgates) return ROUTEPACK_E_INVALID;
    if (dout->type != y->type || dout->n_rows != places->n_tokens || dout->n_cols != y->n_cols) return ROUTEPACK_E_INVALID;
    if (dy) {
        RP_TRY(check_output(dy, y->n_rows, y->n_cols));
        if (dy->type != y->type) return ROUTEPACK_E_INVALID;
        if (y->n_rows > 0 && (!rows || (!dy->data && y->n_cols > 0))) return ROUTEPACK_E_INVALID;
    }
    const bool any = places->n_tokens > 0;
    if (any && !places->data) return ROUTEPACK_E_INVALID;
    if (any && y->n_cols > 0 && (!dout->data || (dgates && !y->data && y->n_rows > 0))) return ROUTEPACK_E_INVALID;
    CombineArgs a = {};
    a.y = y->data;
    a.stride = y->row_stride;
    a.n_rows = y->n_rows;
    a.cols = (int32_t)y->n_cols;
    a.places = static_cast<const int32_t *>(places->data);
    a.place_stride = places->token_stride;
    a.k = top_k;
    a.gates = gates;
    a.gate_stride = gate_stride;
    a.T = places->n_tokens;
    a.dout = dout->data;
    a.dout_stride = dout->row_stride;
    a.rows = rows;
    a.dy = dy && y->n_cols > 0 && y->n_rows > 0 ? dy->data : nullptr;
    a.dgates = dgates;
    return by_type(y->type, [&](auto tag) -> int {
        using T = decltype(tag);
        geometry(a, Vec<T>::W);
        const int nw = a.chunks > 1 ? 4 : 1;
        const int64_t per = nw > 1 ? 1 : 256 / a.lt;
        a.token_groups = (a.T + per - 1) / per;
        const int64_t n = a.token_groups + (a.dy ? (a.n_rows + 255) / 256 : 0);
        if (n == 0) return ROUTEPACK_OK;
        auto few = nw > 1 ? k_spread<T, 8, 4> : k_spread<T, 8, 1>;
        auto many = nw > 1 ? k_spread<T, 32, 4> : k_spread<T, 32, 1>;
        hipLaunchKernelGGL(a.k <= 8 ? few : many, grid_of(n), dim3(256), 0, stream, a);
        return launched();
    });
}
