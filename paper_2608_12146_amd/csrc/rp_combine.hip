// The sum of a token's rows under its gates and its gradients, on gfx950.
//
// Both are streams: out reads every row once; the gradients read it once more
// for the gates' part and write it once, with dout read once a token.  A token
// lies in LT lanes (a power of two, up to a wave), 16 bytes a lane.  8192 tokens x 8
// of 2048 bf16 are summed in 52 us (5.7 TB/s); the gradients of 8192 x 6 of 1447 fp32
// take 142 us (4.3 TB/s).
#include "rp_experts.h"

namespace rp {

struct CombineArgs {
    const void *y;
    int64_t stride;
    int32_t cols, vecs;        // vectors of 16 bytes a row
    int32_t lt, chunks;        // lanes of a token, vectors / lanes
    OrderView order;           // (rows: of the gradients)
    const float *gates;
    int64_t gate_stride;
    void *out;
    // gradients
    const void *dout;
    int64_t dout_stride;
    void *dy;
    float *dgates;
    int64_t token_groups;      // workgroups of tokens; those behind look for rows of no pair
};

// One vector of a row, zeros past its end.  WHOLE: there is no such vector, and all
// stand on 16 bytes.  ONCE: nothing reads it again.
template <class T, bool WHOLE, bool ONCE>
__device__ inline Vec<T> row_vec(const T *row, int32_t cols, int32_t c) {
    constexpr int W = Vec<T>::W;
    Vec<T> x;
    if (WHOLE || c + W <= cols) {
        load16<ONCE>(row + c, x.w);
    } else {
        float v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = c + i < cols ? to_f32(row[c + i]) : 0.0f;
        x.set(v);
    }
    return x;
}

template <class T, bool WHOLE, int N>
__device__ inline void add_rows(const CombineArgs &a, const int32_t *places, const float *gates, int32_t c,
                                float (&sum)[Vec<T>::W]) {
    constexpr int W = Vec<T>::W;
    Vec<T> x[N];
    float g[N];
    bool on[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int64_t r = places[j];
        on[j] = r >= 0 && r < a.order.n_rows;
        g[j] = gates ? gates[j] : 1.0f;
        x[j] = row_vec<T, WHOLE, true>(static_cast<const T *>(a.y) + (on[j] ? r : 0) * a.stride, a.cols, c);
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int w = 0; w < W; ++w) sum[w] = on[j] ? __builtin_fmaf(g[j], x[j].at(w), sum[w]) : sum[w];
}

// ONE: a wave has one token, whose places and gates are read by scalar loads.
template <class T, bool ONE, bool WHOLE>
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
    if (t >= a.order.T || v >= a.vecs) return;
    const int32_t *places = a.order.places + t * a.order.place_stride;
    const float *gates = a.gates ? a.gates + t * a.gate_stride : nullptr;
    float sum[W] = {};
    int j = 0;
    if (a.order.n_rows > 0) {
        for (; j + 4 <= a.order.k; j += 4) add_rows<T, WHOLE, 4>(a, places + j, gates ? gates + j : nullptr, v * W, sum);
        if (j + 2 <= a.order.k) {
            add_rows<T, WHOLE, 2>(a, places + j, gates ? gates + j : nullptr, v * W, sum);
            j += 2;
        }
        if (j < a.order.k) add_rows<T, WHOLE, 1>(a, places + j, gates ? gates + j : nullptr, v * W, sum);
    }
    store_vec<T, WHOLE>(static_cast<T *>(a.out) + t * a.cols, a.cols, v * W, sum);
}

// The sum over aligned groups of lt lanes.
__device__ inline float lanes_sum(float v, int lt) {
    for (int d = 1; d < lt; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// Rows r[0], .. of N choices j, ..: their products with d are added to dots, and
// gate times d is written where the row is the pair's.  The hint that y is read
// and dy written once pays where vectors do not cross lines (8192 tokens x 6 of 1448
// fp32: 150 -> 133 us), and for loads of 16-bit values (1447: 95 -> 80); else it
// costs (1447 fp32: 150 -> 162).
template <class T, bool WHOLE, int N>
__device__ inline void spread_rows(const CombineArgs &a, const int64_t (&r)[N], const bool (&own)[N], const float (&g)[N],
                                   int32_t c, const Vec<T> &d, float *dots) {
    constexpr int W = Vec<T>::W;
    if (a.dgates && a.order.n_rows > 0) {
        Vec<T> y[N];
#pragma unroll
        for (int j = 0; j < N; ++j)  // (no row: the first one, not counted)
            y[j] = row_vec<T, WHOLE, WHOLE || sizeof(T) == 2>(static_cast<const T *>(a.y) + (r[j] >= 0 ? r[j] : 0) * a.stride, a.cols, c);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float sum = dots[j];
#pragma unroll
            for (int w = 0; w < W; ++w) sum = __builtin_fmaf(y[j].at(w), d.at(w), sum);
            dots[j] = r[j] >= 0 ? sum : dots[j];
        }
    }
    if (a.dy) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (!own[j]) continue;
            float x[W];
#pragma unroll
            for (int w = 0; w < W; ++w) x[w] = g[j] * d.at(w);
            T *const to = static_cast<T *>(a.dy) + r[j] * a.cols;
            if constexpr (WHOLE) {
                Vec<T> v;
                v.set(x);
                typedef uint32_t four __attribute__((ext_vector_type(4)));
                __builtin_nontemporal_store(four{v.w[0], v.w[1], v.w[2], v.w[3]}, reinterpret_cast<four *>(to + c));
            } else {
                store_vec<T, false>(to, a.cols, c, x);
            }
        }
    }
}

// Gradients of a token: each vector of dout is held while the same of its k rows
// is read (for the gates) and written.  NW > 0: a token has NW waves, which look
// its rows up once, a lane a choice, and hold them in scalars; NW = 0: a wave has
// several tokens, of lt lanes.
template <class T, int K, int NW, bool WHOLE>
__global__ void __launch_bounds__(256) k_spread(CombineArgs a) {
    constexpr int W = Vec<T>::W;
    __shared__ float part[4][K];
    if (group_index() >= a.token_groups) {  // rows of no pair: zeros
        // (without dy these are the groups that fill the grid's last row: there may be no `rows` either)
        if (!a.dy) return;
        const int lane = threadIdx.x & 63;
        const int64_t r0 = (group_index() - a.token_groups) * 256 + (threadIdx.x & ~63);
        const bool mine = r0 + lane < a.order.n_rows && a.order.pair_of_row(r0 + lane) < 0;
        for (uint64_t m = __ballot(mine); m; m &= m - 1) {
            T *row = static_cast<T *>(a.dy) + (r0 + __builtin_ctzll(m)) * a.cols;
            const float zero[W] = {};
            for (int32_t v = lane; v < a.vecs; v += kWave) store_vec<T, false>(row, a.cols, v * W, zero);
        }
        return;
    }
    const int lt = NW ? kWave : a.lt, lane = threadIdx.x & (lt - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = NW ? group_index() * (4 / (NW ? NW : 1)) + wave / (NW ? NW : 1) : group_index() * (256 / lt) + threadIdx.x / lt;
    const bool live = t < a.order.T;
    const int32_t k = a.order.k;
    float dots[K] = {};
    if (live) {
        const int32_t *places = a.order.places + t * a.order.place_stride;
        const float *gates = a.gates ? a.gates + t * a.gate_stride : nullptr;
        const T *dout = static_cast<const T *>(a.dout) + t * a.dout_stride;
        auto look_up = [&](int j, bool &own, float &g) -> int {
            const int32_t r = places[j];
            const bool on = r >= 0 && r < a.order.n_rows;
            own = on && a.dy && a.order.rows[r] == t * k + j;
            g = gates ? gates[j] : 1.0f;
            return on ? r : -1;
        };
        int mine = -1;
        bool mine_own = false;
        float mine_gate = 0.0f;
        if (NW && lane < k) mine = look_up(lane, mine_own, mine_gate);
        for (int32_t v = lane + (NW ? wave % (NW ? NW : 1) * kWave : 0); v < a.vecs; v += lt * (NW ? NW : 1)) {
            const Vec<T> d = row_vec<T, WHOLE, WHOLE || sizeof(T) == 2>(dout, a.cols, v * W);
            auto batch = [&](auto n_, int j0, float *sums) {
                constexpr int N = decltype(n_)::value;
                int64_t r[N];
                bool own[N];
                float g[N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (NW) {
                        r[j] = __builtin_amdgcn_readlane(mine, j0 + j);
                        own[j] = __builtin_amdgcn_readlane((int)mine_own, j0 + j);
                        g[j] = __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(mine_gate), j0 + j));
                    } else {
                        r[j] = look_up(j0 + j, own[j], g[j]);
                    }
                }
                spread_rows<T, WHOLE, N>(a, r, own, g, v * W, d, sums);
            };
#pragma unroll
            for (int j0 = 0; j0 < K; j0 += 4) {
                const int left = k - j0;
                if (left >= 4) batch(Int<4>(), j0, dots + j0);
                else if (left == 3) batch(Int<3>(), j0, dots + j0);
                else if (left == 2) batch(Int<2>(), j0, dots + j0);
                else if (left == 1) batch(Int<1>(), j0, dots + j0);
            }
        }
    }
    if (!a.dgates) return;
#pragma unroll
    for (int j = 0; j < K; ++j)
        if (j < k) dots[j] = lanes_sum(dots[j], lt);
    if (NW > 1) {
        if (lane == 0)
#pragma unroll
            for (int j = 0; j < K; ++j) part[wave][j] = dots[j];
        __syncthreads();
        if (wave % (NW ? NW : 1) == 0 && live && lane < k) {
            float s = 0.0f;
            for (int w = 0; w < NW; ++w) s += part[wave + w][lane];
            a.dgates[t * k + lane] = s;
        }
    } else if (live && lane == 0) {
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < k) a.dgates[t * k + j] = dots[j];
    }
}

// Rows of whole vectors of 16 bytes, on their boundaries (or none).
template <class T>
bool whole_rows(const void *data, int64_t stride, int64_t cols) {
    constexpr int W = Vec<T>::W;
    return !data || (((uintptr_t)data & 15) == 0 && stride % W == 0 && cols % W == 0);
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
    RP_TRY(check_places(places, top_k, kMaxChoices));
    if (gate_stride < 0) return ROUTEPACK_E_INVALID;
    if (!sizes_fit(places->n_tokens, gate_stride)) return ROUTEPACK_E_UNSUPPORTED;
    RP_TRY(check_output(out, places->n_tokens, y->n_cols));
    if (out->type != y->type) return ROUTEPACK_E_INVALID;
    if (places->n_tokens == 0 || y->n_cols == 0) return ROUTEPACK_OK;
    if (!places->data || !out->data || (!y->data && y->n_rows > 0)) return ROUTEPACK_E_INVALID;
    CombineArgs a = {};
    a.y = y->data;
    a.stride = y->row_stride;
    a.cols = (int32_t)y->n_cols;
    a.order = {nullptr, static_cast<const int32_t *>(places->data), places->token_stride, places->n_tokens, y->n_rows, top_k};
    a.gates = gates;
    a.gate_stride = gate_stride;
    a.out = out->data;
    return by_type(y->type, [&](auto tag) -> int {
        using T = decltype(tag);
        geometry(a, Vec<T>::W);
        const int64_t items = a.order.T * a.chunks, per = 256 / a.lt;
        const bool whole = whole_rows<T>(y->data, a.stride, a.cols) && whole_rows<T>(a.out, a.cols, a.cols);
        auto kern = whole ? (a.lt == kWave ? k_combine<T, true, true> : k_combine<T, false, true>)
                          : (a.lt == kWave ? k_combine<T, true, false> : k_combine<T, false, false>);
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
    RP_TRY(check_places(places, top_k, kMaxChoices));
    if (gate_stride < 0) return ROUTEPACK_E_INVALID;
    if (!sizes_fit(places->n_tokens, gate_stride)) return ROUTEPACK_E_UNSUPPORTED;
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
    a.cols = (int32_t)y->n_cols;
    a.order = {rows, static_cast<const int32_t *>(places->data), places->token_stride, places->n_tokens, y->n_rows, top_k};
    a.gates = gates;
    a.gate_stride = gate_stride;
    a.dout = dout->data;
    a.dout_stride = dout->row_stride;
    a.dy = dy && y->n_cols > 0 && y->n_rows > 0 ? dy->data : nullptr;
    a.dgates = dgates;
    return by_type(y->type, [&](auto tag) -> int {
        using T = decltype(tag);
        geometry(a, Vec<T>::W);
        // A token's waves: as many of four as its vectors of 64 lanes fill evenly (three:
        // one wave, 82 us for 8192 x 6 x 1447 bf16, 90 with two), four where there are
        // many of them or few tokens.
        const bool all_four = a.chunks % 4 == 0 || a.chunks > 8 || (a.order.T < 1024 && a.chunks > 1);
        const int nw = a.lt < kWave ? 0 : all_four ? 4 : a.chunks % 2 == 0 ? 2 : 1;
        const int64_t per = nw ? 4 / nw : 256 / a.lt;
        a.token_groups = (a.order.T + per - 1) / per;
        const int64_t n = a.token_groups + (a.dy ? (a.order.n_rows + 255) / 256 : 0);
        if (n == 0) return ROUTEPACK_OK;
        const bool whole = whole_rows<T>(a.dgates ? a.y : nullptr, a.stride, a.cols) &&
                           whole_rows<T>(a.dout, a.dout_stride, a.cols) && whole_rows<T>(a.dy, a.cols, a.cols);
        auto pick = [&](auto k_, auto whole_) {
            constexpr int K = decltype(k_)::value;
            constexpr bool W = decltype(whole_)::value != 0;
            return nw == 4 ? k_spread<T, K, 4, W> : nw == 2 ? k_spread<T, K, 2, W> : nw == 1 ? k_spread<T, K, 1, W> : k_spread<T, K, 0, W>;
        };
        // (more than 8 choices: the checks cost little beside them)
        const auto kern = top_k > 8 ? pick(Int<32>(), Int<0>()) : whole ? pick(Int<8>(), Int<1>()) : pick(Int<8>(), Int<0>());
        hipLaunchKernelGGL(kern, grid_of(n), dim3(256), 0, stream, a);
        return launched();
    });
}
