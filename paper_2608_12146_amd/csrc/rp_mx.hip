// Matrices into microscaled 4-bit floating point and back, on gfx950.
//
// A lane holds 8 columns, 4 lanes a block of 32, 16 lanes the 128 columns that
// a row is padded to: a lane's codes are one word, the group's scales another.
// The block's exponent is the exponent field of the largest magnitude's bits
// (as integers these order like the magnitudes, NaN above infinity above the
// finite); the conversion instruction divides by the power of two and rounds
// to the nearest code, ties to even, ending at 6.
// Bound by bytes: what is read, and 17/32 of a byte written a value.  Gathered
// into an order, a token is read and converted once, and written to its k rows
// (8192 x 2048 bf16, 8 rows each: 21 us, 70 with a row's conversion each).
#include "rp_experts.h"

namespace rp {

struct QuantizeArgs {
    const void *x;
    int64_t stride, n_in;   // rows of x
    int32_t cols, groups;   // groups of 128 columns a row
    OrderView order;        // rows null: none
    int64_t item_groups;    // workgroups of x's rows; those behind look for rows of no pair
    uint32_t *codes, *scales;
};

// 8 columns from c on, zeros past the row's end.
template <class T>
__device__ inline void load8(const T *row, int32_t cols, int32_t c, float (&v)[8]) {
    constexpr int W = Vec<T>::W;
    if (c + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < 8 / W; ++i) {
            Vec<T> x;
            load16<false>(row + c + i * W, x.w);
#pragma unroll
            for (int w = 0; w < W; ++w) v[i * W + w] = x.at(w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? to_f32(row[c + i]) : 0.0f;
    }
}

template <class T, bool ORDER>
__global__ void __launch_bounds__(256) k_quantize(QuantizeArgs a) {
    if (ORDER && group_index() >= a.item_groups) {  // rows of no pair: zeros
        const int lane = threadIdx.x & 63;
        const int64_t r0 = (group_index() - a.item_groups) * 256 + (threadIdx.x & ~63);
        const bool mine = r0 + lane < a.order.n_rows && a.order.pair_of_row(r0 + lane) < 0;
        for (uint64_t m = __ballot(mine); m; m &= m - 1) {
            const int64_t at = (r0 + __builtin_ctzll(m)) * a.groups;
            for (int64_t i = lane; i < (int64_t)a.groups * 16; i += kWave) a.codes[at * 16 + i] = 0;
            for (int64_t i = lane; i < a.groups; i += kWave) a.scales[at + i] = 0;
        }
        return;
    }
    const int64_t item = group_index() * 16 + (threadIdx.x >> 4), n = a.n_in * a.groups;
    if (item >= n) return;  // (all 16 lanes)
    const int64_t r = n <= UINT32_MAX ? (uint32_t)item / (uint32_t)a.groups : item / a.groups;
    const int32_t g = (int32_t)(item - r * a.groups), lane = threadIdx.x & 15;
    float v[8];
    load8(static_cast<const T *>(a.x) + r * a.stride, a.cols, g * 128 + lane * 8, v);
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        big = u > big ? u : big;
    }
    uint32_t o = across<2>(big);
    big = o > big ? o : big;
    o = across<4>(big);
    big = o > big ? o : big;
    // (subnormal magnitudes have exponent field 0, like those below 2^-125)
    const uint32_t e = big >> 23;
    const bool odd = e == 255;
    const uint32_t s = odd ? 255u : e > 2 ? e - 2 : 0u;
    const float by = scale_of(odd ? 127u : s);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], by, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], by, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], by, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], by, 3);
    w = odd ? 0u : w;
    // the four blocks' scales in one word
    uint32_t all = s << (8 * (lane >> 2));
    all |= across<8>(all);
    all |= across<16>(all);
    auto put = [&](int64_t row) {
        const int64_t at = row * a.groups + g;
        a.codes[at * 16 + lane] = w;
        if (lane == 0) a.scales[at] = all;
    };
    if constexpr (ORDER) {
        for (int j0 = 0; j0 < a.order.k; j0 += 16) {
            const int left = a.order.k - j0 < 16 ? a.order.k - j0 : 16;
            const int mine = lane < left ? (int)a.order.row_of_pair(r, j0 + lane) : -1;
            for (int j = 0; j < left; ++j) {
                const int row = __shfl(mine, j, 16);
                if (row >= 0) put(row);
            }
        }
    } else {
        put(r);
    }
}

struct DequantizeArgs {
    const uint32_t *codes;
    const uint8_t *scales;
    int64_t n_rows;
    int32_t cols, groups;
    void *x;
    bool whole;  // vectors of 16 bytes fill the rows, and stand on their boundaries
};

template <class T>
__global__ void __launch_bounds__(256) k_dequantize(DequantizeArgs a) {
    constexpr int W = Vec<T>::W;
    const int64_t item = group_index() * 16 + (threadIdx.x >> 4), n = a.n_rows * a.groups;
    if (item >= n) return;
    const int64_t r = n <= UINT32_MAX ? (uint32_t)item / (uint32_t)a.groups : item / a.groups;
    const int32_t g = (int32_t)(item - r * a.groups), lane = threadIdx.x & 15, c = g * 128 + lane * 8;
    if (c >= a.cols) return;
    typedef float two __attribute__((ext_vector_type(2)));
    const uint32_t w = a.codes[item * 16 + lane];
    const float by = scale_of(a.scales[item * 4 + (lane >> 2)]);
    const two v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 3)};
    T *row = static_cast<T *>(a.x) + r * a.cols;
#pragma unroll
    for (int i = 0; i < 8 / W; ++i) {
        float y[W];
#pragma unroll
        for (int j = 0; j < W; ++j) y[j] = v[(i * W + j) / 2][j % 2];
        // (whole lines of a large matrix, which leave the cache anyway: with the hint
        // 65536 x 2048 bf16 take 48 us, 70 without)
        if (a.whole) {
            Vec<T> x;
            x.set(y);
            typedef uint32_t four __attribute__((ext_vector_type(4)));
            __builtin_nontemporal_store(four{x.w[0], x.w[1], x.w[2], x.w[3]}, reinterpret_cast<four *>(row + c + i * W));
        } else if (c + i * W < a.cols) {
            store_vec<T, false>(row, a.cols, c + i * W, y);
        }
    }
}

}  // namespace rp

using namespace rp;

extern "C" int routepack_quantize_mx(const routepack_matrix *x, const int32_t *rows, const routepack_ids *places,
                                     int32_t top_k, const routepack_mx *q, hipStream_t stream) {
    RP_TRY(check_matrix(x));
    RP_TRY(check_mx(q, true));
    if (q->n_cols != x->n_cols || (rows && !places) || (places && !rows && q->n_rows > 0)) return ROUTEPACK_E_INVALID;
    if (places) {
        RP_TRY(check_places(places, top_k, 256));
        if (places->n_tokens != x->n_rows || (!places->data && x->n_rows > 0 && q->n_rows > 0)) return ROUTEPACK_E_INVALID;
        if (q->n_rows > INT32_MAX) return ROUTEPACK_E_UNSUPPORTED;
    } else if (q->n_rows != x->n_rows) {
        return ROUTEPACK_E_INVALID;
    }
    if (q->n_rows == 0 || q->n_cols == 0) return ROUTEPACK_OK;
    if (!x->data && x->n_rows > 0) return ROUTEPACK_E_INVALID;
    QuantizeArgs a = {};
    a.x = x->data;
    a.stride = x->row_stride;
    a.n_in = x->n_rows;
    a.cols = (int32_t)x->n_cols;
    a.groups = (int32_t)(padded_cols(x->n_cols) / 128);
    if (places)
        a.order = {rows, static_cast<const int32_t *>(places->data), places->token_stride, x->n_rows, q->n_rows, top_k};
    a.item_groups = (a.n_in * a.groups + 15) / 16;
    a.codes = static_cast<uint32_t *>(q->codes);
    a.scales = static_cast<uint32_t *>(q->scales);
    return by_type(x->type, [&](auto tag) -> int {
        using T = decltype(tag);
        const int64_t n = a.item_groups + (places ? (q->n_rows + 255) / 256 : 0);
        hipLaunchKernelGGL((places ? k_quantize<T, true> : k_quantize<T, false>), grid_of(n), dim3(256), 0, stream, a);
        return launched();
    });
}

extern "C" int routepack_dequantize_mx(const routepack_mx *q, const routepack_matrix *x, hipStream_t stream) {
    RP_TRY(check_mx(q, true));
    RP_TRY(check_output(x, q->n_rows, q->n_cols));
    if (q->n_rows == 0 || q->n_cols == 0) return ROUTEPACK_OK;
    if (!x->data) return ROUTEPACK_E_INVALID;
    DequantizeArgs a = {static_cast<const uint32_t *>(q->codes), static_cast<const uint8_t *>(q->scales), q->n_rows,
                        (int32_t)q->n_cols, (int32_t)(padded_cols(q->n_cols) / 128), x->data, false};
    return by_type(x->type, [&](auto tag) -> int {
        using T = decltype(tag);
        a.whole = a.cols % 8 == 0 && ((uintptr_t)x->data & 15) == 0;
        hipLaunchKernelGGL(k_dequantize<T>, grid_of((a.n_rows * a.groups + 15) / 16), dim3(256), 0, stream, a);
        return launched();
    });
}
