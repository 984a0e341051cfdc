// Matrices into microscaled 4-bit floating point and back, on gfx950.
//
// A lane holds 8 columns, 4 lanes a block of 32, 16 lanes the 128 columns that
// a row is padded to: a lane's codes are one word, the group's scales another.
// The block's exponent is the exponent field of the largest magnitude's bits
// (as integers these order like the magnitudes, NaN above infinity above the
// finite); the conversion instruction divides by the power of two and rounds
// to the nearest code, ties to even, ending at 6.
// Bound by bytes: what is read, and 17/32 of a byte written a value.
#include "rp_experts.h"

namespace rp {

struct QuantizeArgs {
    const void *x;
    int64_t stride, n_in;   // rows of x
    int32_t cols, groups;   // groups of 128 columns a row
    const int32_t *rows;
    int32_t per_row;
    int64_t n_out;
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

template <class T>
__global__ void __launch_bounds__(256) k_quantize(QuantizeArgs a) {
    const int64_t item = group_index() * 16 + (threadIdx.x >> 4), n = a.n_out * a.groups;
    if (item >= n) return;  // (all 16 lanes)
    const int64_t r = n <= UINT32_MAX ? (uint32_t)item / (uint32_t)a.groups : item / a.groups;
    const int32_t g = (int32_t)(item - r * a.groups), lane = threadIdx.x & 15;
    int64_t from = r;
    if (a.rows) {
        const int32_t p = a.rows[r];
        from = p < 0 ? -1 : (int64_t)((uint32_t)p / (uint32_t)a.per_row);
    }
    float v[8];
    uint32_t big = 0;
    if (from >= 0 && from < a.n_in) {
        load8(static_cast<const T *>(a.x) + from * a.stride, a.cols, g * 128 + lane * 8, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t u = __float_as_uint(v[i]) & 0x7FFFFFFFu;
            big = u > big ? u : big;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
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
    const int64_t at = r * a.groups + g;
    a.codes[at * 16 + lane] = odd ? 0u : w;
    // the four blocks' scales in one word
    uint32_t all = s << (8 * (lane >> 2));
    all |= across<8>(all);
    all |= across<16>(all);
    if (lane == 0) a.scales[at] = all;
}

struct DequantizeArgs {
    const uint32_t *codes;
    const uint8_t *scales;
    int64_t n_rows;
    int32_t cols, groups;
    void *x;
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
        if (c + i * W < a.cols) store_vec<T, false>(row, a.cols, c + i * W, y);
    }
}

}  // namespace rp

using namespace rp;

extern "C" int routepack_quantize_mx(const routepack_matrix *x, const int32_t *rows, int32_t per_row,
                                     const routepack_mx *q, hipStream_t stream) {
    RP_TRY(check_matrix(x));
    RP_TRY(check_mx(q, true));
    if (q->n_cols != x->n_cols) return ROUTEPACK_E_INVALID;
    if (rows ? per_row < 1 : q->n_rows != x->n_rows) return ROUTEPACK_E_INVALID;
    if (q->n_rows == 0 || q->n_cols == 0) return ROUTEPACK_OK;
    if (!x->data && x->n_rows > 0) return ROUTEPACK_E_INVALID;
    QuantizeArgs a = {x->data, x->row_stride, x->n_rows, (int32_t)x->n_cols, (int32_t)(padded_cols(x->n_cols) / 128), rows,
                      per_row, q->n_rows, static_cast<uint32_t *>(q->codes), static_cast<uint32_t *>(q->scales)};
    return by_type(x->type, [&](auto tag) -> int {
        using T = decltype(tag);
        hipLaunchKernelGGL(k_quantize<T>, grid_of((a.n_out * a.groups + 15) / 16), dim3(256), 0, stream, a);
        return launched();
    });
}

extern "C" int routepack_dequantize_mx(const routepack_mx *q, const routepack_matrix *x, hipStream_t stream) {
    RP_TRY(check_mx(q, true));
    RP_TRY(check_output(x, q->n_rows, q->n_cols));
    if (q->n_rows == 0 || q->n_cols == 0) return ROUTEPACK_OK;
    if (!x->data) return ROUTEPACK_E_INVALID;
    DequantizeArgs a = {static_cast<const uint32_t *>(q->codes), static_cast<const uint8_t *>(q->scales), q->n_rows,
                        (int32_t)q->n_cols, (int32_t)(padded_cols(q->n_cols) / 128), x->data};
    return by_type(x->type, [&](auto tag) -> int {
        using T = decltype(tag);
        hipLaunchKernelGGL(k_dequantize<T>, grid_of((a.n_rows * a.groups + 15) / 16), dim3(256), 0, stream, a);
        return launched();
    });
}
