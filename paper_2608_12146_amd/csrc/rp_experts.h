// What the experts' operators share: their limits, the checks of their arguments,
// and the order's view of pairs and rows.
#pragma once

#include "rp_internal.h"
#include "rp_route.h"
#include "routepack/experts.h"

namespace rp {

constexpr int kMaxSlots = 2048;
constexpr int64_t kMaxCols = (int64_t)1 << 24, kMaxBytes = (int64_t)1 << 62;

inline int64_t padded_cols(int64_t cols) { return (cols + 127) / 128 * 128; }

// rows * cols elements of up to 16 bytes fit 62 bits.
inline bool sizes_fit(int64_t rows, int64_t cols) { return cols == 0 || rows <= kMaxBytes / 16 / cols; }

inline int check_matrix(const routepack_matrix *x) {
    if (!x || x->n_rows < 0 || x->n_cols < 0 || x->row_stride < 0) return ROUTEPACK_E_INVALID;
    if (x->type < ROUTEPACK_F32 || x->type > ROUTEPACK_F16) return ROUTEPACK_E_INVALID;
    if (x->n_cols > kMaxCols || !sizes_fit(x->n_rows, x->n_cols) || !sizes_fit(x->n_rows, x->row_stride))
        return ROUTEPACK_E_UNSUPPORTED;
    return ROUTEPACK_OK;
}

// An output: dense.
inline int check_output(const routepack_matrix *x, int64_t rows, int64_t cols) {
    RP_TRY(check_matrix(x));
    if (x->n_rows != rows || x->n_cols != cols || x->row_stride != cols) return ROUTEPACK_E_INVALID;
    return ROUTEPACK_OK;
}

// data: whether the call reads or writes its bytes.
inline int check_mx(const routepack_mx *q, bool data) {
    if (!q || q->n_rows < 0 || q->n_cols < 0) return ROUTEPACK_E_INVALID;
    if (q->n_cols > kMaxCols || !sizes_fit(q->n_rows, padded_cols(q->n_cols))) return ROUTEPACK_E_UNSUPPORTED;
    if (data && q->n_rows > 0 && q->n_cols > 0) {
        if (!q->codes || !q->scales) return ROUTEPACK_E_INVALID;
        if ((uintptr_t)q->codes & 15 || (uintptr_t)q->scales & 3) return ROUTEPACK_E_INVALID;
    }
    return ROUTEPACK_OK;
}

// The places of an order, [T][1][k]: k <= most.
inline int check_places(const routepack_ids *p, int32_t k, int32_t most) {
    if (!p || p->type != ROUTEPACK_I32 || p->n_tokens < 0 || p->token_stride < 0 || k < 1) return ROUTEPACK_E_INVALID;
    if (k > most || p->n_tokens > INT32_MAX / k || !sizes_fit(p->n_tokens, p->token_stride)) return ROUTEPACK_E_UNSUPPORTED;
    return ROUTEPACK_OK;
}

// An order's rows and places, on the device.
struct OrderView {
    const int32_t *rows;
    const int32_t *places;
    int64_t place_stride, T, n_rows;
    int32_t k;
    // The pair that stands in row r, if its place is r; else -1.
    __device__ int64_t pair_of_row(int64_t r) const {
        const int32_t p = rows[r];
        if (p < 0) return -1;
        const uint32_t t = (uint32_t)p / (uint32_t)k;
        if (t >= T) return -1;
        return places[t * place_stride + (p - t * (uint32_t)k)] == r ? p : -1;
    }
    // The row of token t's choice j, if it is that row's pair; else -1.
    __device__ int64_t row_of_pair(int64_t t, int j) const {
        const int64_t r = places[t * place_stride + j];
        return r >= 0 && r < n_rows && rows[r] == t * k + j ? r : -1;
    }
};

inline int launched() { return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE; }

// The workgroup's index in a grid of grid_of.
__device__ inline int64_t group_index() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// 2^(x - 127) of a scale byte as the bits of a float (255: an infinity, which
// the conversions take as NaN).
__device__ inline float scale_of(uint32_t x) { return __uint_as_float(x ? x << 23 : 0x00400000u); }

}  // namespace rp
