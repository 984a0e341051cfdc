// The experts' products on matrices in 4 bits, on gfx950: y[r] = w[s] x[r] for the
// rows of slot s, by the block-scaled matrix instructions, which multiply 32
// values of a row with their power of two each.
#include "rp_product.h"

namespace rp {

struct ProductArgs {
    const uint8_t *xc, *xs, *wc, *ws;
    int32_t groups;   // groups of 128 columns
    int32_t N, n_slots, n_tiles;
    int64_t R;
    const int64_t *offsets;
    void *y;
    int64_t tiles;    // workgroups of tiles; those behind clear rows
    int64_t clears;
};

// Few rows a slot: a workgroup holds 16 of a slot's N and passes over its rows,
// 16 RB at a time; the four waves share the columns and add up in LDS.
// Bound by the weights' bytes: each is read once (per pass).
template <class T, int RB>
__global__ void __launch_bounds__(256) k_product_few(ProductArgs a) {
    __shared__ float part[4][RB][4][kWave];
    const int64_t id = group_index();
    if (id >= a.tiles) {
        clear_rows(static_cast<T *>(a.y), a.N, a.offsets, a.n_slots, a.R, id - a.tiles, a.clears);
        return;
    }
    const int64_t index = id / a.n_tiles;
    const int32_t n0 = (int32_t)(id - index * a.n_tiles) * 16;
    int64_t before, total;
    const int32_t s = slot_of_tile<true>(a.offsets, a.n_slots, a.R, 0, index, before, total);
    if (s < 0) return;
    const Segment seg = segment_of(a.offsets, s, a.R);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4, i16 = lane & 15;
    const int32_t n = n0 + i16 < a.N ? n0 + i16 : a.N - 1;
    const int64_t row = (int64_t)s * a.N + n;
    const uint8_t *wc = a.wc + row * a.groups * 64 + q * 16, *ws = a.ws + row * a.groups * 4;
    const int32_t g0 = (int32_t)((int64_t)a.groups * wave / 4), g1 = (int32_t)((int64_t)a.groups * (wave + 1) / 4);
    for (int64_t r0 = seg.begin; r0 < seg.end; r0 += 16 * RB) {
        const uint8_t *xc[RB], *xs[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int64_t r = r0 + b * 16 + i16, x = r < seg.end ? r : seg.end - 1;
            xc[b] = a.xc + x * a.groups * 64 + q * 16;
            xs[b] = a.xs + x * a.groups * 4;
        }
        float4_ sum[RB] = {};
#pragma unroll 4
        for (int32_t g = g0; g < g1; ++g) {
            const int4_ w = *reinterpret_cast<const int4_ *>(wc + (int64_t)g * 64);
            const int wscale = (*reinterpret_cast<const int *>(ws + (int64_t)g * 4) >> (8 * q)) & 255;
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int4_ x = *reinterpret_cast<const int4_ *>(xc[b] + (int64_t)g * 64);
                const int xscale = (*reinterpret_cast<const int *>(xs[b] + (int64_t)g * 4) >> (8 * q)) & 255;
                const int8_ wa = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, xb = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
                sum[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, xb, sum[b], 4, 4, 0, wscale, 0, xscale);
            }
        }
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave][b][i][lane] = sum[b][i];
        __syncthreads();
        // value (n, r) stands in lane (n / 4) 16 + r, element n % 4
        const int n_ = threadIdx.x & 15, r_ = threadIdx.x >> 4, from = (n_ >> 2) * 16 + r_;
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const float v = (part[0][b][n_ & 3][from] + part[1][b][n_ & 3][from]) +
                            (part[2][b][n_ & 3][from] + part[3][b][n_ & 3][from]);
            const int64_t r = r0 + b * 16 + r_;
            if (r < seg.end && n0 + n_ < a.N) static_cast<T *>(a.y)[r * a.N + n0 + n_] = (T)v;
        }
        __syncthreads();
    }
}

}  // namespace rp

using namespace rp;

extern "C" int routepack_expert_product(const routepack_mx *x, const routepack_mx *w, int32_t n_slots,
                                        const int64_t *offsets, const routepack_matrix *y, hipStream_t stream) {
    RP_TRY(check_mx(x, true));
    RP_TRY(check_mx(w, true));
    if (n_slots < 1 || w->n_rows % n_slots != 0 || w->n_cols != x->n_cols) return ROUTEPACK_E_INVALID;
    const int64_t N = w->n_rows / n_slots;
    if (n_slots > kMaxSlots || N > kMaxCols) return ROUTEPACK_E_UNSUPPORTED;
    RP_TRY(check_output(y, x->n_rows, N));
    if (x->n_rows == 0 || N == 0) return ROUTEPACK_OK;
    if (!offsets || !y->data) return ROUTEPACK_E_INVALID;
    ProductArgs a = {};
    a.xc = static_cast<const uint8_t *>(x->codes);
    a.xs = static_cast<const uint8_t *>(x->scales);
    a.wc = static_cast<const uint8_t *>(w->codes);
    a.ws = static_cast<const uint8_t *>(w->scales);
    a.groups = (int32_t)(padded_cols(x->n_cols) / 128);
    a.N = (int32_t)N;
    a.n_slots = n_slots;
    a.R = x->n_rows;
    a.offsets = offsets;
    a.y = y->data;
    a.n_tiles = (int32_t)((N + 15) / 16);
    const int64_t most = a.R < n_slots ? a.R : n_slots;  // slots with rows
    a.tiles = most * a.n_tiles;
    const int64_t pieces = (a.R * N + 65535) / 65536;
    a.clears = pieces < 256 ? pieces : 256;
    return by_type(y->type, [&](auto tag) -> int {
        using T = decltype(tag);
        hipLaunchKernelGGL((k_product_few<T, 2>), grid_of(a.tiles + a.clears), dim3(256), 0, stream, a);
        return launched();
    });
}
