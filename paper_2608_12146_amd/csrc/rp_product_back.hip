// The gradients of the experts' products (rp_product.hip), on gfx950:
//   dx[r][c]    = sum_n dy[r][n] w[s][n][c]   for the rows r of slot s,
//   dw[s][n][c] = sum_r dy[r][n] x[r][c]      over the rows r of slot s.
// A 4-bit value times its power of two is exact in bf16, and dy is split into
// bf16 parts that add up to it (one for bf16, two for fp16, three for fp32), so
// bf16 matrix instructions form exact products and add them in 32 bits.
//
// Both are the same tile program: A is dy, 128 of the output's rows by 64 terms;
// B is the matrix in 4 bits, 64 terms (its rows) by 128 columns, converted on
// the way into LDS.  The terms are B's rows, and A's too in dw: their fragments
// are read through the transposing LDS loads (16 lanes read 4 terms of 16
// columns and each receives a column's 4 terms).
#include "rp_product.h"

namespace rp {

struct BackProductArgs {
    const void *dy;
    int64_t stride;
    const uint8_t *bc, *bs;  // w (dx) or x (dw)
    int32_t groups;          // groups of 128 columns
    int32_t N, C, n_slots;
    int32_t m_tiles, c_tiles;  // of N (dw), of C
    int64_t R;
    const int64_t *offsets;
    void *out;
    int64_t tiles, clears;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4_ __attribute__((ext_vector_type(4)));
typedef short short8_ __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = 128, kTerms = 64;

template <class T> constexpr int kParts = sizeof(T) == 4 ? 3 : __is_same(T, _Float16) ? 2 : 1;

// The first bf16 part of v, by truncation (exact where nothing is left), and
// what is left of v.  Infinities and NaN leave nothing.
__device__ inline uint32_t take_part(float &v) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7F800000u) == 0x7F800000u) {
        v = 0.0f;
        return (u & 0x007FFFFFu) ? 0x7FC0u : u >> 16;
    }
    v -= __uint_as_float(u & 0xFFFF0000u);
    return u >> 16;
}

// 8 values of dy as P vectors of bf16 parts.
template <class T, int P>
__device__ inline void split8(const T *row, int32_t from, int32_t end, bool live, int4_ (&part)[P]) {
    // (a row whose terms do not count is zeros)
    if (P == 1 && live && from + 8 <= end) {
        uint32_t w[4];
        load16<false>(row + from, w);
        part[0] = int4_{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
        return;
    }
    float v[8];
    if (live && from + 8 <= end) {
        constexpr int W = Vec<T>::W;
#pragma unroll
        for (int i = 0; i < 8 / W; ++i) {
            Vec<T> x;
            load16<false>(row + from + i * W, x.w);
#pragma unroll
            for (int j = 0; j < W; ++j) v[i * W + j] = x.at(j);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = live && from + i < end ? to_f32(row[from + i]) : 0.0f;
    }
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = take_part(v[2 * i]), hi = take_part(v[2 * i + 1]);
            part[p][i] = (int)(hi << 16 | lo);
        }
}

// Byte of column c (a multiple of 4) of term row k in a tile of COLS columns: each
// four pieces of 64 bytes of the row, and the four of 16 in each, are exchanged by
// the row, so that the 4 rows of a transposing load, and the 4 rows that 16 lanes
// write, stand in different banks.
template <int COLS>
__device__ inline int term_at(int k, int c) {
    return k * COLS * 2 + (((c >> 5) ^ (k & 3)) << 6) + ((((c >> 3) ^ k) & 3) << 4) + (c & 7) * 2;
}

// The fragment of 32 columns from c0 and 16 terms from k0 on.
template <int COLS>
__device__ inline bf16x8 term_fragment(const char *tile, int k0, int c0) {
    const int lane = threadIdx.x & 63, i = (lane >> 2) & 3, k = k0 + (lane >> 5) * 8 + i;
    const int c = c0 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    typedef __attribute__((address_space(3))) short4_ lds4;
    const short4_ a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(tile + term_at<COLS>(k, c)));
    const short4_ b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(tile + term_at<COLS>(k + 4, c)));
    const short8_ v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, v);
}

template <class T, bool DW, int NB>
__global__ void __launch_bounds__(256, 2) k_product_back(BackProductArgs a) {
    constexpr int P = kParts<T>;
    constexpr int kCols = 64 * NB;  // a wave has 2 x NB matrix tiles, two waves each way
    extern __shared__ __attribute__((aligned(16))) char lds[];
    char *const Bs = lds + P * kTile * kTerms * 2;
    auto As = [&](int p) { return lds + p * kTile * kTerms * 2; };
    const int64_t id = group_index();
    int32_t s, ct;
    int64_t m0;       // first output row: of R (dx), of the slot's N (dw)
    Segment seg;
    if constexpr (DW) {
        if (id >= a.tiles) return;
        const int64_t mt = id / a.c_tiles;
        ct = (int32_t)(id - mt * a.c_tiles);
        s = (int32_t)(mt / a.m_tiles);
        m0 = (mt - (int64_t)s * a.m_tiles) * kTile;
        seg = segment_of(a.offsets, s, a.R);
    } else {
        if (id >= a.tiles) {
            clear_rows(static_cast<T *>(a.out), a.C, a.offsets, a.n_slots, a.R, id - a.tiles, a.clears);
            return;
        }
        const int64_t index = id / a.c_tiles;
        ct = (int32_t)(id - index * a.c_tiles);
        int64_t before;
        const TileMap map(a.offsets, a.n_slots, a.R, kTile);
        if (index >= map.total) return;
        s = map.find(index, a.offsets, a.n_slots, a.R, kTile, seg, before);
        m0 = seg.begin + before * kTile;
    }
    const int c0 = ct * kCols, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int wm = (wave >> 1) * 64, wc = (wave & 1) * 32 * NB;
    // terms [k0, k1), and A's and B's rows of them
    const int64_t k_begin = DW ? seg.begin : 0, k_end = DW ? seg.end : a.N;
    const T *dy = static_cast<const T *>(a.dy);
    const int64_t b_row0 = DW ? 0 : (int64_t)s * a.N;
    int4_ pa[4][P];
    int4_ pb[NB / 2];
    uint32_t sb[NB / 2];
    auto fetch = [&](int64_t k0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DW) {
                const int64_t r = k0 + (t >> 4) + 16 * i;
                split8<T, P>(dy + (r < k_end ? r : 0) * a.stride, (int32_t)m0 + (t & 15) * 8, a.N, r < k_end, pa[i]);
            } else {
                const int64_t r = m0 + (t >> 3) + 32 * i;
                split8<T, P>(dy + (r < seg.end ? r : 0) * a.stride, (int32_t)k0 + (t & 7) * 8, a.N, r < seg.end, pa[i]);
            }
        }
        const int64_t k = k0 + (t >> 2);
#pragma unroll
        for (int i = 0; i < NB / 2; ++i) {
            const int block = ct * (kCols / 32) + (t & 3) + 4 * i;
            pb[i] = int4_{0, 0, 0, 0};
            sb[i] = 127;
            if (k < k_end && block < a.groups * 4) {
                const int64_t row = b_row0 + k;
                pb[i] = *reinterpret_cast<const int4_ *>(a.bc + row * a.groups * 64 + block * 16);
                sb[i] = a.bs[row * a.groups * 4 + block];
            }
        }
    };
    auto store = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                int at;
                if constexpr (DW) at = term_at<kTile>((t >> 4) + 16 * i, (t & 15) * 8);
                else at = ((t >> 3) + 32 * i) * 128 + (((t & 7) ^ ((t >> 4) & 7)) << 4);
                *reinterpret_cast<int4_ *>(As(p) + at) = pa[i][p];
            }
#pragma unroll
        for (int b = 0; b < NB / 2; ++b) {
            const float scale = scale_of(sb[b]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned w = (unsigned)pb[b][i];
                const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1),
                                     __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)};
                const int4_ x = {__builtin_bit_cast(int, v[0]), __builtin_bit_cast(int, v[1]), __builtin_bit_cast(int, v[2]),
                                 __builtin_bit_cast(int, v[3])};
                *reinterpret_cast<int4_ *>(Bs + term_at<kCols>(t >> 2, ((t & 3) + 4 * b) * 32 + i * 8)) = x;
            }
        }
    };
    float16_ sum[2][NB] = {};
    if (k_begin < k_end) fetch(k_begin);
    for (int64_t k0 = k_begin; k0 < k_end; k0 += kTerms) {
        store();
        __syncthreads();
        if (k0 + kTerms < k_end) fetch(k0 + kTerms);
#pragma unroll
        for (int k = 0; k < kTerms; k += 16) {
            bf16x8 b[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) b[n] = term_fragment<kCols>(Bs, k, wc + n * 32);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int p = P - 1; p >= 0; --p) {  // (the smallest parts first)
                    bf16x8 x;
                    if constexpr (DW) {
                        x = term_fragment<kTile>(As(p), k, wm + m * 32);
                    } else {
                        const int row = wm + m * 32 + (lane & 31), chunk = (k >> 3) + (lane >> 5);
                        x = *reinterpret_cast<const bf16x8 *>(As(p) + row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4));
                    }
#pragma unroll
                    for (int n = 0; n < NB; ++n) sum[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, b[n], sum[m][n], 0, 0, 0);
                }
        }
        __syncthreads();
    }
    // value (m, c) of a 32 x 32 tile: column lane % 32, row 8 (i / 4) + 4 (lane / 32) + i % 4
    T *out = static_cast<T *>(a.out);
    const int64_t m_end = DW ? a.N : seg.end, row0 = DW ? (int64_t)s * a.N : 0;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t r = m0 + wm + m * 32 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
                const int c = c0 + wc + n * 32 + (lane & 31);
                if (r < m_end && c < a.C) out[(row0 + r) * a.C + c] = (T)sum[m][n][i];
            }
}

}  // namespace rp

using namespace rp;

extern "C" int routepack_expert_product_backward(const routepack_matrix *dy, const routepack_mx *x,
                                                 const routepack_mx *w, int32_t n_slots, const int64_t *offsets,
                                                 const routepack_matrix *dx, const routepack_matrix *dw,
                                                 hipStream_t stream) {
    if (!dx && !dw) return ROUTEPACK_E_INVALID;
    RP_TRY(check_matrix(dy));
    RP_TRY(check_mx(x, dw != nullptr));
    RP_TRY(check_mx(w, dx != nullptr));
    if (n_slots < 1 || w->n_rows % n_slots != 0 || w->n_cols != x->n_cols) return ROUTEPACK_E_INVALID;
    const int64_t N = w->n_rows / n_slots, C = w->n_cols;
    if (dy->n_rows != x->n_rows || dy->n_cols != N) return ROUTEPACK_E_INVALID;
    if (n_slots > kMaxSlots || N > kMaxCols) return ROUTEPACK_E_UNSUPPORTED;
    if (dx) {
        RP_TRY(check_output(dx, x->n_rows, C));
        if (dx->type != dy->type) return ROUTEPACK_E_INVALID;
    }
    if (dw) {
        RP_TRY(check_output(dw, w->n_rows, C));
        if (dw->type != dy->type) return ROUTEPACK_E_INVALID;
    }
    const bool do_x = dx && dx->n_rows > 0 && C > 0, do_w = dw && dw->n_rows > 0 && C > 0;
    if (!do_x && !do_w) return ROUTEPACK_OK;
    if (!offsets || (do_x && !dx->data) || (do_w && !dw->data)) return ROUTEPACK_E_INVALID;
    if (!dy->data && dy->n_rows > 0 && N > 0) return ROUTEPACK_E_INVALID;
    BackProductArgs a = {};
    a.dy = dy->data;
    a.stride = dy->row_stride;
    a.groups = (int32_t)(padded_cols(C) / 128);
    a.N = (int32_t)N;
    a.C = (int32_t)C;
    a.n_slots = n_slots;
    a.R = x->n_rows;
    a.offsets = offsets;
    return by_type(dy->type, [&](auto tag) -> int {
        using T = decltype(tag);
        constexpr int NB = kParts<T> == 3 ? 2 : 4, lds = kParts<T> * kTile * kTerms * 2 + kTerms * NB * 64 * 2;
        a.c_tiles = (int32_t)((C + NB * 64 - 1) / (NB * 64));
        auto go = [&](auto kern, int64_t n, const BackProductArgs &b) -> int {
            if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(kern),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
                return ROUTEPACK_E_DEVICE;
            hipLaunchKernelGGL(kern, grid_of(n), dim3(256), lds, stream, b);
            return launched();
        };
        if (do_x) {
            BackProductArgs b = a;
            b.bc = static_cast<const uint8_t *>(w->codes);
            b.bs = static_cast<const uint8_t *>(w->scales);
            b.out = dx->data;
            // tiles of 128 rows: each slot may have one that is not full
            const int64_t slots = a.R < n_slots ? a.R : n_slots;
            b.tiles = (a.R / kTile + slots) * a.c_tiles;
            const int64_t pieces = (a.R * C + 65535) / 65536;
            b.clears = pieces < 256 ? pieces : 256;
            RP_TRY(go(k_product_back<T, false, NB>, b.tiles + b.clears, b));
        }
        if (do_w) {
            BackProductArgs b = a;
            b.bc = static_cast<const uint8_t *>(x->codes);
            b.bs = static_cast<const uint8_t *>(x->scales);
            b.out = dw->data;
            b.m_tiles = (int32_t)((N + kTile - 1) / kTile);
            b.tiles = (int64_t)n_slots * b.m_tiles * a.c_tiles;
            RP_TRY(go(k_product_back<T, true, NB>, b.tiles, b));
        }
        return ROUTEPACK_OK;
    });
}
