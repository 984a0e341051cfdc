// The gradients of the experts' products (rp_product.hip), on gfx950:
//   dx[r][c]    = sum_n dy[r][n] w[s][n][c]   for the rows r of slot s,
//   dw[s][n][c] = sum_r dy[r][n] x[r][c]      over the rows r of slot s.
// A 4-bit value times its power of two is exact in bf16, and dy is split into
// bf16 parts that add up to it (one for bf16, two for fp16, three for fp32), so
// bf16 matrix instructions form exact products and add them in 32 bits.  (bf16 ends
// at multiples of 2^-133, and parts of fp32 values below 2^-110 with it.)
//
// Both are the same tile program: A is dy, the output's rows by 64 terms; B is the
// matrix in 4 bits, 64 terms (its rows) by the output's columns, converted on the
// way into LDS.  The terms are B's rows, and A's too in dw: their fragments are
// read through the transposing LDS loads (16 lanes read 4 terms of 16 columns and
// each receives a column's 4 terms).
//
// 24558 rows, 60 x 1408 x 1984 bf16: dx 174 us, dw 207 (1.37e11 operations each,
// 110 us at a large bf16 product's rate).  Bound by LDS (77 and 88 us of its cycles,
// 57 and 59 of the matrix cores') and by the waits between its two phases.
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
    bool whole;                // out's rows are whole vectors of 16 bytes
    int64_t tiles, clears;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4_ __attribute__((ext_vector_type(4)));
typedef short short8_ __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kTerms = 64;

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

// 8 values of dy, in their own type.
template <class T> constexpr int kRaw = 8 * (int)sizeof(T) / 4;
template <class T>
__device__ inline void raw8(const char *at, uint32_t (&raw)[kRaw<T>]) {
#pragma unroll
    for (int i = 0; i < kRaw<T> / 4; ++i) {
        uint32_t w[4];
        load16<false>(at + 16 * i, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) raw[4 * i + j] = w[j];
    }
}
// Those of a row from `from` on, zeros from `end` > 0 on and where the row is not live.
template <class T>
__device__ inline void raw8_cut(const T *row, int32_t from, int32_t end, bool live, uint32_t (&raw)[kRaw<T>]) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool ok = live && from + i < end;
        b[i] = bits_of(row + (ok ? from + i : 0));
        b[i] = ok ? b[i] : 0;
    }
#pragma unroll
    for (int i = 0; i < kRaw<T>; ++i) raw[i] = sizeof(T) == 4 ? b[i] : b[2 * i % 8] | b[(2 * i + 1) % 8] << 16;
}

// 8 values of dy as P vectors of bf16 parts.
template <class T, int P>
__device__ inline void split8(const uint32_t (&raw)[kRaw<T>], int4_ (&part)[P]) {
    if constexpr (P == 1) {
        part[0] = int4_{(int)raw[0], (int)raw[1], (int)raw[2], (int)raw[3]};
        return;
    }
    constexpr int W = Vec<T>::W;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8 / W; ++i) {
        Vec<T> x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x.w[j] = raw[4 * i + j];
#pragma unroll
        for (int j = 0; j < W; ++j) v[i * W + j] = x.at(j);
    }
    // (all finite: no test a value; what is left of an infinity or NaN is NaN)
    float left[8], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        left[i] = v[i] - __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u);
        sum += left[i];
    }
    if (P > 1 && sum == sum) {
        auto top = [](float a, float b) {  // the upper halves, b's above a's
            return (int)__builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            part[0][i] = top(v[2 * i], v[2 * i + 1]);
            part[P > 1 ? 1 : 0][i] = top(left[2 * i], left[2 * i + 1]);
            if (P > 2) {
                const float a = left[2 * i], b = left[2 * i + 1];
                part[P - 1][i] = top(a - __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), b - __uint_as_float(__float_as_uint(b) & 0xFFFF0000u));
            }
        }
        return;
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

// Tiles of 64 MB rows by 32 NB WN columns: 2 x WN waves of MB x NB matrix tiles.
// A wave's blocks of 32 rows alternate with the other row of waves', and the
// upper half of them is left out where it is empty.  One stage of LDS, filled
// between two barriers: two or three workgroups a CU (WAVES a SIMD) cover each
// other's phases (24558 rows, 60 x 1408 x 1984, both gradients: 465 us when this
// was chosen, 517 with two stages, one barrier and one workgroup a CU).
template <class T, int WN, int MB, int NB>
struct BackShape {
    static constexpr int P = kParts<T>, kThreads = 128 * WN, kRows = 64 * MB, kCols = 32 * NB * WN;
    static constexpr int kA = kRows * kTerms * 2, kB = kTerms * kCols * 2, kStage = P * kA + kB;
    static constexpr int kLeave = 2 * WN * 32 * kPitch<T, NB>;
    static constexpr int kLds = kStage > kLeave ? kStage : kLeave;
    // pieces of 8 values of A, and blocks of B, that a thread fetches
    static constexpr int kPieces = kRows * kTerms / 8 / kThreads, kBlocks = kTerms * kCols / 32 / kThreads;
};

template <class T, bool DW, int WN, int MB, int NB>
__device__ __forceinline__ void back_tile(const BackProductArgs &a, int64_t id, char *lds) {
    using G = BackShape<T, WN, MB, NB>;
    constexpr int P = G::P, kRows = G::kRows, kCols = G::kCols;
    int32_t s, ct;
    int64_t m0;       // first output row: of R (dx), of the slot's N (dw)
    Segment seg;
    if constexpr (DW) {
        if (id >= a.tiles) return;
        const int64_t mt = id / a.c_tiles;
        ct = (int32_t)(id - mt * a.c_tiles);
        s = (int32_t)(mt / a.m_tiles);
        m0 = (mt - (int64_t)s * a.m_tiles) * kRows;
        seg = segment_of(a.offsets, s, a.R);
    } else {
        if (id >= a.tiles) {
            clear_rows(static_cast<T *>(a.out), a.C, a.offsets, a.n_slots, a.R, id - a.tiles, a.clears);
            return;
        }
        int64_t before;
        const TileMap map(a.offsets, a.n_slots, a.R, kRows);
        // (workgroups go to the eight XCDs in turn: each XCD gets a run of adjacent tiles)
        const int64_t all = map.total * a.c_tiles, run = (all + 7) / 8, index = (id & 7) * run + (id >> 3);
        if ((id >> 3) >= run || index >= all) return;
        const int64_t tile = index / a.c_tiles;
        ct = (int32_t)(index - tile * a.c_tiles);
        s = map.find(tile, a.offsets, a.n_slots, a.R, kRows, seg, before);
        m0 = seg.begin + before * kRows;
    }
    const int c0 = ct * kCols, t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave / WN, wc = (wave % WN) * 32 * NB;
    const int64_t m_end = DW ? a.N : seg.end;
    const int rows = m_end - m0 < kRows ? (int)(m_end - m0) : kRows;
    // terms [k_begin, k_end), and A's and B's rows of them
    const int64_t k_begin = DW ? seg.begin : 0, k_end = DW ? seg.end : a.N;
    const T *dy = static_cast<const T *>(a.dy);
    const int64_t b_row0 = DW ? 0 : (int64_t)s * a.N;
    // The tile's A: pieces of 8 values, of a row's 64 terms (dx) or of a term's
    // kRows columns (dw); B: blocks of 32 columns, kCols / 32 a term (16 lanes write
    // 4 of 4 terms each to LDS, in different banks).
    constexpr int kAcross = DW ? kRows / 8 : kTerms / 8, kBlocksAcross = kCols / 32;
    constexpr int kAStep = G::kThreads / kAcross, kBStep = G::kThreads / kBlocksAcross;
    const int a_row = t / kAcross, a_piece = t % kAcross;
    const int b_row = ((t >> 2) & 3) + 4 * (t / (4 * kBlocksAcross)), b_block = (t & 3) + 4 * ((t >> 4) % (kBlocksAcross / 4));
    // What a thread fetches stands at fixed distances from a step's first term, in 32
    // bits (rows and pieces past the output's end are its last ones again: nothing of
    // them is kept).  Elsewhere (N ends inside a piece, far rows) values go one by one.
    const bool near = a.stride <= 1 << 22 && (!DW || a.N % 8 == 0 || m0 + kRows <= a.N);
    const int a_col = DW && m0 + a_piece * 8 > a.N - 8 ? a.N - 8 : (DW ? (int)m0 : 0) + a_piece * 8;
    const uint32_t code_row = (uint32_t)a.groups * 64, scale_row = (uint32_t)a.groups * 4;
    const int block = ct * kBlocksAcross + b_block < a.groups * 4 ? ct * kBlocksAcross + b_block : a.groups * 4 - 1;
    uint32_t a_at[G::kPieces];
#pragma unroll
    for (int i = 0; i < G::kPieces; ++i) {
        const int row = a_row + i * kAStep, r = DW || row < rows ? row : rows - 1;
        a_at[i] = (uint32_t)((r * a.stride + a_col) * (int)sizeof(T));
    }
    uint32_t raw[G::kPieces][kRaw<T>];
    int4_ pb[G::kBlocks];
    uint32_t sb[G::kBlocks];
    auto fetch = [&](int64_t k0) __attribute__((always_inline)) {
        const int last = k_end - k0 < kTerms ? (int)(k_end - k0) - 1 : kTerms - 1;  // (term)
        const T *first = dy + (DW ? k0 * a.stride : m0 * a.stride + k0);
        const uint8_t *codes = a.bc + (b_row0 + k0) * code_row, *scales = a.bs + (b_row0 + k0) * scale_row;
        if (near && last == kTerms - 1) {
#pragma unroll
            for (int i = 0; i < G::kPieces; ++i) raw8<T>(reinterpret_cast<const char *>(first) + a_at[i], raw[i]);
        } else if (near && (DW || a.N % 8 == 0)) {
#pragma unroll
            for (int i = 0; i < G::kPieces; ++i) {
                const int row = a_row + i * kAStep;
                const bool ok = DW ? row <= last : a_piece * 8 <= last;
                const uint32_t to = DW ? (uint32_t)((last * a.stride + a_col) * (int)sizeof(T)) : a_at[i] - a_piece * 8 * (int)sizeof(T);
                raw8<T>(reinterpret_cast<const char *>(first) + (ok ? a_at[i] : to), raw[i]);
#pragma unroll
                for (int j = 0; j < kRaw<T>; ++j) raw[i][j] = ok ? raw[i][j] : 0;
            }
        } else {
#pragma unroll
            for (int i = 0; i < G::kPieces; ++i) {
                const int64_t r = (DW ? k0 : m0) + a_row + i * kAStep, end = DW ? k_end : m_end;
                raw8_cut<T>(dy + (r < end ? r : end - 1) * a.stride, (int32_t)(DW ? m0 : k0) + a_piece * 8, a.N, r < end, raw[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < G::kBlocks; ++i) {
            const int row = b_row + i * kBStep, k = row < last ? row : last;
            pb[i] = *reinterpret_cast<const int4_ *>(codes + (k * code_row + block * 16));
            sb[i] = scales[k * scale_row + block];
            if (row > last) {
                pb[i] = int4_{0, 0, 0, 0};
                sb[i] = 127;
            }
        }
    };
    auto store = [&](char *stage) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < G::kPieces; ++i) {
            int4_ part[P];
            split8<T, P>(raw[i], part);
            const int row = a_row + i * kAStep;
            int at;
            if constexpr (DW) at = term_at<kRows>(row, a_piece * 8);
            else at = row * 128 + ((a_piece ^ ((row >> 1) & 7)) << 4);
#pragma unroll
            for (int p = 0; p < P; ++p) *reinterpret_cast<int4_ *>(stage + p * G::kA + at) = part[p];
        }
        char *const to = stage + P * G::kA;
#pragma unroll
        for (int b = 0; b < G::kBlocks; ++b) {
            const float scale = scale_of(sb[b]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned w = (unsigned)pb[b][i];
                const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1),
                                     __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)};
                const int4_ x = {__builtin_bit_cast(int, v[0]), __builtin_bit_cast(int, v[1]), __builtin_bit_cast(int, v[2]),
                                 __builtin_bit_cast(int, v[3])};
                *reinterpret_cast<int4_ *>(to + term_at<kCols>(b_row + b * kBStep, b_block * 32 + i * 8)) = x;
            }
        }
    };
    T *out = static_cast<T *>(a.out) + ((DW ? (int64_t)s * a.N : 0) + m0) * a.C;
    auto run = [&](auto live_) __attribute__((always_inline)) {
        constexpr int kLive = decltype(live_)::value;
        float16_ sum[kLive ? kLive : 1][NB] = {};
        auto multiply = [&](const char *stage, int k) __attribute__((always_inline)) {
            bf16x8 b[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) b[n] = term_fragment<kCols>(stage + P * G::kA, k, wc + n * 32);
#pragma unroll
            for (int m = 0; m < kLive; ++m)
#pragma unroll
                for (int p = P - 1; p >= 0; --p) {  // (the smallest parts first)
                    const int first = (2 * m + wm) * 32;
                    bf16x8 x;
                    if constexpr (DW) {
                        x = term_fragment<kRows>(stage + p * G::kA, k, first);
                    } else {
                        const int row = first + (lane & 31), piece = (k >> 3) + (lane >> 5);
                        x = *reinterpret_cast<const bf16x8 *>(stage + p * G::kA + row * 128 + ((piece ^ ((row >> 1) & 7)) << 4));
                    }
#pragma unroll
                    for (int n = 0; n < NB; ++n) sum[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[n], x, sum[m][n], 0, 0, 0);
                }
        };
        for (int64_t k0 = k_begin;; k0 += kTerms) {  // (fetches what follows what is multiplied)
            if (k0 < k_end) fetch(k0);
            if (kLive && k0 > k_begin) {
#pragma unroll
                for (int k = 0; k < kTerms; k += 16) multiply(lds, k);
            }
            __syncthreads();
            if (k0 >= k_end) break;
            store(lds);
            __syncthreads();
        }
#pragma unroll
        for (int m = 0; m < kLive; ++m) {
            const int first = (2 * m + wm) * 32;
            leave_by_lines<T, NB>(lds + wave * 32 * kPitch<T, NB>, sum[m], out + first * (int64_t)a.C, a.C, rows - first, a.C, c0 + wc, a.whole);
        }
    };
    const int blocks = (rows + 31) / 32, live = c0 + wc < a.C ? (blocks - wm + 1) / 2 : 0;
    if (live > MB / 2) run(Int<MB>());
    else if (live > 0) run(Int<MB / 2>());
    else run(Int<0>());
}

template <class T, bool DW, int WN, int MB, int NB, int WAVES>
__global__ void __launch_bounds__(128 * WN, WAVES) k_product_back(BackProductArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    back_tile<T, DW, WN, MB, NB>(a, group_index(), lds);
}

// Both gradients of a small problem in one launch (100 tokens x 8, 64 x 512 x 512
// bf16: 13.2 us for both; 10.7 and 10.4 in launches of their own).
template <class T, int WN, int MB, int NB, int WAVES>
__global__ void __launch_bounds__(128 * WN, WAVES) k_product_back_both(BackProductArgs x, BackProductArgs w) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int64_t id = group_index(), n = x.tiles + x.clears;
    if (id < n) back_tile<T, false, WN, MB, NB>(x, id, lds);
    else back_tile<T, true, WN, MB, NB>(w, id - n, lds);
}

// The tiles of a gradient.
template <class G, bool DW>
void cut(BackProductArgs &a) {
    a.c_tiles = (a.C + G::kCols - 1) / G::kCols;
    if (DW) {
        a.m_tiles = (a.N + G::kRows - 1) / G::kRows;
        a.tiles = (int64_t)a.n_slots * a.m_tiles * a.c_tiles;
        a.clears = 0;
    } else {
        // each slot may have a tile that is not full; eight runs of equal length
        const int64_t slots = a.R < a.n_slots ? a.R : a.n_slots, pieces = (a.R * a.C + 65535) / 65536;
        a.tiles = ((a.R / G::kRows + slots) * a.c_tiles + 7) / 8 * 8;
        a.clears = pieces < 256 ? pieces : 256;
    }
}

template <class G, class Kernel, class... Args>
int launch_back(Kernel kern, int64_t groups, hipStream_t stream, const Args &...args) {
    if (G::kLds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(kern),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds) != hipSuccess)
        return ROUTEPACK_E_DEVICE;
    hipLaunchKernelGGL(kern, grid_of(groups), dim3(G::kThreads), G::kLds, stream, args...);
    return launched();
}

// Tiles of 128 x 256 where they fill the chip: with parts to multiply on four waves
// of 64 x 128, which read least of LDS (24558 rows, 60 x 1408 x 1984 fp16: dx 396 us
// by eight waves of 64 x 64, 311; dw 384 by tiles of 128 x 128, 341), dx of bf16 on
// eight of 64 x 64, which wait less (194 us, 209 on four).  Else tiles of 128 x 128,
// more of them at a time: for dw, whose sums are short, up to several rounds of the
// chip, and always with bf16 (those rows: 220 us either way; 60000 rows, 128 x 256 x
// 256: 59 us, 85 by the wide ones).  The wide kernels with parts hold all 256
// registers; dw spills 26 (fp16) and 21 (fp32) to scratch, dx one (fp32).
template <class T>
int back_of(BackProductArgs *x, BackProductArgs *w, hipStream_t stream) {
    constexpr int kWaves = kParts<T> == 1 ? 3 : 2;
    using Small = BackShape<T, 2, 2, 2>;
    using Wide = BackShape<T, 2, 2, 4>;
    const BackProductArgs &any = x ? *x : *w;
    const int64_t across = (any.C + 255) / 256, slots = any.R < any.n_slots ? any.R : any.n_slots;
    const bool wide_x = x && any.C > 128 && (any.R / 128 + slots / 2) * across >= 256;
    if (wide_x) {
        if constexpr (kParts<T> == 1) {
            using Eight = BackShape<T, 4, 2, 2>;
            cut<Eight, false>(*x);
            RP_TRY(launch_back<Eight>(k_product_back<T, false, 4, 2, 2, 4>, x->tiles + x->clears, stream, *x));
        } else {
            cut<Wide, false>(*x);
            RP_TRY(launch_back<Wide>(k_product_back<T, false, 2, 2, 4, 2>, x->tiles + x->clears, stream, *x));
        }
    } else if (x) {
        cut<Small, false>(*x);
        const int64_t n = x->tiles + x->clears;
        if (w) {
            cut<Small, true>(*w);
            return launch_back<Small>(k_product_back_both<T, 2, 2, 2, kWaves>, n + w->tiles, stream, *x, *w);
        }
        return launch_back<Small>(k_product_back<T, false, 2, 2, 2, kWaves>, n, stream, *x);
    }
    if constexpr (kParts<T> > 1) {
        if (w && any.C > 128 && (any.N + 127) / 128 * any.n_slots * across >= 4096) {
            cut<Wide, true>(*w);
            return launch_back<Wide>(k_product_back<T, true, 2, 2, 4, 2>, w->tiles, stream, *w);
        }
    }
    if (w) {
        cut<Small, true>(*w);
        return launch_back<Small>(k_product_back<T, true, 2, 2, 2, kWaves>, w->tiles, stream, *w);
    }
    return ROUTEPACK_OK;
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
        BackProductArgs bx = a, bw = a;
        if (do_x) {
            bx.bc = static_cast<const uint8_t *>(w->codes);
            bx.bs = static_cast<const uint8_t *>(w->scales);
            bx.out = dx->data;
            bx.whole = C % (16 / sizeof(T)) == 0 && ((uintptr_t)dx->data & 15) == 0;
        }
        if (do_w) {
            bw.bc = static_cast<const uint8_t *>(x->codes);
            bw.bs = static_cast<const uint8_t *>(x->scales);
            bw.out = dw->data;
            bw.whole = C % (16 / sizeof(T)) == 0 && ((uintptr_t)dw->data & 15) == 0;
        }
        return back_of<T>(do_x ? &bx : nullptr, do_w ? &bw : nullptr, stream);
    });
}
