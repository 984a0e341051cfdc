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

// Many rows a slot: tiles of TM rows by TN of N, four waves of MT x NT matrix
// tiles of 32 x 32, 128 columns (64 bytes a row) a step.
//
// The codes go from memory to LDS without passing registers, S - 1 steps ahead;
// a row's four pieces of 16 bytes are exchanged by the row (the sources are, as
// a wave's 64 pieces land one after the other), so that the 32 rows of a fragment
// stand in different banks.  The scales of kUnit steps are loaded together and
// turned in LDS to a word a row and step.
constexpr int kUnit = 2;  // steps whose scales are loaded together

template <int WM, int WN, int MT, int NT, int S>
struct Shape {
    static constexpr int TM = WM * MT * 32, TN = WN * NT * 32, kRows = TM + TN;
    static constexpr int kStage = kRows * 64, kLds = S * kStage + 2 * kUnit * kRows * 4;
    static constexpr int kLoads = kRows / 64;  // a wave's loads of 1 KiB a step
    static_assert(kRows % 64 == 0 && TM % 16 == 0, "whole loads");
};

__device__ inline uint32_t lds_address(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
}

// 64 lanes' 16 bytes at base + offset to LDS, one after the other from `to` on.
// The compiler knows nothing of the load in flight: whoever reads what it brings
// waits by wait_and_meet.
__device__ inline void load_to_lds(const uint8_t *base, uint32_t offset, uint32_t to) {
    uint32_t m0;  // (the compiler's, given back)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(to), "v"(offset), "s"(base) : "memory");
}

// All but this wave's last N loads have ended, and its LDS accesses; then the
// workgroup's barrier.
template <int N>
__device__ inline void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// A wave's LDS accesses before are done before those after.
__device__ inline void wave_meet() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// 16 bytes of values from column c on, as many as the row has.
template <class T>
__device__ inline void store_cols(T *row, int32_t cols, int32_t c, int4_ v) {
    constexpr int W = 16 / (int)sizeof(T);
    typedef int four __attribute__((ext_vector_type(4), aligned(2)));
    if (c + W <= cols) {
        *reinterpret_cast<four *>(row + c) = v;
    } else {
        typedef T values __attribute__((ext_vector_type(W)));
        const values x = __builtin_bit_cast(values, v);
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (c + i < cols) row[c + i] = x[i];
    }
}

template <class T, int WM, int WN, int MT, int NT, int S>
__global__ void __launch_bounds__(256, 2) k_product_many(ProductArgs a) {
    using G = Shape<WM, WN, MT, NT, S>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int64_t id = group_index();
    if (id >= a.tiles) {
        clear_rows(static_cast<T *>(a.y), a.N, a.offsets, a.n_slots, a.R, id - a.tiles, a.clears);
        return;
    }
    // Workgroups go to the eight XCDs in turn: each XCD gets a run of adjacent
    // tiles, the row tiles of a slot's piece of N next to each other.
    int64_t before, total;
    slot_of_tile<false>(a.offsets, a.n_slots, a.R, G::TM, INT64_MAX, before, total);
    const int64_t all = total * a.n_tiles, run = (all + 7) / 8, index = (id & 7) * run + (id >> 3);
    if ((id >> 3) >= run || index >= all) return;
    // (a slot's tiles: its row tiles times n_tiles)
    const int32_t s = slot_of_tile<false>(a.offsets, a.n_slots, a.R, G::TM, index / a.n_tiles, before, total);
    if (s < 0) return;
    const Segment seg = segment_of(a.offsets, s, a.R);
    const int64_t m_tiles = (seg.end - seg.begin + G::TM - 1) / G::TM;
    // index - (the slot's first) = before * n_tiles + index % n_tiles
    const int64_t within = before * a.n_tiles + index % a.n_tiles;
    const int32_t nt = (int32_t)(within / m_tiles), mt = (int32_t)(within - nt * m_tiles);
    const int64_t r0 = seg.begin + (int64_t)mt * G::TM;
    const int32_t n0 = nt * G::TN;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t code_row = (int64_t)a.groups * 64, scale_row = (int64_t)a.groups * 4;
    // tile row i: x row r0 + i, then w row n0 + (i - TM); past the ends the last one again
    auto x_row = [&](int i) { return r0 + i < seg.end ? i : (int)(seg.end - 1 - r0); };
    auto w_row = [&](int i) { return n0 + i < a.N ? i : a.N - 1 - n0; };
    const uint8_t *xbase = a.xc + r0 * code_row, *wbase = a.wc + ((int64_t)s * a.N + n0) * code_row;
    uint32_t from[G::kLoads];
#pragma unroll
    for (int i = 0; i < G::kLoads; ++i) {
        const int row = ((wave + 4 * i) * 16) + (lane >> 2), piece = (lane & 3) ^ ((row >> 1) & 3);
        const int real = row < G::TM ? x_row(row) : w_row(row - G::TM);
        from[i] = (uint32_t)(real * code_row + piece * 16);
    }
    const uint32_t lds0 = lds_address(lds);
    const int32_t steps = a.groups;
    auto issue = [&](int32_t step) {
        const uint32_t to = lds0 + (uint32_t)(step % S) * G::kStage;
#pragma unroll
        for (int i = 0; i < G::kLoads; ++i) {
            const int load = wave + 4 * i;
            const uint8_t *base = (load * 16 < G::TM ? xbase : wbase) + (int64_t)step * 64;
            load_to_lds(base, from[i], to + load * 1024);
        }
    };
    // scales: a row's word of each step of a unit
    constexpr int kMine = (G::kRows + 255) / 256;
    uint32_t *turned = reinterpret_cast<uint32_t *>(lds + S * G::kStage);
    uint32_t sc[kMine][kUnit];
    auto fetch_scales = [&](int32_t unit) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int row = t + 256 * i;
            if (row >= G::kRows) continue;
            const uint8_t *p = row < G::TM ? a.xs + (r0 + x_row(row)) * scale_row
                                           : a.ws + ((int64_t)s * a.N + n0 + w_row(row - G::TM)) * scale_row;
            typedef uint32_t words __attribute__((ext_vector_type(kUnit), aligned(4)));
            const uint32_t *w = reinterpret_cast<const uint32_t *>(p) + unit * kUnit;
            if ((unit + 1) * kUnit <= steps) {
                const words v = *reinterpret_cast<const words *>(w);
#pragma unroll
                for (int k = 0; k < kUnit; ++k) sc[i][k] = v[k];
            } else {
#pragma unroll
                for (int k = 0; k < kUnit; ++k) sc[i][k] = unit * kUnit + k < steps ? w[k] : 0;
            }
        }
    };
    auto store_scales = [&](int32_t unit) {
        uint32_t *to = turned + (unit & 1) * kUnit * G::kRows;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int row = t + 256 * i;
            if (row >= G::kRows) continue;
#pragma unroll
            for (int k = 0; k < kUnit; ++k) to[k * G::kRows + row] = sc[i][k];
        }
    };
    const int wm = (wave / WN) * MT * 32, wn = G::TM + (wave % WN) * NT * 32, half = lane >> 5, r32 = lane & 31;
    float16_ sum[MT][NT] = {};
    fetch_scales(0);
#pragma unroll
    for (int i = 0; i < S - 1; ++i)
        if (i < steps) issue(i);
    store_scales(0);
    for (int32_t step = 0; step < steps; ++step) {
        // (this step's loads: the oldest of those in flight)
        if (step + S - 2 < steps) wait_and_meet<(S - 2) * G::kLoads>();
        else wait_and_meet<0>();
        if (step + S - 1 < steps) issue(step + S - 1);
        const int32_t unit = step / kUnit;
        if (step % kUnit == 0 && (unit + 1) * kUnit < steps) fetch_scales(unit + 1);
        const char *tile = lds + (step % S) * G::kStage;
        const uint32_t *scale = turned + ((unit & 1) * kUnit + step % kUnit) * G::kRows + r32;
        uint32_t xs[MT], ws[NT];
#pragma unroll
        for (int m = 0; m < MT; ++m) xs[m] = scale[wm + m * 32] >> (8 * half);
#pragma unroll
        for (int n = 0; n < NT; ++n) ws[n] = scale[wn + n * 32] >> (8 * half);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            auto fragment = [&](int first) {
                const int row = first + r32, piece = (2 * k + half) ^ ((row >> 1) & 3);
                const int4_ v = *reinterpret_cast<const int4_ *>(tile + row * 64 + piece * 16);
                return int8_{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
            };
            int8_ x[MT], w[NT];
#pragma unroll
            for (int m = 0; m < MT; ++m) x[m] = fragment(wm + m * 32);
#pragma unroll
            for (int n = 0; n < NT; ++n) w[n] = fragment(wn + n * 32);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (k == 0)
                        sum[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[n], x[m], sum[m][n], 4, 4, 0, (int)ws[n], 0, (int)xs[m]);
                    else
                        sum[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[n], x[m], sum[m][n], 4, 4, 2, (int)ws[n], 2, (int)xs[m]);
                }
        }
        if (step % kUnit == kUnit - 1 && step + 1 < steps) store_scales(unit + 1);
    }
    // A value's row is lane % 32 of x, its column 8 (i / 4) + 4 (lane / 32) + i % 4
    // of w: 32 rows at a time go through this wave's part of LDS, to leave as
    // whole lines.
    wait_and_meet<0>();
    constexpr int kCols = NT * 32, kPitch = kCols * (int)sizeof(T) + 16, kVec = 16 / (int)sizeof(T);
    constexpr int kLanes = kCols / kVec, kRowsAtOnce = kWave / kLanes;
    static_assert(4 * 32 * kPitch <= G::kLds, "the waves' parts fit");
    char *mine = lds + wave * 32 * kPitch;
    T *y = static_cast<T *>(a.y);
    const int32_t c0 = n0 + wn - G::TM;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                typedef T four __attribute__((ext_vector_type(4)));
                const four v = {(T)sum[m][n][4 * g], (T)sum[m][n][4 * g + 1], (T)sum[m][n][4 * g + 2], (T)sum[m][n][4 * g + 3]};
                *reinterpret_cast<four *>(mine + r32 * kPitch + (n * 32 + 8 * g + 4 * half) * sizeof(T)) = v;
            }
        wave_meet();
#pragma unroll
        for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
            const int row = i * kRowsAtOnce + lane / kLanes, c = (lane % kLanes) * kVec;
            const int4_ v = *reinterpret_cast<const int4_ *>(mine + row * kPitch + c * sizeof(T));
            const int64_t r = r0 + wm + m * 32 + row;
            if (r < seg.end) store_cols<T>(y + r * a.N, a.N, c0 + c, v);
        }
        wave_meet();
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
    const int64_t most = a.R < n_slots ? a.R : n_slots;  // slots with rows
    const int64_t pieces = (a.R * N + 65535) / 65536;
    a.clears = pieces < 256 ? pieces : 256;
    return by_type(y->type, [&](auto tag) -> int {
        using T = decltype(tag);
        if (a.R >= 32 * (int64_t)n_slots) {
            using G = Shape<2, 2, 2, 4, 3>;
            const auto kern = k_product_many<T, 2, 2, 2, 4, 3>;
            a.n_tiles = (int32_t)((N + G::TN - 1) / G::TN);
            // (each slot may have a tile that is not full; eight runs of equal length)
            a.tiles = ((a.R / G::TM + most) * a.n_tiles + 7) / 8 * 8;
            if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                    G::kLds) != hipSuccess)
                return ROUTEPACK_E_DEVICE;
            hipLaunchKernelGGL(kern, grid_of(a.tiles + a.clears), dim3(256), G::kLds, stream, a);
            return launched();
        }
        a.n_tiles = (int32_t)((N + 15) / 16);
        a.tiles = most * a.n_tiles;
        hipLaunchKernelGGL((k_product_few<T, 2>), grid_of(a.tiles + a.clears), dim3(256), 0, stream, a);
        return launched();
    });
}
