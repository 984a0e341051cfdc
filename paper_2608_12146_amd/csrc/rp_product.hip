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
    bool whole;       // y's rows are whole vectors of 16 bytes
    int64_t tiles;    // workgroups of tiles; those behind clear rows
    int64_t clears;
};

// Few rows a slot: a wave holds 16 of a slot's N, a workgroup 64, and passes over
// the slot's rows, 16 RB at a time.  A lane loads 16 bytes of a row of w and of x
// for each 128 columns, the scales of 512 columns at once.
// Bound by the weights' bytes: each is read once a pass (512 rows, 256 x 2048 x
// 2048: 89 us).
template <class T, int RB>
__global__ void __launch_bounds__(256) k_product_few(ProductArgs a) {
    const int64_t id = group_index();
    if (id >= a.tiles) {
        clear_rows(static_cast<T *>(a.y), a.N, a.offsets, a.n_slots, a.R, id - a.tiles, a.clears);
        return;
    }
    const int64_t index = id / a.n_tiles;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, i16 = lane & 15;
    const int32_t n0 = (int32_t)(id - index * a.n_tiles) * 64 + wave * 16;
    const TileMap map(a.offsets, a.n_slots, a.R, 0);
    if (index >= map.total || n0 >= a.N) return;
    Segment seg;
    int64_t before;
    const int32_t s = map.find(index, a.offsets, a.n_slots, a.R, 0, seg, before);
    const int32_t n = n0 + i16 < a.N ? n0 + i16 : a.N - 1;
    const int64_t row = (int64_t)s * a.N + n;
    const uint8_t *wc = a.wc + row * a.groups * 64 + q * 16;
    const uint32_t *ws = reinterpret_cast<const uint32_t *>(a.ws + row * a.groups * 4);
    for (int64_t r0 = seg.begin; r0 < seg.end; r0 += 16 * RB) {
        const uint8_t *xc[RB];
        const uint32_t *xs[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int64_t r = r0 + b * 16 + i16, x = r < seg.end ? r : seg.end - 1;
            xc[b] = a.xc + x * a.groups * 64 + q * 16;
            xs[b] = reinterpret_cast<const uint32_t *>(a.xs + x * a.groups * 4);
        }
        float4_ sum[RB] = {};
        // N groups of 128 columns from g on
        auto some = [&](int32_t g, auto n_) __attribute__((always_inline)) {
            constexpr int M = decltype(n_)::value;
            typedef uint32_t words __attribute__((ext_vector_type(M), aligned(4)));
            int4_ w[M], x[RB][M];
            uint32_t wscale[M], xscale[RB][M];
#pragma unroll
            for (int i = 0; i < M; ++i) w[i] = *reinterpret_cast<const int4_ *>(wc + (int64_t)(g + i) * 64);
            const words v = *reinterpret_cast<const words *>(ws + g);
#pragma unroll
            for (int i = 0; i < M; ++i) wscale[i] = v[i];
#pragma unroll
            for (int b = 0; b < RB; ++b) {
#pragma unroll
                for (int i = 0; i < M; ++i) x[b][i] = *reinterpret_cast<const int4_ *>(xc[b] + (int64_t)(g + i) * 64);
                const words u = *reinterpret_cast<const words *>(xs[b] + g);
#pragma unroll
                for (int i = 0; i < M; ++i) xscale[b][i] = u[i];
            }
#pragma unroll
            for (int i = 0; i < M; ++i)
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    const int8_ wa = {w[i][0], w[i][1], w[i][2], w[i][3], 0, 0, 0, 0};
                    const int8_ xb = {x[b][i][0], x[b][i][1], x[b][i][2], x[b][i][3], 0, 0, 0, 0};
                    sum[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, xb, sum[b], 4, 4, 0, (int)(wscale[i] >> (8 * q)), 0,
                                                                              (int)(xscale[b][i] >> (8 * q)));
                }
        };
        int32_t g = 0;
        for (; g + 4 <= a.groups; g += 4) some(g, Int<4>());
        for (; g < a.groups; ++g) some(g, Int<1>());
        // a value's row is lane % 16, its column 4 (lane / 16) + i
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int64_t r = r0 + b * 16 + i16;
            if (r >= seg.end) continue;
            T *y = static_cast<T *>(a.y) + r * a.N + n0 + q * 4;
            typedef T four __attribute__((ext_vector_type(4), aligned(2)));
            const four v = {(T)sum[b][0], (T)sum[b][1], (T)sum[b][2], (T)sum[b][3]};
            if (n0 + q * 4 + 4 <= a.N) {
                *reinterpret_cast<four *>(y) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n0 + q * 4 + i < a.N) y[i] = v[i];
            }
        }
    }
}

// Many rows a slot: tiles of 256 rows by 256 of N, eight waves of 4 x 2 matrix
// tiles of 32 x 32, 256 columns (128 bytes a row) a step.
//
// A wave's blocks of 32 rows alternate with its neighbour's, and blocks that
// the slot's rows leave empty are not multiplied: a part-filled tile costs both
// waves of a SIMD alike, in steps of 32 rows (2).
// The codes go from memory to LDS without passing registers, a step ahead; a
// row's eight pieces of 16 bytes are exchanged by the row (the sources are, as a
// wave's 64 pieces land one after the other), so that the 32 rows of a fragment
// stand in different banks.  The scales of two steps are loaded together and
// turned in LDS to words by row.
// Bound by the loads where a slot has few tiles of rows (65536 rows, 256 x 2048 x
// 2048: 237 us, 227 for the loads alone), else by the phases between them and the
// matrix instructions (65536 rows, 8 x 4096 x 4096: 640 us, 3.4 PFLOP/s; the
// instructions alone, on registers, reach 7.0).
constexpr int kTileRows = 256, kTileCols = 256, kBoth = kTileRows + kTileCols;
constexpr int kStage = kBoth * 128, kWords = 4;  // of scales, two steps
constexpr int kManyLds = 2 * kStage + 2 * kWords * kBoth * 4;

__device__ inline uint32_t lds_address(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
}

// 64 lanes' 16 bytes at base + offset to LDS, one after the other from `to` on.
// The compiler knows nothing of the load in flight: whoever reads what it brings
// waits by wait_and_meet.
__device__ inline void load_to_lds(const uint8_t *base, uint32_t offset, uint32_t to) {
    base = reinterpret_cast<const uint8_t *>(uniform64((int64_t)base));
    to = (uint32_t)__builtin_amdgcn_readfirstlane((int)to);
    uint32_t m0;  // (the compiler's, given back)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(to), "v"(offset), "s"(base) : "memory");
}

// All of this wave's loads have ended, and its LDS accesses; then the
// workgroup's barrier.
__device__ inline void wait_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <class T>
__global__ void __launch_bounds__(512, 1) k_product_many(ProductArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int64_t id = group_index();
    if (id >= a.tiles) {
        clear_rows(static_cast<T *>(a.y), a.N, a.offsets, a.n_slots, a.R, id - a.tiles, a.clears);
        return;
    }
    // Workgroups go to the eight XCDs in turn: each XCD gets a run of adjacent
    // tiles, and within a slot four tiles of N next to each other for each of its
    // row tiles, so that those at work together share both operands.
    const TileMap map(a.offsets, a.n_slots, a.R, kTileRows);
    const int64_t all = map.total * a.n_tiles, run = (all + 7) / 8, index = (id & 7) * run + (id >> 3);
    if ((id >> 3) >= run || index >= all) return;
    Segment seg;
    int64_t before;
    const int32_t s = map.find(index / a.n_tiles, a.offsets, a.n_slots, a.R, kTileRows, seg, before);
    const int64_t m_tiles = (seg.end - seg.begin + kTileRows - 1) / kTileRows;
    const int64_t within = before * a.n_tiles + index % a.n_tiles;  // index less the slot's first
    const int32_t group = (int32_t)(within / (m_tiles * 4)), n_left = a.n_tiles - group * 4;
    const int32_t rest = (int32_t)(within - group * (m_tiles * 4)), n_here = n_left < 4 ? n_left : 4;
    const int32_t mt = rest / n_here, nt = group * 4 + rest - mt * n_here;
    const int64_t r0 = seg.begin + (int64_t)mt * kTileRows;
    const int32_t n0 = nt * kTileCols;
    const int32_t rows = seg.end - r0 < kTileRows ? (int32_t)(seg.end - r0) : kTileRows;
    const int32_t cols = a.N - n0 < kTileCols ? a.N - n0 : kTileCols;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t code_row = (int64_t)a.groups * 64, scale_row = (int64_t)a.groups * 4;
    const uint8_t *xbase = a.xc + r0 * code_row, *wbase = a.wc + ((int64_t)s * a.N + n0) * code_row;
    // Load i of a wave brings 8 rows, of x (i < 4) or w; rows past the end are the
    // last one again, loads of none but those are left out.
    const int piece = (lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7);
    uint32_t from[8], from_last[8];
    int n_x = 0, n_w = 0;
    const bool odd = a.groups & 1;  // the last step has four pieces a row
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int first = ((i & 3) * 8 + wave) * 8, row = first + (lane >> 3), most = (i < 4 ? rows : cols) - 1;
        const uint32_t at = (uint32_t)((row < most ? row : most) * code_row);
        from[i] = at + piece * 16;
        from_last[i] = at + (odd ? piece & 3 : piece) * 16;
        if (first <= most) (i < 4 ? n_x : n_w) += 1;
    }
    const uint32_t lds0 = lds_address(lds);
    const int32_t steps = (a.groups + 1) / 2;
    auto issue = [&](int32_t step) __attribute__((always_inline)) {
        const uint32_t to = lds0 + (step & 1) * kStage + wave * 1024;
        const uint8_t *x = xbase + (int64_t)step * 128, *w = wbase + (int64_t)step * 128;
        const bool last = step + 1 == steps;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n_x) load_to_lds(x, last ? from_last[i] : from[i], to + i * 8192);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n_w) load_to_lds(w, last ? from_last[4 + i] : from[4 + i], to + (4 + i) * 8192);
    };
    // scales: a row's words of two steps a thread
    uint32_t *turned = reinterpret_cast<uint32_t *>(lds + 2 * kStage);
    uint32_t sc[kWords];
    const int srow = t < kTileRows ? (t < rows ? t : rows - 1) : (t - kTileRows < cols ? t - kTileRows : cols - 1);
    const uint32_t *scales = reinterpret_cast<const uint32_t *>(
        t < kTileRows ? a.xs + (r0 + srow) * scale_row : a.ws + ((int64_t)s * a.N + n0 + srow) * scale_row);
    auto fetch_scales = [&](int32_t unit) __attribute__((always_inline)) {
        if ((unit + 1) * kWords <= a.groups) {
            load16<false>(scales + unit * kWords, sc);
        } else {
#pragma unroll
            for (int k = 0; k < kWords; ++k) sc[k] = unit * kWords + k < a.groups ? scales[unit * kWords + k] : 0;
        }
    };
    auto store_scales = [&](int32_t unit) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kWords; ++k) turned[((unit & 1) * kWords + k) * kBoth + t] = sc[k];
    };
    // this wave's blocks: rows (2 m + wm) 32, columns wn + 32 n
    const int wm = wave >> 2, wn = (wave & 3) * 64, half = lane >> 5, r32 = lane & 31;
    const int blocks = (rows + 31) / 32, live = wn < cols ? (blocks - wm + 1) / 2 : 0;
    T *y = static_cast<T *>(a.y);
    // The whole of it for a number of blocks (the accumulators stay where they
    // are): every wave meets the others as often, whatever its number.
    auto multiply = [&](auto live_) __attribute__((always_inline)) {
    constexpr int kLive = decltype(live_)::value;
    float16_ sum[kLive ? kLive : 1][2] = {};
    for (int32_t step = 0; step < steps; ++step) {
        wait_and_meet();
        const int32_t unit = step >> 1;
        if ((unit + 1) * kWords < a.groups) {
            // (before the codes' loads, which a wait for the scales would wait for)
            if (step & 1) store_scales(unit + 1);
            else fetch_scales(unit + 1);
        }
        if (step + 1 < steps) issue(step + 1);
        const char *tile = lds + (step & 1) * kStage;
        const uint32_t *scale = turned + (((step >> 1) & 1) * kWords + (step & 1) * 2) * kBoth + r32;
        const int groups = step + 1 == steps && odd ? 1 : 2;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            if (kLive == 0 || g >= groups) break;
            uint32_t xs[kLive ? kLive : 1], ws[2];
#pragma unroll
            for (int m = 0; m < kLive; ++m) xs[m] = scale[g * kBoth + (2 * m + wm) * 32] >> (8 * half);
#pragma unroll
            for (int n = 0; n < 2; ++n) ws[n] = scale[g * kBoth + kTileRows + wn + n * 32] >> (8 * half);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                auto fragment = [&](int first) {
                    const int row = first + r32, at = (4 * g + 2 * k + half) ^ ((row >> 1) & 7);
                    const int4_ v = *reinterpret_cast<const int4_ *>(tile + row * 128 + at * 16);
                    return int8_{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
                };
                int8_ x[kLive ? kLive : 1], w[2];
#pragma unroll
                for (int n = 0; n < 2; ++n) w[n] = fragment(kTileRows + wn + n * 32);
#pragma unroll
                for (int m = 0; m < kLive; ++m) x[m] = fragment((2 * m + wm) * 32);
#pragma unroll
                for (int m = 0; m < kLive; ++m)
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        if (k == 0)
                            sum[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[n], x[m], sum[m][n], 4, 4, 0, (int)ws[n], 0, (int)xs[m]);
                        else
                            sum[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[n], x[m], sum[m][n], 4, 4, 2, (int)ws[n], 2, (int)xs[m]);
                    }
            }
        }
    }
    wait_and_meet();
    static_assert(8 * 32 * kPitch<T, 2> <= kManyLds, "the waves' parts fit");
#pragma unroll
    for (int m = 0; m < kLive; ++m) {
        const int first = (2 * m + wm) * 32;
        leave_by_lines<T, 2>(lds + wave * 32 * kPitch<T, 2>, sum[m], y + (r0 + first) * a.N, a.N, rows - first, a.N, n0 + wn, a.whole);
    }
    };
    if (steps > 0) {
        fetch_scales(0);
        issue(0);
        store_scales(0);
    }
    switch (live) {
        case 4: multiply(Int<4>()); break;
        case 3: multiply(Int<3>()); break;
        case 2: multiply(Int<2>()); break;
        case 1: multiply(Int<1>()); break;
        default: multiply(Int<0>());
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
    a.whole = N % (y->type == ROUTEPACK_F32 ? 4 : 8) == 0 && ((uintptr_t)y->data & 15) == 0;
    const int64_t most = a.R < n_slots ? a.R : n_slots;  // slots with rows
    const int64_t pieces = (a.R * N + 65535) / 65536;
    a.clears = pieces < 256 ? pieces : 256;
    // Rows a slot on average, and tiles of 256 x 256.  Up to 6 rows the weights'
    // bytes are all there is and many small workgroups stream them best (256 x 2048
    // x 2048, 512 rows: 89 us, 104 by tiles; 2048 rows: 138 and 126); so do they where
    // the tiles would leave half of the chip idle, as long as a slot's rows are few
    // passes (64 x 256 x 256, 2000 rows: 12 and 15 us).
    const int64_t tiles = (a.R / kTileRows + most) * ((N + kTileCols - 1) / kTileCols);
    const bool many = a.R >= 64 * (int64_t)n_slots || (a.R >= 6 * (int64_t)n_slots && tiles >= 128);
    return by_type(y->type, [&](auto tag) -> int {
        using T = decltype(tag);
        if (many) {
            const auto kern = k_product_many<T>;
            a.n_tiles = (int32_t)((N + kTileCols - 1) / kTileCols);
            // (each slot may have a tile that is not full; eight runs of equal length)
            a.tiles = ((a.R / kTileRows + most) * a.n_tiles + 7) / 8 * 8;
            if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                    kManyLds) != hipSuccess)
                return ROUTEPACK_E_DEVICE;
            hipLaunchKernelGGL(kern, grid_of(a.tiles + a.clears), dim3(512), kManyLds, stream, a);
            return launched();
        }
        a.n_tiles = (int32_t)((N + 63) / 64);
        a.tiles = most * a.n_tiles;
        const auto kern = a.R < 8 * (int64_t)n_slots ? k_product_few<T, 1> : k_product_few<T, 2>;
        hipLaunchKernelGGL(kern, grid_of(a.tiles + a.clears), dim3(256), 0, stream, a);
        return launched();
    });
}
