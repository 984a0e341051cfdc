// The balance loss over expert counts (shares of the router's scores against
// the fractions of its choices), on gfx950.
//
// Reading the logits once is the floor.  The tokens are cut into chunks of
// equal length; a workgroup takes one chunk of one layer, keeps running sums of
// the shares in registers (a group of lanes a token) and writes one row of sums
// for each group of the loss that meets its chunk: group g's part of chunk c is
// row c + g (both only grow along the tokens, so no two parts share a row).  A
// second kernel adds every group's rows in their order, a slab of 64 experts a
// workgroup, and forms the slab's part of the loss.  The parts are added in
// their order too, by the last workgroup of a layer to arrive where these are
// few, or by a third kernel.  No floating-point atomics: the result does not
// depend on the launch.
//
// 32768 x 16 x 64 fp32: 22 us for the shares (6 TB/s, part of it from the
// last-level cache) and 7 to 8 us for the loss, which waits for four reads in a
// row (offsets, rows, counts, parts).  131072 x 512 bf16: 24 and 10.5 us;
// logistic scores 40 us for the shares, about 37 of them the issue of 16 vector
// instructions an element, two of a quarter of the others' rate.
#include "rp_internal.h"
#include "rp_route.h"

namespace rp {

struct ShareArgs {
    const void *logits;
    int64_t ts, ls, T, n_chunks;
    int32_t chunk, L, E, n_groups;
    const int64_t *offsets;
    float *rows;        // [n_chunks + n_groups][L][E]
    uint32_t *arrived;  // [L], cleared here
};

__device__ inline int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); }

template <class T, int G, int NV, bool SOFTMAX, bool WHOLE>
__global__ void __launch_bounds__(256) k_share_chunks(ShareArgs a) {
    constexpr int W = 16 / sizeof(T), V = NV * W, SLOTS = 256 / G, EP = G * V;
    __shared__ __align__(16) float part[SLOTS * EP];
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t ch = a.L == 1 ? block : block / a.L;
    const int32_t l = a.L == 1 ? 0 : (int32_t)(block - ch * a.L);
    const int tid = threadIdx.x, c = tid & (G - 1), slot = tid / G;
    if (ch == 0 && tid == 0) a.arrived[l] = 0;
    if (ch >= a.n_chunks) return;
    const int64_t t0 = ch * a.chunk, t1 = t0 + a.chunk < a.T ? t0 + a.chunk : a.T;
    // the first group that ends behind t0
    const int32_t lo = first_where(a.n_groups, [&](int32_t g) { return a.offsets[g + 1] > t0; });
    for (int32_t g = lo; g < a.n_groups; ++g) {
        const int64_t from = a.offsets[g];
        if (from >= t1) break;
        const int64_t b = clamp64(from, t0, t1), e = clamp64(a.offsets[g + 1], t0, t1);
        if (__builtin_expect(b >= e, false)) {  // empty: on to the next group that is not (there may be many)
            g += first_where(a.n_groups - 1 - g, [&](int32_t x) { return a.offsets[g + 2 + (int64_t)x] > e; });
            continue;
        }
        float acc[V];
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] = 0.0f;
        for (int64_t t = b + slot; t < e; t += SLOTS) {
            float z[V];
            load_row<T, G, V, WHOLE>(static_cast<const T *>(a.logits) + t * a.ts + l * a.ls, a.E, c, z);
            float m, inv;
            if constexpr (SOFTMAX) {
                softmax_row<false, G, V>(z, m, inv);
            } else {
                float less[V];
                logistic_row<false, G, V>(z, less, inv);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = __builtin_fmaf(z[v], inv, acc[v]);
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; v += 4)
            *reinterpret_cast<float4 *>(part + slot * EP + elem_of<T, G>(v, c)) =
                make_float4(acc[v], acc[v + 1], acc[v + 2], acc[v + 3]);
        __syncthreads();
        float *dst = a.rows + ((ch + g) * a.L + l) * a.E;
        if constexpr (EP >= 256) {
            for (int x = tid; x < a.E; x += 256) {
                float s = 0.0f;
#pragma unroll 8
                for (int y = 0; y < SLOTS; ++y) s += part[y * EP + x];
                dst[x] = s;
            }
        } else {
            constexpr int P = 256 / EP;
            const int x = tid & (EP - 1), y0 = tid / EP;
            float s = 0.0f;
#pragma unroll 8
            for (int y = y0; y < SLOTS; y += P) s += part[y * EP + x];
            __syncthreads();
            part[tid] = s;
            __syncthreads();
            if (tid < a.E) {
                s = part[tid];
#pragma unroll
                for (int y = 1; y < P; ++y) s += part[y * EP + tid];
                dst[tid] = s;
            }
        }
    }
}

struct LossArgs {
    const float *rows;
    int64_t T;
    int32_t chunk, L, E, n_groups, n_slabs, counts_type;
    const int64_t *offsets;
    const void *counts;
    float *loss, *shares;
    double *parts;  // [L][n_groups][n_slabs][2]
    uint32_t *arrived;
};

// A layer's loss from its parts, by a whole workgroup; `load` reads one.
template <class F>
__device__ inline void add_parts(const LossArgs &a, int32_t l, double *red, F &&load) {
    double total = 0.0;
    for (int64_t y = threadIdx.x; y < a.n_groups; y += blockDim.x) {
        double *part = a.parts + ((int64_t)l * a.n_groups + y) * a.n_slabs * 2;
        double dot = 0.0, sum = 0.0;
        for (int32_t z = 0; z < a.n_slabs; ++z) {
            dot += load(part + 2 * z);
            sum += load(part + 2 * z + 1);
        }
        total += sum > 0.0 ? a.E * dot / sum : 0.0;
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) total += __shfl_xor(total, d, kWave);
    __syncthreads();
    if (lane_id() == 0) red[wave_id()] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int y = 1; y < (int)blockDim.x / kWave; ++y) total += red[y];
        a.loss[l] = (float)(total / a.n_groups);
    }
}

__global__ void __launch_bounds__(1024) k_sum_loss(LossArgs a) {
    __shared__ double red[16];
    const int64_t l = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (l < a.L) add_parts(a, (int32_t)l, red, [](double *p) { return *p; });
}

// R rows abreast of 64 experts.  LAST: the last workgroup of a layer adds its
// parts.
template <int R, bool LAST>
__global__ void __launch_bounds__(64 * R) k_group_loss(LossArgs a) {
    __shared__ double red[R][kWave];
    __shared__ bool last;
    const int64_t n_items = (int64_t)a.n_groups * a.L * a.n_slabs;
    const int64_t item = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (item >= n_items) return;
    const int32_t slab = (int32_t)(item % a.n_slabs);
    const int64_t gl = item / a.n_slabs;
    const int32_t g = (int32_t)(gl / a.L), l = (int32_t)(gl - (int64_t)g * a.L);
    const int lane = lane_id(), r = wave_id();
    const int32_t x = slab * kWave + lane;
    const int64_t b = clamp64(a.offsets[g], 0, a.T), e = clamp64(a.offsets[g + 1], 0, a.T);
    double s = 0.0;
    if (b < e && x < a.E) {
        const int64_t c1 = (e - 1) / a.chunk;
        const int64_t pitch = (int64_t)a.L * a.E;
        const float *p = a.rows + (int64_t)g * pitch + (int64_t)l * a.E + x;
        int64_t ch = b / a.chunk + r;
        constexpr int U = 8;
        for (; ch + (U - 1) * R <= c1; ch += U * R) {
            float y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) y[u] = p[(ch + u * R) * pitch];
#pragma unroll
            for (int u = 0; u < U; ++u) s += (double)y[u];
        }
        for (; ch <= c1; ch += R) s += (double)p[ch * pitch];
    }
    red[r][lane] = s;
    __syncthreads();
    if (r == 0) {
#pragma unroll
        for (int y = 1; y < R; ++y) s += red[y][lane];
        double dot = 0.0, sum = 0.0;
        if (x < a.E) {
            const int64_t at = gl * a.E + x;
            s = b < e ? s / (double)(e - b) : 0.0;
            const double n = (double)(a.counts_type == ROUTEPACK_I32 ? static_cast<const int32_t *>(a.counts)[at]
                                                                     : static_cast<const int64_t *>(a.counts)[at]);
            a.shares[at] = (float)s;
            dot = n * s;
            sum = n;
        }
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            dot += __shfl_xor(dot, d, kWave);
            sum += __shfl_xor(sum, d, kWave);
        }
        if (lane == 0) {
            double *part = a.parts + (((int64_t)l * a.n_groups + g) * a.n_slabs + slab) * 2;
            if constexpr (LAST) {
                __hip_atomic_store(part, dot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(part + 1, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                const uint32_t before =
                    __hip_atomic_fetch_add(a.arrived + l, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
                last = before == (uint32_t)(a.n_groups * a.n_slabs) - 1;
            } else {
                part[0] = dot;
                part[1] = sum;
            }
        }
    }
    if constexpr (LAST) {
        __syncthreads();
        if (last)  // the layer's parts are all there
            add_parts(a, l, &red[0][0], [](double *q) {
                return __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            });
    }
}

}  // namespace rp

using namespace rp;

namespace {

// The workspace: the chunks' rows, the groups' parts of the loss, and a count
// of arrivals a layer (or in `bytes` the error where these do not fit 64 bits).
struct Workspace {
    int64_t n_chunks, parts_at, arrived_at, bytes;
    int32_t chunk;
};
Workspace workspace_of(int64_t T, int32_t L, int32_t E, int32_t n_groups) {
    Workspace w;
    // about 1024 workgroups of 32 tokens and more
    int64_t c = 32;
    while (c < 1024 && (__int128)T * L > c * 1024) c *= 2;
    w.chunk = (int32_t)c;
    w.n_chunks = T / c + (T % c != 0);
    const __int128 rows = ((__int128)w.n_chunks + n_groups) * L * E * 4 + 15;
    const __int128 parts = (__int128)16 * L * n_groups * ((E - 1) / kWave + 1);
    if (rows + parts + (int64_t)4 * L > INT64_MAX) {  // (each addend is below 2^127)
        w.bytes = ROUTEPACK_E_UNSUPPORTED;
        return w;
    }
    w.parts_at = (int64_t)rows & ~(int64_t)15;
    w.arrived_at = w.parts_at + (int64_t)parts;
    w.bytes = w.arrived_at + (int64_t)4 * L;
    return w;
}

}  // namespace

extern "C" int64_t routepack_balance_workspace(const routepack_problem *prob, int64_t n_tokens, int32_t n_groups) {
    if (!prob || prob->n_layers < 0 || prob->n_experts < 1 || n_tokens < 0 || n_groups < 1) return ROUTEPACK_E_INVALID;
    return workspace_of(n_tokens, prob->n_layers, prob->n_experts, n_groups).bytes;
}

extern "C" int routepack_balance_loss(const routepack_problem *prob, const routepack_logits *logits,
                                      int32_t n_groups, const int64_t *offsets, const void *counts,
                                      int32_t counts_type, int32_t score, float *loss, float *shares,
                                      void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    RP_TRY(check_logits(prob, logits, score));
    if (n_groups < 1 || (counts_type != ROUTEPACK_I32 && counts_type != ROUTEPACK_I64)) return ROUTEPACK_E_INVALID;
    const int32_t L = prob->n_layers, E = prob->n_experts;
    if (L == 0) return ROUTEPACK_OK;
    if (!offsets || !counts || !loss || !shares || !workspace || (uintptr_t)workspace % 16) return ROUTEPACK_E_INVALID;
    const Workspace w = workspace_of(logits->n_tokens, L, E, n_groups);
    if (w.bytes < 0) return (int)w.bytes;
    if (workspace_bytes < w.bytes) return ROUTEPACK_E_INVALID;
    float *rows = static_cast<float *>(workspace);
    double *parts = reinterpret_cast<double *>(static_cast<char *>(workspace) + w.parts_at);
    uint32_t *arrived = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + w.arrived_at);
    const ShareArgs a = {logits->data, logits->token_stride, logits->layer_stride, logits->n_tokens, w.n_chunks,
                         w.chunk, L, E, n_groups, offsets, rows, arrived};
    const dim3 grid = grid_of((w.n_chunks > 0 ? w.n_chunks : 1) * L);
    RP_TRY(by_type(logits->type, [&](auto tag) {
        using T = decltype(tag);
        constexpr int kMost = 2 * sizeof(T);  // 32 values a lane
        // rows that fill the lanes exactly go without the checks of every vector
        auto go = [&](auto checked, auto whole, int32_t lanes_hold) {
            hipLaunchKernelGGL(E == lanes_hold ? whole : checked, grid, dim3(256), 0, stream, a);
            return ROUTEPACK_OK;
        };
        if (score == ROUTEPACK_SOFTMAX)
            return by_geometry<T, kMost>(E, [&](auto g, auto nv) {
                return go(k_share_chunks<T, g.value, nv.value, true, false>,
                          k_share_chunks<T, g.value, nv.value, true, true>, g.value * nv.value * Vec<T>::W);
            });
        // logistic rows keep 1 - s too: 16 values a lane while the wave holds the
        // row (131072 x 512 bf16 took 1.3 times as long with 32)
        if (E > 1024)
            return go(k_share_chunks<T, kWave, kMost, false, false>, k_share_chunks<T, kWave, kMost, false, true>,
                      kMaxExperts);
        return by_geometry<T, kMost / 2>(E, [&](auto g, auto nv) {
            return go(k_share_chunks<T, g.value, nv.value, false, false>,
                      k_share_chunks<T, g.value, nv.value, false, true>, g.value * nv.value * Vec<T>::W);
        });
    }));
    const int32_t slabs = (E + kWave - 1) / kWave;
    const LossArgs b = {rows, logits->n_tokens, w.chunk, L, E, n_groups, slabs, counts_type, offsets, counts, loss,
                        shares, parts, arrived};
    const int64_t each = w.n_chunks / n_groups;  // rows of a group, about
    // A workgroup that counts its arrival waits for its stores to reach memory,
    // and the counts of a layer follow one another: up to 64 parts (1000 groups
    // x 4 slabs of 131072 x 256: 116 us, 31 us with the third kernel; 5 x 4 of
    // 8192 x 256: 15.6 us, 17.9 us).
    const bool last = (int64_t)n_groups * slabs <= 64;
    auto go = [&](auto kern, int threads, int64_t n) {
        hipLaunchKernelGGL(kern, grid_of(n, threads), dim3(threads), 0, stream, b);
    };
    const int64_t parts_n = (int64_t)n_groups * L * slabs;
    if (last) {
        if (each >= 64) go(k_group_loss<16, true>, 1024, parts_n);
        else if (each >= 8) go(k_group_loss<4, true>, 256, parts_n);
        else go(k_group_loss<1, true>, 64, parts_n);
    } else {
        if (each >= 64) go(k_group_loss<16, false>, 1024, parts_n);
        else if (each >= 8) go(k_group_loss<4, false>, 256, parts_n);
        else go(k_group_loss<1, false>, 64, parts_n);
        go(k_sum_loss, n_groups > 256 ? 1024 : 256, L);
    }
    return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
}
