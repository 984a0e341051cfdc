// The balance loss over expert counts (shares of the router's scores against
// the fractions of its choices), on gfx950.
//
// The tokens are cut into chunks of equal length; a workgroup takes one chunk
// of one layer and sums the shares of each group that meets it into a row of
// its own (group g's part of chunk c is row c + g: both only grow along the
// tokens, so no two parts share a row).  A second kernel adds every group's
// rows in their order and forms its part of the loss, a third one adds the
// groups.  No atomics: the result does not depend on the launch.
#include "rp_internal.h"
#include "rp_route.h"

namespace rp {

struct ShareArgs {
    const void *logits;
    int64_t ts, ls, T, chunk;
    int32_t L, E, n_groups, score;
    const int64_t *offsets;
    float *rows;  // [n_chunks + n_groups][L][E]
};

__device__ inline int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); }

template <class T, int V>
__global__ void __launch_bounds__(256) k_share_chunks(ShareArgs a) {
    extern __shared__ float part[];  // [4][E]
    const int64_t ch = blockIdx.x;
    const int32_t l = (int32_t)blockIdx.y;
    const int c = lane_id(), wv = wave_id();
    const int64_t t0 = ch * a.chunk, t1 = t0 + a.chunk < a.T ? t0 + a.chunk : a.T;
    // the first group that ends behind t0
    int32_t lo = 0, hi = a.n_groups;
    while (lo < hi) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (a.offsets[mid + 1] > t0) hi = mid;
        else lo = mid + 1;
    }
    for (int32_t g = lo; g < a.n_groups; ++g) {
        const int64_t b = clamp64(a.offsets[g], t0, t1), e = clamp64(a.offsets[g + 1], t0, t1);
        if (a.offsets[g] >= t1) break;
        if (b >= e) continue;
        float acc[V];
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] = 0.0f;
        for (int64_t t = b + wv; t < e; t += 4) {
            float z[V], less[V];
            load_row<T, kWave, V>(static_cast<const T *>(a.logits) + t * a.ts + l * a.ls, a.E, c, z);
            if (a.score == ROUTEPACK_SOFTMAX) softmax_row<kWave, V>(z);
            else logistic_row<kWave, V>(z, less);
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] += z[v];
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int x = elem_of<T, kWave>(v, c);
            if (x < a.E) part[wv * a.E + x] = acc[v];
        }
        __syncthreads();
        float *dst = a.rows + ((ch + g) * a.L + l) * a.E;
        for (int x = threadIdx.x; x < a.E; x += 256)
            dst[x] = (part[x] + part[a.E + x]) + (part[2 * a.E + x] + part[3 * a.E + x]);
    }
}

struct LossArgs {
    const float *rows;
    int64_t T, chunk;
    int32_t L, E, n_groups, counts_type;
    const int64_t *offsets;
    const void *counts;
    float *shares;
    double *parts;  // [L][n_groups]
};

__device__ inline double block_sum(double v, double *red) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d, kWave);
    __syncthreads();
    if (lane_id() == 0) red[wave_id()] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ void __launch_bounds__(256) k_group_loss(LossArgs a) {
    __shared__ double red[4];
    const int64_t item = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (item >= (int64_t)a.n_groups * a.L) return;
    const int32_t g = (int32_t)(item / a.L), l = (int32_t)(item - (int64_t)g * a.L);
    const int64_t b = clamp64(a.offsets[g], 0, a.T), e = clamp64(a.offsets[g + 1], 0, a.T);
    const int64_t at = item * a.E;
    double dot = 0.0, sum = 0.0;
    for (int x = threadIdx.x; x < a.E; x += 256) {
        double s = 0.0;
        if (b < e) {
            for (int64_t ch = b / a.chunk; ch <= (e - 1) / a.chunk; ++ch) s += a.rows[((ch + g) * a.L + l) * a.E + x];
            s /= (double)(e - b);
        }
        const double n = (double)(a.counts_type == ROUTEPACK_I32 ? static_cast<const int32_t *>(a.counts)[at + x]
                                                                 : static_cast<const int64_t *>(a.counts)[at + x]);
        a.shares[at + x] = (float)s;
        dot += n * s;
        sum += n;
    }
    dot = block_sum(dot, red);
    sum = block_sum(sum, red);
    if (threadIdx.x == 0) a.parts[(int64_t)l * a.n_groups + g] = sum > 0.0 ? a.E * dot / sum : 0.0;
}

__global__ void __launch_bounds__(256) k_sum_loss(const double *parts, int32_t n_groups, float *loss) {
    __shared__ double red[4];
    double s = 0.0;
    for (int32_t g = threadIdx.x; g < n_groups; g += 256) s += parts[(int64_t)blockIdx.x * n_groups + g];
    s = block_sum(s, red);
    if (threadIdx.x == 0) loss[blockIdx.x] = (float)(s / n_groups);
}

}  // namespace rp

using namespace rp;

namespace {

int64_t chunk_of(int64_t T, int32_t L) {
    int64_t c = T * L / 2048;
    return c < 16 ? 16 : (c > 1024 ? 1024 : c);
}

// The workspace: the chunks' rows, then the groups' parts of the loss.
struct Workspace {
    int64_t chunk, n_chunks, parts_at, bytes;
};
Workspace workspace_of(int64_t T, int32_t L, int32_t E, int32_t n_groups) {
    Workspace w;
    w.chunk = chunk_of(T, L);
    w.n_chunks = (T + w.chunk - 1) / w.chunk;
    w.parts_at = ((w.n_chunks + n_groups) * L * E * 4 + 15) & ~(int64_t)15;
    w.bytes = w.parts_at + (int64_t)8 * L * n_groups;
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
    if (workspace_bytes < w.bytes) return ROUTEPACK_E_INVALID;
    if (L > 65535 || w.n_chunks > (1 << 23)) return ROUTEPACK_E_UNSUPPORTED;
    float *rows = static_cast<float *>(workspace);
    double *parts = reinterpret_cast<double *>(static_cast<char *>(workspace) + w.parts_at);
    if (w.n_chunks > 0) {
        const ShareArgs a = {logits->data, logits->token_stride, logits->layer_stride, logits->n_tokens, w.chunk,
                             L, E, n_groups, score, offsets, rows};
        by_type(logits->type, [&](auto tag) {
            using T = decltype(tag);
            const dim3 grid((unsigned)w.n_chunks, (unsigned)L);
            if (E <= 512) hipLaunchKernelGGL((k_share_chunks<T, 8>), grid, dim3(256), (size_t)16 * E, stream, a);
            else hipLaunchKernelGGL((k_share_chunks<T, 32>), grid, dim3(256), (size_t)16 * E, stream, a);
            return 0;
        });
    }
    const LossArgs b = {rows, logits->n_tokens, w.chunk, L, E, n_groups, counts_type, offsets, counts, shares, parts};
    hipLaunchKernelGGL(k_group_loss, grid_of((int64_t)n_groups * L), dim3(256), 0, stream, b);
    hipLaunchKernelGGL(k_sum_loss, dim3((unsigned)L), dim3(256), 0, stream, parts, n_groups, loss);
    return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
}
