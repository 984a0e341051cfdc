// Expert demand from recorded ids (Eq. routing-replay-input), on gfx950.
//
// The tokens are cut into chunks of equal length; a workgroup takes one chunk
// of one layer and counts each sample that meets it in LDS.  A sample that
// lies within one chunk is written by plain stores; the parts of one that
// spans chunks are added with integer atomics to a row cleared before.
#include "rp_internal.h"
#include "rp_route.h"

namespace rp {

struct CountArgs {
    const void *ids;
    int64_t ts, ls, T, chunk, n_chunks;
    int32_t type, N, L, E, k;
    const int64_t *offsets;
    int32_t *demand;
};

// A sample's tokens and the first and last chunk that it meets (an empty
// sample meets the chunk of its offset).
struct Span {
    int64_t b, e, first, last;
};
__device__ inline Span span_of(const CountArgs &a, int32_t i) {
    Span s;
    const int64_t b = a.offsets[i], e = a.offsets[i + 1];
    s.b = b < 0 ? 0 : (b > a.T ? a.T : b);
    s.e = e < s.b ? s.b : (e > a.T ? a.T : e);
    s.first = s.b / a.chunk;
    s.first = s.first < a.n_chunks ? s.first : a.n_chunks - 1;
    s.last = s.e > s.b ? (s.e - 1) / a.chunk : s.first;
    return s;
}

// Clears the rows of samples that span chunks (a workgroup per sample).
__global__ void __launch_bounds__(256) k_count_clear(CountArgs a) {
    for (int64_t i = (int64_t)blockIdx.x; i < a.N; i += gridDim.x) {
        const Span s = span_of(a, (int32_t)i);
        if (s.first == s.last) continue;
        int32_t *row = a.demand + i * a.L * a.E;
        for (int64_t x = threadIdx.x; x < (int64_t)a.L * a.E; x += 256) row[x] = 0;
    }
}

__global__ void __launch_bounds__(256) k_count(CountArgs a) {
    extern __shared__ int32_t hist[];  // [E]
    const int64_t ch = blockIdx.x;
    const int32_t l = (int32_t)blockIdx.y;
    int32_t lo = 0, hi = a.N;  // the first sample whose last chunk is ch or later
    while (lo < hi) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (span_of(a, mid).last >= ch) hi = mid;
        else lo = mid + 1;
    }
    const int64_t t0 = ch * a.chunk, t1 = t0 + a.chunk;
    for (int32_t i = lo; i < a.N; ++i) {
        const Span s = span_of(a, i);
        if (s.first > ch) break;
        if (s.last < ch) continue;
        const int64_t b = s.b > t0 ? s.b : t0, e = s.e < t1 ? s.e : t1;
        __syncthreads();
        for (int x = threadIdx.x; x < a.E; x += 256) hist[x] = 0;
        __syncthreads();
        const int64_t n = (e - b) * a.k;
        for (int64_t x = threadIdx.x; x < n; x += 256) {
            const int64_t t = b + x / a.k, j = x % a.k;
            const int32_t id = load_id(a.ids, a.type, t * a.ts + l * a.ls + j, a.E);
            if (id >= 0) atomicAdd(&hist[id], 1);
        }
        __syncthreads();
        int32_t *row = a.demand + ((int64_t)i * a.L + l) * a.E;
        if (s.first == s.last)
            for (int x = threadIdx.x; x < a.E; x += 256) row[x] = hist[x];
        else
            for (int x = threadIdx.x; x < a.E; x += 256)
                if (hist[x]) atomicAdd(&row[x], hist[x]);
    }
}

}  // namespace rp

using namespace rp;

extern "C" int routepack_count_demand(const routepack_problem *prob, const routepack_ids *ids,
                                      const int64_t *offsets, int32_t *demand, hipStream_t stream) {
    if (!prob || !ids) return ROUTEPACK_E_INVALID;
    const int64_t N = prob->n_samples, T = ids->n_tokens;
    const int32_t L = prob->n_layers, E = prob->n_experts, k = prob->top_k;
    if (N < 0 || L < 0 || E < 1 || k < 1 || T < 0) return ROUTEPACK_E_INVALID;
    RP_TRY(check_ids(prob, ids, T));
    if (E > 32768 || L > 65535 || T > INT32_MAX / k) return ROUTEPACK_E_UNSUPPORTED;
    if (N == 0 || L == 0) return ROUTEPACK_OK;
    if (!offsets || !demand) return ROUTEPACK_E_INVALID;
    int64_t chunk = T * L / 4096;
    chunk = chunk < 256 ? 256 : (chunk > 8192 ? 8192 : chunk);
    const int64_t n_chunks = T > 0 ? (T + chunk - 1) / chunk : 1;
    const CountArgs a = {ids->data, ids->token_stride, ids->layer_stride, T, chunk, n_chunks, ids->type, (int32_t)N, L,
                         E, k, offsets, demand};
    if (n_chunks > 1)
        hipLaunchKernelGGL(k_count_clear, dim3((unsigned)(N < 65536 ? N : 65536)), dim3(256), 0, stream, a);
    const size_t lds = (size_t)4 * E;
    if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(k_count),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
        return ROUTEPACK_E_DEVICE;
    hipLaunchKernelGGL(k_count, dim3((unsigned)n_chunks, (unsigned)L), dim3(256), lds, stream, a);
    return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
}
