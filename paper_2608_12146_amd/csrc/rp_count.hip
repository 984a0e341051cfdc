// Expert demand from recorded ids (Eq. routing-replay-input), on gfx950.
//
// Reading the ids once is the floor.  The tokens are cut into chunks of equal
// length and the layers into groups whose counters fit the LDS; a workgroup
// counts what one sample has in one chunk, for one group, with LDS atomics,
// and reads the ids as vectors of 16 bytes.  A thread keeps its place in the row of a
// token (or of several short ones), so the layers that its ids belong to are
// worked out once.  A sample that lies within one chunk is written by plain
// stores; the parts of one that spans chunks are added with integer atomics to
// a row cleared before (integer sums do not depend on their order).
//
// 300007 x 24 x 8 int32: 45 us, 5.2 TB/s.  Byte ids are bound by the LDS:
// 1000000 x 48 x 8 of them, 384 MB, take 101 us, 3.8 TB/s, at 64 atomics in
// about 7 cycles, 4.8 of them lost to lanes that meet in a bank: with a layer's
// counters side by side, lanes of different layers meet as those of one do.
// Two vector instructions an id.  The parts of samples that span chunks write
// 56 MB of additions there, to a demand of 8 MB.
//
// Sample i's part of chunk c is part i + c: both only grow along the tokens,
// so the parts i + (its first chunk) on are its own, up to the next sample's.
#include "rp_internal.h"
#include "rp_route.h"

namespace rp {

struct CountArgs {
    const void *ids;
    int64_t ts, ls;         // strides of tokens and layers
    int64_t T, n_chunks;
    int32_t shift;          // a chunk holds 2^shift tokens
    int32_t N, L, E, k;
    const int64_t *offsets;
    int32_t *demand;
    int32_t group, n_groups;  // layers of a workgroup, and such groups
    int32_t join;           // a row is that many tokens (of one workgroup's layers, or of one layer)
    int64_t row_stride;
    bool layer_runs;        // a row holds ids of one layer only
    int32_t team;           // threads that count one layer then, or all 256
    int32_t pitch, copies;  // words between layers' counters, and copies of them (a power of two)
    int32_t lanes;          // log2 of the lanes that hand over a layer's counters
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
    s.first = s.b >> a.shift;
    s.first = s.first < a.n_chunks ? s.first : a.n_chunks - 1;
    s.last = s.e > s.b ? (s.e - 1) >> a.shift : s.first;
    return s;
}

// Clears the rows of samples that span chunks.
__global__ void __launch_bounds__(256) k_count_clear(CountArgs a) {
    const int64_t row_len = (int64_t)a.L * a.E;
    for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
        const Span s = span_of(a, (int32_t)i);
        if (s.first == s.last) continue;
        int32_t *row = a.demand + i * row_len;
        for (int64_t x = (int64_t)blockIdx.y * 256 + threadIdx.x; x < row_len; x += (int64_t)gridDim.y * 256) row[x] = 0;
    }
}

// The i-th id of a vector.
template <class I>
__device__ inline uint32_t id_at(const uint32_t (&w)[4], int i) {
    if constexpr (sizeof(I) == 1) return w[i / 4] >> (8 * (i % 4)) & 0xFF;
    else if constexpr (sizeof(I) == 2) return (uint32_t)(int32_t)(int16_t)(w[i / 2] >> (16 * (i % 2)));
    else if constexpr (sizeof(I) == 4) return w[i];
    else return w[2 * i + 1] ? UINT32_MAX : w[2 * i];  // (a high word is 0 for an expert)
}
template <class I>
__device__ inline uint32_t id_of(I x) {
    if constexpr (sizeof(I) == 8) return (uint64_t)x >> 32 ? UINT32_MAX : (uint32_t)x;
    else return (uint32_t)(int32_t)x;
}

// W ids a thread (16 bytes; where the row is not of one piece, W = 1).
template <class I, int W>
__global__ void __launch_bounds__(256) k_count(CountArgs a) {
    extern __shared__ int32_t hist[];  // [copies][group][pitch], then [pitch] for what is not this thread's to count
    const int tid = threadIdx.x, lane = lane_id();
    // Workgroups go to the 8 XCDs in turn: 8 parts abreast, and behind them the
    // same parts' other groups of layers, which share lines in their L2.
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t turn = block >> 3;
    const int32_t grp = (int32_t)(turn % a.n_groups);
    const int64_t part = turn / a.n_groups * 8 + (block & 7);
    if (part >= a.n_chunks + a.N) return;
    const int32_t l0 = grp * a.group;
    const int32_t nl = a.group < a.L - l0 ? a.group : a.L - l0;
    // the sample whose part it is: the last one with first part <= part
    const int32_t i = first_where(a.N, [&](int32_t x) { return x + span_of(a, x).first > part; }) - 1;
    if (i < 0) return;
    const Span s = span_of(a, i);
    const int64_t ch = part - i;
    if (ch > s.last) return;
    const int32_t words = a.copies * a.group * a.pitch;
    for (int x = tid; x < words; x += 256) hist[x] = 0;
    const int64_t t0 = ch << a.shift, t1 = t0 + ((int64_t)1 << a.shift);
    const int64_t b = s.b > t0 ? s.b : t0, e = s.e < t1 ? s.e : t1;
    constexpr bool pieces = W > 1;         // (where the row is not of one piece, W is 1)
    const int32_t piece = a.layer_runs ? a.k : nl * a.k;  // ids of one token in a row
    const int32_t len = a.join * piece;    // of a row
    // its places, and the rows that the threads stand on abreast
    const int32_t cols = pieces ? (len + W - 1) / W : len, slots = a.team / cols;
    const int me = tid & (a.team - 1), col = me % cols, slot = me / cols;
    // the thread's ids are at .. at + W of its rows, less those that the place
    // before holds already (the last place is moved back into the row)
    const int32_t want = col * W;
    const int32_t at = want + W <= len || len < W ? want : len - W;
    int32_t *to[W];  // the counters of each id's layer
    const int32_t first = at % piece;
    int32_t l = a.layer_runs ? 0 : first / a.k, j = first - l * a.k;
    const int32_t l_first = l, j_first = j;
    int32_t *const mine = hist + (lane & (a.copies - 1)) * a.group * a.pitch;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const int32_t x = at + w;
        to[w] = x >= want && x < len ? mine + l * a.pitch : hist + words;
        if (!a.layer_runs && ++j == a.k) {
            j = 0;
            l = l + 1 == nl ? 0 : l + 1;
        }
    }
    const I *ids = static_cast<const I *>(a.ids) + (int64_t)l0 * a.ls;
    // (where the row is not of one piece, W is 1: the thread's layer and choice)
    const int64_t place = W == 1 ? (int64_t)l_first * a.ls + j_first : at;
    // an id that is no expert's goes to the word behind the last expert's
    const uint32_t limit = (uint32_t)a.E;
    const int32_t tokens = (int32_t)(e > b ? e - b : 0), full = tokens / a.join;
    __syncthreads();
    for (int32_t q = tid / a.team; q < (a.layer_runs ? nl : 1); q += 256 / a.team) {
        const I *p = ids + b * a.ts + q * a.ls + place;
        const int32_t up = q * a.pitch;  // (rows of one layer are whole vectors: all places are the thread's)
        auto add = [&](uint32_t id, int w) { atomicAdd(to[w] + (up + (id < limit ? id : limit)), 1); };
        int32_t r = slot < slots ? slot : full;
        if constexpr (W == 1) {
            for (; r < full; r += slots) add(id_of<I>(p[r * a.row_stride]), 0);  // (join is 1)
        } else {
            constexpr int U = 4;
            const int32_t whole = len < W ? 0 : full;
            for (; r + (U - 1) * slots < whole; r += U * slots) {
                uint32_t v[U][4];
#pragma unroll
                for (int u = 0; u < U; ++u) load16<true>(p + (int64_t)(r + u * slots) * a.row_stride, v[u]);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int w = 0; w < W; ++w) add(id_at<I>(v[u], w), w);
            }
            for (; r < whole; r += slots) {
                uint32_t v[4];
                load16<true>(p + (int64_t)r * a.row_stride, v);
#pragma unroll
                for (int w = 0; w < W; ++w) add(id_at<I>(v, w), w);
            }
            // what is left, an id a thread: the tokens behind the last row of
            // `join`, or all of a small last group, whose row is shorter than a
            // vector
            const int32_t done = whole * a.join;
            const I *x = ids + (b + done) * a.ts + q * a.ls;
            auto one = [&](int32_t t, int32_t y) {
                const uint32_t id = id_of<I>(x[t * a.ts + y]);
                const int32_t l = a.layer_runs ? q : y / a.k;
                atomicAdd(mine + l * a.pitch + (id < limit ? id : limit), 1);
            };
            if (len >= W) {
                for (int32_t y = me; y < (tokens - done) * piece; y += a.team) one(y / piece, y % piece);
            } else {
                for (int32_t t = me / piece; t < tokens && me < 256 / piece * piece; t += 256 / piece) one(t, me % piece);
            }
        }
    }
    __syncthreads();
    int32_t *row = a.demand + ((int64_t)i * a.L + l0) * a.E;
    const bool alone = s.first == s.last;
    // (few experts: several layers a wave)
    for (int32_t y = tid >> a.lanes; y < nl; y += 256 >> a.lanes)
        for (int32_t x = tid & ((1 << a.lanes) - 1); x < a.E; x += 1 << a.lanes) {
            int32_t n = 0;
            const int32_t *h = hist + y * a.pitch + x;
            for (int32_t z = 0; z < a.copies; ++z, h += a.group * a.pitch) n += *h;
            if (alone) row[y * a.E + x] = n;
            else if (n) atomicAdd(&row[y * a.E + x], n);
        }
}

}  // namespace rp

using namespace rp;

namespace {

int32_t gcd_of(int32_t a, int32_t b) { return b ? gcd_of(b, a % b) : a; }

template <class I>
int count(CountArgs &a, bool layer_runs, bool token_rows, hipStream_t stream) {
    constexpr int W = 16 / sizeof(I);
    constexpr int32_t kWords = 8192;  // 32 KiB of counters: four workgroups a CU and more
    a.pitch = (a.E + 1) | 1;  // (odd: equal experts of several layers stand in different banks)
    const bool pieces = token_rows || layer_runs;
    // Layers of a workgroup: as many as fit the counters and 256 places of a
    // row, but fewer where the chunks of 64 tokens (or the samples, if they are
    // more) would leave less than 512 workgroups; where that is not all of
    // them, such that a token's piece is whole lines of 128 bytes, or whole
    // vectors.
    // Where a layer's tokens follow each other the threads stand on one layer at
    // a time: one layer and copies of its counters, or several layers where a
    // sample has less than 16 KiB in one (300007 x 24 x 8 int32, 71 samples: 48 us
    // by one layer, 61 by seven; 88222 x 27 x 8, 467 samples: 45 and 32 us).
    const int64_t each = a.T / a.N * a.k * (int64_t)sizeof(I);
    int32_t fit = (layer_runs ? kWords / 4 : kWords) / a.pitch;
    if (layer_runs && each > 0) fit = each >= 16384 ? 1 : (fit < 32768 / each ? fit : (int32_t)(32768 / each));
    fit = fit < 1 ? 1 : fit;
    const int32_t places = 256 * (pieces ? W : 1) / a.k;  // (k <= 256)
    a.group = fit < a.L ? fit : a.L;
    a.group = places < a.group ? places : a.group;
    const int64_t along = a.T / 64 > a.N ? a.T / 64 : a.N;
    while (a.group > 1 && (layer_runs || a.group * a.k * (int32_t)sizeof(I) > 64) &&
           along * ((a.L + a.group - 1) / a.group) < (layer_runs ? 2048 : 512))
        a.group = (a.group + 1) / 2;  // (layers one after the other: 289 x 27, 9 samples, 50 us by 27)
    if (a.group < a.L && token_rows) {
        const int32_t line = 128 / gcd_of(128, a.k * (int32_t)sizeof(I)), vec = W / gcd_of(W, a.k);
        const int32_t unit = a.group >= line ? line : (a.group >= vec ? vec : 1);
        const int32_t most = a.group - a.group % unit, n = (a.L + most - 1) / most;
        a.group = ((a.L + n - 1) / n + unit - 1) / unit * unit;  // (the groups about equal)
    }
    a.n_groups = (a.L + a.group - 1) / a.group;
    a.lanes = 0;
    while (a.lanes < 6 && (1 << a.lanes) < a.E) ++a.lanes;
    a.layer_runs = layer_runs;
    // tokens that follow each other without a gap form one row of whole vectors
    const int32_t piece = layer_runs ? a.k : a.group * a.k;
    a.join = 1;
    if (pieces && a.ts == piece && (layer_runs || a.group == a.L)) a.join = W / gcd_of(W, piece);
    if (a.join * piece / W > 256) a.join = 1;
    a.row_stride = a.join * a.ts;
    const bool vectors = pieces && a.join * piece >= W;  // (else an id a thread)
    const int32_t cols = vectors ? (a.join * piece + W - 1) / W : piece;
    if (cols > 256) return ROUTEPACK_E_INTERNAL;  // (never: `places`)
    // several layers: a wave each (131233 x 64 x 3 bytes by layers, 2863 samples:
    // 75 us, 484 with the workgroup on one layer and its odd ids by few threads)
    a.team = layer_runs && a.group > 1 && cols <= kWave ? kWave : 256;
    a.copies = 1;
    while (a.copies < 16 && 2 * a.copies * a.group * a.pitch <= (layer_runs ? kWords : kWords / 2)) a.copies *= 2;
    // Chunks of 64 tokens and more: about 4096 of them, but, where 512 are left,
    // 16 ids for each counter that a workgroup hands over (262144 tokens x 8
    // int32 in one sample: 17 us, 45 us with 4 ids), and 8 samples of the mean
    // length where these are short, since a sample that spans two chunks is
    // cleared and added.
    a.shift = 6;
    while (a.shift < 20) {
        const int64_t n = (a.T * a.n_groups) >> a.shift;
        const bool many = n > 4096, thin = n > 512 && ((int64_t)a.k << a.shift) < 16 * a.E;
        const bool cut = a.shift < 9 && (int64_t)a.N * a.n_groups > 512 && ((int64_t)a.N << a.shift) < 8 * a.T;
        if (!many && !thin && !cut) break;
        ++a.shift;
    }
    // Few ids: one chunk, so no row to clear (64 samples of 16896 tokens, 4
    // layers of 2 byte ids: 8.7 us, and 12.7 us by chunks; at worst, one sample of
    // 256 KiB of ids for one workgroup, 12.2 and 11.2 us).
    if (a.T * piece * (layer_runs ? a.group : 1) * (int64_t)sizeof(I) <= 256 * 1024) a.shift = 31;
    a.n_chunks = a.T > 0 ? (a.T + ((int64_t)1 << a.shift) - 1) >> a.shift : 1;
    if (a.n_chunks > 1) {
        const int64_t row_len = (int64_t)a.L * a.E;
        const int64_t gx = a.N < 65536 ? a.N : 65536;
        int64_t gy = (row_len + 1023) / 1024;
        gy = gy > 16 ? 16 : gy;
        hipLaunchKernelGGL(k_count_clear, dim3((unsigned)gx, (unsigned)gy), dim3(256), 0, stream, a);
    }
    const size_t lds = 4 * ((size_t)a.copies * a.group + 1) * a.pitch;
    const int64_t parts = (a.n_chunks + a.N + 7) / 8 * 8;
    auto go = [&](auto kern) -> int {
        if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(kern),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
            return ROUTEPACK_E_DEVICE;
        hipLaunchKernelGGL(kern, grid_of(parts * a.n_groups), dim3(256), lds, stream, a);
        return hipGetLastError() == hipSuccess ? ROUTEPACK_OK : ROUTEPACK_E_DEVICE;
    };
    if (vectors) return go(k_count<I, W>);
    return go(k_count<I, 1>);
}

}  // namespace

extern "C" int routepack_count_demand(const routepack_problem *prob, const routepack_ids *ids,
                                      const int64_t *offsets, int32_t *demand, hipStream_t stream) {
    if (!prob || !ids) return ROUTEPACK_E_INVALID;
    const int64_t N = prob->n_samples, T = ids->n_tokens;
    const int32_t L = prob->n_layers, E = prob->n_experts, k = prob->top_k;
    if (N < 0 || L < 0 || E < 1 || k < 1 || T < 0) return ROUTEPACK_E_INVALID;
    RP_TRY(check_ids(prob, ids, T));
    if (E > 16384 || k > 256 || T > INT32_MAX / k) return ROUTEPACK_E_UNSUPPORTED;
    if (N == 0 || L == 0) return ROUTEPACK_OK;
    if (!offsets || !demand) return ROUTEPACK_E_INVALID;
    CountArgs a = {};
    a.ids = ids->data;
    a.ts = ids->token_stride;
    a.ls = ids->layer_stride;
    a.T = T;
    a.N = (int32_t)N;
    a.L = L;
    a.E = E;
    a.k = k;
    a.offsets = offsets;
    a.demand = demand;
    const bool token_rows = L == 1 || a.ls == k;   // a token's layers are adjacent
    const bool layer_runs = !token_rows && a.ts == k;  // a layer's tokens are
    switch (ids->type) {
        case ROUTEPACK_U8: return count<uint8_t>(a, layer_runs, token_rows, stream);
        case ROUTEPACK_I16: return count<int16_t>(a, layer_runs, token_rows, stream);
        case ROUTEPACK_I32: return count<int32_t>(a, layer_runs, token_rows, stream);
        default: return count<int64_t>(a, layer_runs, token_rows, stream);
    }
}
