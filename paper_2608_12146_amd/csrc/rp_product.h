// Building blocks of the experts' products: the slots' segments of rows, and
// which of a grid's workgroups has which slot and tile.
#pragma once

#include "rp_experts.h"

namespace rp {

typedef int int4_ __attribute__((ext_vector_type(4)));
typedef int int8_ __attribute__((ext_vector_type(8)));
typedef float float4_ __attribute__((ext_vector_type(4)));
typedef float float16_ __attribute__((ext_vector_type(16)));

// A value that all lanes of a wave have.
__device__ inline int64_t uniform64(int64_t v) {
    return (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
}

struct Segment {
    int64_t begin, end;
};

// Slot s's rows, within [0, R) whatever the offsets say.
__device__ inline Segment segment_of(const int64_t *offsets, int32_t s, int64_t R) {
    int64_t b = offsets[s], e = offsets[s + 1];
    b = b < 0 ? 0 : b > R ? R : b;
    e = e < b ? b : e > R ? R : e;
    return {b, e};
}

// The slot that holds tile `index` of a row of tiles, where a slot of n rows has
// ceil(n / tile) of them (at most one where ONE), and the number of its tiles
// before.  Every wave of a workgroup searches by itself: a lane counts a run of
// adjacent slots.  Returns -1 behind the last tile; `total` is their number.
template <bool ONE>
__device__ inline int32_t slot_of_tile(const int64_t *offsets, int32_t n_slots, int64_t R, int32_t tile, int64_t index,
                                       int64_t &before, int64_t &total) {
    const int lane = threadIdx.x & (kWave - 1);
    const int32_t per = (n_slots + kWave - 1) / kWave, s0 = lane * per;
    auto tiles = [&](int32_t s) -> int64_t {
        if (s >= n_slots) return 0;
        const Segment g = segment_of(offsets, s, R);
        if (ONE) return g.end > g.begin ? 1 : 0;
        return (g.end - g.begin + tile - 1) / tile;
    };
    int64_t mine = 0;
    for (int32_t i = 0; i < per; ++i) mine += tiles(s0 + i);
    int64_t upto = mine;
    for (int d = 1; d < kWave; d <<= 1) {
        const int64_t v = __shfl_up((long long)upto, d, kWave);
        upto += lane >= d ? v : 0;
    }
    total = uniform64(__shfl((long long)upto, kWave - 1, kWave));
    if (index >= total) return -1;
    const uint64_t past = __ballot(upto > index);
    const int owner = __builtin_ctzll(past);
    int64_t at = uniform64(__shfl((long long)(upto - mine), owner, kWave));
    // the owner's run, by all lanes alike
    int32_t s = __builtin_amdgcn_readfirstlane(owner) * per;
    for (;; ++s) {
        const int64_t n = tiles(s);
        if (index < at + n || s + 1 >= n_slots) break;
        at += n;
    }
    before = index - at;
    return s;
}

// Zeros in the rows of no slot: piece `index` of `pieces` of them.
template <class T>
__device__ inline void clear_rows(T *y, int64_t cols, const int64_t *offsets, int32_t n_slots, int64_t R, int64_t index,
                                  int64_t pieces) {
    // (offsets do not decrease: rows before the first slot and behind the last)
    int64_t b = offsets[0], e = offsets[n_slots];
    b = b < 0 ? 0 : b > R ? R : b;
    e = e < b ? b : e > R ? R : e;
    const int64_t head = b * cols, n = head + (R - e) * cols;
    for (int64_t i = index * blockDim.x + threadIdx.x; i < n; i += pieces * blockDim.x)
        y[i < head ? i : e * cols + (i - head)] = (T)0.0f;
}

}  // namespace rp
