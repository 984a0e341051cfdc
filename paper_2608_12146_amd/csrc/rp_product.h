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

// Which slot's segment a tile lies in, where a slot of n rows has ceil(n / tile)
// tiles (one, if any, where tile is 0).  Every wave of a workgroup searches by
// itself: a lane counts a run of adjacent slots, whose offsets it keeps.
struct TileMap {
    static constexpr int kKeep = 4;  // slots of a lane whose offsets stay in registers
    int32_t per;
    int64_t mine, upto;              // tiles of this lane's run, and up to its end
    int64_t total;
    Segment kept[kKeep];

    static __device__ int64_t tiles(const Segment &g, int32_t tile) {
        const int64_t n = g.end - g.begin;
        return tile ? (n + tile - 1) / tile : n > 0;
    }
    __device__ __forceinline__ TileMap(const int64_t *offsets, int32_t n_slots, int64_t R, int32_t tile) {
        const int lane = threadIdx.x & (kWave - 1);
        per = (n_slots + kWave - 1) / kWave;
        mine = 0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const int32_t s = lane * per + i;
            kept[i] = {0, 0};
            if (i < per && s < n_slots) kept[i] = segment_of(offsets, s, R);
        }
#pragma unroll
        for (int i = 0; i < kKeep; ++i) mine += tiles(kept[i], tile);
        for (int i = kKeep; i < per; ++i)
            if (lane * per + i < n_slots) mine += tiles(segment_of(offsets, lane * per + i, R), tile);
        upto = mine;
        for (int d = 1; d < kWave; d <<= 1) {
            const int64_t v = __shfl_up((long long)upto, d, kWave);
            upto += lane >= d ? v : 0;
        }
        total = uniform64(__shfl((long long)upto, kWave - 1, kWave));
    }
    // The slot of tile `index` < total, its segment, and the number of its tiles
    // before.  All results are uniform.
    __device__ __forceinline__ int32_t find(int64_t index, const int64_t *offsets, int32_t n_slots, int64_t R, int32_t tile, Segment &g,
                            int64_t &before) const {
        const int owner = __builtin_amdgcn_readfirstlane(__builtin_ctzll(__ballot(upto > index)));
        int64_t at = uniform64(__shfl((long long)(upto - mine), owner, kWave));
        const int32_t s0 = owner * per;
        int32_t s = s0;
        bool found = false;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const Segment k = {uniform64(__shfl((long long)kept[i].begin, owner, kWave)),
                               uniform64(__shfl((long long)kept[i].end, owner, kWave))};
            const int64_t n = tiles(k, tile);
            if (!found && index < at + n) {
                found = true;
                s = s0 + i;
                g = k;
            }
            at += found ? 0 : n;
        }
        if (!found)
            for (s = s0 + kKeep;; ++s) {
                g = segment_of(offsets, s, R);
                const int64_t n = tiles(g, tile);
                if (index < at + n || s + 1 >= n_slots) break;
                at += n;
            }
        before = index - at;
        return s;
    }
};

// A wave's LDS accesses before are done before those after.
__device__ inline void wave_meet() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// 16 bytes of values from column c on, as many as the row has.  whole: the rows
// are whole vectors of 16 bytes on their boundaries, and large outputs leave the
// caches anyway: a hint that they do (60 x 1408 x 1984 bf16 in dw: 245 -> 223 us;
// vectors that cross lines lose by it).
template <class T>
__device__ inline void store_cols(T *row, int32_t cols, int32_t c, int4_ v, bool whole) {
    constexpr int W = 16 / (int)sizeof(T);
    typedef int four __attribute__((ext_vector_type(4), aligned(2)));
    if (whole) {
        if (c < cols) __builtin_nontemporal_store(v, reinterpret_cast<int4_ *>(row + c));
    } else if (c + W <= cols) {
        *reinterpret_cast<four *>(row + c) = v;
    } else {
        typedef T values __attribute__((ext_vector_type(W)));
        const values x = __builtin_bit_cast(values, v);
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (c + i < cols) row[c + i] = x[i];
    }
}

// 32 rows of NB matrix tiles of 32 columns, from registers to memory through this
// wave's part of LDS, so that they leave as whole lines: lane l holds row l % 32,
// element i of tile n its column 32 n + 8 (i / 4) + 4 (l / 32) + i % 4.  Columns
// c0 .. of rows out, out + stride, ..: as many as `rows` and `cols` have.
template <class T, int NB>
constexpr int kPitch = NB * 32 * (int)sizeof(T) + 16;
template <class T, int NB>
__device__ inline void leave_by_lines(char *mine, const float16_ (&v)[NB], T *out, int64_t stride, int rows, int32_t cols,
                                      int32_t c0, bool whole) {
    constexpr int kVec = 16 / (int)sizeof(T), kLanes = NB * 32 / kVec, kRowsAtOnce = kWave / kLanes;
    const int lane = threadIdx.x & 63, half = lane >> 5, r32 = lane & 31;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            typedef T four __attribute__((ext_vector_type(4)));
            const four x = {(T)v[n][4 * g], (T)v[n][4 * g + 1], (T)v[n][4 * g + 2], (T)v[n][4 * g + 3]};
            *reinterpret_cast<four *>(mine + r32 * kPitch<T, NB> + (n * 32 + 8 * g + 4 * half) * sizeof(T)) = x;
        }
    wave_meet();
#pragma unroll
    for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
        const int row = i * kRowsAtOnce + lane / kLanes, c = (lane % kLanes) * kVec;
        const int4_ x = *reinterpret_cast<const int4_ *>(mine + row * kPitch<T, NB> + c * sizeof(T));
        if (row < rows) store_cols<T>(out + row * stride, cols, c0 + c, x, whole);
    }
    wave_meet();
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
