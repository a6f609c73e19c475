// Packed sequences: where a token or a tile of rows lies in cu_seqlens.  Offsets
// are clipped to [0, T], so what comes out is inside the buffers whatever the
// device data hold.  T < 2^31 (checked on the host).
#pragma once

#include "ris_device.h"

namespace ris {

__device__ __forceinline__ int clip_offset(int64_t v, int64_t T) { return (int)(v < 0 ? 0 : (v > T ? T : v)); }

// Tile `idx` of the tiles of `rows` rows that the sequences are cut into, those
// far into their sequences first: under a causal mask they cost most, and what is
// long goes first so that the end is short.  (More than 64 sequences: one sequence
// after another.)  By the whole wave, idx uniform; false past the last tile.
struct RowTile {
    int first;      // the sequence's first token
    int len;        // its tokens
    int tile;       // its tile: rows [tile * rows, ..)
};
__device__ __forceinline__ bool find_tile(const int64_t* cu, int batch, int64_t T, int rows, uint32_t idx, RowTile& t) {
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < batch; b0 += 64) {
        const int b = b0 + lane;
        int lo = 0, len = 0;
        if (b < batch) {
            lo = clip_offset(cu[b], T);
            len = clip_offset(cu[b + 1], T) - lo;
            if (len < 0) len = 0;
        }
        const uint32_t nt = ((uint32_t)len + rows - 1) / rows;
        const uint32_t upto = wave_inclusive_scan(nt);
        const uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        if (idx < total) {
            int at;
            if (batch > 1 && batch <= 64) {
                // the last level of which more than idx tiles are that far or farther
                uint32_t level = 0, beyond = 0;                  // beyond: tiles above the level
                for (uint32_t bit = 1u << (31 - __builtin_clz(total)); bit; bit >>= 1) {
                    const uint32_t l = level | bit;
                    if (wave_sum_u32(nt > l ? nt - l : 0u) > idx) level = l;
                }
                beyond = wave_sum_u32(nt > level + 1 ? nt - level - 1 : 0u);
                uint64_t on = __ballot(nt > level);
                for (uint32_t i = idx - beyond; i; --i) on &= on - 1;
                at = (int)__builtin_ctzll(on);
                t.tile = (int)level;
            } else {
                at = (int)__builtin_ctzll(__ballot(upto > idx));
                t.tile = __builtin_amdgcn_readlane((int)upto, at) - 1 - (int)idx;
            }
            t.first = __builtin_amdgcn_readlane(lo, at);
            t.len = __builtin_amdgcn_readlane(len, at);
            return true;
        }
        idx -= total;
    }
    return false;
}

// The sequence that owns token t (uniform), by the whole wave: the number of
// the offsets cu[0..batch] that are <= t, less one; -1 and batch: none.  64
// offsets a step.
__device__ __forceinline__ int find_seq(const int64_t* cu, int batch, int64_t t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = batch + 1;
    while (n > 64) {
        const int step = (n + 63) / 64, at = lane * step;
        const int c = __popcll(__ballot(at < n && cu[lo + at] <= t));
        if (c == 0) return lo - 1;
        const int skip = (c - 1) * step + 1;
        n = n - skip < step - 1 ? n - skip : step - 1;
        lo += skip;
    }
    return lo + __popcll(__ballot(lane < n && cu[lo + lane] <= t)) - 1;
}

}  // namespace ris
