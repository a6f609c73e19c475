// Packed sequences: where a token or a tile of rows lies in cu_seqlens.  Offsets
// are clipped to [0, T], so what comes out is inside the buffers whatever the
// device data hold.  T < 2^31 (checked on the host).
#pragma once

#include "ris_device.h"
#include "ris_internal.h"

namespace ris {

__device__ __forceinline__ int clip_offset(int64_t v, int64_t T) { return (int)(v < 0 ? 0 : (v > T ? T : v)); }

// Tile `idx` of the tiles of `rows` rows that the sequences are cut into.  By the
// whole wave, idx uniform; false where there is none.
//
// Up to 64 sequences, tiles far into their sequences come first: under a causal mask
// they cost most, and what is long goes first so that the end is short.  Beyond, the
// tiles of sequence b have the places from cu[b] / rows + b on, as many as it can need
// (some stay empty), so that one search finds idx, the last tile of a sequence first.
struct RowTile {
    int seq;        // the sequence
    int first;      // its first token
    int len;        // its tokens
    int tile;       // its tile: rows [tile * rows, ..)
};
constexpr int kSortedBatch = 64;

// Places of the tiles of T tokens in `batch` sequences.
inline int64_t tile_places(int64_t T, int64_t batch, int rows) {
    return batch <= kSortedBatch ? (T + batch * (rows - 1)) / rows : T / rows + batch;
}

__device__ __forceinline__ bool find_tile(const int64_t* cu, int batch, int64_t T, int rows, uint32_t idx, RowTile& t) {
    const int lane = threadIdx.x & 63;
    if (batch > kSortedBatch) {
        const auto place = [&](int b) { return (uint32_t)clip_offset(cu[b], T) / (uint32_t)rows + (uint32_t)b; };
        // sequences whose first place is at most idx, 64 looked at in a step
        int lo = 0, n = batch;
        while (n > 64) {
            const int step = (n + 63) / 64, at = lane * step;
            const int c = __popcll(__ballot(at < n && place(lo + at) <= idx));
            if (c == 0) {
                n = 0;
                break;
            }
            const int skip = (c - 1) * step + 1;
            n = n - skip < step - 1 ? n - skip : step - 1;
            lo += skip;
        }
        const int b = lo + __popcll(__ballot(lane < n && place(lo + lane) <= idx)) - 1;
        if (b < 0) return false;
        t.seq = b;
        t.first = clip_offset(cu[b], T);
        t.len = clip_offset(cu[b + 1], T) - t.first;
        const uint32_t j = idx - place(b), nt = t.len > 0 ? ((uint32_t)t.len + rows - 1) / rows : 0u;
        t.tile = (int)(nt - 1 - j);
        return j < nt;
    }
    int lo = 0, len = 0;
    if (lane < batch) {
        lo = clip_offset(cu[lane], T);
        len = clip_offset(cu[lane + 1], T) - lo;
        if (len < 0) len = 0;
    }
    const uint32_t nt = ((uint32_t)len + rows - 1) / rows;
    const uint32_t total = wave_sum_u32(nt);
    if (idx >= total) return false;
    int at = 0;
    if (batch == 1) {
        t.tile = (int)(total - 1 - idx);
    } else {
        // the last level of which more than idx tiles are that far or farther
        uint32_t level = 0;
        for (uint32_t bit = 1u << (31 - __builtin_clz(total)); bit; bit >>= 1) {
            const uint32_t l = level | bit;
            if (wave_sum_u32(nt > l ? nt - l : 0u) > idx) level = l;
        }
        uint64_t on = __ballot(nt > level);
        for (uint32_t i = idx - wave_sum_u32(nt > level + 1 ? nt - level - 1 : 0u); i; --i) on &= on - 1;
        at = (int)__builtin_ctzll(on);
        t.tile = (int)level;
    }
    t.seq = at;
    t.first = __builtin_amdgcn_readlane(lo, at);
    t.len = __builtin_amdgcn_readlane(len, at);
    return true;
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

// The same for a lane's token t from a sequence b at or before its own: one step where
// that is b, some 2 log2 of the distance otherwise (thousands of empty sequences).
__device__ __forceinline__ int seq_from(const int64_t* cu, int batch, int b, int64_t t) {
    int step = 1;
    while (b + step <= batch && cu[b + step] <= t) {
        b += step;
        step *= 2;
    }
    for (step >>= 1; step > 0; step >>= 1)
        if (b + step <= batch && cu[b + step] <= t) b += step;
    return b;
}

// Row (of D elements) of head 0 of the place that the block table names for position pos
// of sequence b; -1 where there is none.  Head g's is g << shift rows on.
__device__ __forceinline__ int64_t page_row(const PageMap& m, int b, int64_t pos) {
    if (pos < 0 || pos >= m.places) return -1;
    const int32_t page = m.table[b * m.table_stride + (pos >> m.shift)];
    return page >= 0 && page < m.pages ? (int64_t)page * m.page_rows + (pos & ((1 << m.shift) - 1)) : -1;
}

}  // namespace ris
