// What the kernels of attention over a paged cache share: the tokens of a row tile and the
// keys that they attend to.
#pragma once

#include "packed.h"
#include "ris_internal.h"

namespace ris {
namespace {

// The keys of a row tile: of the tokens at positions pmin .. pmax, as tiles of kKeys keys, of which the
// first `sinks` hold first tokens and the others lie side by side from `near` on.
template <int kKeys>
struct Span {
    int pmin, pmax, lo;       // lo: first key of the window of pmin
    int near, sinks, n;
    __device__ __forceinline__ int key0(int v) const { return kKeys * (v < sinks ? v : near + v - sinks); }
};

// Of tokens at positions a .. z (any; those outside the cache attend to nothing).
template <int kKeys>
__device__ __forceinline__ Span<kKeys> span_of(const PageAttnParams& p, int64_t a, int64_t z) {
    Span<kKeys> s{0, -1, 0, 0, 0, 0};
    if (z < 0 || a >= p.map.places) return s;
    s.pmin = a < 0 ? 0 : (int)a;
    s.pmax = z >= p.map.places ? p.map.places - 1 : (int)z;
    s.lo = s.pmin - p.window + 1 > 0 ? s.pmin - p.window + 1 : 0;
    if (p.window == 0) s.lo = s.pmax + 1;
    const int snk = p.sink < s.pmax + 1 ? p.sink : s.pmax + 1;
    s.near = s.lo <= s.pmax ? s.lo / kKeys : s.pmax / kKeys + 1;
    s.sinks = (snk + kKeys - 1) / kKeys;
    if (s.sinks > s.near) s.sinks = s.near;
    s.n = s.sinks + s.pmax / kKeys + 1 - s.near;
    return s;
}

// Position of a sequence's first new token, near enough to the cache for sums with token
// numbers (below 2^31).
__device__ __forceinline__ int64_t first_pos(const PageAttnParams& p, int b) {
    const int64_t at = p.start ? p.start[b] : 0, far = 1ll << 32;
    return at < -far ? -far : (at > far ? far : at);
}

// The lowest n bits.
__device__ __forceinline__ uint64_t below(int n) { return n <= 0 ? 0ull : (n >= 64 ? ~0ull : (1ull << n) - 1); }

// Tokens of a row tile, and the position of its first one in a sequence whose first new token is
// at position `first`.
__device__ __forceinline__ int tile_tokens(const PageAttnParams& p, const RowTile& t) {
    return t.len - t.tile * p.tokens < p.tokens ? t.len - t.tile * p.tokens : p.tokens;
}
__device__ __forceinline__ int64_t tile_pos(const PageAttnParams& p, int64_t first, const RowTile& t) {
    return first + (int64_t)t.tile * p.tokens;
}

// A factor that may have fallen to 0, for sums that an infinity has to stay in: the least float32
// number in its place, which takes any finite sum (below 2^128) below 2^-21.
__device__ __forceinline__ float kept_infinite(float a) { return fmaxf(a, __uint_as_float(1u)); }

// Four neighbouring elements of out.
__device__ __forceinline__ void store4(const PageAttnParams& p, int64_t at, float a, float b, float c, float d) {
    if (p.out_bf16)
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
    else
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) = f32x4_t{a, b, c, d};
}

}  // namespace
}  // namespace ris
