// What the tiled dense attention kernels share: the place of a row's pieces in a K or
// V tile in LDS, the reference that a row's softmax weights are taken at, and the
// handling of infinities and NaN in V.
#pragma once

#include "ris_device.h"

namespace ris {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

// 16-byte chunk c of row r of a K or V tile lies in place c ^ swizzle(r): 16 rows
// at one chunk (a K read) and 4 rows at four chunks (a transposing V read) both
// spread over all banks.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
    return D == 128 ? ((r & 3) << 2 | (r >> 2 & 3)) : ((r >> 1 & 1) << 2 | (r >> 2 & 3));
}

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

__device__ __forceinline__ bool odd_half(uint32_t u) { return (u & 0x7F80u) == 0x7F80u; }   // infinity or NaN
__device__ __forceinline__ uint32_t finite_only(uint32_t u) {
    return (odd_half(u) ? 0u : u & 0xFFFFu) | (odd_half(u >> 16) ? 0u : u & 0xFFFF0000u);
}
// Whether a tile of N elements holds any such, by the whole wave.
template <int N>
__device__ __forceinline__ bool any_odd(const uint16_t* x) {
    bool odd = false;
#pragma unroll 1
    for (int at = 8 * (threadIdx.x & 63); at < N; at += 8 * 64) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(x + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= finite_only(v[i]) != v[i];
    }
    return __any(odd);
}
template <int N>
__device__ __forceinline__ bool any_odd(const float* x) {
    bool odd = false;
#pragma unroll 1
    for (int at = 4 * (threadIdx.x & 63); at < N; at += 4 * 64) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(x + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= !isfinite(v[i]);
    }
    return __any(odd);
}
// A sum times a factor that may have fallen to 0; an infinity in it stays (kSafe).
template <bool kSafe>
__device__ __forceinline__ float scaled(float x, float a) { return kSafe && !isfinite(x) ? x : x * a; }
// y + x a, the same way in both passes: finite rows have the same bits in either.
template <bool kSafe>
__device__ __forceinline__ float add_scaled(float y, float x, float a) { return kSafe && !isfinite(x) ? y + x : fmaf(x, a, y); }

// A row's reference: the maximum m that its weights 2^((s - m) c) are taken at.  As a
// rule their exponent is one fma, s c - mc, with mc = m c rounded: the row's weights are
// off by one factor then, within 2^0.5 while |mc| < kNearRef.  Beyond, where that factor
// or mc itself may leave float32, a second pass (kSafe) takes the exponents of such rows
// from s - m; other rows keep their bits.
constexpr float kNearRef = 16777216.f;
__device__ __forceinline__ bool far_ref(float mc) { return !(fabsf(mc) < kNearRef); }
// kF32: float32 inputs, where a weight below 2^-126 times a large value counts; the bare
// instruction gives 0 there.  Weights are the square of the half exponent's power, one
// product more (with exp2f 5,000 tokens of 32 heads take 959 us instead of 903).
template <bool kF32>
__device__ __forceinline__ float pow2(float x) { return kF32 ? exp2f(x) : __builtin_amdgcn_exp2f(x); }
template <bool kF32>
struct Ref {
    float m, mc;        // mc: 0 while there is no maximum
    bool apart;         // the row's exponents are taken from differences
    __device__ __forceinline__ void reset() {
        m = -INFINITY;
        mc = 0.f;
    }
    // To the larger of m and mx; the factor for what was summed under the old one.
    template <bool kSafe>
    __device__ __forceinline__ float raise(float mx, float c) {
        const float was = m, wasc = mc;
        m = fmaxf(m, mx);
        mc = m == -INFINITY ? 0.f : m * c;
        return was == -INFINITY ? 0.f : pow2<kF32>(kSafe && apart ? (was - m) * c : wasc - mc);
    }
    template <bool kSafe>
    __device__ __forceinline__ float weight(float s, float c) const {
#pragma clang fp contract(off)              // the square is a number of its own in both passes
        const float f = kF32 ? 0.5f : 1.f;
        const float w = __builtin_amdgcn_exp2f(kSafe && apart ? (m == -INFINITY ? s : s - m) * (f * c) : fmaf(s, f * c, -(f * mc)));
        return kF32 ? w * w : w;
    }
    // After a pass, with the row's sum of weights: references that were far for a while
    // and rose have left a sum that is infinite or NaN.
    __device__ __forceinline__ bool needs_apart(float l) {
        const float sum = pair_sum32(l);
        return apart = far_ref(mc) || !isfinite(sum);
    }
};
// The factor of a partial sum under the reference m (mc) where partial sums of one row
// meet under the largest, top (topc).  Weights of a row apart are taken at m c itself, the others
// at mc, which is up to 2^-1 from it below kNearRef: where the two kinds meet, what an m c is
// over its mc counts as well (none where mc is infinite, and the other one is 2^24 at most then).
__device__ __forceinline__ float over(float m, float mc, bool apart, float c) { return apart && isfinite(mc) ? fmaf(m, c, -mc) : 0.f; }
template <bool kF32>
__device__ __forceinline__ float join_factor(float m, float mc, bool apart, float top, float topc, bool top_apart, float c) {
    if (m == -INFINITY) return 0.f;
    return pow2<kF32>(apart && top_apart ? (m - top) * c : (mc - topc) + (over(m, mc, apart, c) - over(top, topc, top_apart, c)));
}

}  // namespace
}  // namespace ris
