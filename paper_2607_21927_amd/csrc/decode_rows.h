// What the decode kernels share: the key list of a (sequence, kv head) row, and
// the merge of its partials.
#pragma once

#include <float.h>

#include "ris_device.h"
#include "ris_internal.h"

namespace ris {
namespace {

constexpr float kNegBig = -1e30f;   // finite start of ris_decode_attn's running max

struct RowSegs {
    int64_t na, nw, ns;   // anchor entries, window keys, initial keys below the window
    int64_t w_lo;         // window [w_lo, t]; initial tokens [0, ns)
    const int32_t* aidx;  // this row's anchor entries
};

// Key of virtual position v of the row, or -1 (an anchor entry already
// covered by the window or the initial range, or v past the end).
__device__ __forceinline__ int64_t key_of(const RowSegs& r, int64_t v) {
    if (v < r.na) {
        const int64_t j = r.aidx[v];
        return (j >= r.ns && j < r.w_lo) ? j : -1;
    }
    v -= r.na;
    if (v < r.nw) return r.w_lo + v;
    v -= r.nw;
    return v < r.ns ? v : -1;
}

// The three segments of row (b, g).
__device__ __forceinline__ RowSegs row_segs(const DecodeParams& p, int b, int g) {
    const int64_t t = p.pos[b];
    RowSegs r{0, 0, 0, 0, p.anchor_idx};
    if (t >= 0 && t < p.max_len) {
        int64_t lo = 0, hi = 0;
        if (p.anchor_stride > 0) {                         // else there may be no anchor_ptr
            const int64_t* ap = p.anchor_ptr + (int64_t)b * (p.Hkv + 1) + g;
            lo = ap[0];
            hi = ap[1];
        }
        lo = lo < 0 ? 0 : (lo > p.anchor_stride ? p.anchor_stride : lo);
        hi = hi < lo ? lo : (hi > p.anchor_stride ? p.anchor_stride : hi);
        r.na = hi - lo;
        r.aidx = p.anchor_idx + (int64_t)b * p.anchor_stride + lo;
        r.w_lo = p.window > 0 ? (t - p.window + 1 > 0 ? t - p.window + 1 : 0) : t + 1;
        r.nw = t + 1 - r.w_lo;
        r.ns = p.sink < r.w_lo ? p.sink : r.w_lo;
    }
    return r;
}

// A row's output from its weighted sum and the sum of its weights: an empty set
// gives 0.  (ris_decode_attn has always given 0 for a NaN sum too.)
__device__ __forceinline__ float row_out(const DecodeParams& p, float O, float L) {
    return L > 0.f || (p.keep_nan && L != L) ? O / L : 0.f;
}

__device__ __forceinline__ void store_out(const DecodeParams& p, int64_t at, float y) {
    if (p.out_bf16)
        static_cast<uint16_t*>(p.out)[at] = f32_to_bf16(y);
    else
        static_cast<float*>(p.out)[at] = y;
}

// The factor of a sum under the running maximum m where it meets others under M >= m: 2^((m
// - M) unit), the unit being log2 of the weight that 1 in the maxima stands for.  Maxima
// start finite: where nothing is summed any factor will do.
__device__ __forceinline__ float merge_factor(const DecodeParams& p, float m, float M) {
    return __builtin_amdgcn_exp2f((m - M) * p.unit);
}

// A workgroup's partial: its waves' states merged in LDS (`ow`: kDecodeWaves * G *
// D floats, which the waves may still be reading as something else, hence the
// first barrier).  Lane l holds head l % 16's running maximum and its quarter of
// the sum, and output dim 16 db + l % 16 of the heads 4 (l / 16) + i.  A row's only
// partial is its output.
template <int D>
__device__ __forceinline__ void merge_waves(const DecodeParams& p, int row, float* ow, float m_run, float l_run,
                                            const f32x4_t (&o)[D / 16]) {
    constexpr int DB = D / 16;
    __shared__ float2 ml[kDecodeWaves][8];   // the waves' (max, sum) per head
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int li = lane & 15, lg = lane >> 4, G = p.G;
    l_run = quad_sum16(l_run);
    __syncthreads();
    if (lane < G) ml[wave][lane] = make_float2(m_run, l_run);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int h = 4 * lg + i;
        if (h < G) {
#pragma unroll
            for (int db = 0; db < DB; ++db) ow[(wave * G + h) * D + 16 * db + li] = o[db][i];
        }
    }
    __syncthreads();
    const int64_t slot = (int64_t)row * gridDim.x + blockIdx.x;
    float* pml = p.part_ml + slot * G * 2;
    float* po = p.part_o + slot * G * D;
    for (int e = threadIdx.x; e < G * D; e += 64 * kDecodeWaves) {
        const int h = e / D;
        float M = ml[0][h].x;
#pragma unroll
        for (int w = 1; w < kDecodeWaves; ++w) M = fmaxf(M, ml[w][h].x);
        float O = 0.f, L = 0.f;
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) {
            const float c = merge_factor(p, ml[w][h].x, M);
            O += c * ow[w * G * D + e];
            L += c * ml[w][h].y;
        }
        if (gridDim.x == 1) {                                // the row's only partial: its output
            store_out(p, (int64_t)row * G * D + e, row_out(p, O + 0.f, L));
            continue;
        }
        po[e] = O;
        if (e % D == 0) {
            pml[2 * h] = M;
            pml[2 * h + 1] = L;
        }
    }
}

// Merge the workgroups' partials of one (sequence, query head): the threads first find the
// common max and each partial's weight together (in LDS); then D/4 lanes of
// four dims each sum over every kGroups-th partial, and the groups' sums meet
// in LDS.  Latency-bound (a batch of one has 256 partials of 512 bytes a head):
// one thread per dim walking every partial took 48 us there.
constexpr int kCombineThreads = 256;
template <int D>
__global__ __launch_bounds__(kCombineThreads) void k_decode_combine(DecodeParams p, int parts) {
    constexpr int kLanes = D / 4, kGroups = kCombineThreads / kLanes;
    __shared__ float wgt[kDecodeMaxParts / kDecodeWaves];
    __shared__ float red[kCombineThreads / 64][2];
    __shared__ __align__(16) float osum[kGroups][D];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / p.Hq), h = (int)(bh % p.Hq);
    const int g = h / p.G, hh = h - g * p.G;
    const int64_t row = (int64_t)b * p.Hkv + g;
    const int64_t step_ml = p.G, step_o = (int64_t)p.G * D;
    const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + row * parts * step_ml + hh;
    const float* po = p.part_o + row * parts * step_o + (int64_t)hh * D;
    float M = -FLT_MAX;
    for (int i = tid; i < parts; i += kCombineThreads) M = fmaxf(M, ml[i * step_ml].x);
    M = wave_max(M);
    if (lane == 0) red[wv][0] = M;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kCombineThreads / 64; ++w) M = fmaxf(M, red[w][0]);
    float L = 0.f;
    for (int i = tid; i < parts; i += kCombineThreads) {
        const float2 x = ml[i * step_ml];
        const float w = merge_factor(p, x.x, M);
        wgt[i] = w;
        L += w * x.y;
    }
    L = wave_sum(L);
    if (lane == 0) red[wv][1] = L;
    __syncthreads();
    const int grp = tid / kLanes, d4 = 4 * (tid % kLanes);
    f32x4_t O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = grp; i < parts; i += kGroups) O += wgt[i] * *reinterpret_cast<const f32x4_t*>(po + i * step_o + d4);
    *reinterpret_cast<f32x4_t*>(&osum[grp][d4]) = O;
    __syncthreads();
    if (tid < D) {
        L = 0.f;
#pragma unroll
        for (int w = 0; w < kCombineThreads / 64; ++w) L += red[w][1];
        float y = 0.f;
#pragma unroll
        for (int k = 0; k < kGroups; ++k) y += osum[k][tid];
        y = row_out(p, y, L);
        const int64_t at = bh * D + tid;
        store_out(p, at, y);
    }
}

template <int D>
hipError_t launch_decode_combine(const DecodeParams& p, hipStream_t st) {
    hipLaunchKernelGGL(k_decode_combine<D>, dim3((unsigned)((int64_t)p.B * p.Hq)), dim3(kCombineThreads), 0, st, p,
                       p.parts / kDecodeWaves);
    return hipGetLastError();
}

}  // namespace
}  // namespace ris
