// RoPE with long-context scaling: [heads, N, D] rotated into a contiguous
// destination, from a source with any head and token strides (the same
// buffer for an in-place rotation, or e.g. a head's columns of a token-major
// projection output, which fuses the head-major copy with the rotation).
//
// One thread owns one (token, pair i) and walks every head, so the float64
// angle and sincos (needed: a float32 angle at position 65,535 is off by up to
// ~4e-3 rad) are paid once per (token, pair) and amortised over the heads.
// Consecutive threads take consecutive pairs of one token: each wave touches
// contiguous half-rows, x[i] and x[i + D/2].  Elementwise and HBM-bound.
#include "packed.h"
#include "ris_internal.h"

namespace ris {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kManyPairs = 1 << 17;     // pairs from which a lane takes four
constexpr int64_t kManyBlocks = 1024;       // workgroups to which few tokens' heads are dealt

template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_rope(const void* src, int64_t hs, int64_t ts, void* dst,
                                                   int heads, int64_t N, int D, int64_t pos0, RopeTable tab) {
    const int half = D >> 1;
    const int64_t gid = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = gid / half;
    const int i = (int)(gid - t * half);
    if (t >= N) return;
    const double ang = (double)(pos0 + t) * tab.inv_freq[i];
    double sd, cd;
    sincos(ang, &sd, &cd);
    const float c = (float)(cd * tab.mscale);
    const float s = (float)(sd * tab.mscale);
    for (int h = 0; h < heads; ++h) {
        const int64_t in = (int64_t)h * hs + t * ts;      // source row (h, t)
        const int64_t row = ((int64_t)h * N + t) * D;     // destination row
        if constexpr (BF16) {
            const uint16_t* x = static_cast<const uint16_t*>(src) + in;
            uint16_t* y = static_cast<uint16_t*>(dst) + row;
            const float x0 = bf16_to_f32(x[i]), x1 = bf16_to_f32(x[i + half]);
            y[i] = f32_to_bf16(x0 * c - x1 * s);
            y[i + half] = f32_to_bf16(x1 * c + x0 * s);
        } else {
            const float* x = static_cast<const float*>(src) + in;
            float* y = static_cast<float*>(dst) + row;
            const float x0 = x[i], x1 = x[i + half];
            y[i] = x0 * c - x1 * s;
            y[i + half] = x1 * c + x0 * s;
        }
    }
}

// The same on packed sequences, where positions restart: a wave finds the sequence
// of its first token, its lanes go on from there.  The products are written as
// k_rope's compile (one of each two in an fma), so that the bits are the same.
//
// HBM-bound: a lane owns P neighbouring pairs of a token, 8 or 16 bytes an access,
// and loads the next head while it rotates one (64k tokens of 14 heads of 128 in
// bf16, 470 MB: 97 us, 137 with one pair a lane).  With few tokens the angles' latency counts: one pair a
// lane, and the heads are dealt to gridDim.y.
template <bool BF16, int P>
struct RopePairs {
    float lo[P], hi[P];       // dims i .. i + P - 1 and i + D / 2 ..
};

template <bool BF16, int P>
__device__ __forceinline__ void load_pairs(const void* src, int64_t at, int half, RopePairs<BF16, P>& x) {
    if constexpr (BF16) {
        const uint16_t* p = static_cast<const uint16_t*>(src) + at;
        if constexpr (P == 4) {
            const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(p + half);
            const uint32_t u[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                x.lo[2 * k] = __uint_as_float(u[k] << 16);
                x.lo[2 * k + 1] = __uint_as_float(u[k] & 0xFFFF0000u);
                x.hi[2 * k] = __uint_as_float(u[2 + k] << 16);
                x.hi[2 * k + 1] = __uint_as_float(u[2 + k] & 0xFFFF0000u);
            }
        } else {
            x.lo[0] = bf16_to_f32(p[0]);
            x.hi[0] = bf16_to_f32(p[half]);
        }
    } else {
        const float* p = static_cast<const float*>(src) + at;
        if constexpr (P == 4) {
            const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + half);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x.lo[k] = a[k];
                x.hi[k] = b[k];
            }
        } else {
            x.lo[0] = p[0];
            x.hi[0] = p[half];
        }
    }
}

template <bool BF16, int P>
__device__ __forceinline__ void store_pairs(void* dst, int64_t at, int half, const RopePairs<BF16, P>& y) {
    if constexpr (BF16) {
        uint16_t* p = static_cast<uint16_t*>(dst) + at;
        if constexpr (P == 4) {
            *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(y.lo[0], y.lo[1]), pack_bf16x2(y.lo[2], y.lo[3]));
            *reinterpret_cast<uint2*>(p + half) = make_uint2(pack_bf16x2(y.hi[0], y.hi[1]), pack_bf16x2(y.hi[2], y.hi[3]));
        } else {
            p[0] = f32_to_bf16(y.lo[0]);
            p[half] = f32_to_bf16(y.hi[0]);
        }
    } else {
        float* p = static_cast<float*>(dst) + at;
        if constexpr (P == 4) {
            *reinterpret_cast<f32x4_t*>(p) = f32x4_t{y.lo[0], y.lo[1], y.lo[2], y.lo[3]};
            *reinterpret_cast<f32x4_t*>(p + half) = f32x4_t{y.hi[0], y.hi[1], y.hi[2], y.hi[3]};
        } else {
            p[0] = y.lo[0];
            p[half] = y.hi[0];
        }
    }
}

template <bool BF16, int P>
__global__ __launch_bounds__(kThreads) void k_rope_packed(const void* src, int64_t hs, int64_t ts, void* dst, int heads,
                                                          int64_t T, int D, const int64_t* cu, const int64_t* start,
                                                          int batch, RopeTable tab) {
    const int half = D >> 1, lanes = half / P;                    // lanes of a token
    const int64_t gid = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = gid / lanes;
    const int i = P * (int)(gid - t * lanes);
    const int64_t first = (gid - (threadIdx.x & 63)) / lanes;     // of the wave's tokens
    if (first >= T) return;
    int b = find_seq(cu, batch, first);
    b = seq_from(cu, batch, b < 0 ? 0 : b, t);
    if (t >= T || b >= batch || t < cu[b]) return;
    const int64_t from = cu[b] > 0 ? cu[b] : 0;                   // clipped
    const double pos = (double)(t - from + (start ? start[b] : 0));
    float c[P], s[P];
#pragma unroll
    for (int k = 0; k < P; ++k) {
        double sd, cd;
        sincos(pos * tab.inv_freq[i + k], &sd, &cd);
        c[k] = (float)(cd * tab.mscale);
        s[k] = (float)(sd * tab.mscale);
    }
    const int64_t in = t * ts + i, out = t * D + i;
    int h = blockIdx.y;
    RopePairs<BF16, P> x;
    load_pairs<BF16, P>(src, h * hs + in, half, x);
    while (true) {
        const int nh = h + (int)gridDim.y;
        RopePairs<BF16, P> nx = x, y;
        if (nh < heads) load_pairs<BF16, P>(src, nh * hs + in, half, nx);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            y.lo[k] = fmaf(x.lo[k], c[k], -(x.hi[k] * s[k]));
            y.hi[k] = fmaf(x.lo[k], s[k], x.hi[k] * c[k]);
        }
        store_pairs<BF16, P>(dst, h * T * D + out, half, y);
        if (nh >= heads) return;
        h = nh;
        x = nx;
    }
}

// A lane's pairs of a bf16 row as they lie.
template <int P>
struct PairBits {
    uint32_t lo[(P + 1) / 2], hi[(P + 1) / 2];
};
template <int P>
__device__ __forceinline__ PairBits<P> load_bits(const uint16_t* p, int half) {
    PairBits<P> x;
    if constexpr (P == 4) {
        const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(p + half);
        x.lo[0] = a.x; x.lo[1] = a.y; x.hi[0] = b.x; x.hi[1] = b.y;
    } else {
        x.lo[0] = p[0];
        x.hi[0] = p[half];
    }
    return x;
}
template <int P>
__device__ __forceinline__ void store_bits(uint16_t* p, int half, const PairBits<P>& x) {
    if constexpr (P == 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(x.lo[0], x.lo[1]);
        *reinterpret_cast<uint2*>(p + half) = make_uint2(x.hi[0], x.hi[1]);
    } else {
        p[0] = (uint16_t)x.lo[0];
        p[half] = (uint16_t)x.hi[0];
    }
}
template <int P>
__device__ __forceinline__ RopePairs<true, P> values_of(const PairBits<P>& x) {
    RopePairs<true, P> v;
#pragma unroll
    for (int k = 0; k < P; ++k) {
        v.lo[k] = bf16_to_f32((uint16_t)(x.lo[k / 2] >> (16 * (k & 1))));
        v.hi[k] = bf16_to_f32((uint16_t)(x.hi[k / 2] >> (16 * (k & 1))));
    }
    return v;
}

// The new rows of a paged cache: as k_rope_packed, with K rotated into its page, Q into
// rows of its own beside it and V copied, one pass over the projection's output.  A token
// without a place in the cache keeps its Q alone.
// HBM-bound: 2 (Hq + 2 Hkv) D elements a token, each once (65,536 tokens, 12/2 heads of 128: 116 us, 4.6 TB/s, a
// copy's rate; rotating, then copying K and V to their pages would read and write K twice).  Few tokens: one chain
// of offsets, table, angle in float64, load and store (32 tokens 3.5 us in a graph, their heads dealt over workgroups);
// the host's call takes longer, 14.
template <int P>
__global__ __launch_bounds__(kThreads) void k_page_store(PageStoreParams p, RopeTable tab) {
    const int half = p.D >> 1, lanes = half / P;                  // lanes of a token
    const int64_t gid = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = gid / lanes;
    const int i = P * (int)(gid - t * lanes);
    const int64_t first = (gid - (threadIdx.x & 63)) / lanes;     // of the wave's tokens
    if (first >= p.T) return;
    int b = find_seq(p.cu, p.batch, first);
    b = seq_from(p.cu, p.batch, b < 0 ? 0 : b, t);
    if (t >= p.T || b >= p.batch || t < p.cu[b]) return;
    const int64_t from = p.cu[b] > 0 ? p.cu[b] : 0;               // clipped
    const int64_t pos = (int64_t)((uint64_t)(t - from) + (uint64_t)(p.start ? p.start[b] : 0));
    const int64_t row = page_row(p.map, b, pos);
    float c[P], s[P];
    if (p.rotate) {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            double sd, cd;
            sincos((double)pos * tab.inv_freq[i + k], &sd, &cd);
            c[k] = (float)(cd * tab.mscale);
            s[k] = (float)(sd * tab.mscale);
        }
    }
    // heads of Q, then of K, then of V, whose bits stay as they are
    const int turned = p.rotate ? p.Hq + p.Hkv : 0, of_k = p.Hq + p.Hkv, heads = row < 0 ? p.Hq : of_k + p.Hkv;
    const auto source = [&](int h) __attribute__((always_inline)) {
        const void* x = h < p.Hq ? p.Q : (h < of_k ? p.K : p.V);
        const int64_t at = h < p.Hq ? h * p.q_head + t * p.q_token
                                    : (h < of_k ? (h - p.Hq) * p.k_head + t * p.k_token : (h - of_k) * p.v_head + t * p.v_token);
        return static_cast<const uint16_t*>(x) + at + i;
    };
    const auto target = [&](int h) __attribute__((always_inline)) {
        void* y = h < p.Hq ? p.Qout : (h < of_k ? p.Kp : p.Vp);
        const int64_t g = h < of_k ? h - p.Hq : h - of_k;
        return static_cast<uint16_t*>(y) + (h < p.Hq ? h * p.qo_head + t * p.qo_token : (row + (g << p.map.shift)) * p.D) + i;
    };
    int h = blockIdx.y;
    if (h >= heads) return;
    PairBits<P> x = load_bits<P>(source(h), half);
    while (true) {
        const int nh = h + (int)gridDim.y;
        PairBits<P> nx = x;
        if (nh < heads) nx = load_bits<P>(source(nh), half);
        if (h < turned) {
            const RopePairs<true, P> v = values_of<P>(x);
            RopePairs<true, P> y;
#pragma unroll
            for (int k = 0; k < P; ++k) {
                y.lo[k] = fmaf(v.lo[k], c[k], -(v.hi[k] * s[k]));
                y.hi[k] = fmaf(v.lo[k], s[k], v.hi[k] * c[k]);
            }
            store_pairs<true, P>(target(h), 0, half, y);
        } else {
            store_bits<P>(target(h), half, x);
        }
        if (nh >= heads) return;
        h = nh;
        x = nx;
    }
}

}  // namespace

hipError_t launch_page_store(const PageStoreParams& p, const RopeTable& tab, hipStream_t st) {
    const int64_t pairs = p.T * (p.D / 2);
    const bool four = pairs >= kManyPairs;
    const int64_t blocks = (pairs / (four ? 4 : 1) + kThreads - 1) / kThreads;
    const int heads = p.Hq + 2 * p.Hkv;
    int64_t deal = kManyBlocks / blocks;
    deal = deal < 1 ? 1 : (deal > heads ? heads : deal);
    if (deal > 65535) deal = 65535;
    const dim3 grid((unsigned)blocks, (unsigned)deal);
    if (four) hipLaunchKernelGGL(k_page_store<4>, grid, dim3(kThreads), 0, st, p, tab);
    else hipLaunchKernelGGL(k_page_store<1>, grid, dim3(kThreads), 0, st, p, tab);
    return hipGetLastError();
}

hipError_t launch_rope_packed(const void* src, int64_t head_stride, int64_t token_stride, void* dst, int dtype_bf16,
                              int heads, int64_t T, int D, const int64_t* cu, const int64_t* start, int batch,
                              const RopeTable& tab, hipStream_t st) {
    const uintptr_t align = dtype_bf16 ? 8 : 16;                  // of four elements
    const auto whole = [&](const void* p) { return reinterpret_cast<uintptr_t>(p) % align == 0; };
    const int64_t pairs = T * (D / 2);
    const bool four = D % 8 == 0 && head_stride % 4 == 0 && token_stride % 4 == 0 && whole(src) && whole(dst) &&
                      pairs >= kManyPairs;
    const int64_t blocks = (pairs / (four ? 4 : 1) + kThreads - 1) / kThreads;
    int64_t deal = kManyBlocks / blocks;                          // heads side by side where tokens are few
    deal = deal < 1 ? 1 : (deal > heads ? heads : deal);
    if (deal > 65535) deal = 65535;
    const dim3 grid((unsigned)blocks, (unsigned)deal);
    const auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, src, head_stride, token_stride, dst, heads, T, D, cu, start,
                           batch, tab);
    };
    if (dtype_bf16) four ? run(k_rope_packed<true, 4>) : run(k_rope_packed<true, 1>);
    else four ? run(k_rope_packed<false, 4>) : run(k_rope_packed<false, 1>);
    return hipGetLastError();
}

hipError_t launch_rope(const void* src, int64_t head_stride, int64_t token_stride, void* dst, int dtype_bf16,
                       int heads, int64_t N, int D, int64_t pos0, const RopeTable& tab, hipStream_t st) {
    const int64_t work = N * (D / 2);
    const unsigned blocks = (unsigned)((work + kThreads - 1) / kThreads);
    if (dtype_bf16)
        hipLaunchKernelGGL(k_rope<true>, dim3(blocks), dim3(kThreads), 0, st, src, head_stride, token_stride, dst,
                           heads, N, D, pos0, tab);
    else
        hipLaunchKernelGGL(k_rope<false>, dim3(blocks), dim3(kThreads), 0, st, src, head_stride, token_stride, dst,
                           heads, N, D, pos0, tab);
    return hipGetLastError();
}

}  // namespace ris
