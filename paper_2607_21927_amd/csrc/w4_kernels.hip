// Products of a few rows with weights in 4 bits, y = x W^T, and the weights' way into
// and out of their format.
//
// Weights lie in tiles of 16 outputs x 128 inputs, 1 KB of codes that a wave reads in one
// load: lane l holds output l % 16, the block of 32 inputs l / 16, 16 bytes under one scale.
// That is the A operand of four v_mfma_f32_16x16x32_bf16 as it stands, eight codes each
// (their contraction slots 8 (l / 16) .. hold the inputs 32 (l / 16) + 8 s ..); one
// instruction makes two codes bf16, scale included, exactly.  x is the B operand: lane l holds row
// l % 16 at the same inputs.  The waves of a workgroup deal the chunks of 128 inputs among them
// and meet in LDS.  All products are exact, sums are float32.
//
// float32 rows are taken as three bf16 parts, cut off and not rounded, whose sum is the
// float32 value exactly: three products for one.
#include "mxfp4.h"
#include "ris_internal.h"

namespace ris {
namespace {

constexpr int kChunk = 128;       // inputs of a tile

__host__ __device__ inline int64_t tiles_of(int64_t N) { return (N + 15) / 16; }
__host__ __device__ inline int64_t chunks_of(int64_t K) { return (K + kChunk - 1) / kChunk; }
__host__ __device__ inline int64_t quads_of(int64_t K) { return (K + 4 * kChunk - 1) / (4 * kChunk); }

// Eight neighbouring inputs of a row from `at` on as bf16 parts; 0 from K on.
template <bool F32>
struct Part {
    static constexpr int kCount = F32 ? 3 : 1;
    u32x4_t b[kCount];
};

__device__ __forceinline__ uint32_t two(float lo, float hi) {      // the upper halves of both
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

template <bool F32>
__device__ __forceinline__ void load_part(const void* x, int64_t row, int k, int K, Part<F32>& p) {
    if constexpr (!F32) {
        const uint16_t* q = static_cast<const uint16_t*>(x) + row + k;
        if (k + 8 <= K) {
            p.b[0] = *reinterpret_cast<const u32x4_t*>(q);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                p.b[0][i] = (k + 2 * i < K ? q[2 * i] : 0u) | (k + 2 * i + 1 < K ? (uint32_t)q[2 * i + 1] << 16 : 0u);
        }
    } else {
        const float* q = static_cast<const float*>(x) + row + k;
        float f[8];
        if (k + 8 <= K) {
            const f32x4_t a = *reinterpret_cast<const f32x4_t*>(q), b = *reinterpret_cast<const f32x4_t*>(q + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[i] = a[i];
                f[4 + i] = b[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = k + i < K ? q[i] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float v[2] = {f[i], f[i + 1]}, mid[2], low[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (v[e] != v[e]) v[e] = __uint_as_float(0x7FC00000u);       // a NaN's upper half may be an infinity's
                const float r = isfinite(v[e]) ? v[e] - cut(v[e]) : 0.f;
                mid[e] = r;
                low[e] = r - cut(r);
            }
            p.b[0][i / 2] = two(v[0], v[1]);
            p.b[1][i / 2] = two(mid[0], mid[1]);
            p.b[2][i / 2] = two(low[0], low[1]);
        }
    }
}

__device__ __forceinline__ float silu(float g) { return g / (1.f + __expf(-g)); }

// MT tiles of 16 rows of x, NT of 16 outputs (gated: NT of the gate's and the same of the
// other half's), WV waves.
template <bool F32, bool GATED, int MT, int NT, int WV>
__global__ __launch_bounds__(64 * WV) void k_w4_linear(W4Params p) {
    constexpr int NS = GATED ? 2 * NT : NT;             // sets of 16 outputs
    __shared__ __align__(16) f32x4_t sum[WV > 1 ? WV - 1 : 1][NS * MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, lg = lane >> 4;
    const int chunks = (int)chunks_of(p.K), quads = (int)quads_of(p.K);
    const int tiles = (int)tiles_of(GATED ? p.N / 2 : p.N);
    // row blocks of one set of tiles one after another on one XCD
    const int blocks = (p.rows + 16 * MT - 1) / (16 * MT);
    const uint32_t xcd = blockIdx.x & 7u, slot = blockIdx.x >> 3;
    const int t0 = (int)(slot / blocks * 8u + xcd) * NT, m0 = (int)(slot % blocks) * 16 * MT;
    if (t0 >= tiles) return;
    int tile[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
        const int t = t0 + n % NT < tiles ? t0 + n % NT : tiles - 1;
        tile[n] = GATED && n >= NT ? tiles + t : t;
    }
    f32x4_t acc[NS][MT];
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    int64_t row[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int r = m0 + 16 * m + li;
        row[m] = (int64_t)(r < p.rows ? r : p.rows - 1) * p.x_stride;
    }
    for (int kc = wave; kc < chunks; kc += WV) {
        u32x4_t code[NS];
        uint32_t byte[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            code[n] = *reinterpret_cast<const u32x4_t*>(p.C + (((int64_t)tile[n] * chunks + kc) * 64 + lane) * 16);
            byte[n] = p.S[(((int64_t)tile[n] * quads + (kc >> 2)) * 64 + lane) * 4 + (kc & 3)];
        }
        Part<F32> x[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int s = 0; s < 4; ++s) load_part<F32>(p.x, row[m], kc * kChunk + 32 * lg + 8 * s, p.K, x[m][s]);
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const u32x4_t w = decode8(code[n][s], scale_of(byte[n]));
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int i = Part<F32>::kCount - 1; i >= 0; --i)
                        acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(x[m][s].b[i]), acc[n][m], 0, 0, 0);
            }
    }
    if (WV > 1 && wave > 0) {
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) sum[wave - 1][n * MT + m][lane] = acc[n][m];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < WV - 1; ++w)
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[n][m] += sum[w][n * MT + m][lane];
    // lane l holds row l % 16 at the outputs 4 (l / 16) .. of a tile
    const int N = GATED ? p.N / 2 : p.N;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int r = m0 + 16 * m + li, o = 16 * (t0 + n) + 4 * lg;
            if (r >= p.rows || o >= N) continue;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = o + i;
                const auto biased = [&](float v, int col) __attribute__((always_inline)) {
                    if (!p.bias || at >= N) return v;
                    return v + (F32 ? static_cast<const float*>(p.bias)[col] : bf16_to_f32(static_cast<const uint16_t*>(p.bias)[col]));
                };
                y[i] = biased(acc[n][m][i], at);
                if constexpr (GATED) y[i] = silu(y[i]) * biased(acc[NT + n][m][i], N + at);
            }
            const int64_t to = (int64_t)r * p.out_stride + o;
            if constexpr (F32) {
                float* q = static_cast<float*>(p.out) + to;
                if (p.vector_out) {
                    *reinterpret_cast<f32x4_t*>(q) = f32x4_t{y[0], y[1], y[2], y[3]};
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (o + i < N) q[i] = y[i];
                }
            } else {
                uint16_t* q = static_cast<uint16_t*>(p.out) + to;
                if (p.vector_out) {
                    *reinterpret_cast<uint2*>(q) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (o + i < N) q[i] = f32_to_bf16(y[i]);
                }
            }
        }
}

// A workgroup takes 16 outputs and 16 blocks of 32 inputs: four tiles.  Outputs from N on and
// inputs from K on are zeros.
template <bool BF16>
__global__ __launch_bounds__(256) void k_w4_pack(const void* W, int64_t stride, int N, int K, uint8_t* C, uint8_t* S) {
    const int r = threadIdx.x >> 4, blk = threadIdx.x & 15;
    const int64_t t = blockIdx.x, kc = (int64_t)blockIdx.y * 4 + blk / 4, n = 16 * t + r;
    const int64_t chunks = chunks_of(K), quads = quads_of(K);
    if (kc >= chunks) return;
    const int64_t k0 = kc * kChunk + 32 * (blk & 3);
    float x[32];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        x[i] = 0.f;
        if (n < N && k0 + i < K) {
            const int64_t at = n * stride + k0 + i;
            x[i] = BF16 ? bf16_to_f32(static_cast<const uint16_t*>(W)[at]) : static_cast<const float*>(W)[at];
        }
        const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        amax = u > amax ? u : amax;
    }
    const uint32_t byte = scale_byte(amax);
    u32x4_t code = {0u, 0u, 0u, 0u};
    if (byte != kNanScale) {
#pragma unroll
        for (int i = 0; i < 4; ++i) code[i] = encode8(x + 8 * i, scale_of(byte));
    }
    const int64_t lane = 16 * (blk & 3) + r;
    *reinterpret_cast<u32x4_t*>(C + ((t * chunks + kc) * 64 + lane) * 16) = code;
    S[((t * quads + (kc >> 2)) * 64 + lane) * 4 + (kc & 3)] = (uint8_t)byte;
}

template <bool BF16>
__global__ __launch_bounds__(256) void k_w4_load(const uint8_t* C, const uint8_t* S, int N, int K, void* W, int64_t stride,
                                                 int vector) {
    const int r = threadIdx.x >> 4, blk = threadIdx.x & 15;
    const int64_t t = blockIdx.x, kc = (int64_t)blockIdx.y * 4 + blk / 4, n = 16 * t + r;
    const int64_t chunks = chunks_of(K), quads = quads_of(K);
    const int64_t k0 = kc * kChunk + 32 * (blk & 3);
    if (n >= N || k0 >= K) return;
    const int64_t lane = 16 * (blk & 3) + r;
    const u32x4_t code = *reinterpret_cast<const u32x4_t*>(C + ((t * chunks + kc) * 64 + lane) * 16);
    const uint32_t byte = S[((t * quads + (kc >> 2)) * 64 + lane) * 4 + (kc & 3)];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        u32x4_t v = decode8(code[s], scale_of(byte));
        if (byte == kNanScale) v = u32x4_t{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        const int64_t k = k0 + 8 * s, at = n * stride + k;
        if (vector && k + 8 <= K) {
            if constexpr (BF16) {
                *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(W) + at) = v;
            } else {
                f32x4_t* y = reinterpret_cast<f32x4_t*>(static_cast<float*>(W) + at);
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    y[q] = f32x4_t{__uint_as_float(v[2 * q] << 16), __uint_as_float(v[2 * q] & 0xFFFF0000u),
                                   __uint_as_float(v[2 * q + 1] << 16), __uint_as_float(v[2 * q + 1] & 0xFFFF0000u)};
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < K) {
                    const uint16_t h = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
                    if constexpr (BF16) static_cast<uint16_t*>(W)[at + i] = h;
                    else static_cast<float*>(W)[at + i] = bf16_to_f32(h);
                }
        }
    }
}

template <int MT, int NT, int WV>
hipError_t launch_shape(const W4Params& p, hipStream_t st) {
    const int64_t tiles = tiles_of(p.gated ? p.N / 2 : p.N), sets = (tiles + NT - 1) / NT;
    const int64_t blocks = (p.rows + 16 * MT - 1) / (16 * MT);
    const dim3 grid((unsigned)((sets + 7) / 8 * 8 * blocks));
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * WV), 0, st, p); };
    if (p.f32) p.gated ? run(k_w4_linear<true, true, MT, NT, WV>) : run(k_w4_linear<true, false, MT, NT, WV>);
    else p.gated ? run(k_w4_linear<false, true, MT, NT, WV>) : run(k_w4_linear<false, false, MT, NT, WV>);
    return hipGetLastError();
}

}  // namespace

int64_t w4_blocks(const W4Params& p) {
    const int64_t tiles = tiles_of(p.gated ? p.N / 2 : p.N);
    return (tiles + 7) / 8 * 8 * (((int64_t)p.rows + 15) / 16);
}

hipError_t launch_w4_linear(const W4Params& p, hipStream_t st) {
    return p.rows <= 16 ? launch_shape<1, 1, 4>(p, st) : launch_shape<2, 1, 4>(p, st);
}

hipError_t launch_w4_pack(const void* W, int64_t stride, int bf16, int32_t N, int32_t K, uint8_t* C, uint8_t* S, hipStream_t st) {
    const dim3 grid((unsigned)tiles_of(N), (unsigned)quads_of(K));
    if (bf16) hipLaunchKernelGGL(k_w4_pack<true>, grid, dim3(256), 0, st, W, stride, N, K, C, S);
    else hipLaunchKernelGGL(k_w4_pack<false>, grid, dim3(256), 0, st, W, stride, N, K, C, S);
    return hipGetLastError();
}

hipError_t launch_w4_load(const uint8_t* C, const uint8_t* S, int32_t N, int32_t K, void* W, int64_t stride, int bf16,
                          hipStream_t st) {
    const dim3 grid((unsigned)tiles_of(N), (unsigned)quads_of(K));
    const int vector = (reinterpret_cast<uintptr_t>(W) & 15) == 0 && stride % (bf16 ? 8 : 4) == 0;
    if (bf16) hipLaunchKernelGGL(k_w4_load<true>, grid, dim3(256), 0, st, C, S, N, K, W, stride, vector);
    else hipLaunchKernelGGL(k_w4_load<false>, grid, dim3(256), 0, st, C, S, N, K, W, stride, vector);
    return hipGetLastError();
}

}  // namespace ris
