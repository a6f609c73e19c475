// Products of a few rows with weights in 4 bits, y = x W^T, and the weights' way into
// and out of their format.
//
// Weights lie in tiles of 16 outputs x 128 inputs, 1 KB of codes that a wave reads in one
// load: lane l holds output l % 16, the block of 32 inputs l / 16, 16 bytes under one scale.
// That is the A operand of four v_mfma_f32_16x16x32_bf16 as it stands, eight codes each
// (their contraction slots 8 (l / 16) .. hold the inputs 32 (l / 16) + 8 s ..); one
// instruction makes two codes bf16, scale included, exactly.  x is the B operand: lane l holds row
// l % 16 at the same inputs.  All products are exact, sums are float32.
//
// float32 rows are taken as three bf16 parts, cut off and not rounded, whose sum is the
// float32 value exactly from 2^-110 on (the matrix unit keeps subnormal numbers; below, the last
// part lacks bits under 2^-133): three products for one.
//
// Two forms.  k_w4_narrow: a workgroup takes one set of 16 outputs and 16 rows, its waves deal the chunks of
// 128 inputs among them, each reads the rows itself, and meet in LDS: enough workgroups where outputs
// are few, nothing to wait for but the loads.  k_w4_wide: four waves side by side take NT sets each and
// share the rows through LDS, since reading them for every 16 outputs would take longer than the
// weights do.
//
// Bound by the bytes of the weights, N K (1/2 + 1/32), where rows are few, and from some 64 rows on by the matrix
// unit; the unit is fed by decoding: a code is decoded once for the 16 MT rows of a workgroup.  151,936 outputs
// of 1,536 inputs, 64 rows: 45 us, 3.2 TB/s and 0.66 PFLOP/s (matrix unit 26% busy, no bank conflicts).  17,920
// of 1,536, gated, 32 rows: 7.4 us.  1,536 of 8,960 in float32, 5 rows: 10.0 us, of which a third is
// taking rows apart, again for every 16 outputs.  One row of 1,536 inputs, 2,048 outputs: 3.4 us in a graph, a chain of a few loads.
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

// The same as they lie in memory, and into parts.
template <bool F32>
struct Raw {
    u32x4_t v[F32 ? 2 : 1];
};

template <bool F32>
__device__ __forceinline__ void load_raw(const void* x, int64_t row, int k, int K, Raw<F32>& r) {
    if constexpr (!F32) {
        const uint16_t* q = static_cast<const uint16_t*>(x) + row + k;
        if (k + 8 <= K) {
            r.v[0] = *reinterpret_cast<const u32x4_t*>(q);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r.v[0][i] = (k + 2 * i < K ? q[2 * i] : 0u) | (k + 2 * i + 1 < K ? (uint32_t)q[2 * i + 1] << 16 : 0u);
        }
    } else {
        const uint32_t* q = static_cast<const uint32_t*>(x) + row + k;
        if (k + 8 <= K) {
            r.v[0] = *reinterpret_cast<const u32x4_t*>(q);
            r.v[1] = *reinterpret_cast<const u32x4_t*>(q + 4);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) r.v[i / 4][i % 4] = k + i < K ? q[i] : 0u;
        }
    }
}

template <bool F32>
__device__ __forceinline__ Part<F32> parts_of(const Raw<F32>& r) {
    Part<F32> p;
    if constexpr (!F32) {
        p.b[0] = r.v[0];
    } else {
        float v[8], rest[8], odd[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = __uint_as_float(r.v[i / 4][i % 4]);
            rest[i] = v[i] - cut(v[i]);                 // NaN of an infinity
            odd[i & 1] += rest[i];
        }
        if (__any(odd[0] + odd[1] != odd[0] + odd[1])) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (v[i] != v[i]) v[i] = __uint_as_float(0x7FC00000u);       // a NaN's upper half may be an infinity's
                rest[i] = isfinite(v[i]) ? rest[i] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            p.b[0][i / 2] = two(v[i], v[i + 1]);
            p.b[1][i / 2] = two(rest[i], rest[i + 1]);
            p.b[2][i / 2] = two(rest[i] - cut(rest[i]), rest[i + 1] - cut(rest[i + 1]));
        }
    }
    return p;
}

// Where row r keeps its 16-byte places in LDS, place c at c ^ turn(r): 16 rows at one place and four rows at
// four places spread over all banks.
__device__ __forceinline__ int turn(int r) { return (r & 3) << 2 | (r >> 2 & 3); }

__device__ __forceinline__ float silu(float g) { return g / (1.f + __expf(-g)); }

// Where lane `lane` finds its part of a tile, and of chunk kc's scales.
__device__ __forceinline__ const u32x4_t* codes_at(const W4Params& p, int tile, int chunks, int kc, int lane) {
    return reinterpret_cast<const u32x4_t*>(p.C + (((int64_t)tile * chunks + kc) * 64 + lane) * 16);
}
__device__ __forceinline__ uint32_t scale_at(const W4Params& p, int tile, int quads, int kc, int lane) {
    return p.S[(((int64_t)tile * quads + (kc >> 2)) * 64 + lane) * 4 + (kc & 3)];
}

template <bool F32>
__device__ __forceinline__ f32x4_t product(u32x4_t w, const Part<F32>& x, f32x4_t acc) {
#pragma unroll
    for (int i = Part<F32>::kCount - 1; i >= 0; --i)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(x.b[i]), acc, 0, 0, 0);
    return acc;
}

// The outputs 4 (l / 16) .. of tile t of row r (of the first half, and of the second, gated).
template <bool F32, bool GATED>
__device__ __forceinline__ void store_outputs(const W4Params& p, int r, int t, f32x4_t acc, f32x4_t up) {
    const int N = GATED ? p.N / 2 : p.N, o = 16 * t + 4 * ((threadIdx.x & 63) >> 4);
    if (r >= p.rows || o >= N) return;
    const auto biased = [&](float v, int col) __attribute__((always_inline)) {
        if (!p.bias) return v;
        return v + (F32 ? static_cast<const float*>(p.bias)[col] : bf16_to_f32(static_cast<const uint16_t*>(p.bias)[col]));
    };
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = o + i < N ? o + i : N - 1;
        y[i] = biased(acc[i], at);
        if constexpr (GATED) y[i] = silu(y[i]) * biased(up[i], N + at);
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

// Set t of 16 outputs as tiles: itself, and gated the one of the other half.
template <bool GATED>
struct Sets {
    static constexpr int kCount = GATED ? 2 : 1;
    static __device__ __forceinline__ int tile(int t, int i, int sets) { return GATED && i ? sets + t : t; }
};

// 16 rows of x; WV waves, each with a chunk of the rows in LDS at a time and the loads of the next on their way.
template <bool F32, bool GATED, int WV>
__global__ __launch_bounds__(64 * WV) void k_w4_narrow(W4Params p) {
    constexpr int NS = Sets<GATED>::kCount, kParts = Part<F32>::kCount, kPlane = 16 * kChunk, NP = 4, U = 2;
    constexpr int kStage = WV * kParts * kPlane * 2, kMeet = WV * NS * 64 * 16;
    __shared__ __align__(16) uint8_t mem[kStage > kMeet ? kStage : kMeet];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, lg = lane >> 4;
    const int chunks = (int)chunks_of(p.K), quads = (int)quads_of(p.K);
    const int sets = (int)tiles_of(GATED ? p.N / 2 : p.N);
    // row blocks of one set one after another on one XCD
    const int blocks = (p.rows + 15) / 16;
    const uint32_t xcd = blockIdx.x & 7u, slot = blockIdx.x >> 3;
    const int t = (int)(slot / blocks * 8u + xcd), m0 = (int)(slot % blocks) * 16;
    if (t >= sets) return;
    f32x4_t acc[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) acc[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // Piece i of a lane: eight inputs of row lane / 16 + 4 i of a chunk, 16-byte place c of the row at c ^ turn(row).
    // Rows that are not there are not loaded: what is in their place reaches outputs that are not there alone.
    uint16_t* const stage = reinterpret_cast<uint16_t*>(mem) + wave * kParts * kPlane;
    const int have = p.rows - m0, pk = 8 * li;
    const char* const x0 = static_cast<const char*>(p.x) + (int64_t)m0 * p.x_stride * (F32 ? 4 : 2);
    u32x4_t code[U][NS];
    uint32_t byte[U][NS];
    Raw<F32> x[U][NP];
    const auto load = [&](int k, int u) __attribute__((always_inline)) {
        const int kc = k < chunks ? k : chunks - 1;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            code[u][n] = *codes_at(p, Sets<GATED>::tile(t, n, sets), chunks, kc, lane);
            byte[u][n] = scale_at(p, Sets<GATED>::tile(t, n, sets), quads, kc, lane);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i)
            if (4 * i < have) {
                const int r = lg + 4 * i < have ? lg + 4 * i : have - 1;
                load_raw<F32>(x0, r * p.x_stride, kc * kChunk + pk, p.K, x[u][i]);
            }
    };
#pragma unroll
    for (int u = 0; u < U - 1; ++u) load(wave + u * WV, u);
    for (int k0 = wave; k0 < chunks; k0 += U * WV) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kc = k0 + u * WV;
            if (kc >= chunks) break;
            load(kc + (U - 1) * WV, (u + U - 1) % U);
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (4 * i < have) {
                    const Part<F32> b = parts_of<F32>(x[u][i]);
                    const int r = lg + 4 * i;
#pragma unroll
                    for (int e = 0; e < kParts; ++e)
                        *reinterpret_cast<u32x4_t*>(stage + e * kPlane + r * kChunk + 8 * (li ^ turn(r))) = b.b[e];
                }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                Part<F32> b;
#pragma unroll
                for (int e = 0; e < kParts; ++e)
                    b.b[e] = *reinterpret_cast<const u32x4_t*>(stage + e * kPlane + li * kChunk + 8 * ((4 * lg + s) ^ turn(li)));
#pragma unroll
                for (int n = 0; n < NS; ++n)
                    acc[n] = product<F32>(decode8(code[u][n][s], scale_of(byte[u][n])), b, acc[n]);
            }
        }
    }
    f32x4_t* const sum = reinterpret_cast<f32x4_t*>(mem) + lane;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NS; ++n) sum[(wave * NS + n) * 64] = acc[n];
    __syncthreads();
    if (wave > 0) return;
    f32x4_t all[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
        all[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WV; ++w) all[n] += sum[(w * NS + n) * 64];
    }
    store_outputs<F32, GATED>(p, m0 + li, t, all[0], all[NS - 1]);
}

// MT tiles of 16 rows of x in LDS, one chunk of inputs after another, two deep; KW groups of four waves deal the
// chunks among them, a wave has NT sets of 16 outputs.
template <bool F32, bool GATED, int MT, int NT, int KW>
__global__ __launch_bounds__(256 * KW) void k_w4_wide(W4Params p) {
    constexpr int NS = Sets<GATED>::kCount * NT, kParts = Part<F32>::kCount, kPlane = 16 * MT * kChunk;
    constexpr int kStage = 2 * KW * kParts * kPlane * 2, kMeet = (KW - 1) * 4 * NS * MT * 64 * 16;
    __shared__ __align__(16) uint8_t mem[kStage > kMeet ? kStage : kMeet];
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6 & 3), way = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    const int tid = threadIdx.x & 255;
    const int chunks = (int)chunks_of(p.K), quads = (int)quads_of(p.K);
    const int sets = (int)tiles_of(GATED ? p.N / 2 : p.N);
    const int blocks = (p.rows + 16 * MT - 1) / (16 * MT);
    const uint32_t xcd = blockIdx.x & 7u, slot = blockIdx.x >> 3;
    const int t0 = ((int)(slot / blocks * 8u + xcd) * 4 + wave) * NT, m0 = (int)(slot % blocks) * 16 * MT;
    if (t0 - wave * NT >= sets) return;
    int tile[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
        const int t = t0 + n % NT < sets ? t0 + n % NT : sets - 1;
        tile[n] = Sets<GATED>::tile(t, n / NT, sets);
    }
    f32x4_t acc[NS][MT];
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // Piece i of a thread: eight inputs of row tid / 16 + 16 i of a chunk, 16-byte place c of the row at c ^ turn(row).
    uint16_t* const stage = reinterpret_cast<uint16_t*>(mem) + way * 2 * kParts * kPlane;
    const int pr = tid >> 4, pk = 8 * (tid & 15);
    int64_t row[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int r = m0 + 16 * m + pr;
        row[m] = (int64_t)(r < p.rows ? r : p.rows - 1) * p.x_stride;
    }
    const int put = pr * kChunk + 8 * ((tid & 15) ^ turn(pr));
    Raw<F32> x[MT];
    u32x4_t code[NS], next[NS];
    uint32_t byte[NS], next_byte[NS];
    const auto load_x = [&](int kc) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < MT; ++m) load_raw<F32>(p.x, row[m], kc * kChunk + pk, p.K, x[m]);
    };
    const auto load_w = [&](int kc, u32x4_t (&c)[NS], uint32_t (&b)[NS]) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            c[n] = *codes_at(p, tile[n], chunks, kc, lane);
            b[n] = scale_at(p, tile[n], quads, kc, lane);
        }
    };
    const int steps = (chunks + KW - 1) / KW;
    const auto chunk = [&](int i) { return i * KW + way < chunks ? i * KW + way : chunks - 1; };
    load_x(chunk(0));
    load_w(chunk(0), next, next_byte);
    for (int i = 0; i < steps; ++i) {
        uint16_t* const to = stage + (i & 1) * kParts * kPlane;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const Part<F32> b = parts_of<F32>(x[m]);
#pragma unroll
            for (int e = 0; e < kParts; ++e) *reinterpret_cast<u32x4_t*>(to + e * kPlane + 16 * m * kChunk + put) = b.b[e];
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            code[n] = next[n];
            byte[n] = next_byte[n];
        }
        if (i + 1 < steps) {
            load_x(chunk(i + 1));
            load_w(chunk(i + 1), next, next_byte);
        }
        __syncthreads();
        if (i * KW + way >= chunks) continue;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            Part<F32> b[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < kParts; ++e)
                    b[m].b[e] = *reinterpret_cast<const u32x4_t*>(to + e * kPlane + (16 * m + li) * kChunk + 8 * ((4 * lg + s) ^ turn(li)));
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const u32x4_t w = decode8(code[n][s], scale_of(byte[n]));
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[n][m] = product<F32>(w, b[m], acc[n][m]);
            }
        }
    }
    if constexpr (KW > 1) {
        f32x4_t* const sum = reinterpret_cast<f32x4_t*>(mem) + (wave * NS * MT) * 64 + lane;
        __syncthreads();
        if (way > 0) {
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int m = 0; m < MT; ++m) sum[((way - 1) * 4 * NS * MT + n * MT + m) * 64] = acc[n][m];
        }
        __syncthreads();
        if (way > 0) return;
#pragma unroll
        for (int w = 0; w < KW - 1; ++w)
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[n][m] += sum[(w * 4 * NS * MT + n * MT + m) * 64];
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) store_outputs<F32, GATED>(p, m0 + 16 * m + li, t0 + n, acc[n][m], acc[NS - NT + n][m]);
}

// A workgroup takes 16 outputs and 16 blocks of 32 inputs: four tiles.  Outputs from N on and
// inputs from K on are zeros.  Done once for a weight.
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

// Grid of row blocks of `rows` rows beside `sets` sets of outputs, the sets dealt to the XCDs.
int64_t grid_of(const W4Params& p, int64_t sets, int rows) { return (sets + 7) / 8 * 8 * (((int64_t)p.rows + rows - 1) / rows); }

template <bool F32, int WV>
hipError_t narrow(const W4Params& p, hipStream_t st) {
    const dim3 grid((unsigned)grid_of(p, tiles_of(p.gated ? p.N / 2 : p.N), 16));
    if (p.gated) hipLaunchKernelGGL((k_w4_narrow<F32, true, WV>), grid, dim3(64 * WV), 0, st, p);
    else hipLaunchKernelGGL((k_w4_narrow<F32, false, WV>), grid, dim3(64 * WV), 0, st, p);
    return hipGetLastError();
}

template <bool F32, int MT, int NT, int KW>
hipError_t wide(const W4Params& p, hipStream_t st) {
    const int64_t sets = tiles_of(p.gated ? p.N / 2 : p.N);
    constexpr int kGated = NT > 1 ? NT / 2 : 1;             // sets of either half
    if (p.gated) {
        const dim3 grid((unsigned)grid_of(p, (sets + 4 * kGated - 1) / (4 * kGated), 16 * MT));
        hipLaunchKernelGGL((k_w4_wide<F32, true, MT, kGated, KW>), grid, dim3(256 * KW), 0, st, p);
    } else {
        const dim3 grid((unsigned)grid_of(p, (sets + 4 * NT - 1) / (4 * NT), 16 * MT));
        hipLaunchKernelGGL((k_w4_wide<F32, false, MT, NT, KW>), grid, dim3(256 * KW), 0, st, p);
    }
    return hipGetLastError();
}

}  // namespace

// The wide form from 1,024 tiles of outputs on, where the narrow one reads the rows for every 16 outputs (us, bf16, narrow
// and wide: 16 rows, 14,336 outputs of 1,536 inputs 6.9, 6.7, of 4,096 11.4, 12.7, of 8,192 26, 27; 17,920 of 1,536 7.6, 6.8, of
// 4,096 17, 15, of 8,192 32, 28; 64 rows, 17,920 of 1,536 18, 11; float32 16 rows, 14,336 of 4,096 27, 20, 17,920 of 4,096 32, 21).
// The line looks at outputs alone, and that costs one to four rows just above it, where workgroups of the wide form are fewer
// than CUs: one row, 17,920 of 1,536 5.9, 6.8, of 4,096 10.4, 15.4, of 8,192 19.4, 27.8, gated 18.8, 28.7, float32 33, 38, gated
// 24, 38; 28,672 of 4,096 16.3, 17.1, of 8,192 31.8, 32.4; 32,768 of 1,536 8.1, 7.3; 151,936 of 1,536 32, 27, float32 55, 32).
// And for many rows, where the narrow one reads the weights for every 16 of them (1,536 outputs of 8,960 inputs, 256 rows
// 29.6, 33, 512 98, 33; 4,096 of 4,096, 96 rows 15.5, 16.4, 128 18.1, 16.4; float32 128 rows 39, 62, 256 77, 62; 4,096 of
// 4,096, 64 rows 27, 28, 96 36, 28; gated, where a workgroup takes its rows apart for two sets, bf16 128 rows 13.5, 20.8,
// float32 96 rows 23, 28).  Waves of the narrow form: as many as the chunks keep busy where a CU has one workgroup (1,536 of 8,960, 1 row 5.8
// with 16, 6.7 with 8, 9.3 with 4; float32 8.7 with 12, 9.8, 15), fewer where it has several (128 rows 18.3, 17.1, 16.0;
// float32 44, 50, 39).  More than 16 rows to a workgroup save decoding and lose by what they hold in registers and LDS
// (1,536 of 8,960, 64 rows 11.7, with 64 to a workgroup 20.4; float32 30, with 32 to a workgroup 46).
// Ways of the wide form: two, so that few sets keep more waves busy (17,920
// gated, 32 rows 10.1 with one, 7.4 with two, 7.5 with four; 151,936, 64 rows 45.5, 45.3, 65), but one for more than 16
// rows of float32 where a CU has more than one workgroup, and LDS room for no more than one of two ways (one and two ways:
// 1,536 of 8,960, 512 rows 84, 62, 768 115, 114; 151,936, 32 rows 58, 63).  Sets of a wave: two, in bf16 one where
// workgroups would leave half of the CUs empty (two and one: 1,536 of 8,960, 512 rows 41, 33, 768 42, 46; 4,096 of 4,096,
// 256 rows 21.4, 16.9, 512 23, 26).
static int64_t row_tiles(const W4Params& p) { return tiles_of(p.N) * (((int64_t)p.rows + 15) / 16); }
static bool takes_wide(const W4Params& p) {
    return tiles_of(p.N) >= 1024 || row_tiles(p) > (p.f32 ? 1024 : 1536) + (p.gated ? 512 : 0);
}

// Workgroups of the wide form of two sets a wave.
static int64_t wide_groups(const W4Params& p, int rows) {
    const int64_t sets = tiles_of(p.gated ? p.N / 2 : p.N), each = p.gated ? 4 : 8;
    return grid_of(p, (sets + each - 1) / each, rows);
}

int64_t w4_items(const W4Params& p) {
    if (!takes_wide(p)) return grid_of(p, tiles_of(p.gated ? p.N / 2 : p.N), 16) * 1024;
    return wide_groups(p, p.rows <= 16 ? 16 : (p.f32 || p.rows <= 32 ? 32 : 64)) * 512;
}

hipError_t launch_w4_linear(const W4Params& p, hipStream_t st) {
    const int64_t chunks = chunks_of(p.K);
    if (takes_wide(p)) {
        if (p.f32) {
            if (p.rows <= 16) return wide<true, 1, 2, 2>(p, st);
            return wide_groups(p, 32) <= 256 ? wide<true, 2, 2, 2>(p, st) : wide<true, 2, 2, 1>(p, st);
        }
        if (p.rows <= 16) return wide<false, 1, 2, 2>(p, st);
        if (p.rows <= 32) return wide<false, 2, 2, 2>(p, st);
        return wide_groups(p, 64) <= 128 && !p.gated ? wide<false, 4, 1, 2>(p, st) : wide<false, 4, 2, 2>(p, st);
    }
    const int64_t units = row_tiles(p);
    if (p.f32) return units <= 256 && chunks > 8 ? narrow<true, 12>(p, st) : narrow<true, 4>(p, st);
    if (units <= 256 && chunks > 32) return narrow<false, 16>(p, st);
    return units <= 512 && chunks > 8 ? narrow<false, 8>(p, st) : narrow<false, 4>(p, st);
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
