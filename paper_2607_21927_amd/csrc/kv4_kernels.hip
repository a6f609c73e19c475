// Key/value cache in 4 bits: E2M1 codes in blocks of 32 dimensions that share a
// power of two.  gfx950 converts between such codes and bf16 or float32, the
// scale included, one instruction to a pair of values.
//
// Store and load are HBM-bound: a lane owns 8 dimensions of a row of K and of V
// (16 bytes of bf16, 4 of codes), four lanes a block.
//
// Decode is k_decode_partial's pass (a row's set as three disjoint segments, tiles
// of 32 keys dealt to the row's waves, one running softmax per head) over 136
// bytes a key instead of 512 at D = 128.  Both operands of the score product take
// their dimensions in the order in which the codes lie: lane group l / 16 owns the
// D / 4 dimensions from (l / 16) D / 4 on, 16 bytes of codes (D = 128) under one
// scale, and Q is loaded in the same order.  V rows are read whole, become bf16 in
// wave-private LDS and come back transposed.  Weights enter the PV product as bf16, as in
// that pass: off by 2^-8 of themselves at most, their sum taken in float32 before that.
#include "decode_rows.h"
#include "packed.h"

namespace ris {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kNanScale = 255;

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Scale byte of a block whose largest magnitude has these float32 bits: e + 127
// with e the least with amax <= 7 * 2^e (7 / 4 is mantissa 0x600000), -124..125.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    if (amax >= 0x7F800000u) return kNanScale;
    const int e = (int)(amax >> 23) - 2 + ((amax & 0x7FFFFFu) > 0x600000u);
    return (uint32_t)(e < 3 ? 3 : (e > 252 ? 252 : e));
}

// Eight values -> eight codes, the first in the low bits.
__device__ __forceinline__ uint32_t encode8(const float* x, float scale) {
    uint32_t u = 0;
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[0], x[1], scale, 0);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[2], x[3], scale, 1);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[4], x[5], scale, 2);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[6], x[7], scale, 3);
    return u;
}

// Eight codes -> eight bf16 values, exactly.
__device__ __forceinline__ u32x4_t decode8(uint32_t u, float scale) {
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 3))};
}

template <bool BF16>
__device__ __forceinline__ void load8(const void* p, int64_t at, float* x) {
    if constexpr (BF16) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(v[i] << 16);
            x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        }
    } else {
        const f32x4_t* v = reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = v[0][i];
            x[4 + i] = v[1][i];
        }
    }
}

// The cache row of packed token t (in lane order within the wave), or -1.
__device__ __forceinline__ int64_t cache_row(const Kv4Params& p, int64_t first, int64_t t, int h) {
    if (first >= p.T) return -1;
    int b = find_seq(p.cu, p.batch, first);
    b = seq_from(p.cu, p.batch, b < 0 ? 0 : b, t);
    if (t >= p.T || b >= p.batch || t < p.cu[b]) return -1;
    const int64_t from = p.cu[b] > 0 ? p.cu[b] : 0;            // clipped
    const int64_t pos = (int64_t)((uint64_t)(t - from) + (uint64_t)(p.start ? p.start[b] : 0));
    return pos >= 0 && pos < p.max_len ? ((int64_t)b * p.Hkv + h) * p.max_len + pos : -1;
}

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void k_kv4_store(Kv4Params p) {
    constexpr int kLanes = D / 8;              // lanes of a row
    const int lane = threadIdx.x & 63, c = lane % kLanes, h = blockIdx.y;
    const int64_t first = (int64_t)blockIdx.x * (kThreads / kLanes) + (threadIdx.x >> 6) * (64 / kLanes);
    const int64_t t = first + lane / kLanes;
    const int64_t row = cache_row(p, first, t, h);
    if (row < 0) return;                       // all of a row's lanes
    float x[2][8];
    load8<BF16>(p.K, h * p.k_head + t * p.k_token + 8 * c, x[0]);
    load8<BF16>(p.V, h * p.v_head + t * p.v_token + 8 * c, x[1]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t amax = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = __float_as_uint(x[i][e]) & 0x7FFFFFFFu;
            amax = u > amax ? u : amax;
        }
        // the block's four lanes (quad_perm [1,0,3,2], [2,3,0,1])
        uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xB1, 0xF, 0xF, false);
        amax = o > amax ? o : amax;
        o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4E, 0xF, 0xF, false);
        amax = o > amax ? o : amax;
        const uint32_t byte = scale_byte(amax);
        const uint32_t codes = byte == kNanScale ? 0u : encode8(x[i], scale_of(byte));
        reinterpret_cast<uint32_t*>((i ? p.V4 : p.K4) + row * (D / 2))[c] = codes;
        if (c % 4 == 0) p.S[row * (D / 16) + i * (D / 32) + c / 4] = (uint8_t)byte;
    }
}

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void k_kv4_load(Kv4Params p) {
    constexpr int kLanes = D / 8;
    const int lane = threadIdx.x & 63, c = lane % kLanes, h = blockIdx.y;
    const int64_t first = (int64_t)blockIdx.x * (kThreads / kLanes) + (threadIdx.x >> 6) * (64 / kLanes);
    const int64_t t = first + lane / kLanes;
    const int64_t row = cache_row(p, first, t, h);
    if (row < 0) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t u = reinterpret_cast<const uint32_t*>((i ? p.V4 : p.K4) + row * (D / 2))[c];
        const uint32_t byte = p.S[row * (D / 16) + i * (D / 32) + c / 4];
        u32x4_t v = decode8(u, scale_of(byte));
        if (byte == kNanScale) v = u32x4_t{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        const int64_t at = i ? h * p.v_head + t * p.v_token + 8 * c : h * p.k_head + t * p.k_token + 8 * c;
        if constexpr (BF16) {
            *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(i ? p.V : p.K) + at) = v;
        } else {
            f32x4_t* y = reinterpret_cast<f32x4_t*>(static_cast<float*>(i ? p.V : p.K) + at);
#pragma unroll
            for (int q = 0; q < 2; ++q)
                y[q] = f32x4_t{__uint_as_float(v[2 * q] << 16), __uint_as_float(v[2 * q] & 0xFFFF0000u),
                               __uint_as_float(v[2 * q + 1] << 16), __uint_as_float(v[2 * q + 1] & 0xFFFF0000u)};
        }
    }
}

// ---------------------------------------------------------------------------
// Decode
// ---------------------------------------------------------------------------
constexpr int kTileKeys = kDecodeTileKeys;

template <int D>
struct Kv4Tile {
    uint32_t k[2][D / 32], v[2][D / 32];    // D / 8 bytes of codes of a key (16 kb + l % 16) and of a row (16 kb + l / 4)
    uint32_t ks[2], vs[2];                  // their scale bytes
    uint32_t valid;                         // bit 16 kb + i: key slot 16 kb + i is a real key
};

template <int D>
__device__ __forceinline__ void load_codes(const uint8_t* p, uint32_t (&u)[D / 32]) {
    if constexpr (D == 128) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p);
        u[0] = v[0]; u[1] = v[1]; u[2] = v[2]; u[3] = v[3];
    } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        u[0] = v.x; u[1] = v.y;
    }
}

// The codes of the 32 keys from virtual position v0 of the row (uniform) on.  Most
// tiles lie within the anchor or within the window, where a key is one load or none.
template <int D>
__device__ __forceinline__ void load_tile(const RowSegs& r, const uint8_t* Kr, const uint8_t* Vr, const uint8_t* Sr,
                                          int64_t v0, int li, int lg, Kv4Tile<D>& T) {
    const int lane = li + 16 * lg;
    const int row4 = lane >> 2, part = lane & 3;
    uint32_t jk[2], jv[2], vm = 0xFFFFFFFFu;            // max_len <= 2^31: a key fits 32 bits
    if (v0 >= r.na && v0 + kTileKeys <= r.na + r.nw) {
        const uint32_t j0 = (uint32_t)(r.w_lo + (v0 - r.na));
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            jk[kb] = j0 + 16 * kb + li;
            jv[kb] = j0 + 16 * kb + row4;
        }
    } else {
        const bool anchor = v0 + kTileKeys <= r.na;
        vm = 0;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            int64_t j;
            if (anchor) {
                const int a = r.aidx[v0 + 16 * kb + li];
                j = a >= r.ns && a < r.w_lo ? a : -1;
            } else {
                j = key_of(r, v0 + 16 * kb + li);
            }
            vm |= (uint32_t)(__ballot(j >= 0) & 0xFFFFull) << (16 * kb);
            jk[kb] = j >= 0 ? (uint32_t)j : 0u;         // row 0 always exists
            jv[kb] = (uint32_t)__shfl((int)jk[kb], row4);
        }
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        load_codes<D>(Kr + (uint64_t)jk[kb] * (D / 2) + lg * (D / 8), T.k[kb]);
        T.ks[kb] = Sr[(uint64_t)jk[kb] * (D / 16) + lg * D / 128];
        load_codes<D>(Vr + (uint64_t)jv[kb] * (D / 2) + part * (D / 8), T.v[kb]);
        T.vs[kb] = Sr[(uint64_t)jv[kb] * (D / 16) + D / 32 + part * D / 128];
    }
    T.valid = vm;
}

template <int D>
__global__ __launch_bounds__(64 * kDecodeWaves, 4) void k_kv4_decode(DecodeParams p, const uint8_t* S, float slack) {
    constexpr int SL = D / 32;         // k-slices of the score product
    constexpr int DB = D / 16;         // 16-dim blocks of the output
    constexpr int VS = D + 16;         // V row stride in LDS (bf16 elements)
    __shared__ __align__(16) uint16_t vlds[kDecodeWaves * kTileKeys * VS];
    static_assert(kTileKeys * VS * sizeof(uint16_t) >= 8 * D * sizeof(float), "a wave's outputs fit its V slice");

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int li = lane & 15, lg = lane >> 4;
    const int row = blockIdx.y;                       // b * Hkv + g
    const int b = row / p.Hkv, g = row - b * p.Hkv;
    const int G = p.G;
    const int64_t part = (int64_t)blockIdx.x * kDecodeWaves + wave;
    uint16_t* vw = vlds + wave * kTileKeys * VS;

    const RowSegs r = row_segs(p, b, g);
    const int64_t total = r.na + r.nw + r.ns;
    const int64_t stride = (int64_t)p.parts * kTileKeys;
    const uint8_t* Kr = static_cast<const uint8_t*>(p.K) + (int64_t)row * p.max_len * (D / 2);
    const uint8_t* Vr = static_cast<const uint8_t*>(p.V) + (int64_t)row * p.max_len * (D / 2);
    const uint8_t* Sr = S + (int64_t)row * p.max_len * (D / 16);

    // Q^T as the B operand: lane l holds head l % 16, dims (l / 16) D / 4 + 8 s ..
    u32x4_t qf[SL];
    {
        const bool hv = li < G;
        const uint16_t* qp = static_cast<const uint16_t*>(p.Q) +
                             ((int64_t)b * p.Hq + (int64_t)g * G + (hv ? li : 0)) * D + lg * (D / 4);
        const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int s = 0; s < SL; ++s) {
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(qp + 8 * s);
            qf[s] = hv ? v : zero;
        }
    }

    f32x4_t o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const float c = p.unit;
    float m_run = -FLT_MAX, l_run = 0.f;        // maximum in scores: times c it may leave float32

    const int64_t v_first = part * kTileKeys;
    if (v_first < total) {
        Kv4Tile<D> cur;
        load_tile<D>(r, Kr, Vr, Sr, v_first, li, lg, cur);
        for (int64_t v0 = v_first; v0 < total; v0 += stride) {
            // S^T = K Q^T: lane l holds head l % 16 at key slots 16 kb + 4 (l / 16) + i.
            f32x4_t st[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                st[kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                const float sc = scale_of(cur.ks[kb]);
#pragma unroll
                for (int s = 0; s < SL; ++s)
                    st[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(decode8(cur.k[kb][s], sc)),
                                                                      as_bf16x8(qf[s]), st[kb], 0, 0, 0);
            }
            // V rows as bf16 into this wave's LDS, row-major.  A slot without a key
            // has weight 0, which times a NaN would be one: its row is 0.
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const bool ok = (cur.valid >> (16 * kb + (lane >> 2))) & 1u;
                const float sc = scale_of(ok ? cur.vs[kb] : 127u);
                uint16_t* vr = vw + (16 * kb + (lane >> 2)) * VS + (lane & 3) * (D / 4);
#pragma unroll
                for (int s = 0; s < SL; ++s)
                    *reinterpret_cast<u32x4_t*>(vr + 8 * s) = decode8(ok ? cur.v[kb][s] : 0u, sc);
            }
            const uint32_t valid = cur.valid;
            // the next tile's codes take the registers that these have left
            if (v0 + stride < total) load_tile<D>(r, Kr, Vr, Sr, v0 + stride, li, lg, cur);

            // Online softmax over the tile.
            float sc[2][4];
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool ok = (valid >> (16 * kb + 4 * lg + i)) & 1u;
                    sc[kb][i] = ok ? st[kb][i] : -INFINITY;
                    mx = fmaxf(mx, sc[kb][i]);
                }
            mx = quad_max16(mx);
            // The reference moves, and what was summed is rescaled, only where a score
            // exceeds it by 2^8 in weight.
            if (__any(mx > m_run + slack)) {
                const float m_new = fmaxf(m_run, mx);
                const float alpha = merge_factor(p, m_run, m_new);
                m_run = m_new;
                l_run *= alpha;
                // lane l holds the output of heads 4 (l / 16) + i
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = __shfl(alpha, 4 * lg + i);
#pragma unroll
                    for (int db = 0; db < DB; ++db) o[db][i] *= a;
                }
            }
            float pv[2][4];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    pv[kb][i] = __builtin_amdgcn_exp2f((sc[kb][i] - m_run) * c);
                    l_run += pv[kb][i];
                }

            // P as the A operand: head l % 16, k slots 8 (l / 16) + e hold keys
            // 4 (l / 16) + e (e < 4) and 16 + 4 (l / 16) + e - 4 (e >= 4); V as the B
            // operand with the same key order.
            const u32x4_t pk = {pack_bf16x2(pv[0][0], pv[0][1]), pack_bf16x2(pv[0][2], pv[0][3]),
                                pack_bf16x2(pv[1][0], pv[1][1]), pack_bf16x2(pv[1][2], pv[1][3])};
            const uint16_t* v_lo = vw + (lane >> 2) * VS + 4 * (lane & 3);
            const uint16_t* v_hi = v_lo + 16 * VS;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const uint2 a = lds_read_tr16(v_lo + 16 * db);
                const uint2 e = lds_read_tr16(v_hi + 16 * db);
                const u32x4_t vb = {a.x, a.y, e.x, e.y};
                o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(pk), as_bf16x8(vb), o[db], 0, 0, 0);
            }
        }
    }
    merge_waves<D>(p, row, reinterpret_cast<float*>(vlds), m_run, l_run, o);
}

template <int D>
hipError_t launch_d(const DecodeParams& p, const uint8_t* S, hipStream_t st) {
    const dim3 grid((unsigned)(p.parts / kDecodeWaves), (unsigned)(p.B * p.Hkv));
    if (p.parts % kDecodeWaves != 0 || p.parts > kDecodeMaxParts) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_kv4_decode<D>, grid, dim3(64 * kDecodeWaves), 0, st, p, S,
                       fminf(8.0f / p.unit, FLT_MAX));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || grid.x == 1) return e;
    return launch_decode_combine<D>(p, st);
}

}  // namespace

hipError_t launch_kv4_store(const Kv4Params& p, hipStream_t st) {
    const int per = kThreads / (p.D / 8);
    const dim3 grid((unsigned)((p.T + per - 1) / per), (unsigned)p.Hkv);
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, p); };
    if (p.D == 128) p.bf16 ? run(k_kv4_store<128, true>) : run(k_kv4_store<128, false>);
    else p.bf16 ? run(k_kv4_store<64, true>) : run(k_kv4_store<64, false>);
    return hipGetLastError();
}

hipError_t launch_kv4_load(const Kv4Params& p, hipStream_t st) {
    const int per = kThreads / (p.D / 8);
    const dim3 grid((unsigned)((p.T + per - 1) / per), (unsigned)p.Hkv);
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, p); };
    if (p.D == 128) p.bf16 ? run(k_kv4_load<128, true>) : run(k_kv4_load<128, false>);
    else p.bf16 ? run(k_kv4_load<64, true>) : run(k_kv4_load<64, false>);
    return hipGetLastError();
}

hipError_t launch_kv4_decode(const DecodeParams& p, const uint8_t* S, hipStream_t st) {
    return p.D == 128 ? launch_d<128>(p, S, st) : launch_d<64>(p, S, st);
}

}  // namespace ris
