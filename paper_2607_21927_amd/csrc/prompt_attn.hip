// Dense attention over packed prompts, one running softmax per row.
//
// bf16.  A workgroup takes 128 query rows of one head, a wave 32 of them; the
// keys come in tiles of 64 through LDS.  Both products are
// v_mfma_f32_32x32x16_bf16 with the query as the column, S^T = K Q^T and O^T +=
// V^T P^T, so that lane l holds query l mod 32 in the scores and in the output:
// the row's maximum is one exchange with lane l ^ 32, the rescale none, and the
// scores' registers are the PV product's operand as they stand (its contraction
// order is the order in which the score product leaves the keys; V follows it
// through the transposing LDS read).  K and V go from memory to LDS without
// passing registers (16 bytes a lane, whose place in LDS is fixed by the lane:
// the bank swizzle is in the address it loads from), two tiles deep with one
// barrier a tile.
//
// The reference maximum moves only when a score exceeds it by 2^8 in weight, so
// rescales are rare.  Tiles that no row of a wave cuts are computed without a
// mask.  A masked weight is 0, and 0 times an infinity or NaN of V would be NaN:
// a workgroup whose output is not finite goes over its keys once more, with
// such elements of V taken out of the tiles that the mask cuts and added where
// they are attended to.
#include <type_traits>

#include "packed.h"
#include "ris_internal.h"

namespace ris {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kRows = 128;        // query rows of a workgroup
constexpr int kKeys = 64;         // keys of a tile
constexpr int kWaves = 4;

// 16-byte chunk c of row r of a K or V tile lies in place c ^ swizzle(r): 16 rows
// at one chunk (a K read) and 4 rows at four chunks (a transposing V read) both
// spread over all banks.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
    return D == 128 ? ((r & 3) << 2 | (r >> 2 & 3)) : ((r >> 1 & 1) << 2 | (r >> 2 & 3));
}

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

// A lane's part in a tile: 16-byte pieces, piece i at place 256 i + thread of the tile
// in LDS.  Their rows are kStep apart, a multiple of the swizzle's period, so all
// have one chunk and one offset in the row.
template <int D>
struct Piece {
    static constexpr int kCount = kKeys * (D / 8) / (64 * kWaves);
    static constexpr int kStep = kKeys / kCount;
    static_assert(kStep % 16 == 0, "the swizzle repeats every 16 rows");
    int row;            // of piece 0
    uint32_t chunk;     // bytes into the row
    __device__ __forceinline__ Piece() : row((int)threadIdx.x / (D / 8)) {
        chunk = 16u * ((threadIdx.x % (D / 8)) ^ swizzle<D>(row));
    }
};

// Keys [j0, j0 + 64) of x (rows of the sequence, `tok` elements apart) into LDS;
// keys from n on repeat the last one.  (Offsets within a tile fit 32 bits: the host
// refuses rows farther apart.)
template <int D>
__device__ __forceinline__ void load_tile(const Piece<D>& pc, const uint16_t* x, int64_t tok, int j0, int n, uint16_t* lds) {
    uint16_t* to = lds + (threadIdx.x & ~63u) * 8;      // the wave's places
    const char* from = reinterpret_cast<const char*>(x + j0 * tok);
    const uint32_t step = 2u * (uint32_t)tok;
    if (j0 + kKeys <= n) {
        const uint32_t off = pc.row * step + pc.chunk;
#pragma unroll
        for (int i = 0; i < Piece<D>::kCount; ++i)
            __builtin_amdgcn_global_load_lds((gptr_t)(from + (uint64_t)(i * Piece<D>::kStep) * step + off),
                                             (lptr_t)(to + 64 * kWaves * 8 * i), 16, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < Piece<D>::kCount; ++i) {
            const int r = pc.row + i * Piece<D>::kStep < n - j0 ? pc.row + i * Piece<D>::kStep : n - 1 - j0;
            __builtin_amdgcn_global_load_lds((gptr_t)(from + (uint32_t)(r * step + pc.chunk)), (lptr_t)(to + 64 * kWaves * 8 * i),
                                             16, 0, 0);
        }
    }
}

__device__ __forceinline__ bool odd_half(uint32_t u) { return (u & 0x7F80u) == 0x7F80u; }   // infinity or NaN
__device__ __forceinline__ uint32_t finite_only(uint32_t u) {
    return (odd_half(u) ? 0u : u & 0xFFFFu) | (odd_half(u >> 16) ? 0u : u & 0xFFFF0000u);
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void k_prompt_bf16(PromptParams p) {
    constexpr int SL = D / 16;      // contraction steps of the score product
    constexpr int DB = D / 32;      // 32-dim blocks of the output
    // two tiles of K and of V; arrays of their own, so that a load into one is not
    // taken for a write to another
    __shared__ __align__(16) uint16_t k0[kKeys * D], k1[kKeys * D], v0[kKeys * D], v1[kKeys * D];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lq = lane & 31, lh = lane >> 5;
    // The heads of a group take the same tile one after another on one XCD, so
    // that its L2 serves their K and V.
    const uint32_t xcd = blockIdx.x & 7u, slot = blockIdx.x >> 3;
    const uint32_t unit = slot / p.G * 8u + xcd;
    const int g = (int)(unit % p.Hkv), h = g * p.G + (int)(slot % p.G);
    RowTile t;
    if (!find_tile(p.cu, p.batch, p.T, kRows, unit / p.Hkv, t)) return;
    const int n = t.len, q0 = t.tile * kRows + 32 * wave, row = q0 + lq;

    const uint16_t* K = static_cast<const uint16_t*>(p.K) + g * p.k_head + t.first * p.k_token;
    const uint16_t* V = static_cast<const uint16_t*>(p.V) + g * p.v_head + t.first * p.v_token;

    const Piece<D> pc;

    // Q^T as the B operand: lane l holds query l % 32, dims 16 s + 8 (l / 32) ..
    u32x4_t qf[SL];
    {
        const int r = row < n ? row : n - 1;
        const uint16_t* qp = static_cast<const uint16_t*>(p.Q) + h * p.q_head + (t.first + r) * p.q_token + 8 * lh;
#pragma unroll
        for (int s = 0; s < SL; ++s) qf[s] = *reinterpret_cast<const u32x4_t*>(qp + 16 * s);
    }

    const int last = p.causal ? (row < n ? row : n - 1) : n - 1;        // last key of the lane's row
    const int wlast = p.causal ? (q0 + 31 < n ? q0 + 31 : n - 1) : n - 1;
    const int wfull = p.causal ? q0 : n - 1;                            // keys up to here: every row's
    const int kend = p.causal && (t.tile + 1) * kRows < n ? (t.tile + 1) * kRows : n;
    const int tiles = (kend + kKeys - 1) / kKeys;

    f32x16_t o[DB];
    float m = -INFINITY, mc = 0.f, l = 0.f;      // reference maximum in scores; times c, 0 while there is none; sum

    // One tile of keys: kCut where the mask cuts it, kSafe where V may hold
    // infinities or NaN under the mask.
    const auto compute = [&](auto cut, auto safe, const uint16_t* kl, const uint16_t* vl, int j0) __attribute__((always_inline)) {
        constexpr bool kCut = decltype(cut)::value, kSafe = decltype(safe)::value;
        // S^T: lane l holds query l % 32 at keys 32 b + 8 (i / 4) + 4 (l / 32) + i % 4.
        f32x16_t st[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st[b][i] = 0.f;
#pragma unroll
            for (int s = 0; s < SL; ++s) {
                const u32x4_t a = *reinterpret_cast<const u32x4_t*>(kl + (32 * b + lq) * D + 8 * ((2 * s + lh) ^ swizzle<D>(lq)));
                st[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(qf[s]), st[b], 0, 0, 0);
            }
        }
        if constexpr (kCut) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (j0 + 32 * b + 8 * (i / 4) + 4 * lh + i % 4 > last) st[b][i] = -INFINITY;
        }
        float mx = st[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[b][i]);
        mx = pair_max32(mx);
        if (__any(mx > m + p.slack)) {
            const bool none = m == -INFINITY;                      // nothing summed yet: o and l are 0
            m = fmaxf(m, mx);
            const float nc = m == -INFINITY ? 0.f : m * p.c;
            const float al = none ? 0.f : __builtin_amdgcn_exp2f(mc - nc);
            mc = nc;
            l *= al;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= al;
        }
        u32x4_t pf[4];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = __builtin_amdgcn_exp2f(fmaf(st[b][i], p.c, -mc));
                const float y = __builtin_amdgcn_exp2f(fmaf(st[b][i + 1], p.c, -mc));
                l += x + y;
                pf[2 * b + i / 8][i % 8 / 2] = pack_bf16x2(x, y);
            }
        // O^T += V^T P^T over 16 keys at a time: slot e of lane half lh holds
        // key 16 u + 4 lh + e (e < 4) or 16 u + 8 + 4 lh + e - 4.
        const int r0 = 4 * lh + ((lane & 15) >> 2), cq = 2 * (lane >> 4 & 1) + ((lane & 3) >> 1);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int c = 4 * d + cq;
                const uint2 a = lds_read_tr16(vl + (16 * u + r0) * D + 8 * (c ^ swizzle<D>(r0)) + 4 * (lane & 1));
                const uint2 b = lds_read_tr16(vl + (16 * u + r0 + 8) * D + 8 * (c ^ swizzle<D>(r0 + 8)) + 4 * (lane & 1));
                u32x4_t v = {a.x, a.y, b.x, b.y};
                if constexpr (kSafe) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = finite_only(v[i]);
                }
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pf[u]), o[d], 0, 0, 0);
            }
        if constexpr (kSafe) {
            for (int r = 0; r < kKeys; ++r)
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int dim = 32 * d + 8 * (i / 4) + 4 * lh + i % 4;
                        const uint16_t v = vl[r * D + 8 * ((dim >> 3) ^ swizzle<D>(r)) + (dim & 7)];
                        if (odd_half(v) && j0 + r <= last) o[d][i] += bf16_to_f32(v);
                    }
        }
    };
    // All keys: tile `it` is computed from one pair of arrays while tile `it` + 1
    // is on its way into the other.
    const auto pass = [&](auto safe) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        load_tile<D>(pc, K, p.k_token, 0, n, k0);
        load_tile<D>(pc, V, p.v_token, 0, n, v0);
        const auto step = [&](int it, const uint16_t* kl, const uint16_t* vl, uint16_t* kn, uint16_t* vn) __attribute__((always_inline)) {
            const int j0 = it * kKeys;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (it + 1 < tiles) {
                load_tile<D>(pc, K, p.k_token, j0 + kKeys, n, kn);
                load_tile<D>(pc, V, p.v_token, j0 + kKeys, n, vn);
            }
            if (q0 >= n || j0 > wlast) return;
            if (j0 + kKeys - 1 > wfull) compute(std::true_type{}, safe, kl, vl, j0);
            else compute(std::false_type{}, std::false_type{}, kl, vl, j0);
        };
        for (int it = 0; it < tiles; it += 2) {
            step(it, k0, v0, k1, v1);
            if (it + 1 < tiles) step(it + 1, k1, v1, k0, v0);
        }
    };
    pass(std::false_type{});
    float odd = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = fmaf(o[d][i], 0.f, odd);       // NaN if any is not finite
    if (__syncthreads_or(odd != odd && row < n)) {
        m = -INFINITY;
        mc = l = 0.f;
        pass(std::true_type{});
    }
    l = pair_sum32(l);
    if (row >= n) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t at = h * p.o_head + (t.first + row) * p.o_token + 4 * lh;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t e = at + 32 * d + 8 * i;
            const float y0 = o[d][4 * i] * inv, y1 = o[d][4 * i + 1] * inv, y2 = o[d][4 * i + 2] * inv,
                        y3 = o[d][4 * i + 3] * inv;
            if (p.out_bf16)
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + e) = make_uint2(pack_bf16x2(y0, y1), pack_bf16x2(y2, y3));
            else
                *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + e) = f32x4_t{y0, y1, y2, y3};
        }
}

// float32: the same layouts on v_mfma_f32_32x32x2_f32, 32 keys to a tile.  The
// score product takes four dims of a key from one 16-byte read (lane half lh:
// dims 8 s + 4 lh ..), the PV product takes score register i as it stands (its two
// contraction slots are the keys of the lane halves).  64 rows (two waves) to a
// workgroup: the products, 16 times slower than bf16's, hide the rest, and short
// prompts still give many workgroups.
constexpr int kRows32 = 64, kKeys32 = 32, kWaves32 = 2;

template <int D>
__global__ __launch_bounds__(64 * kWaves32, 2) void k_prompt_f32(PromptParams p) {
    constexpr int DB = D / 32;
    constexpr int KS = D + 4;       // K row stride: 16-byte reads of 8 rows meet every bank once
    __shared__ __align__(16) float kl[kKeys32 * KS];
    __shared__ __align__(16) float vl[kKeys32 * D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lq = lane & 31, lh = lane >> 5;
    const uint32_t xcd = blockIdx.x & 7u, slot = blockIdx.x >> 3;
    const uint32_t unit = slot / p.G * 8u + xcd;
    const int g = (int)(unit % p.Hkv), h = g * p.G + (int)(slot % p.G);
    RowTile t;
    if (!find_tile(p.cu, p.batch, p.T, kRows32, unit / p.Hkv, t)) return;
    const int n = t.len, q0 = t.tile * kRows32 + 32 * wave, row = q0 + lq;
    const float* K = static_cast<const float*>(p.K) + g * p.k_head + t.first * p.k_token;
    const float* V = static_cast<const float*>(p.V) + g * p.v_head + t.first * p.v_token;
    f32x4_t qf[D / 8];
    {
        const int r = row < n ? row : n - 1;
        const float* qp = static_cast<const float*>(p.Q) + h * p.q_head + (t.first + r) * p.q_token + 4 * lh;
#pragma unroll
        for (int s = 0; s < D / 8; ++s) qf[s] = *reinterpret_cast<const f32x4_t*>(qp + 8 * s);
    }
    const int last = p.causal ? (row < n ? row : n - 1) : n - 1;
    const int wlast = p.causal ? (q0 + 31 < n ? q0 + 31 : n - 1) : n - 1;
    const int wfull = p.causal ? q0 : n - 1;
    const int kend = p.causal && (t.tile + 1) * kRows32 < n ? (t.tile + 1) * kRows32 : n;
    const int tiles = (kend + kKeys32 - 1) / kKeys32;
    f32x16_t o[DB];
    float m, l;
    for (int safe = 0;; safe = 1) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        m = -INFINITY;
        float mc = 0.f;
        l = 0.f;
        for (int it = 0; it < tiles; ++it) {
            const int j0 = it * kKeys32;
            __syncthreads();
#pragma unroll
            for (int e = threadIdx.x; e < kKeys32 * D / 4; e += 64 * kWaves32) {
                const int r = e / (D / 4), c = 4 * (e % (D / 4)), j = j0 + r < n ? j0 + r : n - 1;
                *reinterpret_cast<f32x4_t*>(kl + r * KS + c) = *reinterpret_cast<const f32x4_t*>(K + j * p.k_token + c);
                *reinterpret_cast<f32x4_t*>(vl + r * D + c) = *reinterpret_cast<const f32x4_t*>(V + j * p.v_token + c);
            }
            __syncthreads();
            if (q0 >= n || j0 > wlast) continue;
            f32x16_t st;
#pragma unroll
            for (int i = 0; i < 16; ++i) st[i] = 0.f;
#pragma unroll
            for (int s = 0; s < D / 8; ++s) {
                const f32x4_t a = *reinterpret_cast<const f32x4_t*>(kl + lq * KS + 8 * s + 4 * lh);
#pragma unroll
                for (int e = 0; e < 4; ++e) st = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], qf[s][e], st, 0, 0, 0);
            }
            const bool cut = j0 + kKeys32 - 1 > wfull;
            if (cut) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (j0 + 8 * (i / 4) + 4 * lh + i % 4 > last) st[i] = -INFINITY;
            }
            float mx = st[0];
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[i]);
            mx = pair_max32(mx);
            if (__any(mx > m + p.slack)) {
                const bool none = m == -INFINITY;
                m = fmaxf(m, mx);
                const float nc = m == -INFINITY ? 0.f : m * p.c;
                const float al = none ? 0.f : __builtin_amdgcn_exp2f(mc - nc);
                mc = nc;
                l *= al;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= al;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                st[i] = __builtin_amdgcn_exp2f(fmaf(st[i], p.c, -mc));
                l += st[i];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = 8 * (i / 4) + 4 * lh + i % 4;
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    float v = vl[r * D + 32 * d + lq];
                    if (safe && cut && !isfinite(v)) v = 0.f;
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, st[i], o[d], 0, 0, 0);
                }
            }
            if (safe && cut)
                for (int r = 0; r < kKeys32; ++r)
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float v = vl[r * D + 32 * d + 8 * (i / 4) + 4 * lh + i % 4];
                            if (!isfinite(v) && j0 + r <= last) o[d][i] += v;
                        }
        }
        float odd = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) odd = fmaf(o[d][i], 0.f, odd);
        if (!__syncthreads_or(odd != odd && row < n && !safe)) break;
    }
    l = pair_sum32(l);
    if (row >= n) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t at = h * p.o_head + (t.first + row) * p.o_token + 4 * lh;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t e = at + 32 * d + 8 * i;
            const float y0 = o[d][4 * i] * inv, y1 = o[d][4 * i + 1] * inv, y2 = o[d][4 * i + 2] * inv,
                        y3 = o[d][4 * i + 3] * inv;
            if (p.out_bf16)
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + e) = make_uint2(pack_bf16x2(y0, y1), pack_bf16x2(y2, y3));
            else
                *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + e) = f32x4_t{y0, y1, y2, y3};
        }
}

}  // namespace

int64_t prompt_blocks(int64_t T, int batch, int Hkv, int G, int in_bf16) {
    const int rows = in_bf16 ? kRows : kRows32;
    const int64_t tiles = (T + (int64_t)batch * (rows - 1)) / rows;     // sequences end inside their last tile
    return (tiles * Hkv + 7) / 8 * 8 * G;
}

hipError_t launch_prompt_attn(const PromptParams& p, hipStream_t st) {
    const dim3 grid((unsigned)prompt_blocks(p.T, p.batch, p.Hkv, p.G, p.in_bf16));
    if (p.in_bf16) {
        if (p.D == 128) hipLaunchKernelGGL(k_prompt_bf16<128>, grid, dim3(64 * kWaves), 0, st, p);
        else hipLaunchKernelGGL(k_prompt_bf16<64>, grid, dim3(64 * kWaves), 0, st, p);
    } else {
        if (p.D == 128) hipLaunchKernelGGL(k_prompt_f32<128>, grid, dim3(64 * kWaves32), 0, st, p);
        else hipLaunchKernelGGL(k_prompt_f32<64>, grid, dim3(64 * kWaves32), 0, st, p);
    }
    return hipGetLastError();
}

}  // namespace ris
