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
// rescales are rare.  A weight of 0, masked or too small for float32, times an infinity
// or NaN of V would be NaN: a workgroup whose output is not finite goes over its keys
// once more, with such elements of V taken out of the tiles and added, whatever their
// weight, where they are attended to.  So does one with a reference far from 0 (see Ref).
//
// Weights enter the PV product as bf16, the type in which the matrix unit takes V (a
// product in float32 would be 16 times slower): each is off by 2^-8 of itself at most, their
// sum is taken in float32 before that.  Nine prompts of 32k tokens are off by 2.1e-3 of the
// outputs' norm, of which rounding the outputs to bf16 alone makes 1.6e-3.
//
// Bound by how well the matrix unit and the vector unit share the waves' time: one prompt
// of 32k tokens keeps them 61% and 39% busy at D = 128 (two waves a SIMD, 1.07 PFLOP/s), 49%
// and 58% at D = 64 (three), LDS 30% and 24%, without bank conflicts, at 1.8 GHz.  At D =
// 128 the next tile's scores stand beside this one's exponentials in one block, the
// products and reads spread through it (1071 -> 1106 TFLOP/s on one machine, 12/2 heads, 32k
// tokens); at D = 64, where exponentials take longer than products, three waves a
// SIMD without that gain more (975 against 937).  Not kept: row sums on v_dot2 (the
// same), the next maximum carried along (the same), raised priority in the PV product
// (-6%), waits placed by hand (the same), 64 rows a wave with each LDS fragment in two
// products (996 against 949 at D = 64 in a kernel of its own; 680 against 1101 at D =
// 128: one wave a SIMD, scores copied out of accumulation registers).
#include <type_traits>

#include "packed.h"
#include "ris_internal.h"

namespace ris {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kRows = 128;        // query rows of a workgroup
constexpr int kNarrowRows = 32;   // of the narrow form's
constexpr int kShortRows = 32;    // of a wave of the short form
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
    __device__ __forceinline__ Piece() : row((int)(threadIdx.x & (64 * kWaves - 1)) / (D / 8)) {
        chunk = 16u * ((threadIdx.x % (D / 8)) ^ swizzle<D>(row));
    }
};

// Keys [j0, j0 + 64) of x (rows of the sequence, `tok` elements apart) into LDS;
// keys from n on repeat the last one.  (Offsets within a tile fit 32 bits: the host
// refuses rows farther apart.)
template <int D>
__device__ __forceinline__ void load_tile(const Piece<D>& pc, const uint16_t* x, int64_t tok, int j0, int n, uint16_t* lds) {
    uint16_t* to = lds + (threadIdx.x & (64 * kWaves - 64)) * 8;      // the wave's places
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

// Four neighbouring elements of out.
__device__ __forceinline__ void store4(const PromptParams& p, int64_t at, float a, float b, float c, float d) {
    if (p.out_bf16)
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
    else
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) = f32x4_t{a, b, c, d};
}

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
// meet under the largest, top (topc); far: one of theirs is.
template <bool kF32>
__device__ __forceinline__ float join_factor(float m, float mc, float top, float topc, bool far, float c) {
    return m == -INFINITY ? 0.f : pow2<kF32>(far ? (m - top) * c : mc - topc);
}

template <int D, int S>
__global__ __launch_bounds__(64 * kWaves * S, D == 64 ? 3 : 2) void k_prompt_bf16(PromptParams p) {
    constexpr int SL = D / 16;      // contraction steps of the score product
    constexpr int DB = D / 32;      // 32-dim blocks of the output
    constexpr bool kPipe = D == 128;
    // two tiles of K and of V; arrays of their own, so that a load into one is not
    // taken for a write to another
    __shared__ __align__(16) uint16_t k0s[S * kKeys * D], k1s[S * kKeys * D], v0s[S * kKeys * D], v1s[S * kKeys * D];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6 & (kWaves - 1);               // wave: row block
    const int group = S == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * kWaves));   // of keys
    const int lq = lane & 31, lh = lane >> 5;
    uint16_t* const k0 = k0s + group * kKeys * D;
    uint16_t* const k1 = k1s + group * kKeys * D;
    uint16_t* const v0 = v0s + group * kKeys * D;
    uint16_t* const v1 = v1s + group * kKeys * D;
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
    Ref<false> ref;
    float l;

    // S^T of a tile: lane l holds query l % 32 at keys 32 b + 8 (i / 4) + 4 (l / 32) + i % 4.
    const auto scores = [&](const uint16_t* kl, f32x16_t (&st)[2]) __attribute__((always_inline)) {
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
    };
    // The tile at j0 from its scores `st` and values `vl`, with the next tile's scores
    // `nx` from `kn` beside it (kMore).  kSafe: V may hold infinities or NaN.
    const auto compute = [&](auto more, auto safe, f32x16_t (&st)[2], f32x16_t (&nx)[2], const uint16_t* kn, const uint16_t* vl,
                             int j0) __attribute__((always_inline)) {
        constexpr bool kMore = decltype(more)::value, kSafe = decltype(safe)::value;
        if (j0 + kKeys - 1 > wfull) {
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
        if (__any(mx > ref.m + p.slack)) {
            const float al = ref.template raise<kSafe>(mx, p.c);
            l *= al;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] = scaled<kSafe>(o[d][i], al);
        }
        if constexpr (kMore) scores(kn, nx);
        u32x4_t pf[4];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = ref.template weight<kSafe>(st[b][i], p.c);
                const float y = ref.template weight<kSafe>(st[b][i + 1], p.c);
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
        if constexpr (kMore) {
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int i = 0; i < 2 * SL; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
            }
#pragma unroll
            for (int i = 0; i < 4 * DB; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            }
        }
        if constexpr (kSafe) {
            if (any_odd<kKeys * D>(vl))
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
    // All of the group's keys, its i-th tile being tile S i + group.  While one is
    // computed, the next is on its way; where kPipe, K of the next is there already for
    // its scores, and K of the one after that and V of the next are on their way.
    const int rounds = (tiles + S - 1) / S;
    const int have = (tiles - group + S - 1) / S;                   // the group's tiles
    const int mine = q0 < n ? (wlast / kKeys + S - group) / S : 0;  // those that the wave's rows attend to
    const auto pass = [&](auto safe) __attribute__((always_inline)) {
        constexpr bool kSafe = decltype(safe)::value;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        ref.reset();
        l = 0.f;
        if (have > 0) {
            load_tile<D>(pc, K, p.k_token, group * kKeys, n, k0);
            load_tile<D>(pc, V, p.v_token, group * kKeys, n, v0);
        }
        if (kPipe && have > 1) load_tile<D>(pc, K, p.k_token, (S + group) * kKeys, n, k1);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        f32x16_t sa[2], sb[2];
        if (kPipe && mine > 0) scores(k0, sa);
        const auto step = [&](int it, f32x16_t (&st)[2], f32x16_t (&nx)[2], uint16_t* kl, const uint16_t* vl, uint16_t* kn,
                              uint16_t* vn) __attribute__((always_inline)) {
            const int j0 = (S * it + group) * kKeys;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (it + 1 < have) load_tile<D>(pc, V, p.v_token, j0 + S * kKeys, n, vn);
            if constexpr (!kPipe) {
                if (it + 1 < have) load_tile<D>(pc, K, p.k_token, j0 + S * kKeys, n, kn);
                if (it < mine) {
                    scores(kl, st);
                    compute(std::false_type{}, safe, st, nx, kn, vl, j0);
                }
                return;
            }
            if (it + 2 < have) load_tile<D>(pc, K, p.k_token, j0 + 2 * S * kKeys, n, kl);
            if (it + 1 < mine) compute(std::true_type{}, safe, st, nx, kn, vl, j0);
            else if (it < mine) compute(std::false_type{}, safe, st, nx, kn, vl, j0);
        };
        for (int it = 0; it < rounds; it += 2) {
            step(it, sa, sb, k0, v0, k1, v1);
            if (it + 1 < rounds) step(it + 1, sb, sa, k1, v1, k0, v0);
        }
        if constexpr (S == 2) {
            // The second group's state joins the first's, through its own tiles' places.
            __syncthreads();
            float* mem[DB] = {};
            uint16_t* const place[4] = {k0s, k1s, v0s, v1s};         // S kKeys D elements each: 64 D floats
#pragma unroll
            for (int d = 0; d < DB; ++d) mem[d] = reinterpret_cast<float*>(place[d]) + wave * 16 * 64 + lane;
            __shared__ float ml[kWaves][3][64];
            if (group == 1) {
                ml[wave][0][lane] = ref.m;
                ml[wave][1][lane] = ref.mc;
                ml[wave][2][lane] = l;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) mem[d][64 * i] = o[d][i];
            }
            __syncthreads();
            if (group == 0) {
                const float m1 = ml[wave][0][lane], mc1 = ml[wave][1][lane], top = fmaxf(ref.m, m1), topc = ref.m < m1 ? mc1 : ref.mc;
                const bool far = far_ref(ref.mc) || far_ref(mc1);
                const float a = join_factor<false>(ref.m, ref.mc, top, topc, far, p.c), a1 = join_factor<false>(m1, mc1, top, topc, far, p.c);
                l = fmaf(ml[wave][2][lane], a1, l * a);
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] = add_scaled<kSafe>(scaled<kSafe>(o[d][i], a), mem[d][64 * i], a1);
            }
        }
    };
    pass(std::false_type{});
    float odd = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = fmaf(o[d][i], 0.f, odd);       // NaN if any is not finite
    if (__syncthreads_or((ref.needs_apart(l) || odd != odd) && row < n)) {
        pass(std::true_type{});
    }
    l = pair_sum32(l);
    if (row >= n || group != 0) return;
    const float inv = 1.f / l;              // every score -inf: 0 / 0, NaN
    const int64_t at = h * p.o_head + (t.first + row) * p.o_token + 4 * lh;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store4(p, at + 32 * d + 8 * i, o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv);
}

// The states of a workgroup's four waves, each over its own keys of the same 32 rows,
// to the rows' outputs (kSafe: after a second pass).  mem: room for [wave][dim
// block][register][lane], a wave's in its K tile's place; ml: 256 floats a wave, kTile
// apart, in its V tile's place.  A wave stores the dims of four registers of every 16 (8 of
// a row's 32).
template <int D, int kTile, bool kSafe, bool kF32>
__device__ __forceinline__ void join_waves(const PromptParams& p, float* mem, float* ml, const Ref<kF32>& ref, float l,
                                           const f32x16_t (&o)[D / 32], const RowTile& t, int row, int h) {
    constexpr int DB = D / 32;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lh = lane >> 5;
    mem += lane;
    ml += lane;
    ml[wave * kTile] = ref.m;
    ml[wave * kTile + 64] = pair_sum32(l);
    ml[wave * kTile + 192] = ref.mc;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) mem[((wave * DB + d) * 16 + i) * 64] = o[d][i];
    __syncthreads();
    if (row >= t.len) return;
    float top = -INFINITY, topc = 0.f, a[kWaves], sum = 0.f;
    bool far = false;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float m = ml[w * kTile], mc = ml[w * kTile + 192];
        topc = top < m ? mc : topc;
        top = fmaxf(top, m);
        far |= kSafe && far_ref(mc);
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        a[w] = join_factor<kF32>(ml[w * kTile], ml[w * kTile + 192], top, topc, far, p.c);
        sum = fmaf(a[w], ml[w * kTile + 64], sum);
    }
    const float inv = 1.f / sum;            // every score -inf: 0 / 0, NaN
    const int64_t at = h * p.o_head + (t.first + row) * p.o_token + 4 * lh + 8 * wave;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) y[i] = add_scaled<kSafe>(y[i], mem[((w * DB + d) * 16 + 4 * wave + i) * 64], a[w]);
        }
        store4(p, at + 32 * d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    }
}

// Whether any lane of the workgroup's waves says so; mem as join_waves' ml.  (The
// library's vote has a shared array of its own, beside which the compiler cannot tell
// K and V tiles apart.)
template <int kTile>
__device__ __forceinline__ bool any_wave(bool x, float* mem) {
    const bool any = __any(x);
    if ((threadIdx.x & 63) == 0) mem[(threadIdx.x >> 6) * kTile + 128] = any ? 1.f : 0.f;
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += mem[w * kTile + 128];
    return sum > 0.f;
}

// The same for batches too small to fill the chip with 128-row workgroups: a
// workgroup takes 32 rows, and its four waves every fourth tile of keys each, in
// places of their own (one K and one V tile a wave, no barrier: the next K tile is
// loaded once the scores have read this one, the next V tile once the output has).
// The waves' states meet at the end, each wave taking a quarter of the output.
//
// The compiler waits for every load before a read of LDS that one of them may write,
// unless it can tell them apart: hence no load under a condition in the loop, tiles that
// are restrict parameters, and one shared array in the kernel (two have marks of their
// own, which these replace).  4 to 10% for one prompt of 1,500 to 3,000 tokens.
template <int D>
__global__ __launch_bounds__(64 * kWaves, D == 128 ? 1 : 2) void k_prompt_narrow(PromptParams p) {
    constexpr int SL = D / 16, DB = D / 32, C = D / 8;
    constexpr int kPieces = kKeys * C / 64, kPer = 64 / C;        // 16-byte pieces of a lane, rows of a piece
    __shared__ __align__(16) uint16_t lds[2 * kWaves * kKeys * D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lq = lane & 31, lh = lane >> 5;
    const uint32_t xcd = blockIdx.x & 7u, slot = blockIdx.x >> 3;
    const uint32_t unit = slot / p.G * 8u + xcd;
    const int g = (int)(unit % p.Hkv), h = g * p.G + (int)(slot % p.G);
    RowTile t;
    if (!find_tile(p.cu, p.batch, p.T, kNarrowRows, unit / p.Hkv, t)) return;
    const int n = t.len, q0 = t.tile * kNarrowRows, row = q0 + lq;
    const uint16_t* K = static_cast<const uint16_t*>(p.K) + g * p.k_head + t.first * p.k_token;
    const uint16_t* V = static_cast<const uint16_t*>(p.V) + g * p.v_head + t.first * p.v_token;
    uint16_t* const kl = lds + wave * kKeys * D;
    uint16_t* const vl = kl + kWaves * kKeys * D;

    const auto load = [&](const uint16_t* x, int64_t tok, int j0, uint16_t* to) __attribute__((always_inline)) {
        const char* from = reinterpret_cast<const char*>(x + j0 * tok);
        const uint32_t step = 2u * (uint32_t)tok;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int r = kPer * i + lane / C, rr = r < n - j0 ? r : n - 1 - j0;
            __builtin_amdgcn_global_load_lds((gptr_t)(from + (uint32_t)(rr * step + 16 * (lane % C ^ swizzle<D>(r)))),
                                             (lptr_t)(to + 64 * 8 * i), 16, 0, 0);
        }
    };
    const int last = p.causal ? (row < n ? row : n - 1) : n - 1;
    const int kend = p.causal && q0 + kNarrowRows < n ? q0 + kNarrowRows : n;
    const int wfull = p.causal ? q0 : n - 1;
    const int tiles = (kend + kKeys - 1) / kKeys;
    u32x4_t qf[SL];
    {
        const int r = row < n ? row : n - 1;
        const uint16_t* qp = static_cast<const uint16_t*>(p.Q) + h * p.q_head + (t.first + r) * p.q_token + 8 * lh;
#pragma unroll
        for (int s = 0; s < SL; ++s) qf[s] = *reinterpret_cast<const u32x4_t*>(qp + 16 * s);
    }
    f32x16_t o[DB];
    Ref<false> ref;
    float l;
    const int r0 = 4 * lh + ((lane & 15) >> 2), cq = 2 * (lane >> 4 & 1) + ((lane & 3) >> 1);
    // kSafe: V may hold infinities or NaN
    const auto pass = [&](auto safe, uint16_t* __restrict__ kt, uint16_t* __restrict__ vt) __attribute__((always_inline)) {
        constexpr bool kSafe = decltype(safe)::value;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        ref.reset();
        l = 0.f;
        // kMore: the wave has a tile after this one
        const auto step = [&](auto more, int it) __attribute__((always_inline)) {
            constexpr bool kMore = decltype(more)::value;
            const int j0 = it * kKeys, jn = j0 + kWaves * kKeys;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kPieces) : "memory");       // K; V may still be on its way
            f32x16_t st[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) st[b][i] = 0.f;
#pragma unroll
                for (int s = 0; s < SL; ++s) {
                    const u32x4_t a = *reinterpret_cast<const u32x4_t*>(kt + (32 * b + lq) * D + 8 * ((2 * s + lh) ^ swizzle<D>(lq)));
                    st[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(qf[s]), st[b], 0, 0, 0);
                }
            }
            if (j0 + kKeys - 1 > wfull) {
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
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // every read of K has returned
            if constexpr (kMore) load(K, p.k_token, jn, kt);
            if (__any(mx > ref.m + p.slack)) {
                const float al = ref.template raise<kSafe>(mx, p.c);
                l *= al;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] = scaled<kSafe>(o[d][i], al);
            }
            u32x4_t pf[4];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float x = ref.template weight<kSafe>(st[b][i], p.c);
                    const float y = ref.template weight<kSafe>(st[b][i + 1], p.c);
                    l += x + y;
                    pf[2 * b + i / 8][i % 8 / 2] = pack_bf16x2(x, y);
                }
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMore ? kPieces : 0) : "memory");      // V; not the next K
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const int c = 4 * d + cq;
                    const uint2 a = lds_read_tr16(vt + (16 * u + r0) * D + 8 * (c ^ swizzle<D>(r0)) + 4 * (lane & 1));
                    const uint2 b = lds_read_tr16(vt + (16 * u + r0 + 8) * D + 8 * (c ^ swizzle<D>(r0 + 8)) + 4 * (lane & 1));
                    u32x4_t v = {a.x, a.y, b.x, b.y};
                    if constexpr (kSafe) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = finite_only(v[i]);
                    }
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pf[u]), o[d], 0, 0, 0);
                }
            if (kSafe && any_odd<kKeys * D>(vt))
                for (int r = 0; r < kKeys; ++r)
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int dim = 32 * d + 8 * (i / 4) + 4 * lh + i % 4;
                            const uint16_t v = vt[r * D + 8 * ((dim >> 3) ^ swizzle<D>(r)) + (dim & 7)];
                            if (odd_half(v) && j0 + r <= last) o[d][i] += bf16_to_f32(v);
                        }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // every read of V has returned
            if constexpr (kMore) load(V, p.v_token, jn, vt);
        };
        if (wave >= tiles) return;
        load(K, p.k_token, wave * kKeys, kt);
        load(V, p.v_token, wave * kKeys, vt);
        int it = wave;
        for (; it + kWaves < tiles; it += kWaves) step(std::true_type{}, it);
        step(std::false_type{}, it);
    };
    pass(std::false_type{}, kl, vl);
    float odd = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = fmaf(o[d][i], 0.f, odd);
    float* const vf = reinterpret_cast<float*>(lds + kWaves * kKeys * D);
    const bool again = any_wave<kKeys * D / 2>((ref.needs_apart(l) || odd != odd) && row < n, vf);
    if (again) {
        __syncthreads();
        pass(std::true_type{}, kl, vl);
        join_waves<D, kKeys * D / 2, true>(p, reinterpret_cast<float*>(lds), vf, ref, l, o, t, row, h);
    } else {
        join_waves<D, kKeys * D / 2, false>(p, reinterpret_cast<float*>(lds), vf, ref, l, o, t, row, h);
    }
}

// The same for many prompts of a few tokens: a tile is 32 neighbouring tokens, of as
// many prompts as they belong to, and a row's keys are the interval from its prompt's
// first token on, so that tiles stay full however short prompts are.  A wave takes one
// tile of one head by itself (heads of a tile side by side on one XCD), 32 keys at a
// time from its rows' first to their last, K and V as in the narrow form.  10,000 prompts
// of 8 tokens (12/2 heads of 128) take 175 us, 1.5 times a copy of their bytes.
constexpr int kShortKeys = 32;

template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void k_prompt_short(PromptParams p) {
    constexpr int SL = D / 16, DB = D / 32, C = D / 8;
    constexpr int kPieces = kShortKeys * C / 64, kPer = 64 / C;
    __shared__ __align__(16) uint16_t lds[2 * kWaves * kShortKeys * D];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lq = lane & 31, lh = lane >> 5;
    const uint32_t unit = (blockIdx.x >> 3) * kWaves + wave, tile = unit / p.Hq * 8u + (blockIdx.x & 7u);
    const int h = (int)(unit % p.Hq), g = h / p.G;
    const int64_t first = (int64_t)tile * kShortRows;
    if (first >= p.T) return;
    const int t = (int)first + lq;                     // the lane's row
    int b = find_seq(p.cu, p.batch, first);
    b = seq_from(p.cu, p.batch, b < 0 ? 0 : b, t);
    const bool in = t < p.T && b < p.batch && p.cu[b] <= t;
    const int lo = in ? clip_offset(p.cu[b], p.T) : (int)p.T;
    const int hi = !in ? -1 : p.causal ? t : clip_offset(p.cu[b + 1], p.T) - 1;
    int from = lo, to = hi;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        from = min(from, __shfl_xor(from, d));
        to = max(to, __shfl_xor(to, d));
    }
    from = __builtin_amdgcn_readfirstlane(from);
    to = __builtin_amdgcn_readfirstlane(to);
    if (to < from) return;                             // no row has a prompt
    const uint16_t* K = static_cast<const uint16_t*>(p.K) + g * p.k_head;
    const uint16_t* V = static_cast<const uint16_t*>(p.V) + g * p.v_head;
    uint16_t* const kl = lds + wave * kShortKeys * D;
    uint16_t* const vl = kl + kWaves * kShortKeys * D;

    const auto load = [&](const uint16_t* x, int64_t tok, int j0, uint16_t* place) __attribute__((always_inline)) {
        const char* at = reinterpret_cast<const char*>(x + j0 * tok);
        const uint32_t step = 2u * (uint32_t)tok;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int r = kPer * i + lane / C, rr = r < to - j0 ? r : to - j0;
            __builtin_amdgcn_global_load_lds((gptr_t)(at + (uint32_t)(rr * step + 16 * (lane % C ^ swizzle<D>(r)))),
                                             (lptr_t)(place + 64 * 8 * i), 16, 0, 0);
        }
    };
    u32x4_t qf[SL];
    {
        const uint16_t* qp = static_cast<const uint16_t*>(p.Q) + h * p.q_head + (in ? t : (int)first) * p.q_token + 8 * lh;
#pragma unroll
        for (int s = 0; s < SL; ++s) qf[s] = *reinterpret_cast<const u32x4_t*>(qp + 16 * s);
    }
    f32x16_t o[DB];
    Ref<false> ref;
    float l;
    const int r0 = 4 * lh + ((lane & 15) >> 2), cq = 2 * (lane >> 4 & 1) + ((lane & 3) >> 1);
    // kSafe: V may hold infinities or NaN
    const auto pass = [&](auto safe, uint16_t* __restrict__ kt, uint16_t* __restrict__ vt) __attribute__((always_inline)) {
        constexpr bool kSafe = decltype(safe)::value;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        ref.reset();
        l = 0.f;
        // kMore: there are keys after this tile's
        const auto step = [&](auto more, int j0) __attribute__((always_inline)) {
            constexpr bool kMore = decltype(more)::value;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kPieces) : "memory");       // K; V may still be on its way
            f32x16_t st;
#pragma unroll
            for (int i = 0; i < 16; ++i) st[i] = 0.f;
#pragma unroll
            for (int s = 0; s < SL; ++s) {
                const u32x4_t a = *reinterpret_cast<const u32x4_t*>(kt + lq * D + 8 * ((2 * s + lh) ^ swizzle<D>(lq)));
                st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(qf[s]), st, 0, 0, 0);
            }
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int j = j0 + 8 * (i / 4) + 4 * lh + i % 4;
                if (j < lo || j > hi) st[i] = -INFINITY;
                mx = fmaxf(mx, st[i]);
            }
            mx = pair_max32(mx);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // every read of K has returned
            if constexpr (kMore) load(K, p.k_token, j0 + kShortKeys, kt);
            if (__any(mx > ref.m + p.slack)) {
                const float al = ref.template raise<kSafe>(mx, p.c);
                l *= al;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] = scaled<kSafe>(o[d][i], al);
            }
            u32x4_t pf[2];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = ref.template weight<kSafe>(st[i], p.c);
                const float y = ref.template weight<kSafe>(st[i + 1], p.c);
                l += x + y;
                pf[i / 8][i % 8 / 2] = pack_bf16x2(x, y);
            }
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMore ? kPieces : 0) : "memory");      // V; not the next K
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const int c = 4 * d + cq;
                    const uint2 a = lds_read_tr16(vt + (16 * u + r0) * D + 8 * (c ^ swizzle<D>(r0)) + 4 * (lane & 1));
                    const uint2 e = lds_read_tr16(vt + (16 * u + r0 + 8) * D + 8 * (c ^ swizzle<D>(r0 + 8)) + 4 * (lane & 1));
                    u32x4_t v = {a.x, a.y, e.x, e.y};
                    if constexpr (kSafe) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = finite_only(v[i]);
                    }
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pf[u]), o[d], 0, 0, 0);
                }
            if (kSafe && any_odd<kShortKeys * D>(vt))
                for (int r = 0; r < kShortKeys; ++r)
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int dim = 32 * d + 8 * (i / 4) + 4 * lh + i % 4;
                            const uint16_t v = vt[r * D + 8 * ((dim >> 3) ^ swizzle<D>(r)) + (dim & 7)];
                            if (odd_half(v) && j0 + r >= lo && j0 + r <= hi) o[d][i] += bf16_to_f32(v);
                        }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // every read of V has returned
            if constexpr (kMore) load(V, p.v_token, j0 + kShortKeys, vt);
        };
        load(K, p.k_token, from, kt);
        load(V, p.v_token, from, vt);
        int j0 = from;
        for (; j0 <= to - kShortKeys; j0 += kShortKeys) step(std::true_type{}, j0);
        step(std::false_type{}, j0);
    };
    pass(std::false_type{}, kl, vl);
    float odd = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = fmaf(o[d][i], 0.f, odd);
    if (__any((ref.needs_apart(l) || odd != odd) && in)) pass(std::true_type{}, kl, vl);
    l = pair_sum32(l);
    if (!in) return;
    const float inv = 1.f / l;              // every score -inf: 0 / 0, NaN
    const int64_t at = h * p.o_head + t * p.o_token + 4 * lh;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store4(p, at + 32 * d + 8 * i, o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv);
}

// float32: the narrow form's plan and the same layouts on v_mfma_f32_32x32x2_f32 (16
// times slower than bf16's: it hides everything else, and so few rows to a workgroup
// keep the chip busy on short prompts), 32 keys to a tile.  The score product takes
// four dims of a key from one 16-byte read (lane half lh: dims 8 s + 4 lh ..), the PV
// product score register i as it stands (its two contraction slots are the keys of
// the lane halves).  16-byte chunk c of row r lies in place c ^ (r % 16).  Bound by the
// matrix unit on many rows (75% busy, 113 of a large product's 154 TFLOP/s for 32 heads
// of 5,000 tokens), by the unequal lengths of few workgroups on less (71 for 4 heads).
constexpr int kKeys32 = 32;

template <int D>
__global__ __launch_bounds__(64 * kWaves, D == 128 ? 1 : 2) void k_prompt_f32(PromptParams p) {
    constexpr int DB = D / 32, C = D / 4;
    constexpr int kPieces = kKeys32 * C / 64, kPer = 64 / C;
    __shared__ __align__(16) float lds[2 * kWaves * kKeys32 * D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lq = lane & 31, lh = lane >> 5;
    const uint32_t xcd = blockIdx.x & 7u, slot = blockIdx.x >> 3;
    const uint32_t unit = slot / p.G * 8u + xcd;
    const int g = (int)(unit % p.Hkv), h = g * p.G + (int)(slot % p.G);
    RowTile t;
    if (!find_tile(p.cu, p.batch, p.T, kNarrowRows, unit / p.Hkv, t)) return;
    const int n = t.len, q0 = t.tile * kNarrowRows, row = q0 + lq;
    const float* K = static_cast<const float*>(p.K) + g * p.k_head + t.first * p.k_token;
    const float* V = static_cast<const float*>(p.V) + g * p.v_head + t.first * p.v_token;
    float* const kl = lds + wave * kKeys32 * D;
    float* const vl = kl + kWaves * kKeys32 * D;

    const auto load = [&](const float* x, int64_t tok, int j0, float* to) __attribute__((always_inline)) {
        const char* from = reinterpret_cast<const char*>(x + j0 * tok);
        const uint32_t step = 4u * (uint32_t)tok;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int r = kPer * i + lane / C, rr = r < n - j0 ? r : n - 1 - j0;
            __builtin_amdgcn_global_load_lds((gptr_t)(from + (uint32_t)(rr * step + 16 * (lane % C ^ (r & 15)))),
                                             (lptr_t)(to + 64 * 4 * i), 16, 0, 0);
        }
    };
    const int last = p.causal ? (row < n ? row : n - 1) : n - 1;
    const int kend = p.causal && q0 + kNarrowRows < n ? q0 + kNarrowRows : n;
    const int wfull = p.causal ? q0 : n - 1;
    const int tiles = (kend + kKeys32 - 1) / kKeys32;
    f32x4_t qf[D / 8];
    {
        const int r = row < n ? row : n - 1;
        const float* qp = static_cast<const float*>(p.Q) + h * p.q_head + (t.first + r) * p.q_token + 4 * lh;
#pragma unroll
        for (int s = 0; s < D / 8; ++s) qf[s] = *reinterpret_cast<const f32x4_t*>(qp + 8 * s);
    }
    f32x16_t o[DB];
    Ref<true> ref;
    float l;
    // kSafe: V may hold infinities or NaN
    const auto pass = [&](auto safe, float* __restrict__ kt, float* __restrict__ vt) __attribute__((always_inline)) {
        constexpr bool kSafe = decltype(safe)::value;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        ref.reset();
        l = 0.f;
        // kMore: the wave has a tile after this one
        const auto step = [&](auto more, int it) __attribute__((always_inline)) {
            constexpr bool kMore = decltype(more)::value;
            const int j0 = it * kKeys32, jn = j0 + kWaves * kKeys32;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kPieces) : "memory");       // K; V may still be on its way
            f32x16_t st;
#pragma unroll
            for (int i = 0; i < 16; ++i) st[i] = 0.f;
#pragma unroll
            for (int s = 0; s < D / 8; ++s) {
                const f32x4_t a = *reinterpret_cast<const f32x4_t*>(kt + lq * D + 4 * ((2 * s + lh) ^ (lq & 15)));
#pragma unroll
                for (int e = 0; e < 4; ++e) st = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], qf[s][e], st, 0, 0, 0);
            }
            if (j0 + kKeys32 - 1 > wfull) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (j0 + 8 * (i / 4) + 4 * lh + i % 4 > last) st[i] = -INFINITY;
            }
            float mx = st[0];
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[i]);
            mx = pair_max32(mx);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // every read of K has returned
            if constexpr (kMore) load(K, p.k_token, jn, kt);
            if (__any(mx > ref.m + p.slack)) {
                const float al = ref.template raise<kSafe>(mx, p.c);
                l *= al;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] = scaled<kSafe>(o[d][i], al);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                st[i] = ref.template weight<kSafe>(st[i], p.c);
                l += st[i];
            }
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMore ? kPieces : 0) : "memory");      // V; not the next K
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = 8 * (i / 4) + 4 * lh + i % 4;
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    float v = vt[r * D + 4 * ((8 * d + lq / 4) ^ (r & 15)) + lq % 4];
                    if (kSafe && !isfinite(v)) v = 0.f;
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, st[i], o[d], 0, 0, 0);
                }
            }
            if (kSafe && any_odd<kKeys32 * D>(vt))
                for (int r = 0; r < kKeys32; ++r)
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int dim = 32 * d + 8 * (i / 4) + 4 * lh + i % 4;
                            const float v = vt[r * D + 4 * (dim / 4 ^ (r & 15)) + dim % 4];
                            if (!isfinite(v) && j0 + r <= last) o[d][i] += v;
                        }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // every read of V has returned
            if constexpr (kMore) load(V, p.v_token, jn, vt);
        };
        if (wave >= tiles) return;
        load(K, p.k_token, wave * kKeys32, kt);
        load(V, p.v_token, wave * kKeys32, vt);
        int it = wave;
        for (; it + kWaves < tiles; it += kWaves) step(std::true_type{}, it);
        step(std::false_type{}, it);
    };
    pass(std::false_type{}, kl, vl);
    float odd = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = fmaf(o[d][i], 0.f, odd);
    float* const vf = lds + kWaves * kKeys32 * D;
    const bool again = any_wave<kKeys32 * D>((ref.needs_apart(l) || odd != odd) && row < n, vf);
    if (again) {
        __syncthreads();
        pass(std::true_type{}, kl, vl);
        join_waves<D, kKeys32 * D, true>(p, lds, vf, ref, l, o, t, row, h);
    } else {
        join_waves<D, kKeys32 * D, false>(p, lds, vf, ref, l, o, t, row, h);
    }
}

// Workgroups of a launch whose row tiles hold `rows`.
int64_t blocks_of(const PromptParams& p, int rows) {
    return (tile_places(p.T, p.batch, rows) * p.Hkv + 7) / 8 * 8 * p.G;
}

// The narrow form while its workgroups are resident at once (one a CU at D = 128, two
// at D = 64) and prompts are longer than a tile of keys.  Below the limit and above it,
// against the 128-row form, us: D = 128, 12/2 heads, one prompt of 512 tokens (192
// workgroups) 9.9 and 16.0; 32/8 heads, of 256 (256) 7.9 and 11.4, of 320 (320) 12.9 and
// 11.6; 16/16 heads, of 512 (256) 10.0 and 16.0; D = 64, 32/4 heads, of 512 (512) 7.8 and
// 11.1, of 800 (832) 14.0 and 13.9.  Few heads of longer prompts would gain beyond it too
// (4/1 heads, one of 3,264: 31 and 49); several prompts lose there (two of 512, 12/2 heads:
// 18.5 and 15.9).
bool narrow(const PromptParams& p) { return p.T > (int64_t)p.batch * kKeys && blocks_of(p, kNarrowRows) <= (p.D == 128 ? 256 : 512); }

// Two groups of waves where long prompts' workgroups do not fill the chip and the
// longest bounds the time.  With them and without, us: one prompt, 12/2 heads of 128, 4,096
// tokens (384 workgroups) 71 and 88, 5,120 (480) 98 and 113, 6,144 (576) 143 and 144, 6,784
// (636) 170 and 166; 32/4 heads of 64, 1,664 (416) 25.5 and 29.1, 2,048 (512) 32.7 and 34.6,
// 2,304 (576) 43.7 and 39.7.  Several prompts turn earlier: 12/2 heads of 128, four of 1,024
// (420) 32.9 and 31.5, three of 1,600 (480) 47.8 and 44.8, seven of 600 (480) 29.9 and 23.3;
// 32/4 heads of 64, two of 900 (512) 22.9 and 19.6.  The limit lies between the two.
bool split(const PromptParams& p) { return p.T >= (int64_t)p.batch * 512 && blocks_of(p, kRows) <= 440; }

// The short form for prompts of a tile of keys or less in the mean that are more than the
// 128-row form's workgroups resident at once.  With it and without, us: 12/2 heads of 128,
// 42 prompts of 20 tokens (576 workgroups) 9.1 and 12.4, 500 of 20 27 and 66, of 64 70 and
// 83, 10,000 of 8 175 and 1,219; 32/4 heads of 64, 500 of 20 32 and 92.  Fewer: 21 of 20
// (288) 8.9 and 7.5; longer: 64 of 100 23.9 and 24.2.  One head to a group, which shares
// nothing there, turns later: 16/16 heads of 128, 32 of 20 (576) 8.9 and 8.1, of 60 (736)
// 12.8 and 10.2, 93 of 20 (1,712) 11.0 and 18.6.
// A long prompt among them, which the host does not see, costs the more the longer it is,
// each wave reading its keys for 32 rows alone: 12/2 heads of 128, one of 10,000 and 499 of
// 20 513 and 363, of 30,000 and 1,000 of 20 4,190 and 2,580, of 63,000 and 1,000 of one token,
// the longest that this rule takes beside 1,000 others, 28,000 and 10,900.
bool brief(const PromptParams& p) { return p.batch > 1 && p.T <= (int64_t)p.batch * kKeys && blocks_of(p, kRows) > 512; }
int64_t brief_blocks(const PromptParams& p) {
    const int64_t tiles = ((p.T + kShortRows - 1) / kShortRows + 7) / 8;       // of an XCD
    return (tiles * p.Hq + kWaves - 1) / kWaves * 8;
}

}  // namespace

int64_t prompt_blocks(const PromptParams& p) {
    if (!p.in_bf16) return blocks_of(p, kNarrowRows);
    return brief(p) ? brief_blocks(p) : blocks_of(p, narrow(p) ? kNarrowRows : kRows);
}

hipError_t launch_prompt_attn(const PromptParams& p, hipStream_t st) {
    const dim3 grid((unsigned)prompt_blocks(p));
    const auto run = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, st, p); };
    if (!p.in_bf16) p.D == 128 ? run(k_prompt_f32<128>, kWaves) : run(k_prompt_f32<64>, kWaves);
    else if (brief(p)) p.D == 128 ? run(k_prompt_short<128>, kWaves) : run(k_prompt_short<64>, kWaves);
    else if (narrow(p)) p.D == 128 ? run(k_prompt_narrow<128>, kWaves) : run(k_prompt_narrow<64>, kWaves);
    else if (split(p)) p.D == 128 ? run(k_prompt_bf16<128, 2>, 2 * kWaves) : run(k_prompt_bf16<64, 2>, 2 * kWaves);
    else p.D == 128 ? run(k_prompt_bf16<128, 1>, kWaves) : run(k_prompt_bf16<64, 1>, kWaves);
    return hipGetLastError();
}

}  // namespace ris
