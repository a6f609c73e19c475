// Attention over a paged cache for one or a few new tokens a sequence: the step form.
//
// A row tile is up to 16 rows, the heads of a group at one or a few tokens.  Its keys come in
// tiles of 32 that are dealt to the waves of one or more workgroups; a wave goes over its own with
// nothing to wait for but its loads: S^T = K Q^T on v_mfma_f32_16x16x32_bf16 with the K
// rows taken from their pages into the operand's layout, O += P V with V passed through
// wave-private LDS and read transposed, as in the contiguous decode.  Lane i looks up the page of key
// i a tile before its loads, which are a tile ahead of the products.
//
// HBM-bound: 4 D bytes a key of a KV head (32 sequences of 41,000 keys on average, 12/2 heads of 128: 229 us for 1.34 GB,
// 5.9 TB/s; one of 33,000, 12.2 us and 4.9 for the second launch, where a wave's chain of table, key and value
// loads is what is left).  The waves of a workgroup meet in LDS, workgroups of one row tile in a second launch.
#include <float.h>

#include "page_rows.h"
#include "softmax_tiles.h"

namespace ris {
namespace {

constexpr int kKeys = 32;         // keys of a tile
constexpr int kMostRows = 16;

template <int D>
struct Tile {
    u32x4_t k[2][D / 32];       // lane: key 16 kb + l % 16, dims 32 s + 8 (l / 16) ..
    u32x4_t v[2][D / 32];       // rows, D / 8 lanes to a row: row 16 kb + (512 / D) s + lane / (D / 8)
    uint32_t live;
};

// Row r's sums over one part of its keys: reference, sum of weights, whether anything was attended to.
struct RowSum {
    float m, l, seen, pad;
};

// The factor of a sum under the reference m where it meets others under M >= m.  References
// start finite: where nothing is summed any factor will do.
__device__ __forceinline__ float meet(const PageAttnParams& p, float m, float M) { return __builtin_amdgcn_exp2f((m - M) * p.c); }

__device__ __forceinline__ void store_out(const PageAttnParams& p, int64_t at, float y) {
    if (p.out_bf16) static_cast<uint16_t*>(p.out)[at] = f32_to_bf16(y);
    else static_cast<float*>(p.out)[at] = y;
}

// kWaves: of a workgroup; kStream: values pass the caches by.
template <int D, int kWaves, bool kStream>
__global__ __launch_bounds__(64 * kWaves, 2) void k_page_step(PageAttnParams p) {
    constexpr int SL = D / 32;         // slices of the score product
    constexpr int DB = D / 16;         // 16-dim blocks of the output
    constexpr int VS = D + 16;         // V row stride in LDS
    __shared__ __align__(16) uint16_t vlds[kWaves * kKeys * VS];
    static_assert(kKeys * VS * sizeof(uint16_t) >= kMostRows * D * sizeof(float), "a wave's outputs fit its V slice");
    __shared__ RowSum sums[kWaves][kMostRows];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int li = lane & 15, lg = lane >> 4;
    const uint32_t groups = (uint32_t)p.parts / kWaves;         // workgroups of a row tile
    const uint32_t unit = blockIdx.x / groups, part = blockIdx.x % groups * kWaves + wave;
    const int g = (int)(unit % p.Hkv);
    RowTile t;
    if (!find_tile(p.cu, p.batch, p.T, p.tokens, unit / p.Hkv, t)) return;
    const int64_t pos0 = tile_pos(p, first_pos(p, t.seq), t);
    const int ntok = tile_tokens(p, t), rows = ntok * p.G;
    const Span<kKeys> s = span_of<kKeys>(p, pos0, pos0 + ntok - 1);
    uint16_t* const vw = vlds + wave * kKeys * VS;

    // the lane's row
    const int tok = li / p.G, head = g * p.G + (li - tok * p.G);
    const bool mine = li < rows;
    const int64_t pq = pos0 + tok;
    const int pos = mine && pq >= 0 && pq < p.map.places ? (int)pq : -1;
    const int from = pos - p.window + 1 > 0 ? pos - p.window + 1 : 0;
    u32x4_t qf[SL];
    {
        const uint16_t* qp = static_cast<const uint16_t*>(p.Q) + (mine ? head : g * p.G) * p.q_head +
                             (int64_t)(t.first + t.tile * p.tokens + (mine ? tok : 0)) * p.q_token + 8 * lg;
        const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(qp + 32 * i);
            qf[i] = mine ? v : zero;
        }
    }

    const uint16_t* const K = static_cast<const uint16_t*>(p.K);
    const uint16_t* const V = static_cast<const uint16_t*>(p.V);
    const int32_t* const table = p.map.table + t.seq * p.map.table_stride;
    const auto look = [&](int v) __attribute__((always_inline)) {
        const int j = s.key0(v) + (lane & 31);
        return v < s.n && j <= s.pmax && (j >= s.lo || j < p.sink) ? table[j >> p.map.shift] : -1;
    };
    // Keys that no row attends to or that have no page are not read: the first live one is in their place.
    const auto load = [&](int v, int page, Tile<D>& x) __attribute__((always_inline)) {
        const bool ok = (uint32_t)page < (uint32_t)p.map.pages;
        const uint64_t live = __ballot(ok);                         // both halves of the wave alike
        x.live = (uint32_t)live;
        uint32_t row = 0;                                           // row 0 always exists
        if (live) {
            const uint32_t slot = (uint32_t)(s.key0(v) + (lane & 31)) & ((1u << p.map.shift) - 1);
            row = (uint32_t)page * p.map.page_rows + ((uint32_t)g << p.map.shift) + slot;
            const uint32_t instead = (uint32_t)__builtin_amdgcn_readlane((int)row, (int)__builtin_ctzll(live));
            row = ok ? row : instead;
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const uint16_t* kp = K + (uint64_t)(uint32_t)__shfl((int)row, 16 * kb + li) * D + 8 * lg;
#pragma unroll
            for (int i = 0; i < SL; ++i) x.k[kb][i] = *reinterpret_cast<const u32x4_t*>(kp + 32 * i);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                const uint32_t r = (uint32_t)__shfl((int)row, 16 * kb + (512 / D) * i + lane / (D / 8));
                const u32x4_t* vp = reinterpret_cast<const u32x4_t*>(V + (uint64_t)r * D + 8 * (lane % (D / 8)));
                x.v[kb][i] = kStream ? __builtin_nontemporal_load(vp) : *vp;
            }
    };

    f32x4_t o[DB];                  // lane: dim 16 db + l % 16 of the rows 4 (l / 16) + i
    float m, l;
    bool seen;
    for (bool safe = false;; safe = true) {
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        m = -FLT_MAX;
        l = 0.f;
        seen = false;
        Tile<D> cur, nxt;
        int page = look((int)part);
        if ((int)part < s.n) load((int)part, page, cur);
        page = look((int)part + p.parts);
        for (int v = (int)part; v < s.n; v += p.parts) {
            if (v + p.parts < s.n) load(v + p.parts, page, nxt);
            page = look(v + 2 * p.parts);
            const int j0 = s.key0(v);
            const uint32_t mask = (uint32_t)(below(pos - j0 + 1) & (~below(from - j0) | below(p.sink - j0))) & cur.live;
            const auto rows_to_lds = [&](bool clean) __attribute__((always_inline)) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < SL; ++i) {
                        u32x4_t x = cur.v[kb][i];
                        if (clean) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[e] = finite_only(x[e]);
                        }
                        *reinterpret_cast<u32x4_t*>(vw + (16 * kb + (512 / D) * i + lane / (D / 8)) * VS + 8 * (lane % (D / 8))) = x;
                    }
            };
            rows_to_lds(false);
            if (safe) {
                // infinities and NaN of V are added where they are attended to, whatever their weight
                uint32_t seen_by[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) seen_by[i] = (uint32_t)__shfl((int)mask, 4 * lg + i);
#pragma unroll 1
                for (int k = 0; k < kKeys; ++k)
#pragma unroll
                    for (int db = 0; db < DB; ++db) {
                        const uint16_t x = vw[k * VS + 16 * db + li];
                        if (odd_half(x))
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (seen_by[i] >> k & 1u) o[db][i] += bf16_to_f32(x);
                    }
                rows_to_lds(true);
            }
            // S^T = K Q^T: lane l holds row l % 16 at keys 16 kb + 4 (l / 16) + i
            f32x4_t st[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                st[kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < SL; ++i)
                    st[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(cur.k[kb][i]), as_bf16x8(qf[i]), st[kb], 0, 0, 0);
            }
            seen |= mask != 0;
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    st[kb][i] = (mask >> (16 * kb + 4 * lg + i)) & 1u ? st[kb][i] : -INFINITY;
                    mx = fmaxf(mx, st[kb][i]);
                }
            mx = quad_max16(mx);
            // The reference moves, and what was summed is rescaled, only where a score exceeds it by 2^8
            // in weight.
            if (__any(mx > m + p.slack)) {
                const float was = m;
                m = fmaxf(m, mx);
                float al = meet(p, was, m);
                l *= al;
                if (safe) al = kept_infinite(al);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = __shfl(al, 4 * lg + i);
#pragma unroll
                    for (int db = 0; db < DB; ++db) o[db][i] *= a;
                }
            }
            float w[2][4];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[kb][i] = __builtin_amdgcn_exp2f((st[kb][i] - m) * p.c);
                    l += w[kb][i];
                }
            // P as the A operand, rounded to bf16 (as the row-tile form's): row l % 16, slots 8 (l / 16) + e hold the keys 4 (l / 16) + e (e < 4) and 16 +
            // 4 (l / 16) + e - 4; V as the B operand with the same key order.
            const u32x4_t pk = {pack_bf16x2(w[0][0], w[0][1]), pack_bf16x2(w[0][2], w[0][3]), pack_bf16x2(w[1][0], w[1][1]),
                                pack_bf16x2(w[1][2], w[1][3])};
            const uint16_t* lo = vw + (lane >> 2) * VS + 4 * (lane & 3);
            const uint16_t* hi = lo + 16 * VS;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const uint2 a = lds_read_tr16(lo + 16 * db), e = lds_read_tr16(hi + 16 * db);
                o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(pk), as_bf16x8(u32x4_t{a.x, a.y, e.x, e.y}), o[db], 0, 0, 0);
            }
            cur = nxt;
        }
        if (safe) break;
        float odd = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) odd = fmaf(o[db][i], 0.f, odd);
        if (!__any(odd != odd)) break;
    }

    // The waves' sums meet.
    l = quad_sum16(l);
    seen &= pos >= 0;
    __syncthreads();
    if (lane < kMostRows) sums[wave][lane] = RowSum{m, l, seen ? 1.f : 0.f, 0.f};
    float* const ow = reinterpret_cast<float*>(vlds);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * lg + i < rows) {
#pragma unroll
            for (int db = 0; db < DB; ++db) ow[(wave * kMostRows + 4 * lg + i) * D + 16 * db + li] = o[db][i];
        }
    __syncthreads();
    const int64_t piece = (int64_t)blockIdx.x * p.part_rows;
    for (int e = threadIdx.x; e < rows * D; e += 64 * kWaves) {
        const int r = e / D;
        RowSum all = sums[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) all.m = fmaxf(all.m, sums[w][r].m);
        float y = 0.f;
        all.l = all.seen = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float a = meet(p, sums[w][r].m, all.m);
            y = add_scaled<true>(y, ow[(w * kMostRows + r) * D + e % D], a);
            all.l = fmaf(sums[w][r].l, a, all.l);
            all.seen += sums[w][r].seen;
        }
        if (groups > 1) {
            p.part_o[(piece + r) * D + e % D] = y;
            if (e % D == 0) reinterpret_cast<RowSum*>(p.part_ml)[piece + r] = all;
        } else {
            const int k = r / p.G;
            const int64_t at = (g * p.G + r - k * p.G) * p.o_head + (int64_t)(t.first + t.tile * p.tokens + k) * p.o_token + e % D;
            store_out(p, at, all.seen > 0.f ? y / all.l : 0.f);       // every score -inf: 0 / 0, NaN
        }
    }
}

// The pieces of one row joined: the threads find the largest reference and each piece's factor
// together, then D / 4 lanes of four dims each sum over every kGroups-th piece.
constexpr int kJoinThreads = 256;
template <int D>
__global__ __launch_bounds__(kJoinThreads) void k_page_step_join(PageAttnParams p) {
    constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes, kJoinWaves = kJoinThreads / 64;
    __shared__ float factor[kMostStepGroups];
    __shared__ float red[kJoinWaves][3];
    __shared__ __align__(16) float osum[kGroups][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int unit = (int)(blockIdx.x / p.part_rows), r = (int)(blockIdx.x % p.part_rows), g = unit % p.Hkv;
    RowTile t;
    if (!find_tile(p.cu, p.batch, p.T, p.tokens, unit / p.Hkv, t)) return;
    if (r >= tile_tokens(p, t) * p.G) return;
    const int n = p.parts / p.part_waves;
    const auto piece = [&](int i) { return ((int64_t)unit * n + i) * p.part_rows + r; };
    const RowSum* sums = reinterpret_cast<const RowSum*>(p.part_ml);
    float m = -FLT_MAX;
    for (int i = tid; i < n; i += kJoinThreads) m = fmaxf(m, sums[piece(i)].m);
    m = wave_max(m);
    if (lane == 0) red[wave][0] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) m = fmaxf(m, red[w][0]);
    float l = 0.f, seen = 0.f;
    for (int i = tid; i < n; i += kJoinThreads) {
        const RowSum x = sums[piece(i)];
        const float a = meet(p, x.m, m);
        factor[i] = a;
        l = fmaf(x.l, a, l);
        seen += x.seen;
    }
    l = wave_sum(l);
    seen = wave_sum(seen);
    if (lane == 0) {
        red[wave][1] = l;
        red[wave][2] = seen;
    }
    __syncthreads();
    const int grp = tid / kLanes, d4 = 4 * (tid % kLanes);
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = grp; i < n; i += kGroups) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(p.part_o + piece(i) * D + d4);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = add_scaled<true>(y[e], x[e], factor[i]);
    }
    *reinterpret_cast<f32x4_t*>(&osum[grp][d4]) = y;
    __syncthreads();
    if (tid >= kLanes) return;
    l = seen = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) {
        l += red[w][1];
        seen += red[w][2];
    }
    y = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kGroups; ++k) y += *reinterpret_cast<const f32x4_t*>(&osum[k][d4]);
    const int k = r / p.G;
    const int64_t at = (g * p.G + r - k * p.G) * p.o_head + (int64_t)(t.first + t.tile * p.tokens + k) * p.o_token + d4;
    if (seen == 0.f) store4(p, at, 0.f, 0.f, 0.f, 0.f);
    else store4(p, at, y[0] / l, y[1] / l, y[2] / l, y[3] / l);
}

// Keys that a row tile may attend to.
int64_t step_keys(const PageAttnParams& p) {
    const int64_t keys = (int64_t)p.window + p.tokens - 1 + p.sink;
    return keys < p.map.places ? keys : p.map.places;
}

// Bytes of keys and values from which the values pass the caches by: more than the last one
// holds (32 sequences as above 255 us through the caches, 232 past them; a cache of less than that stays in
// it from one step to the next).
constexpr int64_t kStreamBytes = 256ll << 20;

// Waves of a row tile for the keys that it may attend to (positions are on the device, so this
// counts the places of the cache under the window).  Up to kSoloTiles, or where row tiles are many, one workgroup that
// writes out itself, of eight waves (48 sequences under a window of 1,024 keys, 32/4 heads
// of 64, 13.3 us, with four 15.4).  Else workgroups
// of four to kTargetWaves in all (32 sequences as above with 2,048 waves 276 us, 4,096 255, 8,192 232, 16,384 240), kMostWaves
// to a row tile (one sequence of 33,000 keys with 1,024 19.3, 512 16.0, 256 17.3, 128 23.2).
constexpr int64_t kSoloTiles = 16, kTargetWaves = 8192, kMostWaves = 512;

template <int D, int kWaves>
hipError_t launch_waves(const PageAttnParams& p, hipStream_t st) {
    const int64_t units = page_attn_blocks(p);
    const dim3 grid((unsigned)(units * (p.parts / kWaves)));
    if (units * step_keys(p) * D * 4 > kStreamBytes)
        hipLaunchKernelGGL((k_page_step<D, kWaves, true>), grid, dim3(64 * kWaves), 0, st, p);
    else
        hipLaunchKernelGGL((k_page_step<D, kWaves, false>), grid, dim3(64 * kWaves), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == kWaves) return e;
    hipLaunchKernelGGL(k_page_step_join<D>, dim3((unsigned)(units * p.part_rows)), dim3(kJoinThreads), 0, st, p);
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const PageAttnParams& p, hipStream_t st) {
    return p.part_waves == 8 ? launch_waves<D, 8>(p, st) : launch_waves<D, 4>(p, st);
}

}  // namespace

// Tokens of a row tile of the step form where the sequences have so few in the mean that a tile holds them, else 0: the row
// tiles of 128 rows.  The step form and those, us: one token after 33,000, 12/2 heads of 128, 16.4 and 21.2, 32/4 of 64 14.1 and
// 17.9; 32 of 41,000 on average 232 and 239; 48 under a window of 1,024, 32/4 of 64, 13.3 and 21.5; 48 of two tokens after 1,000,
// 12/2 heads 19.7 and 22.3, 32/4 14.3 and 21.5; but 32 of one or two after 3,000 34 to 37 and 29, 8 of two after 9,000 31 and 26,
// and 32 of two after 65,000 at most 252 and 248.  The host sees the mean alone: one long chunk among single tokens,
// which the mean hides, is cut into tiles of 16 rows that each read its keys (one of 960 tokens and 63 steps after 9,000, 4/4 heads
// of 128, 249 and 157, as two calls 187; one of 256 and 63, 12/4 heads, 233 and 154; one of 64 and 63, 24/4 heads, 197 and 155).
int32_t page_step_tokens(int64_t T, int32_t batch, int32_t G) {
    const int64_t each = (T + batch - 1) / batch;
    return each * G <= kMostRows ? (int32_t)each : 0;
}

void page_step_waves(PageAttnParams* p) {
    const int64_t tiles = (step_keys(*p) + kKeys - 1) / kKeys, units = page_attn_blocks(*p);
    p->part_waves = 4;
    if (tiles <= kSoloTiles || tiles <= units / 4) {
        p->parts = p->part_waves = tiles <= 4 ? 4 : 8;
        return;
    }
    int64_t waves = (kTargetWaves + units - 1) / units;
    if (waves > tiles) waves = tiles;
    if (waves > kMostWaves) waves = kMostWaves;
    p->parts = (int32_t)((waves + p->part_waves - 1) / p->part_waves * p->part_waves);
}

hipError_t launch_page_step(const PageAttnParams& p, hipStream_t st) {
    return p.D == 128 ? launch_d<128>(p, st) : launch_d<64>(p, st);
}

}  // namespace ris
