// Attention of new tokens over a paged cache, with a sliding window and first tokens that
// stay visible.
//
// A row tile is the query heads of a group at `tokens` neighbouring tokens of a sequence, up to
// 128 rows, so that what a tile's rows attend to is one narrow band whatever the group, and its
// K and V are read once.  The keys come in tiles of 64; those that no row of the tile
// attends to are passed over.  Within a key tile the path is the dense one (prompt
// attention): K and V go from memory to LDS, 16 bytes a lane, two tiles deep; S^T = K Q^T and
// O^T += V^T P^T on v_mfma_f32_32x32x16_bf16, a wave 32 rows, the query as the column.
//
// Pages: lane i of every wave looks up the page of key i of a tile, a tile before it is needed,
// and the lanes that load a row of it take its place from there.  The keys that a row of the tile
// may attend to and whose page there is are a mask of 64 bits (`live`); the others are
// never read: the first live key is loaded in their place.  Rows attend to bits of that
// mask, so that what lies in unwritten places does not reach an output.
#include <type_traits>

#include "packed.h"
#include "ris_internal.h"
#include "softmax_tiles.h"

namespace ris {
namespace {

constexpr int kKeys = 64;         // keys of a tile
constexpr int kWaves = 4;

// A lane's part in a tile, as in prompt attention: 16-byte pieces, piece i at place 256 i
// + thread of the tile in LDS, their rows kStep apart.
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

// The keys of a row tile: of the tokens at positions pmin .. pmax, as key tiles of which the
// first `sinks` hold first tokens and the others lie side by side from `near` on.
struct Span {
    int pmin, pmax, lo;       // lo: first key of the window of pmin
    int near, sinks, n;
    __device__ __forceinline__ int key0(int v) const { return kKeys * (v < sinks ? v : near + v - sinks); }
};

// Of tokens at positions a .. z (any; those outside the cache attend to nothing).
__device__ __forceinline__ Span span_of(const PageAttnParams& p, int64_t a, int64_t z) {
    Span s{0, -1, 0, 0, 0, 0};
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

// Where the lanes' pieces of a key tile lie, and which of its keys are live.
template <int D>
struct Places {
    uint32_t row[Piece<D>::kCount];
    uint64_t live;
};

__device__ __forceinline__ void store4(const PageAttnParams& p, int64_t at, float a, float b, float c, float d) {
    if (p.out_bf16)
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
    else
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) = f32x4_t{a, b, c, d};
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 3 : 2) void k_page_attn(PageAttnParams p) {
    constexpr int SL = D / 16;      // contraction steps of the score product
    constexpr int DB = D / 32;      // 32-dim blocks of the output
    constexpr int NP = Piece<D>::kCount;
    constexpr bool kPipe = D == 128;
    // two tiles of K and of V; arrays of their own, so that a load into one is not
    // taken for a write to another
    __shared__ __align__(16) uint16_t k0[kKeys * D], k1[kKeys * D], v0[kKeys * D], v1[kKeys * D];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lq = lane & 31, lh = lane >> 5;
    const int g = (int)(blockIdx.x % p.Hkv);
    RowTile t;
    if (!find_tile(p.cu, p.batch, p.T, p.tokens, blockIdx.x / p.Hkv, t)) return;
    const int64_t pos0 = first_pos(p, t.seq) + (int64_t)t.tile * p.tokens;       // of the tile's first token
    const int ntok = t.len - t.tile * p.tokens < p.tokens ? t.len - t.tile * p.tokens : p.tokens;
    const Span s = span_of(p, pos0, pos0 + ntok - 1);
    const Piece<D> pc;

    // The lane's row: a token of the tile and a head of the group.
    const int r = 32 * wave + lq, tok = r / p.G, head = g * p.G + (r - tok * p.G);
    const bool mine_row = tok < ntok;
    const int64_t tq = t.first + t.tile * p.tokens + (mine_row ? tok : ntok - 1);
    const int64_t pq = pos0 + tok;
    const int pos = mine_row && pq >= 0 && pq < p.map.places ? (int)pq : -1;
    const int from = pos - p.window + 1 > 0 ? pos - p.window + 1 : 0;         // of the row's window
    // first and last position of the wave's rows
    const uint64_t on = __ballot(pos >= 0 && lh == 0);
    const int wfirst = on ? __builtin_amdgcn_readlane(pos, (int)__builtin_ctzll(on)) : 0;
    const int wlast = on ? __builtin_amdgcn_readlane(pos, 63 - (int)__builtin_clzll(on)) : -1;

    // Q^T as the B operand: lane l holds query l % 32, dims 16 s + 8 (l / 32) ..
    u32x4_t qf[SL];
    {
        const uint16_t* qp = static_cast<const uint16_t*>(p.Q) + (mine_row ? head : g * p.G) * p.q_head + tq * p.q_token + 8 * lh;
#pragma unroll
        for (int i = 0; i < SL; ++i) qf[i] = *reinterpret_cast<const u32x4_t*>(qp + 16 * i);
    }

    const char* const K = static_cast<const char*>(p.K);
    const char* const V = static_cast<const char*>(p.V);
    const int32_t* const table = p.map.table + t.seq * p.map.table_stride;
    // Page of key `lane` of virtual tile v, -1 where no row attends to it.
    const auto look = [&](int v) __attribute__((always_inline)) {
        const int j = s.key0(v) + lane;
        return v < s.n && j <= s.pmax && (j >= s.lo || j < p.sink) ? table[j >> p.map.shift] : -1;
    };
    const auto place = [&](int v, int page, Places<D>& at) __attribute__((always_inline)) {
        const bool ok = (uint32_t)page < (uint32_t)p.map.pages;
        at.live = __ballot(ok);
        uint32_t row = 0;                               // row 0 always exists
        if (at.live) {
            const uint32_t slot = (uint32_t)(s.key0(v) + lane) & ((1u << p.map.shift) - 1);
            row = (uint32_t)page * p.map.page_rows + ((uint32_t)g << p.map.shift) + slot;
            const uint32_t instead = (uint32_t)__builtin_amdgcn_readlane((int)row, (int)__builtin_ctzll(at.live));
            row = ok ? row : instead;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) at.row[i] = (uint32_t)__shfl((int)row, pc.row + i * Piece<D>::kStep);
    };
    const auto load = [&](const char* x, const Places<D>& at, uint16_t* lds) __attribute__((always_inline)) {
        uint16_t* to = lds + 64 * wave * 8;             // the wave's places
#pragma unroll
        for (int i = 0; i < NP; ++i)
            __builtin_amdgcn_global_load_lds((gptr_t)(x + (uint64_t)at.row[i] * (2 * D) + pc.chunk), (lptr_t)(to + 64 * kWaves * 8 * i),
                                             16, 0, 0);
    };

    f32x16_t o[DB];
    Ref<false> ref;
    float l;
    bool seen;                      // the row attends to something

    // S^T of a tile: lane l holds query l % 32 at keys 32 b + 8 (i / 4) + 4 (l / 32) + i % 4.
    const auto scores = [&](const uint16_t* kl, f32x16_t (&st)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st[b][i] = 0.f;
#pragma unroll
            for (int e = 0; e < SL; ++e) {
                const u32x4_t a = *reinterpret_cast<const u32x4_t*>(kl + (32 * b + lq) * D + 8 * ((2 * e + lh) ^ swizzle<D>(lq)));
                st[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(qf[e]), st[b], 0, 0, 0);
            }
        }
    };
    // The tile at j0 from its scores `st` and values `vl`, with the next tile's scores
    // `nx` from `kn` beside it (kMore).  kSafe: V may hold infinities or NaN.
    const auto compute = [&](auto more, auto safe, f32x16_t (&st)[2], f32x16_t (&nx)[2], const uint16_t* kn, const uint16_t* vl,
                             int j0, uint64_t live) __attribute__((always_inline)) {
        constexpr bool kMore = decltype(more)::value, kSafe = decltype(safe)::value;
        uint64_t mask = ~0ull;      // the row's keys
        if (live != ~0ull || j0 + kKeys - 1 > wfirst || (j0 <= wlast - p.window && j0 + kKeys > p.sink)) {
            mask = below(pos - j0 + 1) & (~below(from - j0) | below(p.sink - j0)) & live;
            const uint64_t m = mask >> (4 * lh);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((uint32_t)(m >> (32 * b)) >> (8 * (i / 4) + i % 4) & 1u)) st[b][i] = -INFINITY;
        }
        seen |= mask != 0;
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
                const uint2 e = lds_read_tr16(vl + (16 * u + r0 + 8) * D + 8 * (c ^ swizzle<D>(r0 + 8)) + 4 * (lane & 1));
                u32x4_t v = {a.x, a.y, e.x, e.y};
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
                for (int k = 0; k < kKeys; ++k)
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int dim = 32 * d + 8 * (i / 4) + 4 * lh + i % 4;
                            const uint16_t v = vl[k * D + 8 * ((dim >> 3) ^ swizzle<D>(k)) + (dim & 7)];
                            if (odd_half(v) && (mask >> k & 1)) o[d][i] += bf16_to_f32(v);
                        }
        }
    };
    // The virtual tiles [first, end).  While one is computed, the next is on its way; where
    // kPipe, K of the next is there already for its scores, and K of the one after that and
    // V of the next are on their way.
    const auto pass = [&](auto safe, int first, int end) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        ref.reset();
        l = 0.f;
        seen = false;
        const int n = end - first;
        // those up to the wave's last position
        const int wt = wlast < 0 ? 0 : (wlast / kKeys >= s.near ? s.sinks + wlast / kKeys - s.near + 1
                                                                : (wlast / kKeys + 1 < s.sinks ? wlast / kKeys + 1 : s.sinks));
        const int mine = wt - first < n ? wt - first : n;
        Places<D> cur, nxt;
        int page = look(first), page1 = look(first + 1);
        place(first, page, cur);
        page = look(first + 2);
        place(first + 1, page1, nxt);
        if (n > 0) {
            load(K, cur, k0);
            load(V, cur, v0);
        }
        if (kPipe && n > 1) load(K, nxt, k1);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        f32x16_t sa[2], sb[2];
        if (kPipe && mine > 0) scores(k0, sa);
        const auto step = [&](int it, f32x16_t (&st)[2], f32x16_t (&nx)[2], uint16_t* kl, const uint16_t* vl, uint16_t* kn,
                              uint16_t* vn) __attribute__((always_inline)) {
            const int j0 = s.key0(first + it);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            const uint64_t live = cur.live;
            if (it + 1 < n) {
                load(V, nxt, vn);
                if (!kPipe) load(K, nxt, kn);
            }
            cur = nxt;
            place(first + it + 2, page, nxt);
            page = look(first + it + 3);
            if (kPipe && it + 2 < n) load(K, nxt, kl);
            if constexpr (!kPipe) {
                if (it < mine && live) {
                    scores(kl, st);
                    compute(std::false_type{}, safe, st, nx, kn, vl, j0, live);
                }
                return;
            }
            if (it >= mine) return;
            if (!live) {
                if (it + 1 < mine) scores(kn, nx);
            } else if (it + 1 < mine) {
                compute(std::true_type{}, safe, st, nx, kn, vl, j0, live);
            } else {
                compute(std::false_type{}, safe, st, nx, kn, vl, j0, live);
            }
        };
        for (int it = 0; it < n; it += 2) {
            step(it, sa, sb, k0, v0, k1, v1);
            if (it + 1 < n) step(it + 1, sb, sa, k1, v1, k0, v0);
        }
    };
    pass(std::false_type{}, 0, s.n);
    float odd = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = fmaf(o[d][i], 0.f, odd);       // NaN if any is not finite
    if (__syncthreads_or((ref.needs_apart(l) || odd != odd) && pos >= 0)) pass(std::true_type{}, 0, s.n);
    l = pair_sum32(l);
    if (!mine_row) return;
    seen &= pos >= 0;
    const float inv = seen ? 1.f / l : 0.f;              // every score -inf: 0 / 0, NaN
    const int64_t at = head * p.o_head + tq * p.o_token + 4 * lh;
    if (!seen) {                                         // nothing attended to: zeros
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store4(p, at + 32 * d + 8 * i, o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv);
}

}  // namespace

int64_t page_attn_blocks(const PageAttnParams& p) { return tile_places(p.T, p.batch, p.tokens) * p.Hkv; }

hipError_t launch_page_attn(const PageAttnParams& p, hipStream_t st) {
    const dim3 grid((unsigned)page_attn_blocks(p));
    if (p.D == 128) hipLaunchKernelGGL(k_page_attn<128>, grid, dim3(64 * kWaves), 0, st, p);
    else hipLaunchKernelGGL(k_page_attn<64>, grid, dim3(64 * kWaves), 0, st, p);
    return hipGetLastError();
}

}  // namespace ris
