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

// ---------------------------------------------------------------------------
// Few row tiles: the key tiles of all of them, one after another for each KV head, are
// one line of units that the workgroups cut into equal parts.  A part may begin and end within a
// row tile; such a row tile's pieces are left in the workspace, and a second launch joins
// them.  Lengths and positions are on the device, so every workgroup works the line out.
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 64 * kWaves;
constexpr int kPlanSeqs = kPlanThreads;         // sequences at most
constexpr int kPlanTiles = 4 * kPlanThreads;    // row tiles of a KV head at most
constexpr int kMinUnits = 4;                    // of a part, where there are many workgroups
constexpr int kMostParts = 768;
constexpr int kMostPlanned = 1 << 27;           // and from which: units of all row tiles are counted in 32 bits
constexpr int kSoloKeys = 512;                  // places to which a row tile is one workgroup's

struct Plan {
    uint32_t tile0[kPlanSeqs + 1];      // a sequence's first row tile
    uint32_t unit0[kPlanTiles + 1];     // a row tile's first unit
    uint32_t carry[kWaves];
};

// Sum of v over the threads before this one; total: over all.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* carry, uint32_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t upto = wave_inclusive_scan(v);
    __syncthreads();
    if (lane == 63) carry[wave] = upto;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before += w < wave ? carry[w] : 0u;
        total += carry[w];
    }
    return before + upto - v;
}

// The last of the n ascending entries (the first is at most v) that is at most v: by the whole
// wave, v uniform, n <= 64 * 64.
__device__ __forceinline__ int last_upto(const uint32_t* x, int n, uint32_t v) {
    const int lane = threadIdx.x & 63;
    const int step = (n + 63) / 64;
    const int lo = step * (__popcll(__ballot(lane * step < n && x[lane * step < n ? lane * step : 0] <= v)) - 1);
    const int at = lo + lane;
    return lo + __popcll(__ballot(lane < step && at < n && x[at < n ? at : 0] <= v)) - 1;
}

struct Line {
    uint32_t tiles;         // row tiles of a KV head
    uint32_t head;          // units of a KV head
    uint64_t units;         // of all
    uint32_t parts;
    __device__ __forceinline__ uint64_t first(uint32_t w) const { return w * units / parts; }
    // The part that holds unit u.
    __device__ __forceinline__ uint32_t owner(uint64_t u) const { return (uint32_t)(((u + 1) * parts - 1) / units); }
};

__device__ __forceinline__ int row_tiles(const PageAttnParams& p, int b) {
    const int len = clip_offset(p.cu[b + 1], p.T) - clip_offset(p.cu[b], p.T);
    return len > 0 ? (len + p.tokens - 1) / p.tokens : 0;
}

__device__ __forceinline__ RowTile row_tile(const PageAttnParams& p, int b, int tile) {
    RowTile t;
    t.seq = b;
    t.first = clip_offset(p.cu[b], p.T);
    t.len = clip_offset(p.cu[b + 1], p.T) - t.first;
    t.tile = tile;
    return t;
}

// Positions of the tokens of a row tile.
__device__ __forceinline__ int tile_tokens(const PageAttnParams& p, const RowTile& t) {
    return t.len - t.tile * p.tokens < p.tokens ? t.len - t.tile * p.tokens : p.tokens;
}
__device__ __forceinline__ int64_t tile_pos(const PageAttnParams& p, const RowTile& t) {
    return first_pos(p, t.seq) + (int64_t)t.tile * p.tokens;
}

__device__ __forceinline__ Line make_plan(const PageAttnParams& p, Plan& plan) {
    const int tid = threadIdx.x;
    Line line;
    const uint32_t mine = tid < p.batch ? (uint32_t)row_tiles(p, tid) : 0u;
    const uint32_t at = block_scan(mine, plan.carry, line.tiles);
    if (tid < p.batch) plan.tile0[tid] = at;
    if (tid == 0) plan.tile0[p.batch] = line.tiles;
    __syncthreads();
    // four neighbouring row tiles a thread; one that attends to nothing counts as one unit
    uint32_t n[4] = {0u, 0u, 0u, 0u};
    const uint32_t t0 = 4u * tid;
    if (t0 < line.tiles) {
        int lo = 0, hi = p.batch;               // tile0[lo] <= t0 < tile0[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (plan.tile0[mid] <= t0) lo = mid;
            else hi = mid;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (t0 + i >= line.tiles) break;
            while (plan.tile0[lo + 1] <= t0 + i) ++lo;
            const RowTile t = row_tile(p, lo, (int)(t0 + i - plan.tile0[lo]));
            const int64_t pos = tile_pos(p, t);
            const int units = span_of(p, pos, pos + tile_tokens(p, t) - 1).n;
            n[i] = units > 0 ? (uint32_t)units : 1u;
        }
    }
    uint32_t before = block_scan(n[0] + n[1] + n[2] + n[3], plan.carry, line.head);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (t0 + i < line.tiles) plan.unit0[t0 + i] = before;
        before += n[i];
    }
    if (tid == 0) plan.unit0[line.tiles] = line.head;
    __syncthreads();
    line.units = (uint64_t)line.head * (uint32_t)p.Hkv;
    const uint64_t most = line.units / kMinUnits;
    line.parts = most < 1 ? 1u : (most < (uint64_t)p.parts ? (uint32_t)most : (uint32_t)p.parts);
    return line;
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

template <int D, bool kSplit>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 3 : 2) void k_page_attn(PageAttnParams p) {
    constexpr int SL = D / 16;      // contraction steps of the score product
    constexpr int DB = D / 32;      // 32-dim blocks of the output
    constexpr int NP = Piece<D>::kCount;
    // two tiles of K and of V; arrays of their own, so that a load into one is not
    // taken for a write to another
    __shared__ __align__(16) uint16_t k0[kKeys * D], k1[kKeys * D], v0[kKeys * D], v1[kKeys * D];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lq = lane & 31, lh = lane >> 5;
    const Piece<D> pc;
    // Where a lane reads: chunk c of row r lies at c ^ swizzle(r), so that its places in a tile are
    // one address, a few bits of it turned (bytes; rows 8 apart turn bit 1 of the chunk).
    const uint32_t k_at = 2 * D * lq + 16 * (lh ^ swizzle<D>(lq));
    const int v_row = 4 * lh + ((lane & 15) >> 2);
    const uint32_t v_at = 2 * D * v_row + 16 * ((2 * (lane >> 4 & 1) + ((lane & 3) >> 1)) ^ swizzle<D>(v_row)) + 8 * (lane & 1);

    // The virtual key tiles [begin, end) of row tile t of KV head g (end < 0: all of them): to out,
    // or to piece `piece` of the workspace where that is not negative.
    const auto run = [&](const RowTile& t, int g, int begin, int end, int piece) __attribute__((always_inline)) {
        const int64_t pos0 = tile_pos(p, t);            // of the tile's first token
        const int ntok = tile_tokens(p, t);
        const Span s = span_of(p, pos0, pos0 + ntok - 1);
        if (end < 0) end = s.n;

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
            uint32_t at = k_at;
            asm volatile("" : "+v"(at));            // 16 addresses made here are cheaper than 16 registers
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) st[b][i] = 0.f;
#pragma unroll
                for (int e = 0; e < SL; ++e) {
                    const u32x4_t a = *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const char*>(kl) + 64 * D * b + (at ^ (32 * e)));
                    st[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(qf[e]), st[b], 0, 0, 0);
                }
            }
        };
        // The row's keys of the tile at j0, all of them where `whole`.
        const auto keys_of = [&](int j0, uint64_t live, bool& whole) __attribute__((always_inline)) {
            whole = live == ~0ull && j0 + kKeys - 1 <= wfirst && (j0 > wlast - p.window || j0 + kKeys <= p.sink);
            return whole ? ~0ull : below(pos - j0 + 1) & (~below(from - j0) | below(p.sink - j0)) & live;
        };
        // The tile at j0 from its scores and values `vl`.  safe: the pass over a tile whose outputs were not
        // finite, or whose references were far.
        const auto compute = [&](bool safe, const uint16_t* kl, const uint16_t* vl, int j0, uint64_t live) __attribute__((always_inline)) {
            f32x16_t st[2];
            scores(kl, st);
            bool whole;
            const uint64_t mask = keys_of(j0, live, whole);
            if (!whole) {
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
                const float al = safe ? ref.template raise<true>(mx, p.c) : ref.template raise<false>(mx, p.c);
                l *= al;
                if (safe) {
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] = scaled<true>(o[d][i], al);
                } else {
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] *= al;
                }
            }
            // Exponents are s c - mc; of rows apart, (s - m) c - 0.
            float mc = ref.mc;
            if (safe && ref.apart) {
                const float m = ref.m == -INFINITY ? 0.f : ref.m;
                mc = 0.f;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) st[b][i] -= m;
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
            uint32_t at = v_at;
            asm volatile("" : "+v"(at));
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const char* x = reinterpret_cast<const char*>(vl) + 32 * D * u;
                    const uint2 a = lds_read_tr16(reinterpret_cast<const uint16_t*>(x + (at ^ (64 * d))));
                    const uint2 e = lds_read_tr16(reinterpret_cast<const uint16_t*>(x + 16 * D + (at ^ (64 * d) ^ 32)));
                    const u32x4_t v = {a.x, a.y, e.x, e.y};
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pf[u]), o[d], 0, 0, 0);
                }
        };
        // A weight of 0, masked or too small for float32, times an infinity or NaN of V would be NaN: in the safe
        // pass such elements are added, whatever their weight, where they are attended to, and taken out
        // of the tile before the product.
        const auto take_out = [&](bool attends, uint16_t* vl, int j0, uint64_t live) __attribute__((always_inline)) {
            int half = 4 * lh, tid = threadIdx.x;
            asm volatile("" : "+v"(half), "+v"(tid));       // nothing of this is worth registers in the other pass
            bool odd = false;
#pragma unroll 1
            for (int at = 2 * (tid & 63); at < kKeys * D; at += 2 * 64) {
                const uint32_t x = *reinterpret_cast<const uint32_t*>(vl + at);
                odd |= finite_only(x) != x;
            }
            odd = __any(odd);
            if (odd && attends) {
                bool whole;
                const uint64_t mask = keys_of(j0, live, whole);
#pragma unroll 1
                for (int k = 0; k < kKeys; ++k)
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int dim = 32 * d + 8 * (i / 4) + half + i % 4;
                            const uint16_t v = vl[k * D + 8 * ((dim >> 3) ^ swizzle<D>(k)) + (dim & 7)];
                            if (odd_half(v) && (mask >> k & 1)) o[d][i] += bf16_to_f32(v);
                        }
            }
            __syncthreads();
            if (odd) {
#pragma unroll 1
                for (int at = 2 * tid; at < kKeys * D; at += 2 * 64 * kWaves) {
                    uint32_t* x = reinterpret_cast<uint32_t*>(vl + at);
                    *x = finite_only(*x);
                }
            }
            __syncthreads();
        };
        // The virtual tiles [first, end).  While one is computed, the next is on its way.
        for (bool safe = false;; safe = true) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
            ref.reset();
            l = 0.f;
            seen = false;
            const int n = end - begin;
            // those up to the wave's last position
            const int wt = wlast < 0 ? 0 : (wlast / kKeys >= s.near ? s.sinks + wlast / kKeys - s.near + 1
                                                                    : (wlast / kKeys + 1 < s.sinks ? wlast / kKeys + 1 : s.sinks));
            const int mine = wt - begin < n ? wt - begin : n;
            Places<D> at;
            int page = look(begin);
            place(begin, page, at);
            page = look(begin + 1);
            if (n > 0) {
                load(K, at, k0);
                load(V, at, v0);
            }
            const auto step = [&](int it, const uint16_t* kl, uint16_t* vl, uint16_t* kn, uint16_t* vn) __attribute__((always_inline)) {
                const int j0 = s.key0(begin + it);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                const uint64_t live = at.live;
                place(begin + it + 1, page, at);
                page = look(begin + it + 2);
                if (it + 1 < n) {
                    load(K, at, kn);
                    load(V, at, vn);
                }
                if (safe) take_out(it < mine, vl, j0, live);
                if (it < mine && live) compute(safe, kl, vl, j0, live);
            };
            for (int it = 0; it < n; it += 2) {
                step(it, k0, v0, k1, v1);
                if (it + 1 < n) step(it + 1, k1, v1, k0, v0);
            }
            if (safe) break;
            float odd = 0.f;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) odd = fmaf(o[d][i], 0.f, odd);       // NaN if any is not finite
            if (!__syncthreads_or((ref.needs_apart(l) || odd != odd) && pos >= 0)) break;
        }
        __syncthreads();                // the tiles' places are free
        l = pair_sum32(l);
        if (!mine_row) return;
        seen &= pos >= 0;
        if (kSplit && piece >= 0) {
            const int64_t at = (int64_t)piece * p.part_rows + r;
            if (lh == 0) *reinterpret_cast<f32x4_t*>(p.part_ml + 4 * at) = f32x4_t{ref.m, ref.mc, l, seen ? 1.f : 0.f};
            float* to = p.part_o + at * D + 4 * lh;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4_t*>(to + 32 * d + 8 * i) = f32x4_t{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
            return;
        }
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
    };

    if constexpr (kSplit) {
        __shared__ Plan plan;
        const Line line = make_plan(p, plan);
        // neighbouring parts on one XCD, all XCDs alike
        const uint32_t each = (line.parts + 7) / 8, w = (blockIdx.x & 7u) * each + (blockIdx.x >> 3);
        if ((blockIdx.x >> 3) >= each || w >= line.parts) return;
        const uint64_t stop = line.first(w + 1);
        for (uint64_t u = line.first(w); u < stop;) {
            const uint32_t g = (uint32_t)(u / line.head), at = (uint32_t)(u - (uint64_t)g * line.head);
            const int tile = __builtin_amdgcn_readfirstlane(last_upto(plan.unit0, (int)line.tiles, at));
            const int b = __builtin_amdgcn_readfirstlane(last_upto(plan.tile0, p.batch, (uint32_t)tile));
            const uint32_t begin = at - plan.unit0[tile], all = plan.unit0[tile + 1] - plan.unit0[tile];
            const uint32_t end = begin + (stop - u) < all ? (uint32_t)(begin + (stop - u)) : all;
            const int piece = begin == 0 && end == all ? -1 : 2 * (int)w + (begin == 0);
            run(row_tile(p, b, tile - (int)plan.tile0[b]), (int)g, (int)begin, (int)end, piece);
            u += end - begin;
        }
    } else {
        RowTile t;
        if (!find_tile(p.cu, p.batch, p.T, p.tokens, blockIdx.x / p.Hkv, t)) return;
        run(t, (int)(blockIdx.x % p.Hkv), 0, -1, -1);
    }
}

// The pieces of the row tiles that several parts share, joined: a workgroup takes a row tile of a
// KV head and its rows blockIdx.y, + gridDim.y, ...; the threads find the largest reference and
// each piece's factor together, then D / 4 lanes of four dims each sum over every kGroups-th
// piece.
template <int D>
__global__ __launch_bounds__(kPlanThreads) void k_page_join(PageAttnParams p) {
    constexpr int kLanes = D / 4, kGroups = kPlanThreads / kLanes;
    __shared__ Plan plan;
    __shared__ float factor[kMostParts];
    __shared__ float red[kWaves][4];
    __shared__ __align__(16) float osum[kGroups][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Line line = make_plan(p, plan);
    const uint32_t tile = blockIdx.x / p.Hkv, g = blockIdx.x % p.Hkv;
    if (tile >= line.tiles) return;
    const uint64_t u = (uint64_t)g * line.head + plan.unit0[tile];
    const uint32_t w0 = line.owner(u), n = line.owner(u + (plan.unit0[tile + 1] - plan.unit0[tile]) - 1) - w0 + 1;
    if (n == 1) return;
    const int b = __builtin_amdgcn_readfirstlane(last_upto(plan.tile0, p.batch, tile));
    const RowTile t = row_tile(p, b, (int)(tile - plan.tile0[b]));
    const int rows = tile_tokens(p, t) * p.G;
    // the first piece is the end of part w0, the others begin their parts
    const auto piece = [&](uint32_t i) { return (int64_t)(2 * (w0 + i) + (i == 0)) * p.part_rows; };
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        float top = -INFINITY, topc = 0.f;
        bool far = false;
        for (uint32_t i = tid; i < n; i += kPlanThreads) {
            const f32x4_t ml = *reinterpret_cast<const f32x4_t*>(p.part_ml + 4 * (piece(i) + r));
            topc = top < ml[0] ? ml[1] : topc;
            top = fmaxf(top, ml[0]);
            far |= far_ref(ml[1]);
        }
        const float wtop = wave_max(top);
        const uint64_t has = __ballot(top == wtop);         // none where top is NaN: not raised to one
        topc = __shfl(topc, has ? (int)__builtin_ctzll(has) : 0);
        far = __any(far);
        __syncthreads();
        if (lane == 0) {
            red[wave][0] = wtop;
            red[wave][1] = topc;
            red[wave][2] = far ? 1.f : 0.f;
        }
        __syncthreads();
        top = -INFINITY;
        topc = 0.f;
        far = false;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            topc = top < red[w][0] ? red[w][1] : topc;
            top = fmaxf(top, red[w][0]);
            far |= red[w][2] != 0.f;
        }
        float l = 0.f, seen = 0.f;
        for (uint32_t i = tid; i < n; i += kPlanThreads) {
            const f32x4_t ml = *reinterpret_cast<const f32x4_t*>(p.part_ml + 4 * (piece(i) + r));
            const float a = join_factor<false>(ml[0], ml[1], top, topc, far, p.c);
            factor[i] = a;
            l = fmaf(ml[2], a, l);
            seen += ml[3];
        }
        l = wave_sum(l);
        seen = wave_sum(seen);
        __syncthreads();
        if (lane == 0) {
            red[wave][0] = l;
            red[wave][1] = seen;
        }
        const int grp = tid / kLanes, d4 = 4 * (tid % kLanes);
        __syncthreads();
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (uint32_t i = grp; i < n; i += kGroups) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(p.part_o + (piece(i) + r) * D + d4);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = add_scaled<true>(o[e], x[e], factor[i]);
        }
        *reinterpret_cast<f32x4_t*>(&osum[grp][d4]) = o;
        __syncthreads();
        if (tid < kLanes) {
            l = seen = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                l += red[w][0];
                seen += red[w][1];
            }
            f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kGroups; ++k) y += *reinterpret_cast<const f32x4_t*>(&osum[k][d4]);
            const int tok = r / p.G, h = g * p.G + (r - tok * p.G);
            const int64_t at = h * p.o_head + (int64_t)(t.first + t.tile * p.tokens + tok) * p.o_token + d4;
            if (seen == 0.f) store4(p, at, 0.f, 0.f, 0.f, 0.f);
            else store4(p, at, y[0] / l, y[1] / l, y[2] / l, y[3] / l);
        }
    }
}

}  // namespace

int64_t page_attn_blocks(const PageAttnParams& p) { return tile_places(p.T, p.batch, p.tokens) * p.Hkv; }

// Workgroups that share the units, as many as the card holds at once; 0: a workgroup to a
// row tile.
int32_t page_attn_parts(const PageAttnParams& p) {
    if (p.batch > kPlanSeqs || p.T / p.tokens + p.batch > kPlanTiles) return 0;
    if (p.map.places <= kSoloKeys || p.map.places > kMostPlanned) return 0;
    if (page_attn_blocks(p) >= 1024) return 0;      // they fill the card by themselves
    return p.D == 128 ? 512 : 768;
}

int64_t page_attn_workspace(const PageAttnParams& p) {
    return 2 * (int64_t)p.parts * p.part_rows * (p.D + 4) * (int64_t)sizeof(float);
}

template <int D>
static hipError_t launch_page_attn_d(const PageAttnParams& p, hipStream_t st) {
    const int64_t tiles = page_attn_blocks(p);
    if (p.parts == 0) {
        hipLaunchKernelGGL((k_page_attn<D, false>), dim3((unsigned)tiles), dim3(64 * kWaves), 0, st, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((k_page_attn<D, true>), dim3((unsigned)p.parts), dim3(64 * kWaves), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int64_t deal = 1024 / tiles;                    // rows side by side where row tiles are few
    deal = deal < 1 ? 1 : (deal > p.part_rows ? p.part_rows : deal);
    hipLaunchKernelGGL(k_page_join<D>, dim3((unsigned)tiles, (unsigned)deal), dim3(kPlanThreads), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_page_attn(const PageAttnParams& p, hipStream_t st) {
    return p.D == 128 ? launch_page_attn_d<128>(p, st) : launch_page_attn_d<64>(p, st);
}

}  // namespace ris
