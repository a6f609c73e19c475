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
// Bound by the matrix unit where it is fed: 4 D flops a (query head, key) pair at 0.77 to 0.86 PFLOP/s (2,048 tokens after
// 30,000, 12/2 heads of 128: 453 to 485 us on several machines for 390 GFLOP; 16,384 of three sequences under a window of 4,096:
// 490 to 537 for 413), the unit busy 42% and 38% of the time.  A wave's exponentials and its products follow each other, and of two waves a SIMD
// one is often at a barrier for the next tile (in the first case 71% of the requests for K and V miss
// L2: 18.5 million of 128 bytes, 2.4 GB, a pass).  Weights and values of the next 16 keys are made beside a product.
// Measured and not kept: eight waves of 256 rows with three tiles in LDS, half the reads (438 for 475 there, but 537 for
// 502 under the window and 112 for 92 in a mixed batch); the next tile's scores beside this one's exponentials, with no
// registers left for it (449 -> 489, 496 -> 598); one scalar load of a page for a tile that lies in it
// (455 -> 464, 508 -> 523, mixed 85.7 -> 88.0).
// Softmax weights are rounded to bf16 for the PV product, as in the other attention kernels here: in float32 it would
// run at a sixteenth of the rate, in two bf16 parts at half of it.  An output is off by 2^-8 of the largest value at most for
// it, 2.3e-3 of itself in the root mean square with its own rounding, which alone is 1.7e-3.
#include "page_rows.h"
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

// ---------------------------------------------------------------------------
// Few row tiles: their key tiles, one after another for each KV head, are one line that the
// workgroups cut into equal parts.  A part may begin and end within a row tile; the pieces of such a
// row tile are left in the workspace, and a second launch joins them.  Lengths and positions are on
// the device, so every workgroup works the line out.
//
// (Cutting sequences by slices of their keys, so that neighbouring parts read the same keys at one
// time, gave nothing: 2,048 tokens after 30,000 486 -> 494 us, 600 with 31 other sequences 117 -> 162.
// Nor did counting a key tile for half where one wave's rows read it: 106 for 112, such parts waiting
// for memory.)
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 64 * kWaves;
constexpr int kPlanSeqs = kPlanThreads;         // sequences at most
constexpr int kMostTiles = 1024;                // row tiles of all KV heads
static_assert(kPartList >= 4 * kMostTiles + 1);
constexpr uint32_t kMinUnits = 4;               // of a part, where there are many workgroups
constexpr int kMostParts = 768;
constexpr int kMostPlanned = 1 << 27;           // places up to which the key tiles of all row tiles are counted in 32 bits
constexpr int kSoloKeys = 512;                  // places to which a row tile is one workgroup's

struct Plan {
    uint32_t tile0[kPlanSeqs + 1];      // a sequence's first row tile
    uint32_t unit0[kMostTiles + 1];     // a row tile's first unit
    uint32_t carry[kWaves];
    // a sequence's first new token, its tokens and its first position, near enough to the cache
    int32_t first[kPlanSeqs], len[kPlanSeqs];
    int64_t pos[kPlanSeqs];
    // Row tile `tile` of sequence b.
    __device__ __forceinline__ RowTile row_tile(int b, int tile) const {
        RowTile t;
        t.seq = b;
        t.first = first[b];
        t.len = len[b];
        t.tile = tile;
        return t;
    }
};

// In a piece's fourth number, else 1 where its row attends to something and 0 where not: it does,
// and its weights were taken at m c (see join_factor).
constexpr float kApart = 2.f;

// What the second launch needs of a row tile of a KV head: its pieces are the end of part
// `part` and the beginnings of the parts behind it.
struct Pieces {
    int32_t count, part, seq, tile;
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
    uint32_t head;          // units of a KV head: key tiles of its row tiles
    uint64_t units;         // of all
    uint32_t parts;
    __device__ __forceinline__ uint64_t first(uint32_t w) const { return w * units / parts; }
    // The part that holds unit u.
    __device__ __forceinline__ uint32_t owner(uint64_t u) const { return (uint32_t)(((u + 1) * parts - 1) / units); }
};

__device__ __forceinline__ Line make_plan(const PageAttnParams& p, Plan& plan) {
    const int tid = threadIdx.x;
    Line line;
    uint32_t mine = 0;
    if (tid < p.batch) {
        const int64_t from = p.cu[tid], to = p.cu[tid + 1], pos = first_pos(p, tid);
        plan.first[tid] = clip_offset(from, p.T);
        plan.len[tid] = clip_offset(to, p.T) - plan.first[tid];
        plan.pos[tid] = pos;
        if (plan.len[tid] > 0) mine = (uint32_t)(plan.len[tid] + p.tokens - 1) / (uint32_t)p.tokens;
    }
    const uint32_t at = block_scan(mine, plan.carry, line.tiles);
    // offsets that do not ascend could make more row tiles than there is room for: those are left out
    const uint32_t room = (uint32_t)(kMostTiles / p.Hkv);
    line.tiles = line.tiles < room ? line.tiles : room;
    if (tid < p.batch) plan.tile0[tid] = at < room ? at : room;
    if (tid == 0) plan.tile0[p.batch] = line.tiles;
    __syncthreads();
    // kEach neighbouring row tiles a thread; one that attends to nothing counts as one key tile
    constexpr int kEach = kMostTiles / kPlanThreads;
    uint32_t n[kEach], sum = 0;
    const uint32_t t0 = (uint32_t)kEach * tid;
    int b = 0;
    if (t0 < line.tiles) {
        int hi = p.batch;                       // tile0[b] <= t0 < tile0[hi]
        while (hi - b > 1) {
            const int mid = (b + hi) / 2;
            if (plan.tile0[mid] <= t0) b = mid;
            else hi = mid;
        }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        n[i] = 0;
        if (t0 + i >= line.tiles) continue;
        while (plan.tile0[b + 1] <= t0 + i) ++b;
        const RowTile t = plan.row_tile(b, (int)(t0 + i - plan.tile0[b]));
        const int64_t pos = tile_pos(p, plan.pos[b], t);
        const int tokens = tile_tokens(p, t), keys = span_of<kKeys>(p, pos, pos + tokens - 1).n;
        n[i] = keys > 0 ? (uint32_t)keys : 1u;
        sum += n[i];
    }
    uint32_t before = block_scan(sum, plan.carry, line.head);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (t0 + i < line.tiles) plan.unit0[t0 + i] = before;
        before += n[i];
    }
    if (tid == 0) plan.unit0[line.tiles] = line.head;
    __syncthreads();
    line.units = (uint64_t)line.head * (uint32_t)p.Hkv;
    const uint64_t fill = line.units / kMinUnits;
    line.parts = fill < 1 ? 1u : (fill < (uint64_t)p.parts ? (uint32_t)fill : (uint32_t)p.parts);
    return line;
}

// Where the lanes' pieces of a key tile lie, and which of its keys are live.
template <int D>
struct Places {
    uint32_t row[Piece<D>::kCount];
    uint64_t live;
};

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

    // The virtual key tiles [begin, end) of row tile t, whose tokens' positions begin at pos0, of KV head g
    // (end < 0: all of them): to out
    // where they are all of its, else to piece `piece` of the workspace.
    const auto run = [&](const RowTile& t, int64_t pos0, int g, int begin, int end, int piece) __attribute__((always_inline)) {
        const int ntok = tile_tokens(p, t);
        const Span<kKeys> s = span_of<kKeys>(p, pos0, pos0 + ntok - 1);
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
                float al = safe ? ref.template raise<true>(mx, p.c) : ref.template raise<false>(mx, p.c);
                l *= al;
                if (safe) al = kept_infinite(al);
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= al;
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
            // O^T += V^T P^T over 16 keys at a time, u: slot e of lane half lh holds key 16 u + 4 lh + e (e < 4) or 16 u +
            // 8 + 4 lh + e - 4.  Values and weights of the next 16 keys are made beside a product.
            u32x4_t pf[2], vf[2][DB];
            const auto weigh = [&](int u) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(st[u / 2][8 * (u % 2) + i], p.c, -mc));
                    const float y = __builtin_amdgcn_exp2f(fmaf(st[u / 2][8 * (u % 2) + i + 1], p.c, -mc));
                    l += x + y;
                    pf[u % 2][i / 2] = pack_bf16x2(x, y);
                }
            };
            uint32_t at = v_at;
            asm volatile("" : "+v"(at));
            const auto read = [&](int u) __attribute__((always_inline)) {
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const char* x = reinterpret_cast<const char*>(vl) + 32 * D * u;
                    const uint2 a = lds_read_tr16(reinterpret_cast<const uint16_t*>(x + (at ^ (64 * d))));
                    const uint2 e = lds_read_tr16(reinterpret_cast<const uint16_t*>(x + 16 * D + (at ^ (64 * d) ^ 32)));
                    vf[u % 2][d] = u32x4_t{a.x, a.y, e.x, e.y};
                }
            };
            read(0);
            weigh(0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (u < 3) {
                    read(u + 1);
                    weigh(u + 1);
                }
#pragma unroll
                for (int d = 0; d < DB; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf[u % 2][d]), as_bf16x8(pf[u % 2]), o[d], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
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
        if (kSplit && (begin > 0 || end < s.n)) {
            const int64_t at = (int64_t)piece * p.part_rows + r;
            if (lh == 0) *reinterpret_cast<f32x4_t*>(p.part_ml + 4 * at) = f32x4_t{ref.m, ref.mc, l, seen ? (ref.apart ? kApart : 1.f) : 0.f};
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
        // neighbouring parts on one XCD, all XCDs alike (8, 16 or 32 neighbours at a time to an XCD: 600 tokens with 31
        // steps 89 -> 91 to 94 us, 2,048 after 30,000 473 -> 475 to 478)
        const uint32_t each = (line.parts + 7) / 8, w = (blockIdx.x & 7u) * each + (blockIdx.x >> 3);
        if ((blockIdx.x >> 3) >= each || w >= line.parts) return;
        Pieces* const list = reinterpret_cast<Pieces*>(p.part_list);
        if (w == 0 && threadIdx.x == 0) p.part_list[4 * kMostTiles] = (int32_t)line.tiles;
        const uint64_t stop = line.first(w + 1);
        for (uint64_t u = line.first(w); u < stop;) {
            const uint32_t g = (uint32_t)(u / line.head), at = (uint32_t)(u - (uint64_t)g * line.head);
            const int i = __builtin_amdgcn_readfirstlane(last_upto(plan.unit0, (int)line.tiles, at));
            const int b = __builtin_amdgcn_readfirstlane(last_upto(plan.tile0, p.batch, (uint32_t)i));
            const RowTile t = plan.row_tile(b, i - (int)plan.tile0[b]);
            const uint32_t begin = at - plan.unit0[i], all = plan.unit0[i + 1] - plan.unit0[i];
            const uint32_t end = begin + (stop - u) < all ? (uint32_t)(begin + (stop - u)) : all;
            if (begin == 0 && threadIdx.x == 0)
                list[(uint32_t)i * p.Hkv + g] = Pieces{(int32_t)(line.owner(u + all - 1) - w) + 1, (int32_t)w, b, t.tile};
            run(t, tile_pos(p, plan.pos[b], t), (int)g, (int)begin, (int)end, 2 * (int)w + (begin == 0));
            u += end - begin;
        }
    } else {
        RowTile t;
        if (!find_tile(p.cu, p.batch, p.T, p.tokens, blockIdx.x / p.Hkv, t)) return;
        run(t, tile_pos(p, first_pos(p, t.seq), t), (int)(blockIdx.x % p.Hkv), 0, -1, -1);
    }
}

// The pieces of the row tiles that are in several, joined: a workgroup takes a row tile of a KV
// head and its rows from blockIdx.y on.  Few pieces: a wave a row.  Many: the threads find
// the largest reference and each piece's factor together, then D / 4 lanes of four dims each sum
// over every kGroups-th piece.
constexpr int kFewPieces = 16;

struct RowRef {
    float top = -INFINITY, topc = 0.f, kind = 0.f;
    __device__ __forceinline__ void meet(float m, float mc, float k) {
        kind = top < m ? k : kind;
        topc = top < m ? mc : topc;
        top = fmaxf(top, m);
    }
    // Over the wave.
    __device__ __forceinline__ void join() {
        const float all = wave_max(top);
        const int at = (int)__builtin_ctzll(__ballot(top == all));
        topc = __shfl(topc, at);
        kind = __shfl(kind, at);
        top = all;
    }
    __device__ __forceinline__ float factor(const f32x4_t& ml, float c) const {
        return join_factor<false>(ml[0], ml[1], ml[3] == kApart, top, topc, kind == kApart, c);
    }
};

template <int D>
__global__ __launch_bounds__(kPlanThreads) void k_page_join(PageAttnParams p) {
    constexpr int kLanes = D / 4, kGroups = kPlanThreads / kLanes;
    __shared__ float factor[kMostParts];
    __shared__ float red[kWaves][4];
    __shared__ __align__(16) float osum[kGroups][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t tile = blockIdx.x / p.Hkv, g = blockIdx.x % p.Hkv;
    if (tile >= (uint32_t)p.part_list[4 * kMostTiles]) return;
    const Pieces all = reinterpret_cast<const Pieces*>(p.part_list)[blockIdx.x];
    const int n = all.count;
    if (n == 1) return;
    RowTile t;
    t.seq = all.seq;
    t.first = clip_offset(p.cu[all.seq], p.T);
    t.len = clip_offset(p.cu[all.seq + 1], p.T) - t.first;
    t.tile = all.tile;
    const int rows = tile_tokens(p, t) * p.G;
    const auto piece = [&](int i) __attribute__((always_inline)) { return (int64_t)(2 * (all.part + i) + (i == 0)) * p.part_rows; };
    const auto sums = [&](int i, int r) __attribute__((always_inline)) {
        return *reinterpret_cast<const f32x4_t*>(p.part_ml + 4 * (piece(i) + r));
    };
    const auto place = [&](int r) __attribute__((always_inline)) {
        const int tok = r / p.G, h = (int)g * p.G + (r - tok * p.G);
        return h * p.o_head + (int64_t)(t.first + t.tile * p.tokens + tok) * p.o_token;
    };
    if (n <= kFewPieces) {
        constexpr int kEach = D / 64;           // dims of a lane
        for (int r = (int)blockIdx.y * kWaves + wave; r < rows; r += (int)gridDim.y * kWaves) {
            f32x4_t ml = {-INFINITY, 0.f, 0.f, 0.f};
            if (lane < n) ml = sums(lane, r);
            RowRef ref;
            ref.meet(ml[0], ml[1], ml[3]);
            ref.join();
            const float a = ref.factor(ml, p.c);
            const float l = wave_sum(ml[2] * a), seen = wave_sum(ml[3]);
            float y[kEach] = {};
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                const float* x = p.part_o + (piece(i) + r) * D + kEach * lane;
                const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(a), i));
#pragma unroll
                for (int e = 0; e < kEach; ++e) y[e] = add_scaled<true>(y[e], x[e], f);
            }
            const int64_t at = place(r) + kEach * lane;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const float v = seen == 0.f ? 0.f : y[e] / l;
                if (p.out_bf16) static_cast<uint16_t*>(p.out)[at + e] = f32_to_bf16(v);
                else static_cast<float*>(p.out)[at + e] = v;
            }
        }
        return;
    }
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        RowRef ref;
        for (int i = tid; i < n; i += kPlanThreads) {
            const f32x4_t ml = sums(i, r);
            ref.meet(ml[0], ml[1], ml[3]);
        }
        ref.join();
        __syncthreads();
        if (lane == 0) {
            red[wave][0] = ref.top;
            red[wave][1] = ref.topc;
            red[wave][2] = ref.kind;
        }
        __syncthreads();
        ref = RowRef();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) ref.meet(red[w][0], red[w][1], red[w][2]);
        float l = 0.f, seen = 0.f;
        for (int i = tid; i < n; i += kPlanThreads) {
            const f32x4_t ml = sums(i, r);
            const float a = ref.factor(ml, p.c);
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
        for (int i = grp; i < n; i += kGroups) {
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
            const int64_t at = place(r) + d4;
            if (seen == 0.f) store4(p, at, 0.f, 0.f, 0.f, 0.f);
            else store4(p, at, y[0] / l, y[1] / l, y[2] / l, y[3] / l);
        }
    }
}

}  // namespace

int64_t page_attn_blocks(const PageAttnParams& p) { return tile_places(p.T, p.batch, p.tokens) * p.Hkv; }

// Workgroups that share the units, as many as the card holds at once (2,048 tokens after 30,000 486 us, with 256 679);
// 0: a workgroup to a row tile.
int32_t page_attn_parts(const PageAttnParams& p) {
    if (p.batch > kPlanSeqs) return 0;
    if (p.map.places <= kSoloKeys || p.map.places > kMostPlanned) return 0;
    if ((p.T / p.tokens + p.batch) * p.Hkv >= kMostTiles) return 0;      // they fill the card by themselves
    return p.D == 128 ? 512 : 768;
}

int64_t page_attn_pieces(const PageAttnParams& p) {
    if (!p.step) return 2 * (int64_t)p.parts;
    return p.parts > p.part_waves ? page_attn_blocks(p) * (p.parts / p.part_waves) : 0;        // a row tile's only workgroup writes out itself
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
    int64_t deal = 2048 / tiles;                    // rows side by side where row tiles are few
    deal = deal < 1 ? 1 : (deal > p.part_rows ? p.part_rows : deal);
    hipLaunchKernelGGL(k_page_join<D>, dim3((unsigned)tiles, (unsigned)deal), dim3(kPlanThreads), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_page_attn(const PageAttnParams& p, hipStream_t st) {
    if (p.step) return launch_page_step(p, st);
    return p.D == 128 ? launch_page_attn_d<128>(p, st) : launch_page_attn_d<64>(p, st);
}

}  // namespace ris
