// Log probabilities of given tokens, entropy and the largest logits of a row, in
// one pass over the row: a thread keeps the running maximum m, the sum of
// exp(x - m) and the sum of exp(x - m) (x - m) of what it has read, a wave the
// top_k largest logits as a list over its lanes.  Then log p = x - m - log(sum) and
// the entropy is log(sum) - sum(exp(x - m) (x - m)) / sum.
//
// HBM-bound, and close to it by VALU: 16-byte loads, the exponent's argument as one
// fma in the log2 domain, and a list that few logits reach (see `start_at`).  A row
// is cut into parts where rows are few; each part's workgroup leaves its state and
// list in the workspace, and one wave a row merges them.
#include "ris_device.h"
#include "ris_internal.h"

namespace ris {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kUnroll = 4;          // vectors a thread loads at a time
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFar = -1e30f;      // stands for -inf in products with a weight of 0
// Magnitudes of a maximum up to which its product with log2 e, rounded, may be the
// weights' reference: it is off by half a unit there, and weights by 2^0.5 alike (at 1e30
// by 2^(2^75): infinite or 0).
constexpr float kNear = 8388608.f;

// Keys order logits as they compare, equal ones by descending id: the float's bits
// made monotone, then the id's complement.  NaN ranks first, 0 is no token.
__device__ __forceinline__ uint32_t order_of(float x) {
    uint32_t u = __float_as_uint(x + 0.f);              // -0 is 0
    if (x != x) u = 0x7FFFFFFFu;
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t id) { return (uint64_t)order_of(x) << 32 | (uint32_t)~id; }
constexpr uint64_t kNothing = 0x007FFFFFull << 32 | 0xFFFFFFFFull;   // -inf: keys up to here are not listed

struct State {
    float m, l, u;      // maximum, sum of exp(x - m), sum of exp(x - m) (x - m)
};

__device__ __forceinline__ void add(State& s, float x) {
    if (x > s.m) {
        const float d = s.m - x, a = __builtin_amdgcn_exp2f(d * kLog2e);      // 0 where m is -inf
        s.u = a * fmaf(s.l, fmaxf(d, kFar), s.u);
        s.l *= a;
        s.m = x;
    }
    const float d = x - (s.m == -INFINITY ? 0.f : s.m), w = __builtin_amdgcn_exp2f(d * kLog2e);
    s.l += w;
    s.u = fmaf(w, fmaxf(d, kFar), s.u);
}

// s at the maximum m >= s.m.
__device__ __forceinline__ State raise(State s, float m) {
    const float d = s.m == m ? 0.f : s.m - m, f = __builtin_amdgcn_exp2f(d * kLog2e);
    return State{m, f * s.l, f * fmaf(s.l, fmaxf(d, kFar), s.u)};
}
__device__ __forceinline__ State wave_merge(State s) {
    s = raise(s, wave_max(s.m));
    return State{s.m, wave_sum(s.l), wave_sum(s.u)};
}

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

template <int CTRL, int ROW_MASK = 0xF>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v, uint32_t otherwise) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)otherwise, (int)v, CTRL, ROW_MASK, 0xF, false);
}

// Keys of the wave's lanes into its list: lane i holds the i-th largest, 0 where
// there is none; a key enters above `least`, which is at least the k-th.
__device__ __forceinline__ void insert(uint64_t& list, uint64_t& least, uint64_t key, int k) {
    const int lane = threadIdx.x & 63;
    uint64_t todo = __ballot(key > least);
    while (todo) {
        const int from = (int)__builtin_ctzll(todo);
        const uint64_t v = lane_value(key, from);
        const int at = __popcll(__ballot(list > v));
        // the list one lane on (wave_shr:1)
        const uint64_t up = (uint64_t)dpp_u32<0x138>((uint32_t)(list >> 32), 0) << 32 | dpp_u32<0x138>((uint32_t)list, 0);
        list = lane < at ? list : (lane == at ? v : up);
        const uint64_t kth = lane_value(list, k - 1);
        least = kth > least ? kth : least;
        todo &= __ballot(key > least) & ~(1ull << from);
    }
}

// A lower bound, in its upper 16 bits, of the n-th largest of the lanes' orders.
__device__ __forceinline__ uint32_t nth_largest(uint32_t order, int n) {
    uint32_t t = 0;
    for (uint32_t bit = 0x80000000u; bit > 0x8000u; bit >>= 1)
        if (__popcll(__ballot(order >= (t | bit))) >= n) t |= bit;
    return t;
}

// Largest key over the lanes.
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
    const auto up = [](uint64_t a, uint32_t hi, uint32_t lo) {
        const uint64_t b = (uint64_t)hi << 32 | lo;
        return b > a ? b : a;
    };
#define RIS_STEP(CTRL, MASK) v = up(v, dpp_u32<CTRL, MASK>((uint32_t)(v >> 32), 0), dpp_u32<CTRL, MASK>((uint32_t)v, 0))
    RIS_STEP(0xB1, 0xF);        // quad_perm [1,0,3,2]
    RIS_STEP(0x4E, 0xF);        // quad_perm [2,3,0,1]
    RIS_STEP(0x141, 0xF);       // row_half_mirror
    RIS_STEP(0x140, 0xF);       // row_mirror
    RIS_STEP(0x142, 0xA);       // row_bcast:15
    RIS_STEP(0x143, 0xC);       // row_bcast:31
#undef RIS_STEP
    return lane_value(v, 63);
}

template <bool BF16>
__device__ __forceinline__ float load(const LogprobParams& p, int64_t at) {
    return BF16 ? bf16_to_f32(static_cast<const uint16_t*>(p.logits)[at]) : static_cast<const float*>(p.logits)[at];
}

// log p from the row's state; a row of -inf alone has l = 0.
struct Row {
    float m, log_l;
    __device__ float logprob(float x) const { return x == -INFINITY && log_l == log_l ? x : x - m - log_l; }
};

template <bool BF16>
__device__ __forceinline__ Row finish_row(const LogprobParams& p, int64_t row, State s, int first, int step) {
    const float log_l = __builtin_amdgcn_logf(s.l) * kLn2;
    const Row r{s.m, log_l};
    if (first == 0 && p.entropy) p.entropy[row] = s.l == 0.f ? 0.f : log_l - s.u / s.l;
    for (int i = first; i < p.n_targets; i += step) {
        const int64_t t = p.targets[row * p.n_targets + i];
        p.logprob[row * p.n_targets + i] =
            t < 0 ? 0.f : t >= p.vocab ? NAN : r.logprob(load<BF16>(p, row * p.row_stride + t));
    }
    return r;
}

__device__ __forceinline__ void store_top(const LogprobParams& p, int64_t row, Row r, int i, uint64_t key) {
    p.top_ids[row * p.top_k + i] = key ? (int64_t)(uint32_t)~(uint32_t)key : -1;
    p.top_logprob[row * p.top_k + i] = key ? r.logprob(ordered((uint32_t)(key >> 32))) : -INFINITY;
}

// 16 bytes of logits as floats.
template <bool BF16>
__device__ __forceinline__ void unpack(u32x4_t v, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
            x[2 * i] = __uint_as_float(v[i] << 16);
            x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        } else {
            x[i] = __uint_as_float(v[i]);
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_logprob(LogprobParams p) {
    constexpr int E = BF16 ? 8 : 4;                     // logits of a vector
    constexpr uint32_t kNone = BF16 ? 0xFF80FF80u : 0xFF800000u;      // -inf
    __shared__ State states[kWaves];
    __shared__ uint32_t bound[kWaves][2];
    __shared__ volatile uint32_t shares[kWaves];        // order of the (k / 4)-th logit of a wave's list, 0: none yet
    __shared__ __align__(16) uint64_t lists[kWaves][RIS_MAX_TOP];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = p.top_k;
    const int64_t row = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x % p.parts);
    const int64_t base = row * p.row_stride;
    // The row's whole vectors, from its first 16-byte boundary on, and the logits
    // before and behind them, which part 0 and the last part take.
    const uintptr_t addr = reinterpret_cast<uintptr_t>(p.logits) + base * (BF16 ? 2 : 4);
    const int gap = (int)((16 - (addr & 15)) & 15) / (BF16 ? 2 : 4);
    const int head = gap < p.vocab ? gap : (int)p.vocab;
    const int nv = (int)((p.vocab - head) / E);
    const int per = (nv + p.parts - 1) / p.parts;
    const int v0 = part * per < nv ? part * per : nv, v1 = v0 + per < nv ? v0 + per : nv;
    const u32x4_t* vec = reinterpret_cast<const u32x4_t*>(addr + head * (BF16 ? 2 : 4));

    const int share = k ? (k + kWaves - 1) / kWaves : 1;
    if (tid < kWaves) shares[tid] = 0;
    __syncthreads();
    float m = -INFINITY, b = 0.f;           // running maximum; times log2 e where that is a weight's reference, else 0
    float l = 0.f, u = 0.f;                 // sums of 2^d and of 2^d d, d = x log2 e - b
    uint64_t list = 0, least = kNothing;
    float above = -INFINITY;                // least's logit
    const auto take = [&](const float* x, int n, uint32_t id) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i < n; ++i) top = fmaxf(top, x[i]);
        if (__any(top > m)) {
            const float old = b, was = m;
            m = fmaxf(m, top);
            b = fabsf(m) < kNear ? m * kLog2e : 0.f;
            // under maxima of -kNear and below every weight was 0
            const float d = was > -kNear ? old - b : kFar, a = __builtin_amdgcn_exp2f(d);
            u = a * fmaf(l, d, u);
            l *= a;
        }
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float d = fmaf(x[i], kLog2e, -b), w = __builtin_amdgcn_exp2f(d);
            l += w;
            u = fmaf(w, fmaxf(d, kFar), u);
        }
        // Ids rise from step to step, so what only equals the list's last is left out.
        // (fmaxf passes a NaN over, l does not.)
        if (k && __any(!(top <= above) || l != l)) {
#pragma unroll
            for (int i = 0; i < n; ++i)
                if (__any(!(x[i] < above))) {
                    insert(list, least, key_of(x[i], id + i), k);
                    above = ordered((uint32_t)(least >> 32));
                }
            if (lane == 0) shares[wave] = (uint32_t)(lane_value(list, share - 1) >> 32);
        }
    };
    // Start the list above the orders below t: at least k tokens of the part are known
    // to lie at t or above, and t's own logits enter.  (The order just below 0's is -0's,
    // which as a number is not below 0: that list starts above -2^-126.)
    const auto start_at = [&](uint32_t t) {
        const uint64_t start = ((uint64_t)(t == 0x80000000u ? 0x7F800000u : t) << 32) - 1;
        if (t && start > least) {
            least = start;
            above = ordered((uint32_t)(least >> 32));
        }
    };

    if (part == 0 && head > 0) {
        const float x = tid < head ? load<BF16>(p, base + tid) : -INFINITY;
        if (wave == 0) take(&x, 1, (uint32_t)tid);
    }
    for (int v = v0; v < v1; v += kThreads * kUnroll) {
        u32x4_t r[kUnroll];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const int at = v + i * kThreads + tid;
            r[i] = at < v1 ? vec[at] : u32x4_t{kNone, kNone, kNone, kNone};
        }
        if (k && v == v0) {
            // What the list starts above: the lanes' largest logits of this first piece
            // are as many tokens, so the k-th of a wave's 64, or the least over the
            // waves of the (k / 4)-th, is no more than the row's k-th.  (A few dozen
            // insertions a wave instead of k log(n / k).)
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) {
                float x[E];
                unpack<BF16>(r[i], x);
#pragma unroll
                for (int e = 0; e < E; ++e) top = fmaxf(top, x[e]);
            }
            const uint32_t o = order_of(top);
            const uint32_t all = nth_largest(o, k), some = nth_largest(o, share);
            if (lane == 0) {
                bound[wave][0] = all;
                bound[wave][1] = some;
            }
            __syncthreads();
            uint32_t t = 0, f = 0xFFFFFFFFu;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                t = bound[w][0] > t ? bound[w][0] : t;
                f = bound[w][1] < f ? bound[w][1] : f;
            }
            start_at(f > t ? f : t);
        } else if (k) {
            // The least of the waves' (k / 4)-th listed logits is such a bound too, an old
            // one as well: no wave waits for another.
            uint32_t t = 0xFFFFFFFFu;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t o = shares[w];
                t = o < t ? o : t;
            }
            start_at(__builtin_amdgcn_readfirstlane(t));
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            if (v + i * kThreads + wave * 64 >= v1) break;          // nothing of the wave's is left
            float x[E];
            unpack<BF16>(r[i], x);
            take(x, E, (uint32_t)head + (uint32_t)(v + i * kThreads + tid) * E);
        }
    }
    {
        const int64_t tail = head + (int64_t)nv * E;
        if (part == p.parts - 1 && tail < p.vocab && wave == 0) {
            const float x = tail + tid < p.vocab ? load<BF16>(p, base + tail + tid) : -INFINITY;
            take(&x, 1, (uint32_t)(tail + tid));
        }
    }
    // To natural units at the maximum itself, b being m log2 e rounded.
    State s{m, l, 0.f};
    {
        const float c = fabsf(m) < kNear ? fmaf(m, -kLog2e, b) : 0.f;
        const float f = __builtin_amdgcn_exp2f(c);
        s.u = kLn2 * f * fmaf(l, c, u);
        s.l = l * f;
    }
    s = wave_merge(s);
    if (lane == 0) states[wave] = s;
    if (lane < k) lists[wave][lane] = list;
    __syncthreads();
    {
        float top = states[0].m;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, states[w].m);
        s = State{top, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const State t = raise(states[w], top);
            s.l += t.l;
            s.u += t.u;
        }
    }
    if (!(fabsf(s.m) < kNear) && s.m != -INFINITY) {
        // A maximum far from 0 (a row or part masked as a whole with a large negative
        // number): the sums once more from the differences.
        State t{-INFINITY, 0.f, 0.f};
        const int64_t x0 = part == 0 ? 0 : head + (int64_t)v0 * E;
        const int64_t x1 = part == p.parts - 1 ? p.vocab : head + (int64_t)v1 * E;
        for (int64_t i = x0 + tid; i < x1; i += kThreads) add(t, load<BF16>(p, base + i));
        t = wave_merge(t);
        __syncthreads();
        if (lane == 0) states[wave] = t;
        __syncthreads();
        s = State{s.m, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const State q = raise(states[w], s.m);
            s.l += q.l;
            s.u += q.u;
        }
    }
    Row r{0.f, 0.f};
    if (p.parts == 1) {
        r = finish_row<BF16>(p, row, s, tid, kThreads);
    } else if (tid == 0) {
        float* st = p.part + 4 * (int64_t)blockIdx.x;
        st[0] = s.m;
        st[1] = s.l;
        st[2] = s.u;
    }
    // The waves' lists: a key's rank is its place in its own list and the keys above
    // it in the others.
    if (lane < k) {
        uint64_t* ls = reinterpret_cast<uint64_t*>(p.part + 4 * p.rows * p.parts) + (int64_t)blockIdx.x * k;
        int rank = lane;
        for (int w = 1; w < kWaves; ++w) {
            const uint64_t* other = lists[(wave + w) % kWaves];
            for (int i = 0; i < k; ++i) rank += other[i] > list || (other[i] == 0 && list == 0 && (wave + w) % kWaves < wave);
        }
        if (rank < k) {
            if (p.parts == 1) store_top(p, row, r, rank, list);
            else ls[rank] = list;
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(64) void k_logprob_merge(LogprobParams p) {
    const int lane = threadIdx.x, k = p.top_k;
    const int64_t row = blockIdx.x;
    State s{-INFINITY, 0.f, 0.f};
    if (lane < p.parts) {
        const float* st = p.part + 4 * (row * p.parts + lane);
        s = State{st[0], st[1], st[2]};
    }
    s = wave_merge(s);
    const Row r = finish_row<BF16>(p, row, s, lane, 64);
    // One part's list to a lane; the largest of their heads k times.
    const uint64_t* mine = reinterpret_cast<const uint64_t*>(p.part + 4 * p.rows * p.parts) + (row * p.parts + lane) * k;
    int at = 0;
    uint64_t head = lane < p.parts && k ? mine[0] : 0, next = lane < p.parts && k > 1 ? mine[1] : 0;
    uint64_t best = 0;                                  // lane i: the i-th largest
    for (int i = 0; i < k; ++i) {
        const uint64_t v = wave_max_u64(head);
        if (lane == i) best = v;
        if (v && head == v) {                           // keys differ: one lane's
            head = next;
            next = ++at + 1 < k ? mine[at + 1] : 0;
        }
    }
    if (lane < k) store_top(p, row, r, lane, best);
}

}  // namespace

// Workgroups of a row: ~1024 in all, at least 2048 logits each and 2^25 at most (2^17 terms
// to a thread's sum), at most one per lane of the merging wave.
int32_t logprob_parts(int64_t rows, int64_t vocab) {
    int64_t parts = (1024 + rows - 1) / rows;
    const int64_t most = (vocab + 2047) / 2048, least = (vocab + (1 << 25) - 1) >> 25;
    if (parts > most) parts = most;
    if (parts < least) parts = least;
    return (int32_t)(parts > 64 ? 64 : parts);
}

int64_t logprob_workspace(int64_t rows, int32_t parts, int32_t top_k) {
    return parts == 1 ? 0 : rows * parts * (int64_t)(4 * sizeof(float) + top_k * sizeof(uint64_t));
}

hipError_t launch_logprobs(const LogprobParams& p, hipStream_t st) {
    const dim3 grid((unsigned)(p.rows * p.parts));
    if (p.bf16) hipLaunchKernelGGL(k_logprob<true>, grid, dim3(kThreads), 0, st, p);
    else hipLaunchKernelGGL(k_logprob<false>, grid, dim3(kThreads), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    if (p.bf16) hipLaunchKernelGGL(k_logprob_merge<true>, dim3((unsigned)p.rows), dim3(64), 0, st, p);
    else hipLaunchKernelGGL(k_logprob_merge<false>, dim3((unsigned)p.rows), dim3(64), 0, st, p);
    return hipGetLastError();
}

}  // namespace ris
