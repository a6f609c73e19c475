// Log probabilities of given tokens, entropy and the largest logits of a row, in
// one pass over the row: a thread keeps the running maximum m, the sum of
// exp(x - m) and the sum of exp(x - m) (x - m) of what it has read, a wave the
// top_k largest logits as a list over its lanes.  Then log p = x - m - log(sum) and
// the entropy is log(sum) - sum(exp(x - m) (x - m)) / sum.
//
// A row is cut into parts where rows are few; each part's workgroup leaves its state
// and list in the workspace, and one wave a row merges them.
#include "ris_device.h"
#include "ris_internal.h"

namespace ris {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFar = -1e30f;      // stands for -inf in products with a weight of 0

// Keys order logits as they compare, equal ones by descending id: the float's bits
// made monotone, then the id's complement.  NaN ranks first, 0 is no token.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t id) {
    uint32_t u = __float_as_uint(x + 0.f);              // -0 is 0
    if (x != x) u = 0x7FFFFFFFu;
    u ^= (uint32_t)((int32_t)u >> 31) | 0x80000000u;
    return (uint64_t)u << 32 | (uint32_t)~id;
}
__device__ __forceinline__ float key_logit(uint64_t k) {
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
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

__device__ __forceinline__ State merge(State a, State b) {
    const float m = fmaxf(a.m, b.m);
    const float da = a.m == m ? 0.f : a.m - m, db = b.m == m ? 0.f : b.m - m;
    const float fa = __builtin_amdgcn_exp2f(da * kLog2e), fb = __builtin_amdgcn_exp2f(db * kLog2e);
    return State{m, fa * a.l + fb * b.l,
                 fa * fmaf(a.l, fmaxf(da, kFar), a.u) + fb * fmaf(b.l, fmaxf(db, kFar), b.u)};
}

__device__ __forceinline__ State wave_merge(State s) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s = merge(s, State{__shfl_xor(s.m, o), __shfl_xor(s.l, o), __shfl_xor(s.u, o)});
    return s;
}

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// Keys of the wave's lanes into its list: lane i holds the i-th largest of the
// first k, 0 where there is none; `least` is the k-th.
__device__ __forceinline__ void insert(uint64_t& list, uint64_t& least, uint64_t key, int k) {
    const int lane = threadIdx.x & 63;
    uint64_t todo = __ballot(key > least);
    while (todo) {
        const int from = (int)__builtin_ctzll(todo);
        const uint64_t v = lane_value(key, from);
        const uint64_t up = __shfl_up(list, 1);
        const int at = __popcll(__ballot(list > v));
        list = lane < at ? list : (lane == at ? v : up);
        least = lane_value(list, k - 1);
        if (least < kNothing) least = kNothing;
        todo &= __ballot(key > least) & ~(1ull << from);
    }
}

// The k largest keys of lists of k (descending, 0 after the end), one list to a
// lane, into out[0..k) in order.
template <typename Out>
__device__ __forceinline__ void merge_lists(const uint64_t* lists, int64_t stride, int n, int k, Out out) {
    const int lane = threadIdx.x & 63;
    const uint64_t* mine = lists + lane * stride;
    int at = 0;
    uint64_t head = lane < n ? mine[0] : 0;
    for (int i = 0; i < k; ++i) {
        uint64_t best = head;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint64_t v = __shfl_xor(best, o);
            best = v > best ? v : best;
        }
        out(i, best);
        if (best && head == best) head = ++at < k ? mine[at] : 0;       // keys differ: one lane's
    }
}

__device__ __forceinline__ float load(const LogprobParams& p, int64_t at) {
    return p.bf16 ? bf16_to_f32(static_cast<const uint16_t*>(p.logits)[at]) : static_cast<const float*>(p.logits)[at];
}

// log p from the row's state; a row of -inf alone has l = 0.
struct Row {
    float m, log_l;
    __device__ float logprob(float x) const { return x == -INFINITY && log_l == log_l ? x : x - m - log_l; }
};

__device__ __forceinline__ Row finish_row(const LogprobParams& p, int64_t row, State s, int first, int step) {
    const float log_l = __builtin_amdgcn_logf(s.l) * kLn2;
    const Row r{s.m, log_l};
    if (first == 0 && p.entropy) p.entropy[row] = s.l == 0.f ? 0.f : log_l - s.u / s.l;
    for (int i = first; i < p.n_targets; i += step) {
        const int64_t t = p.targets[row * p.n_targets + i];
        p.logprob[row * p.n_targets + i] = t < 0 ? 0.f : t >= p.vocab ? NAN : r.logprob(load(p, row * p.row_stride + t));
    }
    return r;
}

__device__ __forceinline__ void store_top(const LogprobParams& p, int64_t row, Row r, int i, uint64_t key) {
    if ((threadIdx.x & 63) == 0) {
        p.top_ids[row * p.top_k + i] = key ? (int64_t)(uint32_t)~(uint32_t)key : -1;
        p.top_logprob[row * p.top_k + i] = key ? r.logprob(key_logit(key)) : -INFINITY;
    }
}

__global__ __launch_bounds__(kThreads) void k_logprob(LogprobParams p) {
    __shared__ State states[kWaves];
    __shared__ uint64_t lists[kWaves][RIS_MAX_TOP];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = p.top_k;
    const int64_t row = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x % p.parts);
    const int64_t per = (p.vocab + p.parts - 1) / p.parts;
    const int64_t v0 = part * per, v1 = v0 + per < p.vocab ? v0 + per : p.vocab;
    State s{-INFINITY, 0.f, 0.f};
    uint64_t list = 0, least = kNothing;
    for (int64_t v = v0; v < v1; v += kThreads) {
        const bool in = v + tid < v1;
        const float x = in ? load(p, row * p.row_stride + v + tid) : -INFINITY;
        if (in) add(s, x);
        if (k) insert(list, least, in ? key_of(x, (uint32_t)(v + tid)) : 0, k);
    }
    s = wave_merge(s);
    if (lane == 0) states[wave] = s;
    if (lane < k) lists[wave][lane] = list;
    __syncthreads();
    s = states[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) s = merge(s, states[w]);
    if (p.parts == 1) {
        const Row r = finish_row(p, row, s, tid, kThreads);
        if (wave == 0 && k) merge_lists(lists[0], RIS_MAX_TOP, kWaves, k, [&](int i, uint64_t key) { store_top(p, row, r, i, key); });
        return;
    }
    float* st = p.part + 4 * (int64_t)blockIdx.x;
    if (tid == 0) {
        st[0] = s.m;
        st[1] = s.l;
        st[2] = s.u;
    }
    uint64_t* ls = reinterpret_cast<uint64_t*>(p.part + 4 * p.rows * p.parts) + (int64_t)blockIdx.x * k;
    if (wave == 0 && k) merge_lists(lists[0], RIS_MAX_TOP, kWaves, k, [&](int i, uint64_t key) { if (lane == 0) ls[i] = key; });
}

__global__ __launch_bounds__(64) void k_logprob_merge(LogprobParams p) {
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    State s{-INFINITY, 0.f, 0.f};
    if (lane < p.parts) {
        const float* st = p.part + 4 * (row * p.parts + lane);
        s = State{st[0], st[1], st[2]};
    }
    s = wave_merge(s);
    const Row r = finish_row(p, row, s, lane, 64);
    const uint64_t* ls = reinterpret_cast<const uint64_t*>(p.part + 4 * p.rows * p.parts) + row * p.parts * p.top_k;
    if (p.top_k) merge_lists(ls, p.top_k, p.parts, p.top_k, [&](int i, uint64_t key) { store_top(p, row, r, i, key); });
}

}  // namespace

// Workgroups of a row: ~1024 in all, at least 4096 logits each, at most one per
// lane of the merging wave.
int32_t logprob_parts(int64_t rows, int64_t vocab) {
    int64_t parts = (1024 + rows - 1) / rows;
    const int64_t most = (vocab + 4095) / 4096;
    if (parts > most) parts = most;
    return (int32_t)(parts > 64 ? 64 : parts);
}

int64_t logprob_workspace(int64_t rows, int32_t parts, int32_t top_k) {
    return parts == 1 ? 0 : rows * parts * (int64_t)(4 * sizeof(float) + top_k * sizeof(uint64_t));
}

hipError_t launch_logprobs(const LogprobParams& p, hipStream_t st) {
    hipLaunchKernelGGL(k_logprob, dim3((unsigned)(p.rows * p.parts)), dim3(kThreads), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    hipLaunchKernelGGL(k_logprob_merge, dim3((unsigned)p.rows), dim3(64), 0, st, p);
    return hipGetLastError();
}

}  // namespace ris
