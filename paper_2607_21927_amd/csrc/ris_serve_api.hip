// C ABI of the serving operators (ris_serve.h): argument validation and dispatch.
#include <float.h>
#include <math.h>
#include <stdint.h>

#include "ris_internal.h"
#include "ris_serve.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;      // scores are weighed in the log2 domain

int hip_status(hipError_t e) { return e == hipSuccess ? RIS_OK : RIS_E_HIP; }

bool known_dtype(int32_t d) { return d == RIS_F32 || d == RIS_BF16; }
int64_t elt_bytes(int32_t d) { return d == RIS_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A strided tensor that 16-byte accesses may walk.
bool vector_rows(const void* p, int64_t head, int64_t token, int32_t dtype) {
    const int64_t n = 16 / elt_bytes(dtype);
    return aligned(p, 16) && head >= 0 && token >= 0 && head % n == 0 && token % n == 0;
}

// The same for one that is written: rows that all lie in one place are refused.
bool output_rows(const void* p, int64_t head, int64_t token, int32_t dtype, int64_t heads, int64_t tokens) {
    return vector_rows(p, head, token, dtype) && (heads == 1 || head > 0) && (tokens == 1 || token > 0);
}

// Token offsets fit 32 bits (ris_serve.h's packed sequences).
constexpr int64_t kMaxTokens = 0x7FFFFFFFll;

// Elements between the rows of K or V whose byte offsets within a tile of 64 keys
// fit 32 bits, float32 rows too.
constexpr int64_t kMaxKeyStride = (1ll << 32) / (64 * 4) - 1024;

// Work-items of a launch, which a dispatch counts in 32 bits.
bool fits_dispatch(int64_t blocks, int64_t threads) { return blocks <= 0xFFFFFFFFll / threads; }

int validate_prompt(const ris_prompt_desc* d) {
    if (!d) return RIS_E_ARG;
    if (!known_dtype(d->dtype_in) || !known_dtype(d->dtype_out)) return RIS_E_DTYPE;
    if (d->Hq < 1 || d->Hkv < 1 || d->batch < 1 || d->T < 1) return RIS_E_ARG;
    if (d->Hq % d->Hkv != 0) return RIS_E_SHAPE;
    if (d->D != 64 && d->D != 128) return RIS_E_UNSUPPORTED;
    if (d->causal != 0 && d->causal != 1) return RIS_E_ARG;
    if (!(d->scale >= 0.0f) || !isfinite(d->scale * kLog2e)) return RIS_E_ARG;
    if (d->T > kMaxTokens || d->batch > (1 << 24)) return RIS_E_UNSUPPORTED;
    return RIS_OK;
}

int validate_kv4(const ris_kv4_desc* d) {
    if (!d) return RIS_E_ARG;
    if (!known_dtype(d->dtype)) return RIS_E_DTYPE;
    if (d->Hkv < 1 || d->batch < 1 || d->T < 1) return RIS_E_ARG;
    if (d->max_len < 1 || d->max_len > (1ll << 31)) return RIS_E_ARG;
    if (d->D != 64 && d->D != 128) return RIS_E_UNSUPPORTED;
    if (d->T > kMaxTokens || d->batch > (1 << 24) || d->Hkv > 65535) return RIS_E_UNSUPPORTED;
    return RIS_OK;
}

int kv4_params(const void* K, const void* V, const int64_t* cu, const int64_t* start, const uint8_t* K4, const uint8_t* V4,
               const uint8_t* S, const ris_kv4_desc* d, ris::Kv4Params* p) {
    const int st = validate_kv4(d);
    if (st != RIS_OK) return st;
    if (!K || !V || !cu || !K4 || !V4 || !S) return RIS_E_ARG;
    if (!vector_rows(K, d->k_head, d->k_token, d->dtype) || !vector_rows(V, d->v_head, d->v_token, d->dtype)) return RIS_E_ARG;
    if (!aligned(K4, 16) || !aligned(V4, 16) || !aligned(S, 8)) return RIS_E_ARG;
    p->K = const_cast<void*>(K); p->V = const_cast<void*>(V);
    p->K4 = const_cast<uint8_t*>(K4); p->V4 = const_cast<uint8_t*>(V4); p->S = const_cast<uint8_t*>(S);
    p->cu = cu; p->start = start;
    p->T = d->T; p->max_len = d->max_len;
    p->k_head = d->k_head; p->k_token = d->k_token; p->v_head = d->v_head; p->v_token = d->v_token;
    p->Hkv = d->Hkv; p->D = d->D; p->batch = d->batch;
    p->bf16 = d->dtype == RIS_BF16;
    const int64_t per = 256 / (d->D / 8);
    if (!fits_dispatch((d->T + per - 1) / per, 256)) return RIS_E_UNSUPPORTED;
    return RIS_OK;
}

int validate_kv4_decode(const ris_decode_desc* d) {
    if (!d) return RIS_E_ARG;
    if (!known_dtype(d->dtype_in) || !known_dtype(d->dtype_out)) return RIS_E_DTYPE;
    if (d->dtype_in != RIS_BF16) return RIS_E_UNSUPPORTED;
    if (d->batch < 1 || d->Hq < 1 || d->Hkv < 1) return RIS_E_ARG;
    if (d->Hq % d->Hkv != 0) return RIS_E_SHAPE;
    if (d->Hq / d->Hkv > 8) return RIS_E_UNSUPPORTED;
    if (d->D != 64 && d->D != 128) return RIS_E_UNSUPPORTED;
    if (d->max_len < 1 || d->max_len > (1ll << 31)) return RIS_E_ARG;
    if (d->anchor_stride < 0 || d->anchor_stride > (1ll << 40)) return RIS_E_ARG;
    if (d->window < 0 || d->sink < 0) return RIS_E_ARG;
    if (!(d->scale >= 0.0f) || !isfinite(d->scale * kLog2e)) return RIS_E_ARG;
    if ((int64_t)d->batch * d->Hkv > 65535) return RIS_E_UNSUPPORTED;
    if ((int64_t)d->batch * d->Hq > 0x7FFFFFFFll) return RIS_E_UNSUPPORTED;
    return RIS_OK;
}

// Waves per row for the tiles of a typical row (its share of the anchor slice, window
// and initial tokens).  One workgroup, whose output needs no merge in another launch,
// to kSoloTiles tiles and beyond where rows are many (2 rows of 16 tiles at D = 128:
// 7.3 us with 4 waves, 8.2 with 8, 7.3 with 16; 24 tiles 9.1, 9.1, 8.1; 128 rows of 32
// tiles 11.6, 11.2, 11.1, of 64 19.1, 15.8, 14.0; 256 rows of 64 19.5, 19.8, 21.4; 512 rows
// of 128 48, 53, 54).  Else a wave to a tile up to kWaves in all: rows of one length
// are fastest with 2048 (64 rows of 65,536 keys 105 us with 2048, 110 with 4096, 111 with
// 8192), rows of lengths between a quarter and all of that with 8192 (87, 81, 80).  A row
// takes kMostWaves at most (2 rows of 33,000 keys: 11.9 us, 12.9 with twice as many).
// Positions are on the device, so this counts what the cache may hold: sequences of 500
// tokens (12/2 heads of 128) take 7.1 us for one and 8.6 for 32 in a cache of 516 rows, 8.1
// and 11.1 in one of 65,536.
constexpr int64_t kSoloTiles = 16, kWaves = 4096, kMostWaves = 512;
int64_t kv4_decode_waves(const ris_decode_desc& d) {
    const int64_t win = d.window < d.max_len ? d.window : d.max_len;
    const int64_t snk = d.sink < d.max_len ? d.sink : d.max_len;
    int64_t keys = (d.anchor_stride + d.Hkv - 1) / d.Hkv + win + snk;
    if (keys > d.max_len) keys = d.max_len;
    const int64_t tiles = (keys + ris::kDecodeTileKeys - 1) / ris::kDecodeTileKeys;
    const int64_t rows = (int64_t)d.batch * d.Hkv;
    if (tiles <= kSoloTiles || tiles <= rows / 4) return ris::kDecodeWaves;
    int64_t waves = (kWaves + rows - 1) / rows;
    if (waves > tiles) waves = tiles;
    if (waves > kMostWaves) waves = kMostWaves;
    return (waves + ris::kDecodeWaves - 1) / ris::kDecodeWaves * ris::kDecodeWaves;
}

int64_t kv4_decode_workspace(const ris_decode_desc& d) {
    return (int64_t)d.batch * d.Hq * (kv4_decode_waves(d) / ris::kDecodeWaves) * (d.D + 2) * (int64_t)sizeof(float);
}

int validate_logprob(const ris_logprob_desc* d) {
    if (!d) return RIS_E_ARG;
    if (!known_dtype(d->dtype)) return RIS_E_DTYPE;
    if (d->rows < 1 || d->vocab < 1 || d->vocab > 0x7FFFFFFFll) return RIS_E_ARG;
    if (d->n_targets < 0 || d->n_targets > 65536 || d->top_k < 0 || d->top_k > RIS_MAX_TOP) return RIS_E_ARG;
    if (d->row_stride < d->vocab || d->row_stride > (1ll << 40)) return RIS_E_ARG;
    if (d->rows > 0xFFFFFFFFll || !fits_dispatch(d->rows * ris::logprob_parts(d->rows, d->vocab), 256)) return RIS_E_UNSUPPORTED;
    return RIS_OK;
}

constexpr int64_t kMostPlaces = 1ll << 30;      // of a sequence in a paged cache: positions fit 32 bits

int page_map(const ris_page_map& m, int32_t Hkv, int32_t D, ris::PageMap* out) {
    if (m.page < 1 || m.page > 65536 || (m.page & (m.page - 1)) || m.max_pages < 1) return RIS_E_ARG;
    if (m.pages < 1 || m.pages > 0x7FFFFFFFll || m.table_stride < m.max_pages) return RIS_E_ARG;
    if (m.page_stride < (int64_t)Hkv * m.page * D || m.page_stride % D != 0) return RIS_E_ARG;
    if ((int64_t)m.max_pages * m.page > kMostPlaces || m.page_stride / D > 0xFFFFFFFFll / m.pages ||
        m.table_stride > (1ll << 32))
        return RIS_E_UNSUPPORTED;
    out->table = nullptr;
    out->table_stride = m.table_stride;
    out->page_rows = (uint32_t)(m.page_stride / D);
    out->pages = (int32_t)m.pages;
    out->places = m.max_pages * m.page;
    out->shift = 31 - __builtin_clz((unsigned)m.page);
    return RIS_OK;
}

int validate_page_store(const ris_page_store_desc* d, ris::PageMap* map) {
    if (!d) return RIS_E_ARG;
    if (!known_dtype(d->dtype)) return RIS_E_DTYPE;
    if (d->dtype != RIS_BF16) return RIS_E_UNSUPPORTED;
    if (d->Hq < 0 || d->Hkv < 1 || d->batch < 1 || d->T < 1) return RIS_E_ARG;
    if (d->D != 64 && d->D != 128) return RIS_E_UNSUPPORTED;
    if (d->T > kMaxTokens || d->batch > (1 << 24) || d->Hq > 65535 || d->Hkv > 65535) return RIS_E_UNSUPPORTED;
    if (!fits_dispatch((d->T * (d->D / 2) + 255) / 256, 256)) return RIS_E_UNSUPPORTED;
    return page_map(d->map, d->Hkv, d->D, map);
}

// The descriptor resolved, all but the pointers.
int page_attn_params(const ris_page_attn_desc* d, ris::PageAttnParams* p) {
    if (!d) return RIS_E_ARG;
    if (!known_dtype(d->dtype_in) || !known_dtype(d->dtype_out)) return RIS_E_DTYPE;
    if (d->dtype_in != RIS_BF16) return RIS_E_UNSUPPORTED;
    if (d->Hq < 1 || d->Hkv < 1 || d->batch < 1 || d->T < 1) return RIS_E_ARG;
    if (d->Hq % d->Hkv != 0) return RIS_E_SHAPE;
    if (d->Hq / d->Hkv > ris::kPageRows) return RIS_E_UNSUPPORTED;
    if (d->D != 64 && d->D != 128) return RIS_E_UNSUPPORTED;
    if (d->window < 0 || d->sink < 0) return RIS_E_ARG;
    if (!(d->scale >= 0.0f) || !isfinite(d->scale * kLog2e)) return RIS_E_ARG;
    if (d->T > kMaxTokens || d->batch > (1 << 24) || d->Hkv > 65535) return RIS_E_UNSUPPORTED;
    const int st = page_map(d->map, d->Hkv, d->D, &p->map);
    if (st != RIS_OK) return st;
    p->T = d->T;
    p->q_head = d->q_head; p->q_token = d->q_token; p->o_head = d->o_head; p->o_token = d->o_token;
    p->Hq = d->Hq; p->Hkv = d->Hkv; p->G = d->Hq / d->Hkv; p->D = d->D;
    p->batch = d->batch;
    p->tokens = ris::page_step_tokens(d->T, d->batch, p->G);
    p->step = p->tokens > 0;
    if (!p->step) p->tokens = ris::kPageRows / p->G;
    p->window = d->window; p->sink = d->sink;
    p->out_bf16 = d->dtype_out == RIS_BF16;
    p->c = (d->scale > 0.0f ? d->scale : 1.0f / sqrtf((float)d->D)) * kLog2e;
    p->slack = fminf(8.0f / p->c, FLT_MAX);       // -inf + slack stays -inf
    if (p->step) ris::page_step_waves(p);
    else p->parts = ris::page_attn_parts(*p);
    p->part_rows = (int32_t)(d->T < p->tokens ? d->T : p->tokens) * p->G;
    const int64_t blocks = ris::page_attn_blocks(*p);
    if (!fits_dispatch(blocks, 256) || (p->step && !fits_dispatch(blocks * p->parts, 64)) ||
        (ris::page_attn_pieces(*p) > 0 && !fits_dispatch(blocks * p->part_rows, 256)))
        return RIS_E_UNSUPPORTED;
    return RIS_OK;
}

int64_t page_attn_workspace(const ris::PageAttnParams& p) {
    const int64_t pieces = ris::page_attn_pieces(p);
    return pieces > 0 ? (pieces * p.part_rows * (p.D + 4) + ris::kPartList) * (int64_t)sizeof(float) : 0;
}

// Sizes of 4-bit weights whose tiles a launch can count.
int w4_sizes(int32_t dtype, int64_t N, int64_t K) {
    if (!known_dtype(dtype)) return RIS_E_DTYPE;
    if (N < 1 || K < 1) return RIS_E_ARG;
    if (N > (1ll << 27) || K > (1ll << 24)) return RIS_E_UNSUPPORTED;
    return RIS_OK;
}

int w4_rows(const void* W, int32_t dtype, int64_t N, int64_t K, int64_t row_stride, const uint8_t* C, const uint8_t* S) {
    const int st = w4_sizes(dtype, N, K);
    if (st != RIS_OK) return st;
    if (!W || !C || !S || !aligned(W, (uintptr_t)elt_bytes(dtype)) || !aligned(C, 16)) return RIS_E_ARG;
    if (row_stride < K || row_stride > (1ll << 40)) return RIS_E_ARG;
    return RIS_OK;
}

}  // namespace

extern "C" {

int ris_rope_packed(const void* src, int64_t head_stride, int64_t token_stride, void* x, int32_t dtype, int32_t heads,
                    int64_t T, int32_t D, const int64_t* cu_seqlens, const int64_t* start, int32_t batch,
                    const ris_rope_desc* desc, void* stream) {
    if (!src || !x || !cu_seqlens || !desc) return RIS_E_ARG;
    if (head_stride < 0 || token_stride < 0) return RIS_E_ARG;
    if (!known_dtype(dtype)) return RIS_E_DTYPE;
    if (heads < 1 || T < 1 || batch < 1) return RIS_E_ARG;
    if (D < 2 || (D & 1) || D / 2 > ris::kMaxRopeHalf) return RIS_E_SHAPE;
    if (T > kMaxTokens || batch > (1 << 24) || !fits_dispatch((T * (D / 2) + 255) / 256, 256)) return RIS_E_UNSUPPORTED;
    if (desc->kind != RIS_ROPE_PLAIN && !(desc->factor > 0.0)) return RIS_E_ARG;
    ris::RopeTable tab;
    const int st = ris::make_rope_table(desc, D, 1, &tab);
    if (st != RIS_OK) return st;
    return hip_status(ris::launch_rope_packed(src, head_stride, token_stride, x, dtype == RIS_BF16, heads, T, D, cu_seqlens,
                                              start, batch, tab, static_cast<hipStream_t>(stream)));
}

int ris_prompt_attn(const void* Q, const void* K, const void* V, const int64_t* cu_seqlens, void* out,
                    const ris_prompt_desc* desc, void* stream) {
    const int st = validate_prompt(desc);
    if (st != RIS_OK) return st;
    if (!Q || !K || !V || !cu_seqlens || !out) return RIS_E_ARG;
    const ris_prompt_desc& d = *desc;
    if (!vector_rows(Q, d.q_head, d.q_token, d.dtype_in) || !vector_rows(K, d.k_head, d.k_token, d.dtype_in) ||
        !vector_rows(V, d.v_head, d.v_token, d.dtype_in) ||
        !output_rows(out, d.o_head, d.o_token, d.dtype_out, d.Hq, d.T))
        return RIS_E_ARG;
    if (d.k_token > kMaxKeyStride || d.v_token > kMaxKeyStride) return RIS_E_UNSUPPORTED;
    ris::PromptParams p;
    p.Q = Q; p.K = K; p.V = V; p.cu = cu_seqlens; p.out = out;
    p.T = d.T;
    p.q_head = d.q_head; p.q_token = d.q_token; p.k_head = d.k_head; p.k_token = d.k_token;
    p.v_head = d.v_head; p.v_token = d.v_token; p.o_head = d.o_head; p.o_token = d.o_token;
    p.Hq = d.Hq; p.Hkv = d.Hkv; p.G = d.Hq / d.Hkv; p.D = d.D;
    p.batch = d.batch; p.causal = d.causal;
    p.in_bf16 = d.dtype_in == RIS_BF16; p.out_bf16 = d.dtype_out == RIS_BF16;
    p.c = (d.scale > 0.0f ? d.scale : 1.0f / sqrtf((float)d.D)) * kLog2e;
    p.slack = fminf(8.0f / p.c, FLT_MAX);       // -inf + slack stays -inf
    if (!fits_dispatch(ris::prompt_blocks(p), 256)) return RIS_E_UNSUPPORTED;
    return hip_status(ris::launch_prompt_attn(p, static_cast<hipStream_t>(stream)));
}

int ris_kv4_store(const void* K, const void* V, const int64_t* cu_seqlens, const int64_t* start, uint8_t* K4, uint8_t* V4,
                  uint8_t* S, const ris_kv4_desc* desc, void* stream) {
    ris::Kv4Params p;
    const int st = kv4_params(K, V, cu_seqlens, start, K4, V4, S, desc, &p);
    if (st != RIS_OK) return st;
    return hip_status(ris::launch_kv4_store(p, static_cast<hipStream_t>(stream)));
}

int ris_kv4_load(const uint8_t* K4, const uint8_t* V4, const uint8_t* S, const int64_t* cu_seqlens, const int64_t* start,
                 void* K, void* V, const ris_kv4_desc* desc, void* stream) {
    ris::Kv4Params p;
    const int st = kv4_params(K, V, cu_seqlens, start, K4, V4, S, desc, &p);
    if (st != RIS_OK) return st;
    if (!output_rows(K, p.k_head, p.k_token, desc->dtype, p.Hkv, p.T) || !output_rows(V, p.v_head, p.v_token, desc->dtype, p.Hkv, p.T))
        return RIS_E_ARG;
    return hip_status(ris::launch_kv4_load(p, static_cast<hipStream_t>(stream)));
}

int64_t ris_kv4_decode_workspace_bytes(const ris_decode_desc* desc) {
    const int st = validate_kv4_decode(desc);
    if (st != RIS_OK) return st;
    return kv4_decode_workspace(*desc);
}

int ris_kv4_decode_attn(const void* Q, const uint8_t* K4, const uint8_t* V4, const uint8_t* S, const int64_t* pos,
                        const int64_t* anchor_ptr, const int32_t* anchor_idx, void* out, void* workspace,
                        int64_t workspace_bytes, const ris_decode_desc* desc, void* stream) {
    const int st = validate_kv4_decode(desc);
    if (st != RIS_OK) return st;
    if (!Q || !K4 || !V4 || !S || !pos || !out || !workspace) return RIS_E_ARG;
    if (desc->anchor_stride > 0 && (!anchor_ptr || !anchor_idx)) return RIS_E_ARG;
    if (!aligned(Q, 16) || !aligned(K4, 16) || !aligned(V4, 16) || !aligned(S, 8) || !aligned(workspace, 16)) return RIS_E_ARG;
    if (workspace_bytes < kv4_decode_workspace(*desc)) return RIS_E_CAPACITY;
    const ris_decode_desc& d = *desc;
    ris::DecodeParams p;
    p.Q = Q; p.K = K4; p.V = V4;
    p.pos = pos; p.anchor_ptr = anchor_ptr; p.anchor_idx = anchor_idx;
    p.out = out;
    p.max_len = d.max_len; p.anchor_stride = d.anchor_stride;
    p.B = d.batch; p.Hq = d.Hq; p.Hkv = d.Hkv; p.G = d.Hq / d.Hkv; p.D = d.D;
    p.out_bf16 = d.dtype_out == RIS_BF16;
    p.window = d.window; p.sink = d.sink;
    p.keep_nan = 1;
    p.parts = (int32_t)kv4_decode_waves(d);
    p.kv_bytes = 0;
    p.scale = d.scale > 0.0f ? d.scale : 1.0f / sqrtf((float)d.D);
    p.unit = p.scale * kLog2e;
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = p.part_o + (int64_t)d.batch * d.Hq * (p.parts / ris::kDecodeWaves) * d.D;
    return hip_status(ris::launch_kv4_decode(p, S, static_cast<hipStream_t>(stream)));
}

int64_t ris_logprobs_workspace_bytes(const ris_logprob_desc* desc) {
    const int st = validate_logprob(desc);
    if (st != RIS_OK) return st;
    return ris::logprob_workspace(desc->rows, ris::logprob_parts(desc->rows, desc->vocab), desc->top_k);
}

int ris_logprobs(const void* logits, const int64_t* targets, float* logprob, float* entropy, int64_t* top_ids,
                 float* top_logprob, void* workspace, int64_t workspace_bytes, const ris_logprob_desc* desc, void* stream) {
    const int st = validate_logprob(desc);
    if (st != RIS_OK) return st;
    const ris_logprob_desc& d = *desc;
    if (!logits || !aligned(logits, (uintptr_t)elt_bytes(d.dtype))) return RIS_E_ARG;
    if (d.n_targets > 0 && (!targets || !logprob)) return RIS_E_ARG;
    if (d.top_k > 0 && (!top_ids || !top_logprob)) return RIS_E_ARG;
    ris::LogprobParams p;
    p.parts = ris::logprob_parts(d.rows, d.vocab);
    const int64_t need = ris::logprob_workspace(d.rows, p.parts, d.top_k);
    if (need > 0 && (!workspace || !aligned(workspace, 16))) return RIS_E_ARG;
    if (workspace_bytes < need) return RIS_E_CAPACITY;
    p.logits = logits; p.targets = targets; p.logprob = logprob; p.entropy = entropy;
    p.top_ids = top_ids; p.top_logprob = top_logprob;
    p.part = static_cast<float*>(workspace);
    p.rows = d.rows; p.vocab = d.vocab; p.row_stride = d.row_stride;
    p.n_targets = d.n_targets; p.top_k = d.top_k; p.bf16 = d.dtype == RIS_BF16;
    return hip_status(ris::launch_logprobs(p, static_cast<hipStream_t>(stream)));
}

int ris_page_store(const void* Q, void* Qout, const void* K, const void* V, const int64_t* cu_seqlens, const int64_t* start,
                   const int32_t* table, void* Kp, void* Vp, const ris_page_store_desc* desc, const ris_rope_desc* rope,
                   void* stream) {
    ris::PageStoreParams p;
    int st = validate_page_store(desc, &p.map);
    if (st != RIS_OK) return st;
    const ris_page_store_desc& d = *desc;
    if (!K || !V || !cu_seqlens || !table || !Kp || !Vp || (d.Hq > 0 && (!Q || !Qout))) return RIS_E_ARG;
    if (!vector_rows(K, d.k_head, d.k_token, d.dtype) || !vector_rows(V, d.v_head, d.v_token, d.dtype) || !aligned(Kp, 16) ||
        !aligned(Vp, 16))
        return RIS_E_ARG;
    if (d.Hq > 0 && (!vector_rows(Q, d.q_head, d.q_token, d.dtype) ||
                     !output_rows(Qout, d.qo_head, d.qo_token, d.dtype, d.Hq, d.T)))
        return RIS_E_ARG;
    ris::RopeTable tab = {};
    if (rope) {
        if (rope->kind != RIS_ROPE_PLAIN && !(rope->factor > 0.0)) return RIS_E_ARG;
        st = ris::make_rope_table(rope, d.D, 1, &tab);
        if (st != RIS_OK) return st;
    }
    p.Q = Q; p.Qout = Qout; p.K = K; p.V = V; p.Kp = Kp; p.Vp = Vp;
    p.cu = cu_seqlens; p.start = start;
    p.map.table = table;
    p.T = d.T;
    p.q_head = d.q_head; p.q_token = d.q_token; p.qo_head = d.qo_head; p.qo_token = d.qo_token;
    p.k_head = d.k_head; p.k_token = d.k_token; p.v_head = d.v_head; p.v_token = d.v_token;
    p.Hq = d.Hq; p.Hkv = d.Hkv; p.D = d.D; p.batch = d.batch;
    p.rotate = rope != nullptr;
    return hip_status(ris::launch_page_store(p, tab, static_cast<hipStream_t>(stream)));
}

int64_t ris_page_attn_workspace_bytes(const ris_page_attn_desc* desc) {
    ris::PageAttnParams p;
    const int st = page_attn_params(desc, &p);
    return st == RIS_OK ? page_attn_workspace(p) : st;
}

int ris_page_attn(const void* Q, const void* Kp, const void* Vp, const int32_t* table, const int64_t* cu_seqlens,
                  const int64_t* start, void* out, void* workspace, int64_t workspace_bytes, const ris_page_attn_desc* desc,
                  void* stream) {
    ris::PageAttnParams p;
    const int st = page_attn_params(desc, &p);
    if (st != RIS_OK) return st;
    if (!Q || !Kp || !Vp || !table || !cu_seqlens || !out) return RIS_E_ARG;
    if (!vector_rows(Q, p.q_head, p.q_token, RIS_BF16) || !aligned(Kp, 16) || !aligned(Vp, 16) ||
        !output_rows(out, p.o_head, p.o_token, desc->dtype_out, p.Hq, p.T))
        return RIS_E_ARG;
    const int64_t need = page_attn_workspace(p);
    if (need > 0 && (!workspace || !aligned(workspace, 16))) return RIS_E_ARG;
    if (workspace_bytes < need) return RIS_E_CAPACITY;
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = p.part_o + ris::page_attn_pieces(p) * p.part_rows * p.D;
    p.part_list = reinterpret_cast<int32_t*>(p.part_ml + ris::page_attn_pieces(p) * p.part_rows * 4);
    p.Q = Q; p.K = Kp; p.V = Vp; p.cu = cu_seqlens; p.start = start; p.out = out;
    p.map.table = table;
    return hip_status(ris::launch_page_attn(p, static_cast<hipStream_t>(stream)));
}

int ris_w4_pack(const void* W, int32_t dtype, int64_t N, int64_t K, int64_t row_stride, uint8_t* C, uint8_t* S, void* stream) {
    const int st = w4_rows(W, dtype, N, K, row_stride, C, S);
    if (st != RIS_OK) return st;
    return hip_status(ris::launch_w4_pack(W, row_stride, dtype == RIS_BF16, (int32_t)N, (int32_t)K, C, S,
                                          static_cast<hipStream_t>(stream)));
}

int ris_w4_load(const uint8_t* C, const uint8_t* S, void* W, int32_t dtype, int64_t N, int64_t K, int64_t row_stride, void* stream) {
    const int st = w4_rows(W, dtype, N, K, row_stride, C, S);
    if (st != RIS_OK) return st;
    return hip_status(ris::launch_w4_load(C, S, (int32_t)N, (int32_t)K, W, row_stride, dtype == RIS_BF16,
                                          static_cast<hipStream_t>(stream)));
}

int ris_w4_linear(const void* x, const uint8_t* C, const uint8_t* S, const void* bias, void* out, const ris_w4_desc* desc,
                  void* stream) {
    if (!desc) return RIS_E_ARG;
    const ris_w4_desc& d = *desc;
    const int st = w4_sizes(d.dtype, d.N, d.K);
    if (st != RIS_OK) return st;
    if (d.gated != 0 && d.gated != 1) return RIS_E_ARG;
    if (d.gated && d.N % 32 != 0) return RIS_E_SHAPE;
    if (d.rows < 1 || d.rows > kMaxTokens) return RIS_E_ARG;
    const int64_t cols = d.gated ? d.N / 2 : d.N, e = elt_bytes(d.dtype);
    if (d.x_stride < d.K || d.x_stride > (1ll << 40) || d.out_stride < cols || d.out_stride > (1ll << 40)) return RIS_E_ARG;
    if (!x || !C || !S || !out || !vector_rows(x, 0, d.x_stride, d.dtype) || !aligned(C, 16) || !aligned(out, (uintptr_t)e) ||
        !aligned(bias, (uintptr_t)e))
        return RIS_E_ARG;
    ris::W4Params p;
    p.x = x; p.C = C; p.S = S; p.bias = bias; p.out = out;
    p.x_stride = d.x_stride; p.out_stride = d.out_stride;
    p.rows = (int32_t)d.rows; p.N = (int32_t)d.N; p.K = (int32_t)d.K;
    p.f32 = d.dtype == RIS_F32; p.gated = d.gated;
    p.vector_out = cols % 4 == 0 && d.out_stride % 4 == 0 && aligned(out, (uintptr_t)(4 * e));
    if (ris::w4_items(p) > 0xFFFFFFFFll) return RIS_E_UNSUPPORTED;
    return hip_status(ris::launch_w4_linear(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
