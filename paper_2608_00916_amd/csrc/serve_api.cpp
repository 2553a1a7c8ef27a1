// C ABI of the 8-bit serving operators (declared in include/moe.h): argument
// checks, workspace layouts and launch sequences.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "api.hpp"
#include "launch.hpp"
#include "serve.hpp"

using namespace moe;

namespace {

int check_k(int32_t K) {
  if (K < 1 || K > MOE_I8_MAX_K) return fail(MOE_ERR_ARG, "K=%d must be in [1, %d]", K, MOE_I8_MAX_K);
  if (K % 16 != 0) return fail(MOE_ERR_SHAPE, "K=%d must be a multiple of 16", K);
  return MOE_OK;
}

int check_pitch(const char* name, int64_t ld, int64_t least, int multiple) {
  if (ld < least) return fail(MOE_ERR_ARG, "%s=%lld is less than %lld", name, static_cast<long long>(ld),
                              static_cast<long long>(least));
  if (ld % multiple != 0) return fail(MOE_ERR_SHAPE, "%s=%lld must be a multiple of %d", name,
                                      static_cast<long long>(ld), multiple);
  return MOE_OK;
}

int check_i8_dims(const moe_i8_dims* d) {
  if (d == nullptr) return fail(MOE_ERR_ARG, "dims is NULL");
  if (d->M < 1 || d->N < 1) return fail(MOE_ERR_ARG, "M, N must be positive (M=%d N=%d)", d->M, d->N);
  if (d->flags & ~MOE_F_OUT_FP32) return fail(MOE_ERR_ARG, "unknown flags 0x%x", d->flags);
  // tiles are numbered in 32 bits
  if (cdiv64(d->M, 64) * cdiv64(d->N, 64) > (1ll << 30)) return fail(MOE_ERR_ARG, "M=%d x N=%d too large", d->M, d->N);
  return check_k(d->K);
}

int check_weights(const moe_i8_experts* w) {
  if (w == nullptr) return fail(MOE_ERR_ARG, "w is NULL");
  return check_ptrs({{"w.w_gate", w->w_gate}, {"w.w_up", w->w_up}, {"w.w_down", w->w_down}, {"w.s_gate", w->s_gate},
                     {"w.s_up", w->s_up}, {"w.s_down", w->s_down}});
}

struct LinearWs {
  int8_t* q;
  float* scale;
  size_t bytes;
};

LinearWs linear_layout(const moe_i8_dims* d, void* base) {
  Carve c(base);
  LinearWs w;
  w.q = c.take<int8_t>(static_cast<size_t>(d->M) * d->K);
  w.scale = c.take<float>(d->M);
  w.bytes = c.off;
  return w;
}

// Scratch of the routed rows: the SwiGLU activation, its int8 rows.
struct RowsWs {
  float* a;
  float* a_top;
  int8_t* a8;
  float* sa;
};

RowsWs take_rows(Carve& c, size_t R, size_t F) {
  RowsWs w;
  w.a = c.take<float>(R * F);
  w.a_top = c.take<float>(R * (F / kI8Cols));
  w.a8 = c.take<int8_t>(R * F);
  w.sa = c.take<float>(R);
  return w;
}

struct ExpertsWs {
  int32_t *offsets, *tile_start;
  int2* tile_desc;
  int8_t* x8;
  float* sx;
  RowsWs rows;
  size_t bytes;
};

ExpertsWs experts_layout(const moe_experts_dims* d, void* base) {
  const size_t R = d->rows, E = d->E;
  Carve c(base);
  ExpertsWs w;
  w.offsets = c.take<int32_t>(E + 1);
  w.tile_start = c.take<int32_t>(E + 1);
  w.tile_desc = c.take<int2>(static_cast<size_t>(max_row_tiles(d->rows, d->E)));
  w.x8 = c.take<int8_t>(R * d->H);
  w.sx = c.take<float>(R);
  w.rows = take_rows(c, R, d->F);
  w.bytes = c.off;
  return w;
}

struct InferWs {
  float *logits, *router_part, *gates;
  int32_t *topk_idx, *counts, *offsets, *tile_start, *row_token, *row_of, *perm;
  int2* tile_desc;
  int8_t* x8;
  float* sx;
  RowsWs rows;
  bf16_t* o;
  size_t bytes;
};

InferWs infer_layout(const moe_dims* d, void* base) {
  const size_t T = d->T, E = d->E, k = d->top_k, R = T * k;
  Carve c(base);
  InferWs w;
  w.logits = c.take<float>(T * E);
  w.router_part = c.take<float>(static_cast<size_t>(router_part_floats(d->T, d->E)));
  w.gates = c.take<float>(R);
  w.topk_idx = c.take<int32_t>(R);
  w.counts = c.take<int32_t>(E);
  w.offsets = c.take<int32_t>(E + 1);
  w.tile_start = c.take<int32_t>(E + 1);
  w.row_token = c.take<int32_t>(R);
  w.row_of = c.take<int32_t>(R);
  w.perm = c.take<int32_t>(static_cast<size_t>(permute_ws_ints(d->T, d->E)));
  w.tile_desc = c.take<int2>(static_cast<size_t>(max_row_tiles(d->T * d->top_k, d->E)));
  w.x8 = c.take<int8_t>(T * d->H);
  w.sx = c.take<float>(T);
  w.rows = take_rows(c, R, d->F);
  w.o = c.take<bf16_t>(R * d->H);
  w.bytes = c.off;
  return w;
}

int check_experts_i8(const moe_experts_dims* d) {
  if (int rc = check_experts_dims(d)) return rc;
  if (d->flags != 0) return fail(MOE_ERR_ARG, "flags 0x%x: the 8-bit experts take none", d->flags);
  if (d->H > MOE_I8_MAX_K || d->F > MOE_I8_MAX_K)
    return fail(MOE_ERR_ARG, "H=%d or F=%d exceeds %d", d->H, d->F, MOE_I8_MAX_K);
  return MOE_OK;
}

int check_infer_i8(const moe_dims* d) {
  if (int rc = check_dims(d)) return rc;
  if (d->H > MOE_I8_MAX_K || d->F > MOE_I8_MAX_K)
    return fail(MOE_ERR_ARG, "H=%d or F=%d exceeds %d", d->H, d->F, MOE_I8_MAX_K);
  return MOE_OK;
}

// The expert products on routed rows; x8 row rows[r], or r where rows is null.
int expert_products(const I8Rows& rt, const int8_t* x8, const float* sx, const int32_t* rows, const moe_i8_experts* w,
                    int H, int F, const RowsWs& ws, bf16_t* o, hipStream_t s) {
  hipError_t e = launch_i8_gateup(rt, x8, sx, rows, *w, H, F, ws.a, ws.a_top, s);
  if (e != hipSuccess) return hip_status(e, "gate/up");
  e = launch_i8_requant(ws.a, ws.a_top, rt.rows_cap, F, rt.offsets + rt.E, ws.a8, ws.sa, s);
  if (e != hipSuccess) return hip_status(e, "activation rows");
  e = launch_i8_down(rt, ws.a8, ws.sa, *w, H, F, o, s);
  return hip_status(e, "down");
}

// Whether n and m int32 at a and b share memory without being the same.
bool shifted(const int32_t* a, int64_t n, const int32_t* b, int64_t m) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x != y && x < y + m * sizeof(int32_t) && y < x + n * sizeof(int32_t);
}

bool block_size_ok(int32_t n) { return n == 16 || n == 32 || n == 64 || n == 128; }

int check_cache(const moe_kv_cache* c) {
  if (c == nullptr) return fail(MOE_ERR_ARG, "cache is NULL");
  if (c->n_blocks < 1 || c->kv_heads < 1 || c->kv_heads > 65535)
    return fail(MOE_ERR_ARG, "n_blocks=%d must be positive, kv_heads=%d in [1, 65535]", c->n_blocks, c->kv_heads);
  if (!block_size_ok(c->block_tokens))
    return fail(MOE_ERR_SHAPE, "block_tokens=%d must be 16, 32, 64 or 128", c->block_tokens);
  if (c->head_dim != 64 && c->head_dim != 128) return fail(MOE_ERR_SHAPE, "head_dim=%d must be 64 or 128", c->head_dim);
  if (static_cast<int64_t>(c->n_blocks) * c->block_tokens > 0x7fffffffll)
    return fail(MOE_ERR_ARG, "n_blocks=%d x block_tokens=%d exceeds 2^31 - 1 slots", c->n_blocks, c->block_tokens);
  return check_ptrs({{"cache.k", c->k}, {"cache.v", c->v}, {"cache.k_scale", c->k_scale}, {"cache.v_scale", c->v_scale}});
}

int check_batch_dims(const moe_kv_cache* c, const moe_kv_batch* b) {
  if (b == nullptr) return fail(MOE_ERR_ARG, "batch is NULL");
  if (b->B < 1 || b->W < 1 || b->T < 0)
    return fail(MOE_ERR_ARG, "B, W must be positive, T not negative (B=%d W=%d T=%d)", b->B, b->W, b->T);
  if (static_cast<int64_t>(b->W) * c->block_tokens > (1ll << 30) || b->B > (1 << 24))
    return fail(MOE_ERR_ARG, "B=%d exceeds 2^24 or W=%d 2^30 tokens", b->B, b->W);
  return MOE_OK;
}

int check_batch(const moe_kv_cache* c, const moe_kv_batch* b) {
  if (int rc = check_batch_dims(c, b)) return rc;
  return check_ptrs({{"row_start", b->row_start}, {"kv_len", b->kv_len}, {"block_table", b->block_table}});
}

int check_attn(const moe_kv_cache* c, const moe_kv_batch* b, const moe_kv_attn* a) {
  if (a == nullptr) return fail(MOE_ERR_ARG, "attention arguments are NULL");
  if (a->heads < 1 || a->heads % c->kv_heads != 0)
    return fail(MOE_ERR_SHAPE, "heads=%d must be a positive multiple of kv_heads=%d", a->heads, c->kv_heads);
  if (a->max_q < 1 || a->max_kv < 1) return fail(MOE_ERR_ARG, "max_q=%d and max_kv=%d must be positive", a->max_q, a->max_kv);
  if (!std::isfinite(a->scale)) return fail(MOE_ERR_ARG, "scale is not finite");
  if (a->flags & ~MOE_F_CAUSAL) return fail(MOE_ERR_ARG, "unknown flags 0x%x", a->flags);
  // workgroups and a request's rows are numbered in 32 bits
  const int64_t group = a->heads / c->kv_heads;
  if (std::min(a->max_q, b->T) * group > (1ll << 30) || (b->T * group / 16 + b->B) * c->kv_heads > (1ll << 30))
    return fail(MOE_ERR_ARG, "T=%d x heads=%d too large", b->T, a->heads);
  return MOE_OK;
}

}  // namespace

extern "C" {

int moe_i8_quant_rows(int32_t rows, int32_t K, const void* x, int64_t ldx, int8_t* q, float* scale, void* stream) {
  if (rows < 1) return fail(MOE_ERR_ARG, "rows=%d must be positive", rows);
  if (int rc = check_k(K)) return rc;
  if (int rc = check_pitch("ldx", ldx, K, 8)) return rc;
  if (int rc = check_ptrs({{"x", x}, {"q", q}, {"scale", scale}})) return rc;
  return hip_status(launch_i8_quant_rows(static_cast<const bf16_t*>(x), ldx, rows, K, nullptr, q, scale,
                                         static_cast<hipStream_t>(stream)),
                    "quant rows");
}

int moe_i8_quant_weight(int32_t E, int32_t K, int32_t N, const void* w, int8_t* q, float* scale, void* stream) {
  if (E < 1 || E > 65535 || N < 1) return fail(MOE_ERR_ARG, "E=%d must be in [1, 65535], N=%d positive", E, N);
  if (int rc = check_k(K)) return rc;
  if (int rc = check_ptrs({{"w", w}, {"q", q}, {"scale", scale}})) return rc;
  return hip_status(launch_i8_quant_weight(static_cast<const bf16_t*>(w), E, K, N, q, scale,
                                           static_cast<hipStream_t>(stream)),
                    "quant weight");
}

int moe_i8_matmul(const moe_i8_dims* d, const int8_t* a, const float* a_scale, const int8_t* b, const float* b_scale,
                  void* out, int64_t ldo, void* stream) {
  if (int rc = check_i8_dims(d)) return rc;
  if (int rc = check_pitch("ldo", ldo, d->N, 1)) return rc;
  if (int rc = check_ptrs({{"a", a}, {"a_scale", a_scale}, {"b", b}, {"b_scale", b_scale}, {"out", out}})) return rc;
  return hip_status(launch_i8_matmul(a, a_scale, b, b_scale, d->M, d->N, d->K, out, ldo, d->flags & MOE_F_OUT_FP32,
                                     static_cast<hipStream_t>(stream)),
                    "int8 product");
}

size_t moe_i8_linear_workspace_bytes(const moe_i8_dims* d) {
  if (check_i8_dims(d) != MOE_OK) return 0;
  return linear_layout(d, nullptr).bytes;
}

int moe_i8_linear(const moe_i8_dims* d, const void* x, int64_t ldx, const int8_t* b, const float* b_scale, void* out,
                  int64_t ldo, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_i8_dims(d)) return rc;
  if (int rc = check_pitch("ldx", ldx, d->K, 8)) return rc;
  if (int rc = check_pitch("ldo", ldo, d->N, 1)) return rc;
  if (int rc = check_ptrs({{"x", x}, {"b", b}, {"b_scale", b_scale}, {"out", out}, {"ws", ws}})) return rc;
  const LinearWs w = linear_layout(d, ws);
  if (ws_bytes < w.bytes) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, w.bytes);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bf16_t* xb = static_cast<const bf16_t*>(x);
  if (launch_i8_linear_fused(xb, ldx, b, b_scale, d->M, d->N, d->K, out, ldo, d->flags & MOE_F_OUT_FP32, s))
    return hip_status(hipGetLastError(), "int8 product");
  hipError_t e = launch_i8_quant_rows(xb, ldx, d->M, d->K, nullptr, w.q, w.scale, s);
  if (e != hipSuccess) return hip_status(e, "quant rows");
  e = launch_i8_matmul(w.q, w.scale, b, b_scale, d->M, d->N, d->K, out, ldo, d->flags & MOE_F_OUT_FP32, s);
  return hip_status(e, "int8 product");
}

size_t moe_experts_i8_workspace_bytes(const moe_experts_dims* d) {
  if (check_experts_i8(d) != MOE_OK) return 0;
  return experts_layout(d, nullptr).bytes;
}

int moe_experts_i8(const moe_experts_dims* d, const void* xp, const int32_t* counts, const moe_i8_experts* w, void* o,
                   void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_experts_i8(d)) return rc;
  if (int rc = check_ptrs({{"xp", xp}, {"counts", counts}, {"o", o}, {"ws", ws}})) return rc;
  if (int rc = check_weights(w)) return rc;
  const ExpertsWs l = experts_layout(d, ws);
  if (ws_bytes < l.bytes) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, l.bytes);
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = launch_offsets_from_counts(counts, d->E, d->rows, l.offsets, l.tile_start, l.tile_desc, s);
  if (e != hipSuccess) return hip_status(e, "offsets");
  e = launch_i8_quant_rows(static_cast<const bf16_t*>(xp), d->H, d->rows, d->H, l.offsets + d->E, l.x8, l.sx, s);
  if (e != hipSuccess) return hip_status(e, "quant rows");
  return expert_products({d->rows, d->E, l.offsets}, l.x8, l.sx, nullptr, w, d->H, d->F, l.rows,
                         static_cast<bf16_t*>(o), s);
}

size_t moe_infer_i8_workspace_bytes(const moe_dims* d) {
  if (check_infer_i8(d) != MOE_OK) return 0;
  return infer_layout(d, nullptr).bytes;
}

int moe_infer_i8(const moe_dims* d, const void* x, const void* w_r, const moe_i8_experts* w, const uint8_t* token_mask,
                 void* y, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_infer_i8(d)) return rc;
  if (int rc = check_ptrs({{"x", x}, {"w_r", w_r}, {"y", y}, {"ws", ws}})) return rc;
  if (int rc = check_weights(w)) return rc;
  const bool masked = d->flags & MOE_F_MASK;
  if (masked && token_mask == nullptr) return fail(MOE_ERR_ARG, "MOE_F_MASK set but token_mask is NULL");
  const InferWs l = infer_layout(d, ws);
  if (ws_bytes < l.bytes) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, l.bytes);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int T = d->T, H = d->H, E = d->E, F = d->F, k = d->top_k;
  const bf16_t* xb = static_cast<const bf16_t*>(x);
  hipError_t e = launch_router_fwd(xb, static_cast<const bf16_t*>(w_r), masked ? token_mask : nullptr, T, H, E, k,
                                   l.logits, l.router_part, l.topk_idx, l.gates, nullptr, l.perm, l.row_token, s);
  if (e != hipSuccess) return hip_status(e, "router");
  e = launch_permute(l.topk_idx, xb, T, H, E, k, l.counts, l.offsets, l.tile_start, l.tile_desc, l.row_token, l.row_of,
                     nullptr, l.perm, s);
  if (e != hipSuccess) return hip_status(e, "permute");
  // a token is rounded once, and its k rows read that
  e = launch_i8_quant_rows(xb, H, T, H, nullptr, l.x8, l.sx, s);
  if (e != hipSuccess) return hip_status(e, "quant rows");
  if (int rc = expert_products({T * k, E, l.offsets}, l.x8, l.sx, l.row_token, w, H, F, l.rows, l.o, s)) return rc;
  return hip_status(launch_combine(l.o, l.gates, l.row_of, T, H, k, static_cast<bf16_t*>(y), s), "combine");
}

int moe_kv_plan(const moe_kv_plan_dims* d, const int32_t* old_len, const int32_t* new_len, int32_t* block_table,
                const int32_t* free_ids, const int32_t* n_free, int32_t* row_start, int32_t* kv_len,
                int32_t* positions, int32_t* slots, int32_t* seq, int32_t* state, void* stream) {
  if (d == nullptr) return fail(MOE_ERR_ARG, "dims is NULL");
  if (d->B < 1 || d->W < 1 || d->T < 0 || d->n_blocks < 1 || d->free_cap < 0)
    return fail(MOE_ERR_ARG, "B, W, n_blocks must be positive, T, free_cap not negative (B=%d W=%d n_blocks=%d T=%d free_cap=%d)",
                d->B, d->W, d->n_blocks, d->T, d->free_cap);
  if (!block_size_ok(d->block_tokens))
    return fail(MOE_ERR_SHAPE, "block_tokens=%d must be 16, 32, 64 or 128", d->block_tokens);
  if (static_cast<int64_t>(d->n_blocks) * d->block_tokens > 0x7fffffffll ||
      static_cast<int64_t>(d->W) * d->block_tokens > 0x7fffffffll)
    return fail(MOE_ERR_ARG, "n_blocks=%d or W=%d x block_tokens=%d exceeds 2^31 - 1 slots", d->n_blocks, d->W,
                d->block_tokens);
  if (int rc = check_ptrs({{"old_len", old_len}, {"new_len", new_len}, {"block_table", block_table},
                           {"n_free", n_free}, {"row_start", row_start}, {"kv_len", kv_len}, {"state", state}}))
    return rc;
  if (d->free_cap > 0)
    if (int rc = check_ptrs({{"free_ids", free_ids}})) return rc;
  if (d->T > 0)
    if (int rc = check_ptrs({{"positions", positions}, {"slots", slots}, {"seq", seq}})) return rc;
  if (shifted(kv_len, d->B, old_len, d->B) || shifted(kv_len, d->B, new_len, d->B))
    return fail(MOE_ERR_ARG, "kv_len overlaps old_len or new_len without being it");
  return hip_status(launch_kv_plan(*d, old_len, new_len, block_table, free_ids, n_free, row_start, kv_len, positions,
                                   slots, seq, state, static_cast<hipStream_t>(stream)),
                    "cache plan");
}

int moe_kv_append(const moe_kv_cache* c, const moe_kv_batch* b, const void* k, const void* v, int64_t ld,
                  void* stream) {
  if (int rc = check_cache(c)) return rc;
  if (int rc = check_batch(c, b)) return rc;
  if (b->T == 0) return ok();
  if (int rc = check_pitch("ld", ld, static_cast<int64_t>(c->kv_heads) * c->head_dim, 8)) return rc;
  if (int rc = check_ptrs({{"k", k}, {"v", v}})) return rc;
  return hip_status(launch_kv_append(*c, *b, static_cast<const bf16_t*>(k), static_cast<const bf16_t*>(v), ld,
                                     static_cast<hipStream_t>(stream)),
                    "cache append");
}

int moe_kv_read(const moe_kv_cache* c, int32_t B, int32_t W, const int32_t* block_table, const int32_t* kv_start,
                int32_t total, void* k_out, void* v_out, void* stream) {
  if (int rc = check_cache(c)) return rc;
  const moe_kv_batch b{B, total, W, kv_start, kv_start, block_table};
  if (int rc = check_batch_dims(c, &b)) return rc;
  if (int rc = check_ptrs({{"block_table", block_table}, {"kv_start", kv_start}})) return rc;
  if (total == 0) return ok();
  if (int rc = check_ptrs({{"k_out", k_out}, {"v_out", v_out}})) return rc;
  return hip_status(launch_kv_read(*c, B, W, block_table, kv_start, total, static_cast<bf16_t*>(k_out),
                                   static_cast<bf16_t*>(v_out), static_cast<hipStream_t>(stream)),
                    "cache read");
}

size_t moe_kv_attention_workspace_bytes(const moe_kv_cache* c, const moe_kv_batch* b, const moe_kv_attn* a) {
  if (check_cache(c) != MOE_OK || check_batch_dims(c, b) != MOE_OK || check_attn(c, b, a) != MOE_OK) return 0;
  return kv_attention_ws(*c, *b, *a);
}

int moe_kv_attention(const moe_kv_cache* c, const moe_kv_batch* b, const moe_kv_attn* a, const void* q, int64_t ldq,
                     void* out, int64_t ldo, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_cache(c)) return rc;
  if (int rc = check_batch(c, b)) return rc;
  if (int rc = check_attn(c, b, a)) return rc;
  if (b->T == 0) return ok();
  const int64_t row = static_cast<int64_t>(a->heads) * c->head_dim;
  if (int rc = check_pitch("ldq", ldq, row, 8)) return rc;
  if (int rc = check_pitch("ldo", ldo, row, 8)) return rc;
  if (int rc = check_ptrs({{"q", q}, {"out", out}, {"ws", ws}})) return rc;
  const size_t need = kv_attention_ws(*c, *b, *a);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  return hip_status(launch_kv_attention(*c, *b, *a, static_cast<const bf16_t*>(q), ldq, static_cast<bf16_t*>(out), ldo,
                                        ws, static_cast<hipStream_t>(stream)),
                    "cache attention");
}

}  // extern "C"
