// C ABI of a decoding step's operators (declared in include/moe.h): argument
// checks, workspace layouts and launch sequences.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "api.hpp"
#include "launch.hpp"
#include "serve.hpp"
#include "step.hpp"

using namespace moe;

namespace {

// ---- norms
int check_norm(const moe_norm_dims* d) {
  if (d == nullptr) return fail(MOE_ERR_ARG, "dims is NULL");
  if (d->T < 1 || d->H < 1 || d->H > MOE_NORM_MAX_H)
    return fail(MOE_ERR_ARG, "T=%d must be positive, H=%d in [1, %d]", d->T, d->H, MOE_NORM_MAX_H);
  if (d->H % 8 != 0) return fail(MOE_ERR_SHAPE, "H=%d must be a multiple of 8", d->H);
  if (d->flags & ~MOE_F_DW_FP32) return fail(MOE_ERR_ARG, "unknown flags 0x%x", d->flags);
  if (!(d->eps >= FLT_MIN) || !std::isfinite(d->eps))
    return fail(MOE_ERR_ARG, "eps=%g must be a positive normal number", static_cast<double>(d->eps));
  return MOE_OK;
}

int check_rows(const char* name, int64_t ld, int64_t H) {
  if (ld < H) return fail(MOE_ERR_ARG, "ld of %s: %lld is less than %lld", name, static_cast<long long>(ld),
                          static_cast<long long>(H));
  if (ld > (1ll << 31)) return fail(MOE_ERR_ARG, "ld of %s: %lld exceeds 2^31", name, static_cast<long long>(ld));
  if (ld % 8 != 0) return fail(MOE_ERR_SHAPE, "ld of %s: %lld must be a multiple of 8", name, static_cast<long long>(ld));
  return MOE_OK;
}

// A stretch of memory that a call reads or writes.
struct Span {
  const char* name;
  const void* p;  // null: not given
  int64_t bytes;
  bool whole;  // rows of H bf16 without gaps: what may be written in place
};
Span span_rows(const char* name, const void* p, int64_t T, int64_t H, int64_t ld) {
  return {name, p, ((T - 1) * ld + H) * 2, ld == H || T == 1};
}
bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p != nullptr && b.p != nullptr && x < y + b.bytes && y < x + a.bytes;
}
// Whether an output overlaps another or an input other than, in `in_place`
// rows, as that input itself.
int check_spans(std::initializer_list<Span> in, std::initializer_list<Span> out) {
  for (const Span& o : out) {
    for (const Span& i : in)
      if (overlap(o, i) && !(o.p == i.p && o.whole && i.whole))
        return fail(MOE_ERR_ARG, "%s overlaps %s", o.name, i.name);
    for (const Span& p : out)
      if (&p != &o && overlap(o, p)) return fail(MOE_ERR_ARG, "%s overlaps %s", o.name, p.name);
  }
  return MOE_OK;
}

struct NormBwdWs {
  float* part;
  size_t bytes;
};
NormBwdWs norm_layout(const moe_norm_dims* d, void* base) {
  Carve c(base);
  NormBwdWs w;
  w.part = c.take<float>(static_cast<size_t>(norm_bwd_parts(d->T, d->H)) * d->H);
  w.bytes = c.off;
  return w;
}

// ---- the expert layer for a few tokens
int check_decode(const moe_dims* d) {
  if (int rc = check_dims(d)) return rc;
  if (d->T > MOE_DECODE_MAX_T) return fail(MOE_ERR_ARG, "T=%d exceeds %d", d->T, MOE_DECODE_MAX_T);
  if (d->F > (1 << 24) || d->H > (1 << 24)) return fail(MOE_ERR_ARG, "H=%d or F=%d exceeds 2^24", d->H, d->F);
  return MOE_OK;
}
int check_decode_i8(const moe_dims* d) {
  if (int rc = check_decode(d)) return rc;
  if (d->H > MOE_I8_MAX_K || d->F > MOE_I8_MAX_K)
    return fail(MOE_ERR_ARG, "H=%d or F=%d exceeds %d", d->H, d->F, MOE_I8_MAX_K);
  return MOE_OK;
}

struct DecodeWs {
  DecodeRows rows;
  int32_t* row_token;
  bf16_t* a;   // bf16 experts: the activation's summands,
  float* gu;   // or the ranges' G and U
  float *a32, *top, *sx, *sa;  // int8 experts
  int8_t *x8, *a8;
  float* o;
  size_t bytes;
};
DecodeWs decode_layout(const moe_dims* d, bool i8, void* base) {
  const size_t T = d->T, E = d->E, R = T * d->top_k, RF = R * d->F;
  Carve c(base);
  DecodeWs w{};
  w.rows = {nullptr, nullptr, nullptr, nullptr, nullptr, d->T, d->H, d->E, d->F, d->top_k};
  w.rows.part = c.take<float>(T * E + static_cast<size_t>(router_part_floats(d->T, d->E)));
  w.rows.gates = c.take<float>(R);
  w.rows.topk_idx = c.take<int32_t>(R);
  w.rows.counts = c.take<int32_t>(E);
  w.row_token = c.take<int32_t>(R);
  if (i8) {
    w.x8 = c.take<int8_t>(T * d->H);
    w.sx = c.take<float>(T);
    w.a32 = c.take<float>(RF);
    w.top = c.take<float>(RF / 16);
    w.a8 = c.take<int8_t>(RF);
    w.sa = c.take<float>(R);
  } else if (const int ranges = decode_ranges(d->T, d->E, d->F, d->top_k); ranges > 1) {
    w.gu = c.take<float>(2 * ranges * RF);
  } else {
    w.a = c.take<bf16_t>(kDecodeParts * RF);
  }
  w.o = c.take<float>(R * d->H);
  w.bytes = c.off;
  return w;
}

// A call of fewer tokens may use more, where their product is split over K:
// what a size query returns is enough for up to its T.
size_t decode_bytes(const moe_dims* d, bool i8) {
  size_t most = decode_layout(d, i8, nullptr).bytes;
  if (i8) return most;
  moe_dims e = *d;
  for (e.T = d->T - 1; e.T > 0; --e.T) {
    if (!decode_fused(e.T)) e.T = kDecodeFusedT;
    if (decode_ranges(e.T, e.E, e.F, e.top_k) > 1) most = std::max(most, decode_layout(&e, i8, nullptr).bytes);
  }
  return most;
}

// Router and, but for the fewest tokens, the selection.
hipError_t route(const DecodeWs& l, const bf16_t* x, const bf16_t* w_r, hipStream_t s) {
  const DecodeRows& r = l.rows;
  if (const hipError_t e = launch_decode_router(r, x, w_r, l.x8, l.sx, s); e != hipSuccess || decode_fused(r.T)) return e;
  // one chunk of counts: the tokens are fewer than the selection's chunk
  static_assert(MOE_DECODE_MAX_T <= kPermChunk, "counts of one chunk");
  return launch_topk(r.mask, r.T, r.E, r.k, r.part, r.part + static_cast<int64_t>(r.T) * r.E, r.topk_idx, r.gates, nullptr,
                     r.counts, l.row_token, s);
}

// ---- sampling
int check_sample(const moe_sample_dims* d) {
  if (d == nullptr) return fail(MOE_ERR_ARG, "dims is NULL");
  if (d->B < 1 || d->B > 65535 || d->V < 1 || d->V > MOE_SAMPLE_MAX_V)
    return fail(MOE_ERR_ARG, "B=%d must be in [1, 65535], V=%d in [1, %d]", d->B, d->V, MOE_SAMPLE_MAX_V);
  if (d->flags & ~MOE_F_LOGITS_FP32) return fail(MOE_ERR_ARG, "unknown flags 0x%x", d->flags);
  return MOE_OK;
}
int check_given(std::initializer_list<std::pair<const char*, const void*>> ps) {
  for (const auto& p : ps)
    if (p.second != nullptr)
      if (int rc = check_ptrs({p})) return rc;
  return MOE_OK;
}

int check_elements(std::initializer_list<std::pair<const char*, const void*>> ps, int size, bool required) {
  for (const auto& p : ps) {
    if (p.second == nullptr && required) return fail(MOE_ERR_ARG, "%s is NULL", p.first);
    if (reinterpret_cast<uintptr_t>(p.second) % size != 0)
      return fail(MOE_ERR_ALIGN, "%s is not aligned to its elements", p.first);
  }
  return MOE_OK;
}

}  // namespace

extern "C" {

int moe_norm_fwd(const moe_norm_dims* d, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* w,
                 void* h, void* y, int8_t* q, float* scale, void* stream) {
  if (int rc = check_norm(d)) return rc;
  if (int rc = check_rows("x", ldx, d->H)) return rc;
  if (residual != nullptr)
    if (int rc = check_rows("residual", ldr, d->H)) return rc;
  if (int rc = check_ptrs({{"x", x}, {"w", w}})) return rc;
  if (int rc = check_given({{"residual", residual}, {"h", h}, {"y", y}, {"q", q}, {"scale", scale}})) return rc;
  if (h != nullptr && residual == nullptr) return fail(MOE_ERR_ARG, "h without a residual");
  if (y == nullptr && q == nullptr) return fail(MOE_ERR_ARG, "y and q are both NULL");
  if ((q == nullptr) != (scale == nullptr)) return fail(MOE_ERR_ARG, "q and scale go together");
  if (q != nullptr && d->H % 16 != 0) return fail(MOE_ERR_SHAPE, "H=%d must be a multiple of 16 for int8 rows", d->H);
  const int64_t T = d->T, H = d->H;
  if (int rc = check_spans({span_rows("x", x, T, H, ldx), span_rows("residual", residual, T, H, ldr), {"w", w, 2 * H, false}},
                           {span_rows("h", h, T, H, H), span_rows("y", y, T, H, H), {"q", q, T * H, false},
                            {"scale", scale, T * 4, false}}))
    return rc;
  const NormFwd a{static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(residual), ldx, ldr,
                  static_cast<const bf16_t*>(w), static_cast<bf16_t*>(h), static_cast<bf16_t*>(y), q, scale, d->T, d->H,
                  d->eps};
  return hip_status(launch_norm_fwd(a, static_cast<hipStream_t>(stream)), "norm");
}

size_t moe_norm_bwd_workspace_bytes(const moe_norm_dims* d) {
  if (check_norm(d) != MOE_OK) return 0;
  return norm_layout(d, nullptr).bytes;
}

int moe_norm_bwd(const moe_norm_dims* d, const void* h, int64_t ldh, const void* w, const void* dy, int64_t lddy,
                 const void* dh, int64_t lddh, void* dx, void* dw, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_norm(d)) return rc;
  if (int rc = check_rows("h", ldh, d->H)) return rc;
  if (int rc = check_rows("dy", lddy, d->H)) return rc;
  if (dh != nullptr)
    if (int rc = check_rows("dh", lddh, d->H)) return rc;
  if (int rc = check_ptrs({{"h", h}, {"w", w}, {"dy", dy}, {"dx", dx}, {"dw", dw}, {"ws", ws}})) return rc;
  if (int rc = check_given({{"dh", dh}})) return rc;
  const NormBwdWs l = norm_layout(d, ws);
  if (ws_bytes < l.bytes) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, l.bytes);
  const int64_t T = d->T, H = d->H;
  Span in_h = span_rows("h", h, T, H, ldh);
  in_h.whole = false;  // dx must not replace what a later call may need
  if (int rc = check_spans({in_h, span_rows("dy", dy, T, H, lddy), span_rows("dh", dh, T, H, lddh), {"w", w, 2 * H, false}},
                           {span_rows("dx", dx, T, H, H), {"dw", dw, H * (d->flags & MOE_F_DW_FP32 ? 4 : 2), false},
                            {"ws", ws, static_cast<int64_t>(l.bytes), false}}))
    return rc;
  const NormBwd a{static_cast<const bf16_t*>(h), static_cast<const bf16_t*>(dy), static_cast<const bf16_t*>(dh), ldh, lddy,
                  lddh, static_cast<const bf16_t*>(w), static_cast<bf16_t*>(dx), dw, (d->flags & MOE_F_DW_FP32) != 0, l.part,
                  d->T, d->H, d->eps};
  return hip_status(launch_norm_bwd(a, static_cast<hipStream_t>(stream)), "norm backward");
}

size_t moe_decode_workspace_bytes(const moe_dims* d) {
  if (check_decode(d) != MOE_OK) return 0;
  return decode_bytes(d, false);
}

int moe_decode(const moe_dims* d, const void* x, const void* w_r, const void* w_gate, const void* w_up,
               const void* w_down, const uint8_t* token_mask, void* y, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_decode(d)) return rc;
  if (int rc = check_ptrs({{"x", x}, {"w_r", w_r}, {"w_gate", w_gate}, {"w_up", w_up}, {"w_down", w_down}, {"y", y},
                           {"ws", ws}}))
    return rc;
  const bool masked = d->flags & MOE_F_MASK;
  if (masked && token_mask == nullptr) return fail(MOE_ERR_ARG, "MOE_F_MASK set but token_mask is NULL");
  DecodeWs l = decode_layout(d, false, ws);
  if (const size_t need = decode_bytes(d, false); ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  l.rows.mask = masked ? token_mask : nullptr;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bf16_t* xb = static_cast<const bf16_t*>(x);
  hipError_t e = route(l, xb, static_cast<const bf16_t*>(w_r), s);
  if (e != hipSuccess) return hip_status(e, "router");
  e = launch_decode_gateup(l.rows, xb, static_cast<const bf16_t*>(w_gate), static_cast<const bf16_t*>(w_up), l.a, l.gu, s);
  if (e != hipSuccess) return hip_status(e, "gate/up");
  e = launch_decode_down(l.rows, l.a, l.gu, static_cast<const bf16_t*>(w_down), l.o, s);
  if (e != hipSuccess) return hip_status(e, "down");
  return hip_status(launch_decode_combine(l.rows, l.o, static_cast<bf16_t*>(y), s), "combine");
}

size_t moe_decode_i8_workspace_bytes(const moe_dims* d) {
  if (check_decode_i8(d) != MOE_OK) return 0;
  return decode_bytes(d, true);
}

int moe_decode_i8(const moe_dims* d, const void* x, const void* w_r, const moe_i8_experts* w, const uint8_t* token_mask,
                  void* y, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_decode_i8(d)) return rc;
  if (int rc = check_ptrs({{"x", x}, {"w_r", w_r}, {"y", y}, {"ws", ws}})) return rc;
  if (w == nullptr) return fail(MOE_ERR_ARG, "w is NULL");
  if (int rc = check_ptrs({{"w.w_gate", w->w_gate}, {"w.w_up", w->w_up}, {"w.w_down", w->w_down}, {"w.s_gate", w->s_gate},
                           {"w.s_up", w->s_up}, {"w.s_down", w->s_down}}))
    return rc;
  const bool masked = d->flags & MOE_F_MASK;
  if (masked && token_mask == nullptr) return fail(MOE_ERR_ARG, "MOE_F_MASK set but token_mask is NULL");
  DecodeWs l = decode_layout(d, true, ws);
  if (ws_bytes < l.bytes) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, l.bytes);
  l.rows.mask = masked ? token_mask : nullptr;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bf16_t* xb = static_cast<const bf16_t*>(x);
  hipError_t e = route(l, xb, static_cast<const bf16_t*>(w_r), s);
  if (e != hipSuccess) return hip_status(e, "router");
  e = launch_decode_gateup_i8(l.rows, l.x8, l.sx, *w, l.a32, l.top, s);
  if (e != hipSuccess) return hip_status(e, "gate/up");
  e = launch_decode_down_i8(l.rows, l.a32, l.top, l.a8, l.sa, *w, l.o, s);
  if (e != hipSuccess) return hip_status(e, "down");
  return hip_status(launch_decode_combine(l.rows, l.o, static_cast<bf16_t*>(y), s), "combine");
}

size_t moe_sample_workspace_bytes(const moe_sample_dims* d) {
  if (check_sample(d) != MOE_OK) return 0;
  return sample_ws(d->B, d->V);
}

int moe_sample(const moe_sample_dims* d, const void* logits, int64_t ld, const float* temperature,
               const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* token,
               float* logprob, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_sample(d)) return rc;
  if (ld < d->V) return fail(MOE_ERR_ARG, "ld=%lld is less than %d", static_cast<long long>(ld), d->V);
  if (ld > (1ll << 31)) return fail(MOE_ERR_ARG, "ld=%lld exceeds 2^31", static_cast<long long>(ld));
  // logits, settings and outputs are read and written by the element: any slice of a tensor will do
  const int size = d->flags & MOE_F_LOGITS_FP32 ? 4 : 2;
  if (int rc = check_elements({{"logits", logits}}, size, true)) return rc;
  if (int rc = check_elements({{"u", u}, {"token", token}}, 4, true)) return rc;
  if (int rc = check_elements({{"temperature", temperature}, {"top_k", top_k}, {"top_p", top_p}, {"min_p", min_p},
                               {"logprob", logprob}}, 4, false))
    return rc;
  if (int rc = check_ptrs({{"ws", ws}})) return rc;
  const size_t need = sample_ws(d->B, d->V);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  const SampleArgs a{logits, ld, (d->flags & MOE_F_LOGITS_FP32) != 0, d->B, d->V, temperature, top_p, min_p, top_k, u,
                     token, logprob};
  return hip_status(launch_sample(a, ws, static_cast<hipStream_t>(stream)), "sample");
}

}  // extern "C"
