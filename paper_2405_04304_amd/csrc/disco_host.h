// What the files of the C boundary share: error texts, the handles behind the opaque types and the workspace of a forward.
#pragma once
#include "../../include/disco.h"
#include "disco_internal.h"

#include <cstdarg>
#include <cstdio>
#include <vector>

namespace disco {

inline thread_local char g_err[512] = "";

inline int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return code;
}

inline int hip_fail(hipError_t e, const char* what) {
  return fail(DISCO_EHIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace disco

#define HIP_TRY(expr, what) do { hipError_t e__ = (expr); if (e__ != hipSuccess) return hip_fail(e__, what); } while (0)

struct disco_model {
  disco_model_desc d;
  disco_model_weights w;
  std::vector<disco_layer_weights> layers;
  int d_q, d_kv, d_qkv;
  // one launch per forward (RMSNorm / rotary / SwiGLU family with shapes the persistent kernel tiles)
  bool persist_ok, persist_big;
  std::vector<disco::FwdLayer> fwd_layers;      // copied into every workspace by disco_workspace_init
  int loop_steps;                        // draft-loop steps the workspace holds panel versions for (1: none beyond one forward)
};

struct disco_kv {
  const disco_model* model;
  disco::bf16_t* pages;
  int32_t* dev_page_table;   // inside the caller's buffer, or nullptr for the identity order
  float* dev_rope;           // inside the caller's buffer: [capacity][d_head / 2][cos, sin] (family B), else nullptr
  bool rope_ready;           // the table is written by the first forward that uses the cache, on its stream
  int page_tokens, n_pages, capacity, len;
  size_t layer_stride;       // elements between layers
};

namespace disco {

struct Ws {
  float* h; float* q; bf16_t* xn; bf16_t* xattn; bf16_t* xact; float* part; float* gpart; size_t gpart_bytes; float* logits;
  float* ssq; int* gemm_counters; int* attn_counters; int n_counters; float* clf_scratch;
  uint32_t* gate; int32_t* sl_count; int32_t* tok_next;
  int* head_ready; unsigned* abort_word;     // fused QKV + attention launch: per-head counters, sticky failure flag
  // LayerNorm family: per-tile sums beside ssq, and the correction vectors of the deferred norms (W . g, W . b) of
  // every matrix that reads a normalised row: per layer [wg | wb] of the QKV matrix (2 d_qkv floats) and of the MLP
  // input matrix (2 d_ff), then the LM head's (2 vocab); written by disco_workspace_init
  float* sum; float* ln_vec; size_t ln_layer_stride;
  // persistent forward: panel versions (a fresh address per phase and step), the layer table, barrier words
  bf16_t* xn_v; bf16_t* xattn_v; bf16_t* xact_v; float* q_v; size_t xn_stride, xattn_stride, xact_stride;
  FwdLayer* fwd_layers; unsigned* bar;
  size_t total;
};

// Carve the workspace; with base == nullptr only the total is meaningful.
inline Ws carve(const disco_model* m, int max_block, int max_ctx, void* base) {
  (void)max_block;  // buffers are sized for DISCO_MAX_BLOCK tokens
  const disco_model_desc& d = m->d;
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) { void* r = p ? p + off : nullptr; off += round_up(bytes, 256); return r; };
  Ws w;
  w.h = static_cast<float*>(take(sizeof(float) * 16 * d.d_model));
  w.q = static_cast<float*>(take(sizeof(float) * 16 * m->d_q));
  w.xn = static_cast<bf16_t*>(take(sizeof(bf16_t) * 2 * 16 * d.d_model));
  w.xattn = static_cast<bf16_t*>(take(sizeof(bf16_t) * 2 * 16 * m->d_q));
  w.xact = static_cast<bf16_t*>(take(sizeof(bf16_t) * 2 * 16 * d.d_ff));
  // partial tiles and ticket counters of split row groups: sized for the widest matrix of the model
  int max_rows = d.vocab;
  if (m->d_qkv > max_rows) max_rows = m->d_qkv;
  if (2 * d.d_ff > max_rows) max_rows = 2 * d.d_ff;
  if (d.d_model > max_rows) max_rows = d.d_model;
  const int max_tiles = max_rows / 16;
  w.gpart_bytes = sizeof(float) * GEMM_MAX_SPLIT * 256 * (size_t)max_tiles;
  w.gpart = static_cast<float*>(take(w.gpart_bytes));
  w.logits = static_cast<float*>(take(sizeof(float) * 16 * (size_t)d.vocab));
  w.ssq = static_cast<float*>(take(sizeof(float) * 16 * (size_t)(d.d_model / 16)));
  w.sum = nullptr; w.ln_vec = nullptr; w.ln_layer_stride = 2 * ((size_t)m->d_qkv + d.d_ff);
  if (d.family == DISCO_FAMILY_A) {
    w.sum = static_cast<float*>(take(sizeof(float) * 16 * (size_t)(d.d_model / 16)));
    w.ln_vec = static_cast<float*>(take(sizeof(float) * (w.ln_layer_stride * d.n_layers + 2 * (size_t)d.vocab)));
  }
  w.n_counters = max_tiles + d.n_heads;
  w.gemm_counters = static_cast<int*>(take(sizeof(int) * (size_t)w.n_counters));
  w.attn_counters = w.gemm_counters ? w.gemm_counters + max_tiles : nullptr;
  w.clf_scratch = static_cast<float*>(take(CLASSIFY_SCRATCH_BYTES));
  w.gate = static_cast<uint32_t*>(take(256));
  w.sl_count = reinterpret_cast<int32_t*>(w.gate ? w.gate + 16 : nullptr);
  w.tok_next = reinterpret_cast<int32_t*>(w.gate ? w.gate + 32 : nullptr);
  w.abort_word = w.gate ? w.gate + 48 : nullptr;
  w.head_ready = static_cast<int*>(take(sizeof(int) * QKV_ATTN_READY_SLOT * (size_t)d.n_heads));
  w.xn_stride = (size_t)2 * 16 * d.d_model + 2 * (size_t)d.d_model;      // two panels + d floats of sums of squares
  w.xattn_stride = (size_t)2 * 16 * m->d_q; w.xact_stride = (size_t)2 * 16 * d.d_ff;
  w.xn_v = w.xattn_v = w.xact_v = nullptr; w.q_v = nullptr; w.fwd_layers = nullptr; w.bar = nullptr;
  if (m->persist_ok) {
    const size_t steps = (size_t)m->loop_steps, L = (size_t)d.n_layers;
    w.xn_v = static_cast<bf16_t*>(take(sizeof(bf16_t) * w.xn_stride * (2 * L + 1) * steps));
    w.xattn_v = static_cast<bf16_t*>(take(sizeof(bf16_t) * w.xattn_stride * L * steps));
    w.xact_v = static_cast<bf16_t*>(take(sizeof(bf16_t) * w.xact_stride * L * steps));
    w.q_v = static_cast<float*>(take(sizeof(float) * 16 * m->d_q * L * steps));
    w.fwd_layers = static_cast<FwdLayer*>(take(sizeof(FwdLayer) * L));
    w.bar = static_cast<unsigned*>(take(sizeof(unsigned) * FWD_BAR_WORDS));
  }
  // the only buffer whose size depends on max_ctx goes last, so that every other offset (the ticket
  // counters above all) is the same for every call on this workspace
  const int n_splits = (max_ctx + DISCO_MAX_BLOCK + ATTN_SPLIT_LEN - 1) / ATTN_SPLIT_LEN;
  w.part = static_cast<float*>(take(sizeof(float) * (size_t)d.n_heads * n_splits * 16 * (d.d_head + 2)));
  w.total = off;
  return w;
}

}  // namespace disco
