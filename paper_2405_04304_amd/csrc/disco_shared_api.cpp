// C boundary of the operators for several sequences that continue one prompt: argument checks on the host, then the launches of
// disco_shared.hip.
#include "disco_host.h"
#include "disco_shared.h"

#include <cmath>

using namespace disco;

namespace {

constexpr int MOST_SEQS = 65535, MOST_HEADS = 1024, MOST_POSITIONS = 1 << 30;

// The sizes of a cache (pointers apart), and the kernels' view of it.
int check_shape(const disco_shared_kv* kv) {
  if (!kv) return fail(DISCO_EINVAL, "null argument");
  if (kv->d_head != 64 && kv->d_head != 128) return fail(DISCO_EINVAL, "d_head %d unsupported (64 or 128)", kv->d_head);
  if (kv->page_tokens < 4 || kv->page_tokens % 4 || kv->page_tokens > 1 << 20) return fail(DISCO_EINVAL, "the page size must be a positive multiple of 4");
  if (kv->n_kv_heads < 1 || kv->n_kv_heads > MOST_HEADS) return fail(DISCO_EINVAL, "%d K / V heads", kv->n_kv_heads);
  if (kv->n_seqs < 0 || kv->n_seqs > MOST_SEQS) return fail(DISCO_EINVAL, "%d sequences outside [0, %d]", kv->n_seqs, MOST_SEQS);
  if (kv->prefix_len < 0 || kv->prefix_len > MOST_POSITIONS || kv->n_prefix_pages < 0) return fail(DISCO_EINVAL, "bad prompt length");
  if (kv->table_ld < 1 || kv->n_pages < 1 || (int64_t)kv->table_ld * kv->page_tokens > MOST_POSITIONS) return fail(DISCO_EINVAL, "bad page tables");
  return DISCO_OK;
}

int check_cache(const disco_shared_kv* kv, bool prefix) {
  if (!kv->dev_pages || !kv->dev_tables) return fail(DISCO_EINVAL, "null argument");
  if (!aligned(kv->dev_pages, 16) || !aligned(kv->dev_tables, 4) || !aligned(kv->dev_lens, 4)) return fail(DISCO_EINVAL, "misaligned pointer");
  if (prefix && kv->prefix_len > 0) {
    if (!kv->dev_prefix) return fail(DISCO_EINVAL, "null argument");
    if (!aligned(kv->dev_prefix, 16) || !aligned(kv->dev_prefix_table, 4)) return fail(DISCO_EINVAL, "misaligned pointer");
    if (!kv->dev_prefix_table && ((int64_t)kv->prefix_len + kv->page_tokens - 1) / kv->page_tokens > kv->n_prefix_pages)
      return fail(DISCO_ECAP, "a prompt of %d positions in %d pages", kv->prefix_len, kv->n_prefix_pages);
  }
  return DISCO_OK;
}

SharedKv device_view(const disco_shared_kv& k) {
  SharedKv v{};
  v.prefix = static_cast<const bf16_t*>(k.dev_prefix); v.prefix_table = k.dev_prefix_table; v.n_prefix_pages = k.n_prefix_pages; v.prefix_len = k.prefix_len;
  v.pages = static_cast<bf16_t*>(k.dev_pages); v.tables = k.dev_tables; v.lens = k.dev_lens; v.n_pages = k.n_pages; v.table_ld = k.table_ld;
  v.n_seqs = k.n_seqs; v.pt = k.page_tokens; v.nkv = k.n_kv_heads; v.dh = k.d_head;
  v.pt_shift = (k.page_tokens & (k.page_tokens - 1)) == 0 ? __builtin_ctz((unsigned)k.page_tokens) : -1;
  return v;
}

int check_heads(int n_heads, const disco_shared_kv* kv) {
  if (n_heads < 1 || n_heads > MOST_HEADS || n_heads % kv->n_kv_heads) return fail(DISCO_EINVAL, "n_heads must be a multiple of n_kv_heads, at most %d", MOST_HEADS);
  return DISCO_OK;
}

// Rows of 16-byte pieces: type, pointer, row stride.
int check_rows(int dtype, const void* p, int64_t ld, int64_t width, const char* what) {
  if (dtype != DISCO_F32 && dtype != DISCO_BF16) return fail(DISCO_EINVAL, "unknown element type %d", dtype);
  if (!p) return fail(DISCO_EINVAL, "null argument");
  if (!aligned(p, 16)) return fail(DISCO_EINVAL, "%s misaligned", what);
  if (ld < width || ld % (dtype == DISCO_F32 ? 4 : 8)) return fail(DISCO_EINVAL, "row stride of %s: at least %lld elements and a multiple of 16 bytes", what, (long long)width);
  return DISCO_OK;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

int check_attn(const disco_shared_kv* kv, int n_tok, int n_heads, int max_len) {
  int rc = check_shape(kv);
  if (rc == DISCO_OK) rc = check_heads(n_heads, kv);
  if (rc) return rc;
  if (n_tok < 1 || n_tok > DISCO_MAX_BLOCK) return fail(DISCO_EINVAL, "%d tokens outside [1, %d]", n_tok, DISCO_MAX_BLOCK);
  if (max_len < 0) return fail(DISCO_EINVAL, "negative length");
  return DISCO_OK;
}

SharedAttnPlan attn_plan(const disco_shared_kv* kv, bool fp32, int n_tok, int n_heads, int max_len) {
  const int cap = kv->table_ld * kv->page_tokens;
  return shared_attn_plan(kv->n_seqs, n_tok, n_heads, kv->n_kv_heads, kv->d_head, fp32, kv->prefix_len, max_len == 0 || max_len > cap ? cap : max_len);
}

// A launch has fewer than 2^32 threads: elements of the rows (four a thread where parts are put together, two or more where rows are appended), and
// workgroups of up to 256.
constexpr double MOST_ELEMENTS = 8589934592.0, MOST_WORKGROUPS = 16777216.0;
bool launchable(const disco_shared_kv* kv, int n_tok, int n_heads, const SharedAttnPlan& p) {
  const double n = (double)kv->n_kv_heads * ((double)p.prefix_tiles * p.prefix_splits + (double)kv->n_seqs * p.own_tiles * p.own_splits);
  return n < MOST_WORKGROUPS && (double)kv->n_seqs * n_tok * n_heads * kv->d_head <= MOST_ELEMENTS;
}

}  // namespace

int disco_rope_table(float* dev_table, int n_pos, int d_head, float base, disco_stream s) {
  if (n_pos < 0 || n_pos > MOST_POSITIONS || d_head < 2 || d_head % 2 || !(base > 0.f) || !std::isfinite(base)) return fail(DISCO_EINVAL, "bad rotary table");
  if (n_pos == 0) return DISCO_OK;
  if (!dev_table) return fail(DISCO_EINVAL, "null argument");
  if (!aligned(dev_table, 16)) return fail(DISCO_EINVAL, "misaligned pointer");
  HIP_TRY(launch_rope_fill(dev_table, n_pos, d_head, base, static_cast<hipStream_t>(s)), "rotary table launch");
  return DISCO_OK;
}

int disco_append(const disco_shared_kv* kv, const void* dev_qkv, int dtype, int64_t ld_qkv, int n_rows, int n_heads, const int32_t* dev_seq,
                 const int32_t* dev_pos, const float* dev_rope, int n_rope, const float* dev_q_gain, const float* dev_k_gain, float eps,
                 void* dev_q, int64_t ld_q, disco_stream s) {
  int rc = check_shape(kv);
  if (rc == DISCO_OK) rc = check_heads(n_heads, kv);
  if (rc) return rc;
  if (n_rows < 0 || n_rows > 1 << 24) return fail(DISCO_EINVAL, "%d rows outside [0, 2^24]", n_rows);
  if ((dev_seq == nullptr) != (dev_pos == nullptr)) return fail(DISCO_EINVAL, "sequences and positions of the rows come together");
  if (n_rows == 0) return DISCO_OK;
  if (kv->n_seqs == 0) return fail(DISCO_EINVAL, "rows without sequences");
  if (!dev_seq && (!kv->dev_lens || n_rows % kv->n_seqs)) return fail(DISCO_EINVAL, "rows without sequences of their own need dev_lens and as many for every sequence");
  if ((rc = check_cache(kv, false))) return rc;
  const int64_t width = (int64_t)(n_heads + 2 * kv->n_kv_heads) * kv->d_head, q_width = (int64_t)n_heads * kv->d_head;
  if ((double)n_rows * width > MOST_ELEMENTS) return fail(DISCO_EINVAL, "%d rows of %lld elements: more than 2^33 in one call", n_rows, (long long)width);
  if ((rc = check_rows(dtype, dev_qkv, ld_qkv, width, "dev_qkv")) || (rc = check_rows(dtype, dev_q, ld_q, q_width, "dev_q"))) return rc;
  const size_t es = dtype == DISCO_F32 ? 4 : 2;
  if (overlap(dev_qkv, es * ((size_t)ld_qkv * (n_rows - 1) + width), dev_q, es * ((size_t)ld_q * (n_rows - 1) + q_width)))
    return fail(DISCO_EINVAL, "dev_q overlaps dev_qkv");
  if (!aligned(dev_seq, 4) || !aligned(dev_pos, 4) || !aligned(dev_rope, 16) || !aligned(dev_q_gain, 16) || !aligned(dev_k_gain, 16))
    return fail(DISCO_EINVAL, "misaligned pointer");
  if (dev_rope && n_rope < (int64_t)kv->prefix_len + (int64_t)kv->table_ld * kv->page_tokens)
    return fail(DISCO_ECAP, "rotary table of %d positions, %lld in the prompt and a table's pages", n_rope,
                (long long)kv->prefix_len + (long long)kv->table_ld * kv->page_tokens);
  if ((dev_q_gain || dev_k_gain) && !(eps > 0.f)) return fail(DISCO_EINVAL, "eps must be positive");
  AppendArgs a{};
  a.kv = device_view(*kv); a.qkv = dev_qkv; a.ld = ld_qkv; a.rows = n_rows; a.nq = n_heads; a.seq = dev_seq; a.pos = dev_pos;
  a.n_tok = dev_seq ? 1 : n_rows / kv->n_seqs; a.rope = dev_rope; a.q_gain = dev_q_gain; a.k_gain = dev_k_gain; a.eps = eps;
  a.q = dev_q; a.ld_q = ld_q;
  HIP_TRY(launch_append(a, dtype == DISCO_F32, static_cast<hipStream_t>(s)), "append launch");
  return DISCO_OK;
}

size_t disco_attn_shared_bytes(const disco_shared_kv* kv, int n_tok, int n_heads, int max_len) {
  if (check_attn(kv, n_tok, n_heads, max_len)) return 0;
  size_t n = 0;                      // (the two types' plans differ: room for either)
  for (int fp32 = 0; kv->n_seqs && fp32 < 2; ++fp32) {
    const size_t m = attn_plan(kv, fp32 != 0, n_tok, n_heads, max_len).bytes;
    n = m > n ? m : n;
  }
  return round_up(n < 256 ? 256 : n, 256);
}

int disco_attn_shared(const disco_shared_kv* kv, const void* dev_q, int dtype, int64_t ld_q, int n_tok, int n_heads, float scale, void* dev_out,
                      int64_t ld_out, float* dev_lse, int max_len, void* dev_ws, size_t ws_bytes, disco_stream s) {
  int rc = check_attn(kv, n_tok, n_heads, max_len);
  if (rc) return rc;
  if (!(scale > 0.f) || !std::isfinite(scale)) return fail(DISCO_EINVAL, "scale must be positive");
  if (kv->n_seqs == 0) return DISCO_OK;
  if (!kv->dev_lens) return fail(DISCO_EINVAL, "null argument");
  if ((rc = check_cache(kv, true))) return rc;
  const int64_t width = (int64_t)n_heads * kv->d_head, n_rows = (int64_t)kv->n_seqs * n_tok;
  if ((rc = check_rows(dtype, dev_q, ld_q, width, "dev_q")) || (rc = check_rows(dtype, dev_out, ld_out, width, "dev_out"))) return rc;
  if (!aligned(dev_lse, 4)) return fail(DISCO_EINVAL, "misaligned pointer");
  const size_t es = dtype == DISCO_F32 ? 4 : 2;
  if (overlap(dev_q, es * ((size_t)ld_q * (n_rows - 1) + width), dev_out, es * ((size_t)ld_out * (n_rows - 1) + width)))
    return fail(DISCO_EINVAL, "dev_out overlaps dev_q");
  SharedAttnArgs a{};
  a.plan = attn_plan(kv, dtype == DISCO_F32, n_tok, n_heads, max_len);
  if (!launchable(kv, n_tok, n_heads, a.plan)) return fail(DISCO_EINVAL, "more workgroups than a launch takes");
  if (a.plan.bytes > 0) {
    if (!dev_ws || !aligned(dev_ws, 256)) return fail(DISCO_EINVAL, "workspace null or not 256-byte aligned");
    if (ws_bytes < a.plan.bytes) return fail(DISCO_EINVAL, "workspace of %zu bytes, %zu needed", ws_bytes, a.plan.bytes);
    a.part = static_cast<float*>(dev_ws);
    a.ml = reinterpret_cast<float2*>(a.part + (size_t)a.plan.parts * n_rows * width);
  }
  a.kv = device_view(*kv); a.q = dev_q; a.ld_q = ld_q; a.n_tok = n_tok; a.nq = n_heads; a.scale = scale; a.out = dev_out; a.ld_out = ld_out; a.lse = dev_lse;
  HIP_TRY(launch_shared_attn(a, dtype == DISCO_F32, static_cast<hipStream_t>(s)), "attention launch");
  return DISCO_OK;
}

static int check_beams(int n_groups, int n_beams, int vocab, int k) {
  if (n_groups < 0 || n_groups > MOST_SEQS || n_beams < 1 || n_beams > DISCO_MAX_BEAMS) return fail(DISCO_EINVAL, "%d groups of %d beams", n_groups, n_beams);
  if ((int64_t)n_groups * n_beams > MOST_SEQS) return fail(DISCO_EINVAL, "%d groups of %d beams", n_groups, n_beams);
  if (vocab < 1 || vocab > DISCO_BEAM_MAX_VOCAB) return fail(DISCO_EINVAL, "vocab %d outside [1, %d]", vocab, DISCO_BEAM_MAX_VOCAB);
  if (k < 1 || k > DISCO_BEAM_MAX_K) return fail(DISCO_EINVAL, "k %d outside [1, %d]", k, DISCO_BEAM_MAX_K);
  return DISCO_OK;
}

static int beam_units(int rows, int vocab) { const int n = beam_unit_logits(rows, vocab); return (vocab + n - 1) / n; }

size_t disco_beam_select_bytes(int n_groups, int n_beams, int vocab, int k) {
  if (check_beams(n_groups, n_beams, vocab, k)) return 0;
  const size_t rows = (size_t)n_groups * n_beams, per_row = (size_t)beam_units((int)rows, vocab);
  return round_up(rows * per_row * (8 + 8 * (size_t)k) + 256, 256);
}

int disco_beam_select(const void* dev_logits, int dtype, int64_t ld_logits, int n_groups, int n_beams, int vocab, int k, const float* dev_scores,
                      const int32_t* dev_done, int end_token, int32_t* dev_tokens, int32_t* dev_parents, float* dev_scores_out,
                      int32_t* dev_done_out, void* dev_ws, size_t ws_bytes, disco_stream s) {
  const int rc = check_beams(n_groups, n_beams, vocab, k);
  if (rc) return rc;
  if (dtype != DISCO_F32 && dtype != DISCO_BF16) return fail(DISCO_EINVAL, "unknown element type %d", dtype);
  if (end_token < -1 || end_token >= vocab) return fail(DISCO_EINVAL, "end token %d outside [-1, vocab)", end_token);
  if (dev_done && end_token < 0) return fail(DISCO_EINVAL, "finished beams need an end token");
  if (n_groups == 0) return DISCO_OK;
  if (!dev_logits || !dev_scores || !dev_tokens || !dev_parents || !dev_scores_out || !dev_ws) return fail(DISCO_EINVAL, "null argument");
  if (ld_logits < vocab) return fail(DISCO_EINVAL, "row stride %lld below vocab", (long long)ld_logits);
  if (!aligned(dev_logits, dtype == DISCO_F32 ? 4 : 2) || !aligned(dev_scores, 4) || !aligned(dev_done, 4) || !aligned(dev_tokens, 4) || !aligned(dev_parents, 4) ||
      !aligned(dev_scores_out, 4) || !aligned(dev_done_out, 4) || !aligned(dev_ws, 256))
    return fail(DISCO_EINVAL, "misaligned pointer");
  // (a group's results are written while another's scores are read)
  const size_t in = 4 * (size_t)n_groups * n_beams, out = 4 * (size_t)n_groups * k;
  const void* outs[4] = {dev_tokens, dev_parents, dev_scores_out, dev_done_out};
  for (int i = 0; i < 4; ++i) {
    if (!outs[i]) continue;
    bool shared = overlap(outs[i], out, dev_scores, in) || (dev_done && overlap(outs[i], out, dev_done, in));
    for (int j = 0; j < i; ++j) shared |= overlap(outs[i], out, outs[j], out);
    if (shared) return fail(DISCO_EINVAL, "a result overlaps dev_scores, dev_done or another result");
  }
  const size_t need = disco_beam_select_bytes(n_groups, n_beams, vocab, k), rows = (size_t)n_groups * n_beams, per_row = (size_t)beam_units((int)rows, vocab);
  if (ws_bytes < need) return fail(DISCO_EINVAL, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  BeamSelectArgs a{};
  a.logits = dev_logits; a.ld = ld_logits; a.n_groups = n_groups; a.n_beams = n_beams; a.vocab = vocab; a.k = k; a.scores = dev_scores; a.done = dev_done;
  a.end_token = end_token; a.tokens = dev_tokens; a.parents = dev_parents; a.scores_out = dev_scores_out; a.done_out = dev_done_out;
  a.cand = static_cast<unsigned long long*>(dev_ws); a.stats = reinterpret_cast<float2*>(a.cand + rows * per_row * k); a.units = (int)per_row;
  HIP_TRY(launch_beam_select(a, dtype == DISCO_F32, static_cast<hipStream_t>(s)), "beam selection launch");
  return DISCO_OK;
}

int disco_beam_reorder(void* dev_pages, int n_layers, int64_t layer_stride, int n_pages, int64_t page_elems, const int32_t* dev_tables,
                       int32_t* dev_tables_out, int table_ld, const int32_t* dev_parents, int n_groups, int n_beams, int len, int page_tokens, disco_stream s) {
  if (n_groups < 0 || n_groups > MOST_SEQS || n_beams < 1 || n_beams > DISCO_MAX_BEAMS || (int64_t)n_groups * n_beams > MOST_SEQS)
    return fail(DISCO_EINVAL, "%d groups of %d beams", n_groups, n_beams);
  if (table_ld < 1 || page_tokens < 4 || page_tokens % 4 || (int64_t)table_ld * page_tokens > MOST_POSITIONS) return fail(DISCO_EINVAL, "bad page tables");
  if (len < 0 || (int64_t)len > (int64_t)table_ld * page_tokens) return fail(DISCO_ECAP, "%d positions in tables of %d pages", len, table_ld);
  if (n_layers < 1 || n_layers > 65535 || n_pages < 1 || page_elems < 8 || page_elems % 8 || layer_stride < 0 || layer_stride % 8 ||
      (n_layers > 1 && layer_stride / page_elems < n_pages))
    return fail(DISCO_EINVAL, "bad page pool");
  if ((double)n_layers * n_beams * ((double)page_elems / 32768 + 1) >= MOST_WORKGROUPS) return fail(DISCO_EINVAL, "more copies than a launch takes");
  if (n_groups == 0) return DISCO_OK;
  if (!dev_pages || !dev_tables || !dev_tables_out || !dev_parents) return fail(DISCO_EINVAL, "null argument");
  if (!aligned(dev_pages, 16) || !aligned(dev_tables, 4) || !aligned(dev_tables_out, 4) || !aligned(dev_parents, 4)) return fail(DISCO_EINVAL, "misaligned pointer");
  const size_t tb = sizeof(int32_t) * (size_t)n_groups * n_beams * table_ld;
  if (overlap(dev_tables, tb, dev_tables_out, tb)) return fail(DISCO_EINVAL, "dev_tables_out overlaps dev_tables");
  BeamReorderArgs a{};
  a.pages = static_cast<bf16_t*>(dev_pages); a.n_layers = n_layers; a.layer_stride = layer_stride; a.n_pages = n_pages; a.page_elems = page_elems;
  a.tables = dev_tables; a.tables_out = dev_tables_out; a.table_ld = table_ld; a.parents = dev_parents; a.n_groups = n_groups; a.n_beams = n_beams;
  a.full = len / page_tokens; a.live = len % page_tokens;
  HIP_TRY(launch_beam_reorder(a, static_cast<hipStream_t>(s)), "reorder launch");
  return DISCO_OK;
}

// ---- a decoding step of a model for several sequences ------------------------------------------------

namespace {

// Workspace of a step: an ordinary one first (max_ctx 0), then the rows and parts of the operators above.
struct StepWs { Ws base; float* qkv; float* q; void* attn; size_t attn_bytes, total; };
StepWs carve_step(const disco_model* m, const disco_shared_kv& k, void* ws) {
  StepWs w;
  w.base = carve(m, DISCO_MAX_BLOCK, 0, ws);
  char* p = static_cast<char*>(ws);
  size_t off = w.base.total;
  auto take = [&](size_t bytes) { void* r = p ? p + off : nullptr; off += round_up(bytes, 256); return r; };
  w.qkv = static_cast<float*>(take(sizeof(float) * 16 * m->d_qkv));
  w.q = static_cast<float*>(take(sizeof(float) * 16 * m->d_q));
  w.attn_bytes = disco_attn_shared_bytes(&k, 1, m->d.n_heads, 0);
  w.attn = take(w.attn_bytes);
  w.total = off;
  return w;
}

// The caller's sequences behind the prompt that kv holds, for layer l.
int check_step(const disco_model* m, const disco_kv* kv, const disco_shared_kv* seqs, disco_shared_kv* out) {
  if (!m || !kv || !seqs) return fail(DISCO_EINVAL, "null argument");
  if (kv->model != m) return fail(DISCO_ESTATE, "KV cache belongs to another model");
  *out = *seqs;
  out->dev_prefix = kv->pages; out->dev_prefix_table = kv->dev_page_table; out->n_prefix_pages = kv->n_pages; out->prefix_len = kv->len;
  if (seqs->n_kv_heads != m->d.n_kv_heads || seqs->d_head != m->d.d_head || seqs->page_tokens != kv->page_tokens)
    return fail(DISCO_EINVAL, "the sequences' pages have another shape than the model's cache");
  const int rc = check_shape(out);
  if (rc) return rc;
  if (seqs->n_seqs < 1 || seqs->n_seqs > DISCO_MAX_BLOCK) return fail(DISCO_EINVAL, "%d sequences outside [1, %d]", seqs->n_seqs, DISCO_MAX_BLOCK);
  return DISCO_OK;
}

}  // namespace

size_t disco_step_workspace_bytes(const disco_model* m, const disco_kv* kv_prompt, const disco_shared_kv* seqs) {
  disco_shared_kv k;
  return check_step(m, kv_prompt, seqs, &k) ? 0 : carve_step(m, k, nullptr).total;
}

int disco_step(const disco_model* m, disco_kv* kv_prompt, const disco_shared_kv* seqs, int64_t layer_stride, int len, const int32_t* dev_tokens,
               float* dev_logits, void* dev_ws, size_t ws_bytes, disco_stream st) {
  disco_shared_kv k;
  int rc = check_step(m, kv_prompt, seqs, &k);
  if (rc) return rc;
  const disco_model_desc& d = m->d;
  const int n = k.n_seqs, cap = k.table_ld * k.page_tokens, pos = k.prefix_len + len - 1, n_tiles = d.d_model / 16;
  const bool fam_a = d.family == DISCO_FAMILY_A;
  hipStream_t s = static_cast<hipStream_t>(st);
  if (!dev_tokens || !dev_logits || !dev_ws || !k.dev_lens) return fail(DISCO_EINVAL, "null argument");
  if ((rc = check_cache(&k, true))) return rc;
  if (!aligned(dev_tokens, 4) || !aligned(dev_logits, 16) || !aligned(dev_ws, 256)) return fail(DISCO_EINVAL, "misaligned pointer");
  if (len < 1 || len > cap) return fail(DISCO_ECAP, "%d own positions, tables hold %d", len, cap);
  if (fam_a && pos >= d.max_pos) return fail(DISCO_ECAP, "position table of %d rows exceeded", d.max_pos);
  if (!fam_a && kv_prompt->capacity < k.prefix_len + cap)
    return fail(DISCO_ECAP, "the prompt's cache has a rotary table for %d positions, %d + %d needed", kv_prompt->capacity, k.prefix_len, cap);
  const int64_t page_elems = (int64_t)2 * k.n_kv_heads * k.page_tokens * k.d_head;
  if (layer_stride < 0 || layer_stride % 8 || (d.n_layers > 1 && layer_stride / page_elems < k.n_pages)) return fail(DISCO_EINVAL, "bad page pool");
  const StepWs ws = carve_step(m, k, dev_ws);
  if (ws_bytes < ws.total) return fail(DISCO_EINVAL, "workspace of %zu bytes, %zu needed", ws_bytes, ws.total);
  // An empty prompt's table may be unwritten.  Every step writes it then (the same values): another stream's step does not wait for this one's.
  if (kv_prompt->dev_rope && !kv_prompt->rope_ready)
    HIP_TRY(launch_rope_fill(kv_prompt->dev_rope, kv_prompt->capacity, d.d_head, d.rope_base, s), "rotary table launch");
  const Ws& b = ws.base;
  const int split_o = gemm_split_for(d.d_model, m->d_q / 32, n), split_dn = gemm_split_for(d.d_model, d.d_ff / 32, n);

  // every norm is applied inside the matrix that reads the row, as in the forwards of one sequence
  auto normed_input = [&](GemmArgs& g, const float* ln_vec, int n_rows) {
    g.M = n; g.X = b.xn; g.KT = d.d_model / 32; g.planes = b.gpart; g.counters = b.gemm_counters; g.n_rows = n_rows;
    g.ssq = b.ssq; g.n_ssq = n_tiles; g.d_in = d.d_model; g.eps = d.norm_eps;
    if (fam_a) { g.sum = b.sum; g.wg = ln_vec; g.wb = ln_vec + n_rows; }
  };
  auto residual_update = [&](const void* w, const bf16_t* x, int kdim, int split, const float* next_gain, const char* what) -> int {
    GemmArgs g{};
    g.M = n; g.W = static_cast<const bf16_t*>(w); g.X = x; g.KT = kdim / 32; g.n_rows = d.d_model; g.h = b.h; g.ld_out = d.d_model; g.only_row = -1;
    g.n_split = split; g.planes = b.gpart; g.counters = b.gemm_counters;
    g.Xout = b.xn; g.KT_out = d.d_model / 32; g.gain = next_gain; g.ssq_out = b.ssq; g.n_ssq_out = n_tiles;
    if (fam_a) g.sum_out = b.sum;
    HIP_TRY(launch_gemm(g, EPI_PARTIAL, s), what);
    return DISCO_OK;
  };

  BeamEmbedArgs e{};
  e.tokens = dev_tokens; e.rows = n; e.vocab = d.vocab; e.d = d.d_model; e.tok_emb = static_cast<const bf16_t*>(m->w.tok_emb); e.tok_stride = m->w.tok_emb_stride;
  e.pos_row = fam_a ? static_cast<const bf16_t*>(m->w.pos_emb) + (size_t)pos * d.d_model : nullptr;
  e.gain = m->layers[0].norm1_g; e.h = b.h; e.panels = b.xn; e.ssq = b.ssq; e.sum = fam_a ? b.sum : nullptr; e.n_slots = n_tiles;
  HIP_TRY(launch_beam_embed(e, s), "embedding launch");
  AppendArgs ap{};
  ap.qkv = ws.qkv; ap.ld = m->d_qkv; ap.rows = n; ap.nq = d.n_heads; ap.n_tok = 1; ap.rope = kv_prompt->dev_rope; ap.q = ws.q; ap.ld_q = m->d_q;
  SharedAttnArgs at{};
  at.plan = attn_plan(&k, true, 1, d.n_heads, 0);
  if (!launchable(&k, 1, d.n_heads, at.plan)) return fail(DISCO_EINVAL, "more workgroups than a launch takes");
  at.q = ws.q; at.ld_q = m->d_q; at.n_tok = 1; at.nq = d.n_heads; at.scale = 1.0f / sqrtf((float)d.d_head); at.panels = b.xattn;
  at.part = static_cast<float*>(ws.attn); at.ml = reinterpret_cast<float2*>(at.part + (size_t)at.plan.parts * n * m->d_q);
  for (int l = 0; l < d.n_layers; ++l) {
    const disco_layer_weights& L = m->layers[l];
    const float* next_g = l + 1 == d.n_layers ? m->w.normf_g : m->layers[l + 1].norm1_g;
    const float* ln_l = fam_a ? b.ln_vec + b.ln_layer_stride * l : nullptr;
    k.dev_prefix = kv_prompt->pages + (size_t)l * kv_prompt->layer_stride;
    k.dev_pages = static_cast<bf16_t*>(seqs->dev_pages) + (size_t)l * layer_stride;
    ap.kv = at.kv = device_view(k);
    GemmArgs g{};
    normed_input(g, ln_l, m->d_qkv);
    g.W = static_cast<const bf16_t*>(L.wqkv); g.out = ws.qkv; g.ld_out = m->d_qkv; g.only_row = -1;
    HIP_TRY(launch_gemm(g, EPI_STORE, s), "qkv launch");
    HIP_TRY(launch_append(ap, true, s), "append launch");
    HIP_TRY(launch_shared_attn(at, true, s), "attention launch");
    if ((rc = residual_update(L.wo, b.xattn, m->d_q, split_o, L.norm2_g, "o-proj launch"))) return rc;
    GemmArgs u{};
    normed_input(u, fam_a ? ln_l + 2 * (size_t)m->d_qkv : nullptr, fam_a ? d.d_ff : 2 * d.d_ff);
    u.W = static_cast<const bf16_t*>(L.w_in); u.grp = 1; u.Xout = b.xact; u.KT_out = d.d_ff / 32;
    HIP_TRY(launch_gemm(u, fam_a ? EPI_GELU : EPI_SWIGLU, s), "mlp-in launch");
    if ((rc = residual_update(L.w_out, b.xact, d.d_ff, split_dn, next_g, "mlp-out launch"))) return rc;
  }
  GemmArgs lm{};
  normed_input(lm, fam_a ? b.ln_vec + b.ln_layer_stride * d.n_layers : nullptr, d.vocab);
  lm.W = static_cast<const bf16_t*>(m->w.wlm); lm.out = dev_logits; lm.ld_out = d.vocab; lm.only_row = -1;
  HIP_TRY(launch_gemm(lm, EPI_STORE, s), "lm-head launch");
  return DISCO_OK;
}
