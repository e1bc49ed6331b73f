// Launcher interface between the boundary of the operators for several sequences behind one prompt (disco_shared_api.cpp) and
// their gfx950 kernels (disco_shared.hip).  Nothing here is exported.
#pragma once
#include "disco_internal.h"

namespace disco {

// One layer of the paged cache: the prompt's pages and every sequence's own.  Page: [K | V][kv head] blocks of pt x dh bf16, K blocks
// [token][channel], V blocks [channel][token].
struct SharedKv {
  const bf16_t* prefix; const int32_t* prefix_table; int n_prefix_pages, prefix_len;
  bf16_t* pages; const int32_t* tables; const int32_t* lens; int n_pages, table_ld, n_seqs;
  int pt, nkv, dh;
  int pt_shift;                      // log2 of pt, or -1
};

struct AppendArgs {
  SharedKv kv;
  const void* qkv; int64_t ld; int rows, nq;
  const int32_t* seq; const int32_t* pos;
  int n_tok;                         // seq == nullptr: row i is token i % n_tok of sequence i / n_tok
  const float* rope;
  const float* q_gain; const float* k_gain; float eps;
  void* q; int64_t ld_q;
};
hipError_t launch_append(const AppendArgs& a, bool fp32, hipStream_t s);

// Ranges and launches of an attention call.
constexpr int ATTN_MAX_PARTS = 256;
struct SharedAttnPlan {
  bool fused;                        // every workgroup walks the prompt before its sequence's own positions: one launch, one part
  int few_rows, few_waves;           // rows (16 or 32) and wavefronts of a workgroup that is not one of 128 rows
  bool prefix_many, own_many;        // workgroups of 128 rows
  int prefix_tiles, prefix_splits, prefix_len;    // row tiles of a kv head, ranges, positions of a range
  int own_tiles, own_splits, own_len;
  int parts;                         // partial results of a row
  size_t bytes;                      // of the partial results (0 with one part)
};
SharedAttnPlan shared_attn_plan(int n_seqs, int n_tok, int nq, int nkv, int dh, bool fp32, int prefix_len, int max_len);

struct SharedAttnArgs {
  SharedKv kv;
  const void* q; int64_t ld_q; int n_tok, nq; float scale;
  void* out; int64_t ld_out; float* lse;
  bf16_t* panels;                    // fp32, up to sixteen rows: the result goes here instead of `out`, as the next matrix' input
  float* part; float2* ml;           // [part][kv head][row][channel] and their (maximum in log2 units, sum)
  SharedAttnPlan plan;
};
hipError_t launch_shared_attn(const SharedAttnArgs& a, bool fp32, hipStream_t s);

constexpr int DISCO_BEAM_MAX_ROWS = 64;
int beam_unit_logits(int rows, int vocab);   // logits of a unit
struct BeamSelectArgs {
  const void* logits; int64_t ld; int n_groups, n_beams, vocab, k;
  const float* scores; const int32_t* done; int end_token;
  int32_t* tokens; int32_t* parents; float* scores_out; int32_t* done_out;
  float2* stats;                     // [row][unit]: maximum, sum of exponentials
  unsigned long long* cand;          // [row][unit][k]: (order key, ~index), descending, 0 behind the last
  int units;
};
hipError_t launch_beam_select(const BeamSelectArgs& a, bool fp32, hipStream_t s);

struct BeamReorderArgs {
  bf16_t* pages; int n_layers; int64_t layer_stride; int n_pages; int64_t page_elems;
  const int32_t* tables; int32_t* tables_out; int table_ld; const int32_t* parents;
  int n_groups, n_beams, full, live;
};
hipError_t launch_beam_reorder(const BeamReorderArgs& a, hipStream_t s);

struct BeamEmbedArgs {
  const int32_t* tokens; int rows, vocab, d;
  const bf16_t* tok_emb; int64_t tok_stride; const bf16_t* pos_row;   // pos_row: the position's row of the position table, or nullptr
  const float* gain; float* h; bf16_t* panels; float* ssq; float* sum; int n_slots;
};
hipError_t launch_beam_embed(const BeamEmbedArgs& a, hipStream_t s);

}  // namespace disco
