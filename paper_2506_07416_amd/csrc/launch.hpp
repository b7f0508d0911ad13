// Host-side launch entry points of the device kernels, called by api.hip after
// argument validation. Each returns the HIP error of its launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/litevlm.h"
#include "viewsel.hpp"

namespace litevlm {

struct ViewOffsets {
  int32_t off[LITEVLM_MAX_VIEWS + 1];
};

hipError_t launch_patch_select(int B, int N, int S, const ViewOffsets& vo, const float* logit,
                               const float* lexical, float w, float tau, uint8_t* view_keep,
                               uint8_t* token_keep, int32_t* n_visual_kept, hipStream_t stream);

// Workspace of the scoring step, carved from one caller buffer:
//   rowpart  float2 [B][Hkv][ns1][R]  per-key-split (max, sum) of each text row
//   acc      u64    [B][V_full]       fixed-point column sums of sweep 2
// with R = (Hq/Hkv)*n_query rows per KV group (the last n_query text tokens
// are the query rows); ns1 (key splits of sweep 1) is a function of the shape.
struct ScoreWorkspace {
  size_t rowpart_off, acc_off, total;
};
ScoreWorkspace score_workspace_layout(int B, int S, int V_full, int Hq, int Hkv, int n_query);

struct ScoreArgs {
  int dtype, B, S, V_full, Hq, Hkv, D;
  int query_rows;  // the last query_rows text tokens are the query rows (1..T)
  const void* q;
  const void* k;
  const void* v;
  float logit_scale_log2;  // softmax_scale*q_scale*k_scale*log2(e)
  const uint8_t* token_keep;
  double keep_ratio;
  float* scores;
  int32_t* kept_index;
  int32_t* cu_seqlens;
  void* qc;
  void* kc;
  void* vc;
  void* workspace;
  // in-call patch selection (vs.N > 0, token_keep NULL): the keep flags come
  // from the view scores, and the selection's outputs are written (each may be NULL)
  ViewSel vs{};
  uint8_t* view_keep = nullptr;
  uint8_t* token_keep_out = nullptr;
  int32_t* n_visual_kept = nullptr;
};
hipError_t launch_token_score_topk(const ScoreArgs& a, hipStream_t stream);

// Row gather behind the compaction: rows kept_index[r] of each sample of q, k,
// v (qvec / kvvec 16-byte pieces per row) into packed qc, kc, vc (each may be
// NULL, kvvec may be 0).
void launch_gather(int B, int S, const int32_t* kept_index, const int32_t* cu_seqlens, const void* q,
                   const void* k, const void* v, void* qc, void* kc, void* vc, int qvec, int kvvec,
                   hipStream_t stream);
hipError_t launch_gather_hidden(int B, int S, int row_bytes, const void* hidden, const int32_t* kept_index,
                                const int32_t* cu_seqlens, void* out, hipStream_t stream);

struct AttnArgs {
  int in_dtype, out_dtype, B, Hq, Hkv, D, max_seqlen, causal;
  const void* q;
  const void* k;
  const void* v;
  const int32_t* cu_seqlens;
  float logit_scale_log2;  // softmax_scale*q_scale*k_scale*log2(e)
  float out_scale;         // v_scale
  void* o;
};
// Whether the work items of the launch (row tiles of the bound x heads x samples)
// can be counted in an int.
bool prefill_attn_fits(int in_dtype, int B, int Hq, int max_seqlen);
hipError_t launch_prefill_attn(const AttnArgs& a, hipStream_t stream);

// Workspace of the decode step: per (sample, query head, key split) the
// unnormalised output float [D] and the split's (max, sum) float2. The split
// length and count follow from the shape and the host bound max_seqlen.
struct DecodeLayout {
  int split_len, nsplit;
  size_t part_o_off, part_ml_off, total;
};
DecodeLayout decode_layout(int in_dtype, int B, int Hq, int Hkv, int D, int max_seqlen);

struct DecodeArgs {
  int in_dtype, out_dtype, B, Hq, Hkv, D, max_seqlen;
  const void* q1;
  const void* k1;
  const void* v1;
  const void* kc;
  const void* vc;
  const int32_t* cu_seqlens;
  float logit_scale_log2;  // softmax_scale*q_scale*k_scale*log2(e)
  float out_scale;         // v_scale
  void* o;
  void* workspace;
};
hipError_t launch_decode_attn(const DecodeArgs& a, hipStream_t stream);

struct TsmArgs {
  int B, S, V_full, Dm, Hq, Hkv, D;
  const void* hidden;
  const uint8_t* token_keep;
  const void* w_q;
  const void* w_k;
  float eps, rope_theta;
  void* q;
  void* k;
};
hipError_t launch_tsm_qk(const TsmArgs& a, hipStream_t stream);

// Patch Selection Module: parameter count and workspace carving.
struct PsmLayout {
  size_t layer_params, params;
  size_t h_off, q_off, k_off, v_off, att_off, ff_off, cu_off, fold_off, total;
};
PsmLayout psm_layout(int B, int T, int d, int d_ff, int n_views, int n_layers);

struct PsmArgs {
  int B, T, d, n_heads, d_ff, n_views, n_layers;
  const float* emb;
  const float* params;
  float* view_logit;
  void* workspace;
};
hipError_t launch_psm_forward(const PsmArgs& a, hipStream_t stream);

// Rows of K and V into (k_in, v_in) or out of (k_out, v_out) the 4-bit cache.
struct Cache4RowsArgs {
  int dtype, B, Hkv, D, cap, max_rows;
  const void* k_in;
  const void* v_in;
  void* k_out;
  void* v_out;
  const int32_t* cu;
  const int32_t* start;
  void* cache;
  float* weight;
};
hipError_t launch_cache4_append(const Cache4RowsArgs& a, hipStream_t stream);
hipError_t launch_cache4_read(const Cache4RowsArgs& a, hipStream_t stream);

// Workspace of the attention over the 4-bit cache, and how the rows of a KV head
// (the queries of its heads) and the keys are dealt to workgroups:
//   part_o   float  [B][Hkv][rows][nsplit][D]  unnormalised outputs of the key splits
//   part_ml  float2 [B][Hkv][rows][nsplit]     their (reference, sum)
//   stat     float2 [B][Hkv][weight rows]      (reference, 1 / sum) of the rows that add weight
//   logit    float  [B][Hkv][weight rows][lpad] their logits, where they are kept
// Each part may be missing; a call that takes one launch has none (total 0).
struct Cache4AttnLayout {
  int tiles, blocks, nsplit, split_len, lpad;
  bool keep, whole;  // logits kept; and the weights added by the first kernel
  size_t part_o_off, part_ml_off, stat_off, logit_off, total;
};
Cache4AttnLayout cache4_attn_layout(int dtype, int B, int Hq, int Hkv, int D, int max_q, int max_len,
                                    int weight_rows);

struct Cache4AttnArgs {
  int dtype, B, Hq, Hkv, D, cap, max_q, max_len, weight_rows;
  const void* q;
  const int32_t* cu_q;
  const void* cache;
  const int32_t* lengths;
  float scale_log2;  // softmax_scale*log2(e)
  void* o;
  const float* weight_in;
  float* weight_out;
  void* workspace;
};
hipError_t launch_cache4_attn(const Cache4AttnArgs& a, hipStream_t stream);

struct Cache4EvictArgs {
  int B, Hkv, D, cap, cap_out, max_len, budget, recent;
  const void* cache;
  const float* weight;
  const int32_t* lengths;
  void* cache_out;
  float* weight_out;
  int32_t* lengths_out;
  int32_t* kept_index;
};
hipError_t launch_cache4_evict(const Cache4EvictArgs& a, hipStream_t stream);

// Workspace of the draft verification: per (sample, chunk of the vocabulary) two
// sums in 64 bits, and per sample the accepted drafts; nothing (total 0) where one
// workgroup takes a sample.
struct VerifyLayout {
  bool one;
  int chunks;
  size_t acc_off, total;
};
VerifyLayout verify_layout(int B, int V);

struct VerifyArgs {
  int dtype, B, max_draft, V;
  const int32_t* draft;
  const int32_t* n_draft;
  const void* target;
  const void* proposal;
  const float* u;
  const float* r;
  const int32_t* lengths;
  int32_t* tokens;
  int32_t* n_accepted;
  int32_t* lengths_out;
  void* workspace;
};
hipError_t launch_verify_draft(const VerifyArgs& a, hipStream_t stream);

hipError_t launch_tsm_fold_gain(const void* w, const float* gamma, void* w_out, int rows, int cols,
                                hipStream_t stream);

}  // namespace litevlm
