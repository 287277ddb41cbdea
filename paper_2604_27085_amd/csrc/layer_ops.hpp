// Launchers of the layer operators beside the stage calls: rotary positions, cross attention, the router's balance loss.  Every function only
// enqueues on `st` and returns the launch status.
#pragma once
#include "common.hpp"

// Rotary positions in other layouts and scalings.  Turns of pair i a position: base^(-2i/rot) f / 2 pi with f = 1 / factor, or by parts
// keep + (1 - keep) / factor, keep = clamp((trained_len base^(-2i/rot) / 2 pi - slow) / (fast - slow), 0, 1); log2_base_step = 2 log2(base) / rot.
struct RopeScale { double log2_base_step, inv_factor, trained_len, slow, inv_span, amplitude; int by_parts; };
hipError_t k_rope_table_scaled(hipStream_t st, float2* cs, int n_pos, int rot, const RopeScale& r);
struct RotateArgs {
  const bf16 *in_q, *in_k;
  bf16 *out_q, *out_k;
  long ld_in_q, ld_in_k, ld_out_q, ld_out_k;
  const float2* cs;
  const int* pos;                  // [T] or NULL: t % seq
  int n_pos, T, seq, a, k, d, rot, bwd;
  int nunits, nrot, tokens_per_block, first;    // set by the launcher; first: the launch's first token
};
// layout 0: pairs (i, i + rot/2);  1: pairs (2i, 2i+1).
hipError_t k_rope(hipStream_t st, int layout, const RotateArgs& p);

// Balance loss of a router with its gradient (balance.hip).
struct BalanceArgs {
  const float* logits;             // [T, E]
  const int* idx;                  // [T, top_k]
  const unsigned char* mask;       // [T] or NULL
  const float* dlogits_in;         // [T, E] or NULL; may be dlogits
  float* dlogits;                  // [T, E] or NULL
  int *counts, *tokens;            // [groups, E], [groups + 1]
  float* loss;                     // [3]
  int seq, E, top_k;
  float coef, z_coef, grad_scale;
  int *hist, *tok;                 // from here on set by the launcher
  float2* part;
  int groups, slices, chunks, rows_per_block, total_given, first;    // first: the launch's first group
};
size_t k_moe_balance_scratch(int T, int seq, int E);
hipError_t k_moe_balance(hipStream_t st, BalanceArgs p, int T, void* scratch);

// Attention of seq_q queries a sequence to seq_kv keys of another (cross_attention.hip).
struct CrossArgs {
  const bf16 *q, *k, *v, *dout, *o_in;
  bf16 *o, *dq, *dk, *dv;
  float* lse;                      // forward, or NULL
  const float* lse_in;
  float* delta;                    // [batch, a, seq_q]: written by dQ, read by dK/dV
  long ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;
  const int *q_len, *kv_len;       // [batch] or NULL
  int batch, seq_q, seq_kv, a, kh;
  float scale, scale_log2e, inv_scale;
  float* part;                     // from here on set by the launcher
  float2* part_ml;
  int splits;
};
// Scratch with which the calls split as they like to; with less they split less.
void k_cross_attn_scratch(const CrossArgs& p, int d, size_t* fwd_bytes, size_t* bwd_bytes);
hipError_t k_cross_attn_fwd(hipStream_t st, const CrossArgs& p, int d, void* scratch, size_t bytes);
hipError_t k_cross_attn_bwd(hipStream_t st, const CrossArgs& p, int d, void* scratch, size_t bytes);
