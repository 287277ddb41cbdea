// Launchers of the operators for training on packed documents: the plan of a packed row, attention with a span of keys for every query, the gated
// linear recurrence, the embedding with its gradient, dropout.  Every function only enqueues on `st` and returns the launch status.
#pragma once
#include "common.hpp"

// What the documents of packed rows make of every token (packing.hip).
struct PackArgs {
  const int *starts, *prefix;      // [n_docs + 1], [n_docs] or NULL
  int2* span;                      // each of the three [T] or NULL
  int* pos;
  unsigned char* first;
  int n_docs, window, T, seq;
};
hipError_t k_pack_plan(hipStream_t st, const PackArgs& p);

// y = res + x stay / share (packing.hip); groups of eight elements, n8 a row.  stay: 16 bits of the generator below `keep`.
struct DropoutArgs {
  const bf16 *x, *res;             // res or NULL
  bf16* y;
  long ldx, ldr, ldy, groups;
  const unsigned long long* step;  // or NULL
  unsigned long long seed, offset;
  uint32_t n8, keep;
  float scale;
};
hipError_t k_dropout(hipStream_t st, const DropoutArgs& p);

// Embedding (embedding.hip).
hipError_t k_embed_fwd(hipStream_t st, const bf16* table, long ldt, const int* ids, float scale, bf16* x, long ldx, int T, int V, int h);
struct EmbedGrad {
  const bf16* dx;
  const int* ids;
  float* dtable;
  long lddx, ldt;
  float scale;
  int accumulate, T, V, h;
};
size_t k_embed_scratch(int T, int V, int h);
hipError_t k_embed_bwd(hipStream_t st, const EmbedGrad& p, void* scratch);

// Gated linear recurrence (scan.hip).
struct ScanArgs {
  const bf16 *x, *g, *dy;
  bf16 *y, *dx, *dg;
  long ldx, ldg, ldy, lddy, lddx, lddg;
  const unsigned char* first;      // [batch * seq] or NULL
  const int* len;                  // [batch] or NULL
  const float *h0, *dlast;         // [batch, c] or NULL
  float *last, *dh0;               // [batch, c] or NULL
  float* states;                   // [batch, chunks, c]: the state that every chunk starts from; written by the forward call, or NULL
  int batch, seq, c;
  int chunks, blocks;              // from here on set by the launcher; blocks: of channels
  unsigned* counter;
  unsigned long long* words;       // [batch, chunks, c]
};
void k_scan_sizes(int batch, int seq, int c, size_t* states, size_t* scratch);
hipError_t k_scan_fwd(hipStream_t st, int weight, const ScanArgs& p, void* scratch);
hipError_t k_scan_bwd(hipStream_t st, int weight, const ScanArgs& p, void* scratch);

// Attention in which every query sees a span of the keys (span_attention.hip).
struct SpanArgs {
  const bf16 *q, *k, *v, *dout, *o_in, *rest_in;
  bf16 *o, *rest, *dq, *dk, *dv;   // rest, rest_in or NULL: what o's rounding left over, laid out as o
  float* lse;                      // forward, or NULL
  const float* lse_in;
  float* delta;                    // [batch, a, seq_q]: written by dQ, read by dK/dV
  long ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;
  const int2* span;                // [batch, seq_q] first key, key behind the last
  const int* q_pos;                // [batch, seq_q] or NULL: t + seq_kv - seq_q
  const float* slopes;             // [a] or NULL
  int batch, seq_q, seq_kv, a, kh;
  float scale, cap;                // cap 0: none
  int4* tiles;                     // from here on set by the launcher
  float* part;
  float4* part_ml;
  int splits;
  int2* ranges;                    // [batch * key tiles] row tiles that see any of its keys
  int* sums;                       // [batch * key tiles + 1]
  int4* pieces;                    // [parts]
  int parts;                       // pieces of a key head's (key tile, row tile) pairs, or 0
};
void k_span_attn_scratch(const SpanArgs& p, int d, size_t* fwd_bytes, size_t* bwd_bytes);
size_t k_span_attn_least(const SpanArgs& p);      // what the backward call cannot do without
hipError_t k_span_attn_fwd(hipStream_t st, const SpanArgs& p, int d, void* scratch, size_t bytes);
hipError_t k_span_attn_bwd(hipStream_t st, const SpanArgs& p, int d, void* scratch, size_t bytes);
