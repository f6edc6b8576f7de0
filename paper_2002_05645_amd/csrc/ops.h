// Arguments and launchers of the single operations whose kernels are compiled in translation units of their own: attention
// over sequences of different lengths (seq_attention_variant.hip), dropout and token log probabilities (token_ops.hip).
// The entry points in l2l.hip check everything; a launcher only launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

struct SeqAttnArgs {
  const void *q, *k, *v, *o, *dout;   // o, dout: backward only
  void *out, *dq, *dk, *dv;           // out: forward only
  float* lse;                         // [heads][rows]; written forward, read backward
  float* nlse2;                       // backward, [heads][rows]: -lse / scale (16-bit formats) ...
  float* delta;                       // ... and rowsum(dO O) (16-bit formats: negated), left by the dQ kernel for the dK / dV kernel
  uint32_t* bounds;                   // backward in fp16 by two kernels, [heads][rows]: at the first of each 32 rows of a sequence their largest kept |dO| (low half, as bf16) and |D|
  long long ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;   // row strides in elements
  const int32_t *first, *len;         // device, per sequence, or null
  int heads, kv_heads, d, sequences, max_len, causal;
  long long rows;
  float scale;                        // > 0
  uint32_t drop;                      // of 256; 0 = no dropout
  uint64_t seed, site;
  const uint64_t* step;
  // Splits over the long axis: of a query block's keys (forward, dQ) and of a key block's queries and query
  // heads (dK / dV).  Above 1 the kernels leave fp32 partial results that a second kernel adds up.
  int splits_fwd, splits_dq, splits_dkv;
  int in_one;                         // backward: one kernel for all three gradients; splits_dkv then divides the query heads of a key head
  float* part;                        // [split][rows][heads d]; dK / dV: [split][2][rows][kv_heads d], dV first
  float *part_m, *part_sum;           // forward, [split][heads][rows]: the maximum (of the scores before their scale) and the sum that a part's rows are relative to
  int by_group;                       // 1: an XCD takes the query heads that share a key head one after the other
  int32_t* bad;                       // bit 1: a sequence did not fit rows or max_len
};

// X(padded head width)
#define L2L_SEQ_ATTN_WIDTHS(X) X(32) X(64) X(96) X(128)
#define L2L_SEQ_ATTN_DECLARE(dp)                                      \
  void l2l_seq_attn_fwd_v##dp(const SeqAttnArgs&, hipStream_t);       /* bf16 */ \
  void l2l_seq_attn_fwd_h##dp(const SeqAttnArgs&, hipStream_t);       /* fp16 */ \
  void l2l_seq_attn_fwd_f##dp(const SeqAttnArgs&, hipStream_t);       /* fp32 */ \
  void l2l_seq_attn_bwd_v##dp(const SeqAttnArgs&, hipStream_t);       \
  void l2l_seq_attn_bwd_h##dp(const SeqAttnArgs&, hipStream_t);       \
  void l2l_seq_attn_bwd_f##dp(const SeqAttnArgs&, hipStream_t);
L2L_SEQ_ATTN_WIDTHS(L2L_SEQ_ATTN_DECLARE)
#undef L2L_SEQ_ATTN_DECLARE

struct DropoutArgs {
  const void *x, *bias, *resid;   // bias, resid: or null
  void* y;
  long long ldx, ldr, ldy;
  int rows, n;
  uint32_t drop;                  // of 65536; 0 = keep everything
  uint64_t seed, site;
  const uint64_t* step;
  float* dbias;                   // backward: [n] or null
  float* part;                    // [dropout_row_blocks][n]
  int accumulate;
};
// row blocks of the column sums: the rows a workgroup walks
int dropout_row_blocks(int rows, int n);
void l2l_launch_dropout(const DropoutArgs&, int dtype, hipStream_t);

struct LogprobArgs {
  const void* logits;
  long long ld;
  const int32_t* ids;
  int rows, vocab, top;
  float *logp, *entropy, *lse;
  int32_t* top_ids;
  float* top_logp;
  void* work;
  int splits;                     // workgroups per row
  int32_t* bad;
  // backward
  const float *dlogp, *dentropy;
  void* dlogits;
  long long ldd;
};
int logprob_splits(int rows, int vocab);
size_t logprob_work_bytes(int rows, int splits, int top);
void l2l_launch_logprobs(const LogprobArgs&, int dtype, hipStream_t);
void l2l_launch_logprobs_bwd(const LogprobArgs&, int dtype, hipStream_t);
