// Attention with a sliding window, sinks and a relative position bias: the
// arguments of its kernels and their launchers.  See attn_op_kernels.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "recycle_stage.h"

// A launch holds fewer than 2^32 threads: workgroups of 256.
constexpr long ATTN_OP_MAX_GROUPS = (1L << 24) - 1;

// Distances in tokens at which the last bucket of a side has to begin at the latest.
constexpr int ATTN_OP_MAX_FAR = 1024;
constexpr int ATTN_OP_MAX_BUCKETS = 128;

// [batch, token, head, head_dim] in elements; the head_dim elements are contiguous.
struct AttnOpView {
  void* p;
  long b, t, h;
};

struct AttnOpArgs {
  AttnOpView q, k, v, o, dout, dq, dk, dv;
  const int* lengths;  // tokens of each sequence, or null: all s
  int batch, s, spad, heads, kv_heads, group, d;
  // token j is in the window of token i iff -left <= j - i <= right
  int causal, left, right, sinks;
  int seen;  // no row sees more tokens
  float scale, sl2;  // of the products, and with log2(e)
  // relative position bias [heads, buckets]; distances of `far` or more share
  // the last bucket of their side
  const void* bias;
  int bias_f32, buckets, far;
  // row statistics [batch, heads, spad]: reference score (q.k, or with a bias in base 2)
  // and log2 of the sum of exponentials relative to it, and (bf16) what the rounding of
  // o drops
  float *m, *l;
  void* rest;
  float* drow;   // [batch, heads, spad] rowsum(dO o O)
  float* bpart;  // [batch, heads, bias_blocks, buckets] shares of the bias gradient, by query block
  int bias_blocks;
  void* dbias;
  // fp32, and grids of few blocks of 128 rows, take 32 rows a workgroup instead, whose four
  // waves share the other side's blocks.
  int split_f, split_q, split_k;  // forward, dq, dk and dv
  // Every query sees the sinks.  Their keys (sink_rows: up to a multiple of 32)
  // are handled twice: with the other keys for the queries whose window holds
  // them, and by workgroups of 32 keys and chunk_len queries for the others; the
  // shares of dK and dV are added up afterwards.  (chunks 0: one chunk would do and
  // blocks are of 32 keys; the sinks' own block visits every query.)
  float* spart;
  int sink_rows, chunks, chunk_len;
  // The heads of a key head in `parts` workgroups of the dk and dv kernel where
  // that has few: their shares [batch, kv_heads, parts, 2, part_rows, columns].
  float* gpart;
  int parts, part_rows;
  unsigned short first[ATTN_OP_MAX_BUCKETS];  // first distance of each bucket of a side
  unsigned char bucket[ATTN_OP_MAX_FAR];      // of distances below `far`, one side
};

#define ATTN_OP_DECL(NAME)                                        \
  hipError_t attn_op_fwd_##NAME(const AttnOpArgs& a, hipStream_t st); \
  hipError_t attn_op_bwd_##NAME(const AttnOpArgs& a, hipStream_t st);
ATTN_OP_DECL(bf16_32)
ATTN_OP_DECL(bf16_64)
ATTN_OP_DECL(bf16_96)
ATTN_OP_DECL(bf16_128)
ATTN_OP_DECL(f32_32)
ATTN_OP_DECL(f32_64)
ATTN_OP_DECL(f32_96)
ATTN_OP_DECL(f32_128)
#undef ATTN_OP_DECL

// Checks a configuration and sets the arguments that follow from it (operators.cpp).
rc_status attn_op_check(const rc_attention& c, AttnOpArgs& a);

// dbias (+)= the sum of n gradients of count floats, in order.
constexpr int ATTN_OP_MAX_SHARES = 32;
struct AttnOpShares {
  const float* p[ATTN_OP_MAX_SHARES];
};
hipError_t attn_op_add_dbias(const AttnOpShares& shares, int n, long count, float* out, int accumulate, hipStream_t st);

// What one attention needs, in bytes, and its launches.  The arguments' scratch
// pointers are set from `saved` (null: nothing is kept for a backward pass) and
// `work`.
size_t attn_op_saved_bytes(const AttnOpArgs& a, int elt);
size_t attn_op_work_bytes(const AttnOpArgs& a);
void attn_op_plan(AttnOpArgs& a, int elt, int window, int max_distance);
hipError_t attn_op_forward(AttnOpArgs a, int elt, void* saved, hipStream_t st);
hipError_t attn_op_backward(AttnOpArgs a, int elt, const void* saved, void* work, hipStream_t st);
