// Operators on the caller's tensors behind the C ABI: argument checks, then launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <utility>
#include <vector>

#include "adamw_op.h"
#include "attn_op.h"
#include "operators_common.h"

rc_status attn_op_check(const rc_attention& c, AttnOpArgs& a) {
  if (c.dtype != RC_FP32 && c.dtype != RC_BF16) return rc_set_error(RC_ERR_INVALID_ARG, "unknown dtype");
  if (c.batch < 1 || c.seq_len < 1 || c.heads < 1 || c.kv_heads < 1 || c.head_dim < 1)
    return rc_set_error(RC_ERR_INVALID_ARG, "attention sizes must be positive");
  if (c.heads % c.kv_heads) return rc_set_error(RC_ERR_INVALID_ARG, "heads must be a multiple of kv_heads");
  if (c.causal != 0 && c.causal != 1) return rc_set_error(RC_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (c.window < 0 || c.sinks < 0) return rc_set_error(RC_ERR_INVALID_ARG, "window and sinks must not be negative");
  if (!(c.scale > 0.f) || !std::isfinite(c.scale * 1.4426950408889634f))
    return rc_set_error(RC_ERR_INVALID_ARG, "scale must be finite and above zero");
  if (c.buckets) {
    const int side = c.causal ? c.buckets : c.buckets / 2;
    if (c.buckets < 0 || side < 2 || (!c.causal && c.buckets % 2))
      return rc_set_error(RC_ERR_INVALID_ARG, "buckets: at least 2 (causal), or an even number of at least 4");
    if (c.max_distance <= side / 2)
      return rc_set_error(RC_ERR_INVALID_ARG, "max_distance must exceed the distances with a bucket each (" +
                                          std::to_string(side / 2) + ")");
    if (c.bias_dtype != RC_FP32 && c.bias_dtype != RC_BF16)
      return rc_set_error(RC_ERR_INVALID_ARG, "unknown bias_dtype");
    if (c.buckets > ATTN_OP_MAX_BUCKETS || c.max_distance > ATTN_OP_MAX_FAR)
      return rc_set_error(RC_ERR_UNSUPPORTED, "at most " + std::to_string(ATTN_OP_MAX_BUCKETS) +
                                          " buckets and a max_distance of " + std::to_string(ATTN_OP_MAX_FAR));
  }
  if (c.head_dim % 8 || c.head_dim > 128)
    return rc_set_error(RC_ERR_UNSUPPORTED, "head_dim must be a multiple of 8, at most 128");
  if (c.seq_len > (1 << 24)) return rc_set_error(RC_ERR_UNSUPPORTED, "seq_len exceeds 2^24");
  a = {};
  a.batch = c.batch;
  a.s = c.seq_len;
  a.heads = c.heads;
  a.kv_heads = c.kv_heads;
  a.d = c.head_dim;
  a.causal = c.causal;
  a.sinks = c.sinks;
  a.scale = c.scale;
  a.buckets = c.buckets;
  a.bias_f32 = c.bias_dtype == RC_FP32;
  attn_op_plan(a, c.dtype == RC_FP32 ? 4 : 2, c.window, c.max_distance);
  // workgroups a batch and head: of the kernels over queries, over keys, and over the sinks' rows
  // (bf16 grids take 32 tokens a workgroup only where that is few workgroups)
  const int rows = c.dtype == RC_FP32 ? 32 : 128;
  const long units =
      std::max((a.s + rows - 1) / rows + (long)a.sink_rows / 32 * a.chunks, (std::min(a.sinks, a.s) + 7L) / 8);
  if (units * a.batch > (ATTN_OP_MAX_GROUPS - a.heads) / a.heads)
    return rc_set_error(RC_ERR_UNSUPPORTED, "more than 2^24 - 1 blocks of " + std::to_string(rows) + " tokens of a head");
  return RC_OK;
}

namespace {

rc_status attention_args(const rc_attention* c, AttnOpArgs& a) {
  if (!c) return fail(RC_ERR_INVALID_ARG, "null attention");
  return attn_op_check(*c, a);
}

// A view of n heads; an output's elements must each have a place of their own.
rc_status view_args(const rc_view* v, const char* name, const rc_attention* c, int heads, bool output, AttnOpView& to) {
  if (!v || !v->data) return fail(RC_ERR_INVALID_ARG, std::string("null ") + name);
  const int elt = elt_of(c->dtype), unit = 16 / elt;
  if ((uintptr_t)v->data % 16 || v->batch_stride % unit || v->token_stride % unit || v->head_stride % unit)
    return fail(RC_ERR_INVALID_ARG, std::string(name) + ": data and strides must be multiples of 16 bytes");
  if (v->batch_stride < 0 || v->token_stride < 0 || v->head_stride < 0)
    return fail(RC_ERR_INVALID_ARG, std::string(name) + ": negative stride");
  if (elt == 2 && v->token_stride > (0x7fffffffL / 2 - c->head_dim) / std::max(1, c->seq_len - 1))
    return fail(RC_ERR_UNSUPPORTED, std::string(name) + ": a head's tokens span 2^31 bytes or more");
  if (elt == 4 && c->seq_len > 1 && v->token_stride >= 1L << 24)
    return fail(RC_ERR_UNSUPPORTED, std::string(name) + ": a token_stride of 2^24 elements or more");
  if (output) {
    std::pair<int64_t, int64_t> dims[3] = {
        {v->batch_stride, c->batch}, {v->token_stride, c->seq_len}, {v->head_stride, heads}};
    std::sort(dims, dims + 3);
    int64_t span = c->head_dim;
    for (const auto& d : dims) {
      if (d.second == 1) continue;
      if (d.first < span) return fail(RC_ERR_INVALID_ARG, std::string(name) + ": elements of the output overlap");
      span += d.first * (d.second - 1);
    }
  }
  to = {v->data, (long)v->batch_stride, (long)v->token_stride, (long)v->head_stride};
  return RC_OK;
}

rc_status bias_args(const rc_attention* c, const void* bias, const int32_t* lengths, AttnOpArgs& a) {
  if ((c->buckets != 0) != (bias != nullptr))
    return fail(RC_ERR_INVALID_ARG, c->buckets ? "null bias with buckets" : "a bias without buckets");
  if ((uintptr_t)bias % elt_of(c->bias_dtype) || (uintptr_t)lengths % 4)
    return fail(RC_ERR_INVALID_ARG, "bias or lengths not aligned to their elements");
  a.bias = bias;
  a.lengths = lengths;
  return RC_OK;
}

rc_status moment_args(const rc_adamw_tensor& t, int state_bits, const std::string& name) {
  if (!t.exp_avg || !t.exp_avg_sq) return fail(RC_ERR_INVALID_ARG, name + "null array");
  const bool scales = t.exp_avg_scale && t.exp_avg_sq_scale, none = !t.exp_avg_scale && !t.exp_avg_sq_scale;
  if (state_bits == 8 ? !scales : !none)
    return fail(RC_ERR_INVALID_ARG, name + "8-bit moments have scales, 32-bit ones have none");
  if (state_bits == 32 && ((uintptr_t)t.exp_avg | (uintptr_t)t.exp_avg_sq) % 4)
    return fail(RC_ERR_INVALID_ARG, name + "an array is not aligned to its elements");
  return RC_OK;
}

// Whether the destinations of the moments overlap each other or the moments.
bool read_overlaps(const rc_adamw_tensor* t, int n, int state_bits, float* const* m, float* const* v) {
  using Span = std::pair<uintptr_t, uintptr_t>;
  std::vector<Span> out;
  out.reserve(2 * (size_t)n);
  for (int i = 0; i < n; ++i)
    for (const float* p : {m[i], v[i]})
      if (t[i].count) out.emplace_back((uintptr_t)p, (uintptr_t)(p + t[i].count));
  std::sort(out.begin(), out.end());
  for (size_t i = 1; i < out.size(); ++i)
    if (out[i].first < out[i - 1].second) return true;
  auto meets = [&](const void* p, int64_t bytes) {
    const uintptr_t at = (uintptr_t)p;
    const auto next = std::upper_bound(out.begin(), out.end(), Span(at, UINTPTR_MAX));
    return (next != out.end() && next->first < at + bytes) || (next != out.begin() && next[-1].second > at);
  };
  for (int i = 0; i < n; ++i) {
    if (!t[i].count) continue;
    const int64_t bytes = t[i].count * (state_bits / 8), blocks = (t[i].count + ADAMW_BLOCK - 1) / ADAMW_BLOCK;
    if (meets(t[i].exp_avg, bytes) || meets(t[i].exp_avg_sq, bytes)) return true;
    if (state_bits == 8 && (meets(t[i].exp_avg_scale, blocks) || meets(t[i].exp_avg_sq_scale, blocks))) return true;
  }
  return false;
}

}  // namespace

extern "C" {

rc_status rc_attention_memory(const rc_attention* c, size_t* saved_bytes, size_t* work_bytes) {
  return guarded([&]() -> rc_status {
    if (!saved_bytes || !work_bytes) return fail(RC_ERR_INVALID_ARG, "null output pointer");
    AttnOpArgs a;
    TRY(attention_args(c, a));
    *saved_bytes = attn_op_saved_bytes(a, elt_of(c->dtype));
    *work_bytes = attn_op_work_bytes(a);
    return RC_OK;
  });
}

rc_status rc_attention_forward(const rc_attention* c, const rc_view* q, const rc_view* k, const rc_view* v,
                               const void* bias, const int32_t* lengths, const rc_view* o, void* saved,
                               void* hip_stream) {
  return guarded([&]() -> rc_status {
    AttnOpArgs a;
    TRY(attention_args(c, a));
    TRY(view_args(q, "q", c, c->heads, false, a.q));
    TRY(view_args(k, "k", c, c->kv_heads, false, a.k));
    TRY(view_args(v, "v", c, c->kv_heads, false, a.v));
    TRY(view_args(o, "o", c, c->heads, true, a.o));
    TRY(bias_args(c, bias, lengths, a));
    if (o->data == q->data || o->data == k->data || o->data == v->data)
      return fail(RC_ERR_INVALID_ARG, "o must not be one of the inputs");
    if ((uintptr_t)saved % 256) return fail(RC_ERR_INVALID_ARG, "saved must be 256-byte aligned");
    OnDevice on((hipStream_t)hip_stream);
    if (on.err != hipSuccess) return hip_result(on.err, "device of the stream");
    return hip_result(attn_op_forward(a, elt_of(c->dtype), saved, (hipStream_t)hip_stream), "attention forward");
  });
}

rc_status rc_attention_backward(const rc_attention* c, const rc_view* q, const rc_view* k, const rc_view* v,
                                const void* bias, const int32_t* lengths, const rc_view* o, const void* saved,
                                const rc_view* dout, const rc_view* dq, const rc_view* dk, const rc_view* dv,
                                void* dbias, void* work, void* hip_stream) {
  return guarded([&]() -> rc_status {
    AttnOpArgs a;
    TRY(attention_args(c, a));
    TRY(view_args(q, "q", c, c->heads, false, a.q));
    TRY(view_args(k, "k", c, c->kv_heads, false, a.k));
    TRY(view_args(v, "v", c, c->kv_heads, false, a.v));
    TRY(view_args(o, "o", c, c->heads, false, a.o));
    TRY(view_args(dout, "dout", c, c->heads, false, a.dout));
    TRY(view_args(dq, "dq", c, c->heads, true, a.dq));
    TRY(view_args(dk, "dk", c, c->kv_heads, true, a.dk));
    TRY(view_args(dv, "dv", c, c->kv_heads, true, a.dv));
    TRY(bias_args(c, bias, lengths, a));
    if (c->buckets && !dbias) return fail(RC_ERR_INVALID_ARG, "null dbias with buckets");
    if ((uintptr_t)dbias % elt_of(c->bias_dtype)) return fail(RC_ERR_INVALID_ARG, "dbias not aligned to its elements");
    const void* in[5] = {q->data, k->data, v->data, o->data, dout->data};
    const void* outs[3] = {dq->data, dk->data, dv->data};
    for (int i = 0; i < 3; ++i) {
      for (const void* x : in)
        if (outs[i] == x) return fail(RC_ERR_INVALID_ARG, "a gradient must not be one of the inputs");
      if (outs[i] == outs[(i + 1) % 3]) return fail(RC_ERR_INVALID_ARG, "two gradients share their memory");
    }
    if (!saved || !work || ((uintptr_t)saved | (uintptr_t)work) % 256)
      return fail(RC_ERR_INVALID_ARG, "saved and work must be given, 256-byte aligned");
    a.dbias = dbias;
    OnDevice on((hipStream_t)hip_stream);
    if (on.err != hipSuccess) return hip_result(on.err, "device of the stream");
    return hip_result(attn_op_backward(a, elt_of(c->dtype), saved, work, (hipStream_t)hip_stream),
                      "attention backward");
  });
}

rc_status rc_adamw_step(const rc_adamw_tensor* tensors, int32_t n, const rc_adam_config* adam, int32_t state_bits,
                        int64_t step, float grad_scale, void* hip_stream) {
  return guarded([&]() -> rc_status {
    if (n < 0 || (n > 0 && !tensors) || !adam) return fail(RC_ERR_INVALID_ARG, "null argument or negative count");
    if (state_bits != 32 && state_bits != 8) return fail(RC_ERR_INVALID_ARG, "state_bits must be 32 or 8");
    if (step < 1) return fail(RC_ERR_INVALID_ARG, "step numbers start at 1");
    if (!(adam->beta1 >= 0.f && adam->beta1 < 1.f && adam->beta2 >= 0.f && adam->beta2 < 1.f))
      return fail(RC_ERR_INVALID_ARG, "beta1 and beta2 must lie in [0, 1)");
    for (int i = 0; i < n; ++i) {
      const rc_adamw_tensor& t = tensors[i];
      const std::string name = "tensor " + std::to_string(i) + ": ";
      if (t.count < 0 || t.count > ADAMW_MAX_COUNT) return fail(RC_ERR_INVALID_ARG, name + "count out of range");
      if (t.grad_dtype != RC_FP32 && t.grad_dtype != RC_BF16)
        return fail(RC_ERR_INVALID_ARG, name + "unknown grad_dtype");
      if (t.count == 0) continue;
      if (!t.param || !t.grad) return fail(RC_ERR_INVALID_ARG, name + "null array");
      TRY(moment_args(t, state_bits, name));
      if ((uintptr_t)t.param % 4 || (uintptr_t)t.grad % elt_of(t.grad_dtype) || (uintptr_t)t.copy % 2)
        return fail(RC_ERR_INVALID_ARG, name + "an array is not aligned to its elements");
    }
    OnDevice on((hipStream_t)hip_stream);
    if (on.err != hipSuccess) return hip_result(on.err, "device of the stream");
    return hip_result(adamw_tensors(tensors, n, state_bits, adamw_hyper(*adam, step, grad_scale), (hipStream_t)hip_stream),
                      "AdamW step");
  });
}

rc_status rc_adamw_read(const rc_adamw_tensor* tensors, int32_t n, int32_t state_bits, float* const* exp_avg,
                        float* const* exp_avg_sq, void* hip_stream) {
  return guarded([&]() -> rc_status {
    if (n < 0 || (n > 0 && (!tensors || !exp_avg || !exp_avg_sq)))
      return fail(RC_ERR_INVALID_ARG, "null argument or negative count");
    if (state_bits != 32 && state_bits != 8) return fail(RC_ERR_INVALID_ARG, "state_bits must be 32 or 8");
    for (int i = 0; i < n; ++i) {
      const rc_adamw_tensor& t = tensors[i];
      const std::string name = "tensor " + std::to_string(i) + ": ";
      if (t.count < 0 || t.count > ADAMW_MAX_COUNT) return fail(RC_ERR_INVALID_ARG, name + "count out of range");
      if (t.count == 0) continue;
      TRY(moment_args(t, state_bits, name));
      if (!exp_avg[i] || !exp_avg_sq[i] || ((uintptr_t)exp_avg[i] | (uintptr_t)exp_avg_sq[i]) % 4)
        return fail(RC_ERR_INVALID_ARG, name + "null or misaligned destination");
    }
    if (read_overlaps(tensors, n, state_bits, exp_avg, exp_avg_sq))
      return fail(RC_ERR_INVALID_ARG, "destinations overlap each other or the moments");
    OnDevice on((hipStream_t)hip_stream);
    if (on.err != hipSuccess) return hip_result(on.err, "device of the stream");
    return hip_result(adamw_read(tensors, n, state_bits, exp_avg, exp_avg_sq, (hipStream_t)hip_stream), "AdamW read");
  });
}

}  // extern "C"
