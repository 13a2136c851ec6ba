// Dropout, layer norm and linear layers on the caller's tensors behind the C ABI:
// argument checks, then launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>
#include <vector>

#include "common.h"
#include "linear_op.h"
#include "operators_common.h"
#include "rows_op.h"

namespace {

static_assert((int)RC_ACT_GELU == ACT_GELU && (int)RC_ACT_RELU == ACT_RELU && (int)RC_ACT_SILU == ACT_SILU, "activations");

constexpr int64_t MAX_ROWS = 0x7fffffff, MAX_COLS = 1 << 29, MAX_ELEMENTS = 1LL << 46;
// Widths of a linear layer: the products count rows and columns in 32 bits, up to a
// tile past the last one, and the bias gradient's bytes of a row (fp32) in 32 unsigned.
constexpr int32_t MAX_WIDTH = 1 << 30;

bool known(int dtype) { return dtype == RC_FP32 || dtype == RC_BF16; }

// The memory that a tensor of the call takes: rows of `width` bytes, `step` apart.
struct Span {
  const char* data;
  int64_t step, width, rows;
  bool output;
  const char* name;
};

// Whether two spans share a byte.  Spans of one step are compared by their places
// within it (columns of one matrix); of others, by their ends.
bool meet(const Span& a, const Span& b) {
  const uintptr_t pa = (uintptr_t)a.data, pb = (uintptr_t)b.data;
  const uintptr_t ea = pa + (a.rows - 1) * a.step + a.width, eb = pb + (b.rows - 1) * b.step + b.width;
  if (pa >= eb || pb >= ea) return false;
  if (a.step != b.step || a.step <= 0 || a.rows == 1 || b.rows == 1) return true;
  const int64_t d = (int64_t)(pb - pa), at = ((d % a.step) + a.step) % a.step;
  return at < a.width || at + b.width > a.step;
}

// Collects the tensors of a call as they are checked, then refuses overlaps.
struct Tensors {
  std::vector<Span> spans;

  rc_status overlap() const {
    for (size_t i = 0; i < spans.size(); ++i)
      for (size_t j = 0; j < spans.size(); ++j)
        if (i != j && spans[i].output && meet(spans[i], spans[j]))
          return fail(RC_ERR_INVALID_ARG, std::string(spans[i].name) + " overlaps " + spans[j].name);
    return RC_OK;
  }

  // A [rows, cols] matrix; unit: what data and stride are multiples of, in bytes.
  rc_status matrix(const rc_matrix* m, const char* name, int elt, int64_t rows, int64_t cols, bool needed, bool output,
                   int unit, RowsView& to) {
    to = {nullptr, 0};
    if (!m || !m->data) {
      if (needed && rows > 0) return fail(RC_ERR_INVALID_ARG, std::string("null ") + name);
      return RC_OK;
    }
    if (rows == 0) return RC_OK;
    const int64_t stride = rows > 1 ? m->row_stride : cols;
    if ((uintptr_t)m->data % unit || stride * elt % unit)
      return fail(RC_ERR_INVALID_ARG, std::string(name) + ": data and row_stride must be multiples of " +
                                          std::to_string(unit) + " bytes");
    if (stride < 0 || stride > MAX_ELEMENTS / rows) return fail(RC_ERR_INVALID_ARG, std::string(name) + ": row_stride out of range");
    if (output && rows > 1 && stride < cols)
      return fail(RC_ERR_INVALID_ARG, std::string(name) + ": rows of the output overlap");
    to = {m->data, (long)stride};
    spans.push_back({(const char*)m->data, stride * elt, cols * elt, rows, output, name});
    return RC_OK;
  }

  rc_status vector(const void* p, const char* name, int elt, int64_t n, bool output, int unit) {
    if (!p || n == 0) return RC_OK;
    if ((uintptr_t)p % unit)
      return fail(RC_ERR_INVALID_ARG, std::string(name) + (unit == elt ? ": not aligned to its elements" : ": not aligned to 16 bytes"));
    spans.push_back({(const char*)p, 0, n * elt, 1, output, name});
    return RC_OK;
  }

  rc_status work(void* p, size_t bytes) {
    if (!bytes) return RC_OK;
    if (!p || (uintptr_t)p % 256) return fail(RC_ERR_INVALID_ARG, "work must be given, 256-byte aligned");
    spans.push_back({(const char*)p, 0, (int64_t)bytes, 1, true, "work"});
    return RC_OK;
  }
};

rc_status rows_args(const rc_rows* r) {
  if (!r) return fail(RC_ERR_INVALID_ARG, "null sizes");
  if (!known(r->dtype)) return fail(RC_ERR_INVALID_ARG, "unknown dtype");
  if (!known(r->param_dtype)) return fail(RC_ERR_INVALID_ARG, "unknown param_dtype");
  if (r->rows < 0 || r->rows > MAX_ROWS || r->cols < 1 || r->cols > MAX_COLS)
    return fail(RC_ERR_INVALID_ARG, "rows must lie in 0 .. 2^31 - 1, cols in 1 .. 2^29");
  return RC_OK;
}

rc_status drop_args(const rc_dropout* d, DropArgs& to) {
  to = DropArgs{};
  if (!d) return RC_OK;
  if (!(d->p >= 0.f && d->p <= 1.f)) return fail(RC_ERR_INVALID_ARG, "p must lie in 0 .. 1");
  if (d->reserved) return fail(RC_ERR_INVALID_ARG, "reserved must be 0");
  if ((uintptr_t)d->step % 8) return fail(RC_ERR_INVALID_ARG, "step not aligned to its elements");
  to.threshold = (uint32_t)std::floor((double)d->p * 65536.0 + 0.5);
  to.on = to.threshold > 0;
  to.scale = to.threshold < 65536 ? (float)(65536.0 / (65536.0 - to.threshold)) : 0.f;
  to.seed = d->seed;
  to.offset = d->offset;
  to.step = d->step;
  return RC_OK;
}

rc_status flag(int x, const char* name) {
  return x == 0 || x == 1 ? RC_OK : fail(RC_ERR_INVALID_ARG, std::string(name) + " must be 0 or 1");
}

rc_status norm_args(const rc_rows* r, const rc_dropout* drop, NormArgs& a) {
  a = NormArgs{};
  TRY(rows_args(r));
  if (r->cols > NORM_MAX_COLS)
    return fail(RC_ERR_UNSUPPORTED, "more than " + std::to_string(NORM_MAX_COLS) + " columns");
  TRY(drop_args(drop, a.drop));
  a.rows = r->rows;
  a.cols = (int)r->cols;
  a.params_f32 = r->param_dtype == RC_FP32;
  return RC_OK;
}

rc_status linear_args(const rc_linear* l, LinearArgs& a) {
  a = LinearArgs{};
  if (!l) return fail(RC_ERR_INVALID_ARG, "null linear");
  if (!known(l->dtype)) return fail(RC_ERR_INVALID_ARG, "unknown dtype");
  if (!known(l->bias_dtype)) return fail(RC_ERR_INVALID_ARG, "unknown bias_dtype");
  if (l->rows < 0 || l->rows > MAX_ROWS || l->in < 1 || l->out < 1)
    return fail(RC_ERR_INVALID_ARG, "rows must lie in 0 .. 2^31 - 1, in and out be positive");
  if (l->activation < RC_ACT_NONE || l->activation > RC_ACT_SILU) return fail(RC_ERR_INVALID_ARG, "unknown activation");
  TRY(flag(l->by_out, "by_out"));
  if (l->in % 8 || l->out % 8) return fail(RC_ERR_UNSUPPORTED, "in and out must be multiples of 8");
  if (l->in > MAX_WIDTH || l->out > MAX_WIDTH) return fail(RC_ERR_UNSUPPORTED, "in or out above 2^30");
  a.elt = elt_of(l->dtype);
  if (a.elt == 2 && 2LL * l->in * l->out > 0x7fffffffLL)
    return fail(RC_ERR_UNSUPPORTED, "a weight of 2^31 bytes or more");
  if ((int64_t)l->in * l->out >= 1LL << 40) return fail(RC_ERR_UNSUPPORTED, "a weight of 2^40 elements or more");
  a.rows = l->rows;
  a.in = l->in;
  a.out = l->out;
  a.by_out = l->by_out;
  a.act = l->activation;
  a.bias_f32 = l->bias_dtype == RC_FP32;
  return RC_OK;
}

struct LinearTensors : Tensors {
  const rc_linear* l;
  int elt;
  LinearTensors(const rc_linear* l, int elt) : l(l), elt(elt) {}
  rc_status at(const rc_matrix* m, const char* name, int64_t cols, bool needed, bool output, RowsView& to) {
    TRY(matrix(m, name, elt, l->rows, cols, needed, output, 16, to));
    // (the kernels bound their reads by rows of at least a row's length)
    if (to.data && to.stride < cols) return fail(RC_ERR_INVALID_ARG, std::string(name) + ": rows overlap");
    if (elt == 2 && to.stride >= 1L << 21)
      return fail(RC_ERR_UNSUPPORTED, std::string(name) + ": a row_stride of 2^21 elements or more");
    return RC_OK;
  }
  rc_status weight(const rc_matrix* m, RowsView& to) {
    const int64_t rows = l->by_out ? l->out : l->in, cols = l->by_out ? l->in : l->out;
    TRY(matrix(m, "weight", elt, rows, cols, true, false, 16, to));
    if (to.stride < cols) return fail(RC_ERR_INVALID_ARG, "weight: rows overlap");
    if (elt == 2 && to.stride * rows * 2 > 0x7fffffffL)
      return fail(RC_ERR_UNSUPPORTED, "weight: spans 2^31 bytes or more");
    return RC_OK;
  }
};

#define ON_DEVICE(stream)                  \
  OnDevice on((hipStream_t)(stream));      \
  if (on.err != hipSuccess) return hip_result(on.err, "device of the stream")

}  // namespace

extern "C" {

rc_status rc_dropout_memory(const rc_rows* r, size_t* work_bytes) {
  return guarded([&]() -> rc_status {
    if (!work_bytes) return fail(RC_ERR_INVALID_ARG, "null output pointer");
    TRY(rows_args(r));
    *work_bytes = dropout_work_bytes(r->rows, (int)r->cols);
    return RC_OK;
  });
}

rc_status rc_dropout_forward(const rc_rows* r, const rc_dropout* drop, const rc_matrix* x, const void* bias,
                             const rc_matrix* residual, const rc_matrix* y, void* hip_stream) {
  return guarded([&]() -> rc_status {
    DropoutArgs a{};
    TRY(rows_args(r));
    if (!drop) return fail(RC_ERR_INVALID_ARG, "null dropout");
    TRY(drop_args(drop, a.drop));
    const int elt = elt_of(r->dtype), pelt = elt_of(r->param_dtype);
    Tensors t;
    TRY(t.matrix(x, "x", elt, r->rows, r->cols, true, false, elt, a.x));
    TRY(t.matrix(residual, "residual", elt, r->rows, r->cols, false, false, elt, a.more));
    TRY(t.matrix(y, "y", elt, r->rows, r->cols, true, true, elt, a.y));
    TRY(t.vector(bias, "bias", pelt, r->cols, false, pelt));
    TRY(t.overlap());
    a.rows = r->rows;
    a.cols = (int)r->cols;
    a.bias = bias;
    a.bias_f32 = r->param_dtype == RC_FP32;
    ON_DEVICE(hip_stream);
    return hip_result(dropout_rows(a, elt, (hipStream_t)hip_stream), "dropout");
  });
}

rc_status rc_dropout_backward(const rc_rows* r, const rc_dropout* drop, const rc_matrix* dy,
                              const rc_matrix* derivative, const rc_matrix* dx, float* dbias, int32_t accumulate,
                              void* work, void* hip_stream) {
  return guarded([&]() -> rc_status {
    DropoutArgs a{};
    TRY(rows_args(r));
    if (!drop) return fail(RC_ERR_INVALID_ARG, "null dropout");
    TRY(drop_args(drop, a.drop));
    TRY(flag(accumulate, "accumulate"));
    const int elt = elt_of(r->dtype);
    Tensors t;
    TRY(t.matrix(dy, "dy", elt, r->rows, r->cols, true, false, elt, a.x));
    TRY(t.matrix(derivative, "derivative", elt, r->rows, r->cols, false, false, elt, a.more));
    TRY(t.matrix(dx, "dx", elt, r->rows, r->cols, dbias == nullptr, true, elt, a.y));
    TRY(t.vector(dbias, "dbias", 4, r->cols, true, 4));
    if (dbias) TRY(t.work(work, dropout_work_bytes(r->rows, (int)r->cols)));
    TRY(t.overlap());
    a.rows = r->rows;
    a.cols = (int)r->cols;
    a.more_factor = 1;
    a.sums = dbias;
    a.accumulate = accumulate;
    a.work = (float*)work;
    ON_DEVICE(hip_stream);
    return hip_result(dropout_rows(a, elt, (hipStream_t)hip_stream), "dropout backward");
  });
}

rc_status rc_layer_norm_memory(const rc_rows* r, size_t* work_bytes) {
  return guarded([&]() -> rc_status {
    NormArgs a;
    if (!work_bytes) return fail(RC_ERR_INVALID_ARG, "null output pointer");
    TRY(norm_args(r, nullptr, a));
    *work_bytes = norm_work_bytes(a.rows, a.cols);
    return RC_OK;
  });
}

rc_status rc_layer_norm_forward(const rc_rows* r, float eps, const rc_dropout* drop, const rc_matrix* x,
                                const void* in_bias, const rc_matrix* residual, const void* weight, const void* bias,
                                const rc_matrix* total, const rc_matrix* y, float* stats, void* hip_stream) {
  return guarded([&]() -> rc_status {
    NormArgs a;
    TRY(norm_args(r, drop, a));
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(RC_ERR_INVALID_ARG, "eps must be finite and not negative");
    const int elt = elt_of(r->dtype), pelt = elt_of(r->param_dtype);
    const bool added = drop || in_bias || (residual && residual->data);
    if (!added && total && total->data)
      return fail(RC_ERR_INVALID_ARG, "total without a residual, a dropout or an in_bias is x");
    Tensors t;
    TRY(t.matrix(x, "x", elt, r->rows, r->cols, true, false, elt, a.x));
    TRY(t.matrix(residual, "residual", elt, r->rows, r->cols, false, false, elt, a.residual));
    TRY(t.matrix(total, "total", elt, r->rows, r->cols, added, true, elt, a.total));
    TRY(t.matrix(y, "y", elt, r->rows, r->cols, true, true, elt, a.y));
    TRY(t.vector(in_bias, "in_bias", pelt, r->cols, false, pelt));
    TRY(t.vector(weight, "weight", pelt, r->cols, false, pelt));
    TRY(t.vector(bias, "bias", pelt, r->cols, false, pelt));
    TRY(t.vector(stats, "stats", 4, 2 * r->rows, true, 4));
    TRY(t.overlap());
    a.eps = eps;
    a.bias = in_bias;
    a.weight = weight;
    a.shift = bias;
    a.stats = stats;
    ON_DEVICE(hip_stream);
    return hip_result(norm_forward(a, elt, (hipStream_t)hip_stream), "layer norm");
  });
}

rc_status rc_layer_norm_backward(const rc_rows* r, const rc_dropout* drop, const rc_matrix* dy,
                                 const rc_matrix* dtotal_in, const rc_matrix* total, const float* stats,
                                 const void* weight, const rc_matrix* dtotal, const rc_matrix* dx, float* dweight,
                                 float* dbias, float* din_bias, int32_t accumulate, void* work, void* hip_stream) {
  return guarded([&]() -> rc_status {
    NormArgs a;
    TRY(norm_args(r, drop, a));
    TRY(flag(accumulate, "accumulate"));
    const int elt = elt_of(r->dtype), pelt = elt_of(r->param_dtype);
    const bool sums = dweight || dbias || din_bias;
    Tensors t;
    TRY(t.matrix(dy, "dy", elt, r->rows, r->cols, true, false, elt, a.dy));
    TRY(t.matrix(dtotal_in, "dtotal_in", elt, r->rows, r->cols, false, false, elt, a.dtotal_in));
    TRY(t.matrix(total, "total", elt, r->rows, r->cols, true, false, elt, a.total));
    TRY(t.matrix(dtotal, "dtotal", elt, r->rows, r->cols, false, true, elt, a.dtotal));
    TRY(t.matrix(dx, "dx", elt, r->rows, r->cols, false, true, elt, a.dx));
    if (!sums && r->rows > 0 && !a.dtotal.data && !a.dx.data) return fail(RC_ERR_INVALID_ARG, "no gradient is asked for");
    if (r->rows > 0 && !stats) return fail(RC_ERR_INVALID_ARG, "null stats");
    TRY(t.vector(stats, "stats", 4, 2 * r->rows, false, 4));
    TRY(t.vector(weight, "weight", pelt, r->cols, false, pelt));
    TRY(t.vector(dweight, "dweight", 4, r->cols, true, 4));
    TRY(t.vector(dbias, "dbias", 4, r->cols, true, 4));
    TRY(t.vector(din_bias, "din_bias", 4, r->cols, true, 4));
    if (sums) TRY(t.work(work, norm_work_bytes(a.rows, a.cols)));
    TRY(t.overlap());
    a.weight = weight;
    a.stats = const_cast<float*>(stats);
    a.dweight = dweight;
    a.dshift = dbias;
    a.dbias = din_bias;
    a.accumulate = accumulate;
    a.work = (float*)work;
    ON_DEVICE(hip_stream);
    return hip_result(norm_backward(a, elt, (hipStream_t)hip_stream), "layer norm backward");
  });
}

rc_status rc_linear_memory(const rc_linear* l, size_t* forward_work, size_t* input_work, size_t* weight_work) {
  return guarded([&]() -> rc_status {
    LinearArgs a;
    TRY(linear_args(l, a));
    float one;
    a.dbias = &one;   // with a bias gradient
    if (forward_work) *forward_work = linear_forward_work(a);
    if (input_work) *input_work = linear_input_work(a);
    if (weight_work) *weight_work = linear_weight_work(a);
    return RC_OK;
  });
}

rc_status rc_linear_forward(const rc_linear* l, const rc_matrix* x, const rc_matrix* weight, const void* bias,
                            const rc_matrix* residual, const rc_matrix* y, const rc_matrix* derivative, void* work,
                            void* hip_stream) {
  return guarded([&]() -> rc_status {
    LinearArgs a;
    TRY(linear_args(l, a));
    if (a.act == ACT_NONE && derivative && derivative->data)
      return fail(RC_ERR_INVALID_ARG, "a derivative without an activation");
    LinearTensors t(l, a.elt);
    TRY(t.at(x, "x", l->in, true, false, a.x));
    TRY(t.weight(weight, a.w));
    TRY(t.at(residual, "residual", l->out, false, false, a.residual));
    TRY(t.at(y, "y", l->out, true, true, a.y));
    TRY(t.at(derivative, "derivative", l->out, false, true, a.slope));
    TRY(t.vector(bias, "bias", elt_of(l->bias_dtype), l->out, false, elt_of(l->bias_dtype)));
    TRY(t.work(work, linear_forward_work(a)));
    TRY(t.overlap());
    a.bias = bias;
    a.work = work;
    ON_DEVICE(hip_stream);
    return hip_result(linear_forward(a, (hipStream_t)hip_stream), "linear");
  });
}

rc_status rc_linear_backward_input(const rc_linear* l, const rc_matrix* dy, const rc_matrix* weight,
                                   const rc_matrix* before, const rc_matrix* dx, void* work, void* hip_stream) {
  return guarded([&]() -> rc_status {
    LinearArgs a;
    TRY(linear_args(l, a));
    LinearTensors t(l, a.elt);
    TRY(t.at(dy, "dy", l->out, true, false, a.dy));
    TRY(t.weight(weight, a.w));
    TRY(t.at(before, "before", l->in, false, false, a.before));
    TRY(t.at(dx, "dx", l->in, true, true, a.dx));
    TRY(t.work(work, linear_input_work(a)));
    TRY(t.overlap());
    a.work = work;
    ON_DEVICE(hip_stream);
    return hip_result(linear_backward_input(a, (hipStream_t)hip_stream), "linear backward, input");
  });
}

rc_status rc_linear_backward_weight(const rc_linear* l, const rc_matrix* x, const rc_matrix* dy, float* dweight,
                                    float* dbias, int32_t accumulate, void* work, void* hip_stream) {
  return guarded([&]() -> rc_status {
    LinearArgs a;
    TRY(linear_args(l, a));
    TRY(flag(accumulate, "accumulate"));
    if (!dweight) return fail(RC_ERR_INVALID_ARG, "null dweight");
    LinearTensors t(l, a.elt);
    TRY(t.at(x, "x", l->in, true, false, a.x));
    TRY(t.at(dy, "dy", l->out, true, false, a.dy));
    TRY(t.vector(dweight, "dweight", 4, (int64_t)l->in * l->out, true, 16));
    TRY(t.vector(dbias, "dbias", 4, l->out, true, 4));
    a.dw = dweight;
    a.dbias = dbias;
    a.accumulate = accumulate;
    a.work = work;
    TRY(t.work(work, linear_weight_work(a)));
    TRY(t.overlap());
    ON_DEVICE(hip_stream);
    return hip_result(linear_backward_weight(a, (hipStream_t)hip_stream), "linear backward, weight");
  });
}

}  // extern "C"
