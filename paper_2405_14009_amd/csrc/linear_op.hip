// Launches of the linear operator (kernels: gemm_*.h).  The bf16 kernels reach
// 2^31 - 1 bytes of an operand from its base, so calls of more rows run in parts.
#include "linear_op.h"

#include <algorithm>

#include "gemm.h"
#include "gemm_plan.h"
#include "linear_few.h"

namespace {

constexpr long MAX_PART = 1L << 20;   // rows of a launch

// Rows of a part: whole blocks of 256, as the launch's largest tiles are.
long part_rows(int elt, long stride_a, long stride_b) {
  if (elt == 4) return MAX_PART;
  const long most = 0x7fffffffL / (2 * std::max(1L, std::max(stride_a, stride_b)));
  return std::min(MAX_PART, std::max(256L, most / 256 * 256));
}

template <class F>
hipError_t parts(long rows, long each, F f) {
  for (long r = 0; r < rows || r == 0; r += each) {
    const hipError_t e = f(r, std::min(each, rows - r));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

const void* at(const RowsView& v, long row, int elt) {
  return v.data ? (const char*)v.data + row * v.stride * elt : nullptr;
}
void* at(RowsView& v, long row, int elt) { return v.data ? (char*)v.data + row * v.stride * elt : nullptr; }

hipError_t gemm(int elt, const GemmParams& p, hipStream_t s) { return elt == 2 ? gemm_bf16(p, s) : gemm_f32(p, s); }

GemmWork work_of(int elt, long m, long n, long k, bool tn) {
  return elt == 2 ? gemm_bf16_work(m, n, 1, k, tn) : gemm_f32_work(m, n, 1, k, true);
}

// Whether a product of n columns over k is the reading of its weight (plan_stream).
// kcontig: weights whose reduced dimension is the contiguous one.  Below 32 MB, with
// those 64 MB, one unsplit launch is as fast.
bool streams(int elt, long rows, long n, long k, bool kcontig) {
  return elt == 2 && rows <= 64 && n * k >= (kcontig ? 32L << 20 : 16L << 20);
}

// Floats of split workspace for a product over `rows`, sized for operands without
// gaps between their rows (a call with others runs in more parts, which split
// within that room).  Small products of few rows are not split: one launch of 32x32
// tiles takes no longer than two (1 row over 4096 x 1024: 9 and 15 us, of which each
// launch takes the host 3.5) until its chain of k-tiles is the longer one.
long split_floats(int elt, long rows, long n, long k, bool kcontig) {
  if (streams(elt, rows, n, k, kcontig)) return plan_stream(rows, n, k, GEMM_SPLIT_MAX_FLOATS, 256).split_floats;
  if (elt == 2 && rows <= 32 && (kcontig ? k <= 8192 : k <= 4096 && n <= 2048)) return 0;
  const long each = part_rows(elt, k, 0);
  const long full = std::min(rows, each), rest = rows > each ? rows % each : 0;
  long f = work_of(elt, std::max(1L, full), n, k, false).split_floats;
  if (rest) f = std::max(f, work_of(elt, rest, n, k, false).split_floats);
  return f;
}

GemmParams params(long m, int n, long k, int epi) {
  GemmParams p{};
  p.M = (int)m;
  p.N = n;
  p.K = (int)k;
  p.batch = p.heads = 1;
  p.epi = epi;
  p.wide = 1;
  return p;
}

// A launch's rows of the weight's gradient, and what its column sums take.  The
// bias gradient is the column sums of dy, which the bf16 products form on their
// way (it is their right operand, or, by_out, their left one: 4001 x 8192 x 2048
// by_out 117 us so, 123 with a kernel of its own over dy, 112 without the sums); fp32
// products leave them to a kernel of their own.
bool sums_in_product(const LinearArgs& a) { return a.dbias && a.elt == 2; }

struct WeightWork {
  long split, sums;
};
// Few tokens: no tiles.
bool few(const LinearArgs& a) {
  return a.rows > 0 && a.rows <= few_tokens_most(a.elt) && std::max(a.in, a.out) <= FEW_MOST_ROWS;
}
WeightWork weight_work(const LinearArgs& a) {
  if (few(a)) return {0, 0};
  const long each = part_rows(a.elt, a.in, a.out);
  const long m = a.by_out ? a.out : a.in, n = a.by_out ? a.in : a.out;
  const long full = std::max(1L, std::min(a.rows, each)), rest = a.rows > each ? a.rows % each : 0;
  WeightWork w{0, 0};
  for (long k : {full, rest})
    if (k) {
      const GemmWork g = work_of(a.elt, m, n, k, true);
      w.split = std::max(w.split, g.split_floats);
      w.sums = std::max(w.sums, a.by_out ? g.colsum_a_floats : g.colsum_floats);
    }
  if (!sums_in_product(a)) w.sums = a.dbias ? (long)(dropout_work_bytes(a.rows, a.out) / sizeof(float)) : 0;
  w.split = (w.split + 3) & ~3L;
  return w;
}

}  // namespace

size_t linear_forward_work(const LinearArgs& a) {
  return sizeof(float) * (size_t)split_floats(a.elt, a.rows, a.out, a.in, a.by_out);
}
size_t linear_input_work(const LinearArgs& a) {
  return sizeof(float) * (size_t)split_floats(a.elt, a.rows, a.in, a.out, !a.by_out);
}
size_t linear_weight_work(const LinearArgs& a) {
  const WeightWork w = weight_work(a);
  return sizeof(float) * (size_t)(w.split + w.sums);
}

hipError_t linear_forward(const LinearArgs& args, hipStream_t s) {
  LinearArgs a = args;
  if (a.rows == 0) return hipSuccess;
  const long each = part_rows(a.elt, a.x.stride, 0);
  const long split = split_floats(a.elt, a.rows, a.out, a.in, a.by_out);
  return parts(a.rows, each, [&](long r, long m) {
    GemmParams p = params(m, a.out, a.in, EPI_LINEAR);
    p.A = at(a.x, r, a.elt);
    p.lda = a.x.stride;
    p.a_kcontig = 1;
    p.B = a.w.data;
    p.ldb = a.w.stride;
    p.b_kcontig = a.by_out;
    p.stream = streams(a.elt, a.rows, p.N, p.K, p.b_kcontig);
    p.C = at(a.y, r, a.elt);
    p.ldc = a.y.stride;
    p.bias = (const float*)a.bias;
    p.bias_bf16 = !a.bias_f32;
    p.act = a.act;
    p.resid = at(a.residual, r, a.elt);
    p.ld_resid = a.residual.stride;
    p.C2 = at(a.slope, r, a.elt);
    p.ldc2 = a.slope.stride;
    p.split_work = (float*)a.work;
    p.split_floats = split;
    return gemm(a.elt, p, s);
  });
}

hipError_t linear_backward_input(const LinearArgs& args, hipStream_t s) {
  LinearArgs a = args;
  if (a.rows == 0) return hipSuccess;
  const long each = part_rows(a.elt, a.dy.stride, 0);
  const long split = split_floats(a.elt, a.rows, a.in, a.out, !a.by_out);
  return parts(a.rows, each, [&](long r, long m) {
    GemmParams p = params(m, a.in, a.out, a.before.data ? EPI_GELU_BWD : EPI_STORE);
    p.A = at(a.dy, r, a.elt);
    p.lda = a.dy.stride;
    p.a_kcontig = 1;
    p.B = a.w.data;
    p.ldb = a.w.stride;
    p.b_kcontig = !a.by_out;
    p.stream = streams(a.elt, a.rows, p.N, p.K, p.b_kcontig);
    p.C = at(a.dx, r, a.elt);
    p.ldc = a.dx.stride;
    p.aux = at(a.before, r, a.elt);
    p.ld_aux = a.before.stride;
    p.split_work = (float*)a.work;
    p.split_floats = split;
    return gemm(a.elt, p, s);
  });
}

hipError_t linear_backward_weight(const LinearArgs& args, hipStream_t s) {
  LinearArgs a = args;
  if (few(a)) {
    const int m = a.by_out ? a.out : a.in, n = a.by_out ? a.in : a.out;
    return few_tokens({(int)a.rows, m, n, a.by_out ? a.dy : a.x, a.by_out ? a.x : a.dy, a.dw, a.dbias, !a.by_out,
                       a.accumulate}, a.elt, s);
  }
  const long each = part_rows(a.elt, a.x.stride, a.dy.stride);
  const WeightWork w = weight_work(a);
  float* const sums = (float*)a.work + w.split;
  const bool fused = sums_in_product(a);
  hipError_t e = parts(a.rows, each, [&](long r, long k) {
    const int accumulate = a.accumulate || r > 0;
    GemmParams p = params(a.by_out ? a.out : a.in, a.by_out ? a.in : a.out, k, EPI_F32_ACC);
    const RowsView &left = a.by_out ? a.dy : a.x, &right = a.by_out ? a.x : a.dy;
    p.A = at(left, r, a.elt);
    p.lda = left.stride;
    p.B = at(right, r, a.elt);
    p.ldb = right.stride;
    p.C = a.dw;
    p.ldc = p.N;
    p.accumulate = accumulate;
    p.split_work = (float*)a.work;
    p.split_floats = w.split;
    int rows = 0;
    if (fused) {
      p.colsum_work = sums;
      p.colsum_floats = w.sums;
      p.colsum_rows = &rows;
      p.colsum_a = a.by_out;
    }
    const hipError_t g = gemm(a.elt, p, s);
    if (g != hipSuccess || !fused) return g;
    return rows_finish(sums, rows, 1, a.out, a.out, &a.dbias, accumulate, s);
  });
  if (e != hipSuccess || !a.dbias || fused) return e;
  DropoutArgs d{};
  d.rows = a.rows;
  d.cols = a.out;
  d.x = a.dy;
  d.sums = a.dbias;
  d.accumulate = a.accumulate;
  d.work = sums;
  return dropout_rows(d, a.elt, s);
}
