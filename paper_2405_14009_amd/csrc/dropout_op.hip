// Dropout of a matrix, y = residual + D(x + bias) or D(x) * derivative, and the
// column sums that the operators over rows share.
//
// Bound by memory.  A thread owns a group of eight columns and walks down the
// rows of its workgroup, ROWS of them in flight; workgroups are as wide as the
// matrix (up to 256 groups) and share out the rest of their threads over rows.
#include <algorithm>

#include "rows_op_kernels.h"

namespace {

constexpr int NT = 256;

struct Grid {
  int lanes;       // threads across (a power of two up to NT)
  int wide, deep;  // workgroups across and down
  long rows;       // rows of a workgroup
};

// Rows of a workgroup: enough workgroups to fill the card eight times over, or,
// where column sums are kept, twice (each stores a row of them; 2048 x 4096 bf16:
// 11.4 us so, 12.4 with eight rows in flight, 11.6 with twice the workgroups).
// Sums of up to 512 rows are one workgroup's down, of 64 columns if need be, which
// stores them itself (128 x 256 fp32: 7 us, where the second launch alone takes the
// host 3.5).
Grid grid_of(long rows, int cols, bool sums) {
  Grid g;
  const int groups = (cols + 7) / 8;
  g.lanes = 1;
  while (g.lanes < NT && g.lanes < groups) g.lanes *= 2;
  auto steps = [&] { return std::max(1L, (rows * g.lanes + NT - 1) / NT); };   // NT / lanes rows side by side
  bool alone = false;
  if (sums && rows <= 512) {
    while (g.lanes > 8 && steps() > 16) g.lanes /= 2;
    alone = steps() <= 16;
  }
  g.wide = (groups + g.lanes - 1) / g.lanes;
  const long want = alone ? 1 : std::max(1L, (sums ? 512L : 2048L) / g.wide);
  g.rows = (steps() + want - 1) / want * (NT / g.lanes);
  g.deep = (int)std::max(1L, (rows + g.rows - 1) / g.rows);
  return g;
}

template <class E, bool TAIL, bool SUMS>
__global__ __launch_bounds__(NT) void dropout_k(DropoutArgs a, int lanes, long rows_each, int stride) {
  typedef Columns<E, TAIL> C;
  constexpr int ROWS = 4;
  const int lane = threadIdx.x & (lanes - 1), at = threadIdx.x / lanes, step = NT / lanes;
  const int group = (int)blockIdx.x * lanes + lane;
  const bool in = 8 * group < a.cols;
  const long r1 = min(a.rows, ((long)blockIdx.y + 1) * rows_each);
  Philox rng;
  if (a.drop.on) rng.init(a.drop);
  float bias[8], sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = sum[e] = 0.f;
  if (in && a.bias) param_floats<TAIL>(load_params<TAIL>(a.bias, a.bias_f32, group, a.cols), a.bias_f32, group, a.cols, bias);
  if (in) {
    for (long r = (long)blockIdx.y * rows_each + at; r < r1; r += (long)ROWS * step) {
      Raw8<E> x[ROWS], m[ROWS];
#pragma unroll
      for (int u = 0; u < ROWS; ++u) {
        const long q = r + (long)u * step;
        if (q < r1) {
          x[u] = C::load((const E*)a.x.data + q * a.x.stride, group, a.cols);
          if (a.more.data) m[u] = C::load((const E*)a.more.data + q * a.more.stride, group, a.cols);
        }
      }
#pragma unroll
      for (int u = 0; u < ROWS; ++u) {
        const long q = r + (long)u * step;
        if (q < r1) {
          float f[8], g[8];
          C::floats(x[u], group, a.cols, f);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] += bias[e];
          if (a.drop.on) drop8(rng, a.drop, group, q, f);
          if (a.more.data) {
            C::floats(m[u], group, a.cols, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = a.more_factor ? f[e] * g[e] : f[e] + g[e];
          }
          if (a.y.data) C::store((E*)a.y.data + q * a.y.stride, group, a.cols, f);
          if constexpr (SUMS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += f[e];
          }
        }
      }
    }
  }
  if constexpr (SUMS) {
    __shared__ float red[NT][9];
#pragma unroll
    for (int e = 0; e < 8; ++e) red[threadIdx.x][e] = sum[e];
    __syncthreads();
    // column c of the workgroup: its row sets in order
    for (int i = threadIdx.x; i < 8 * lanes; i += NT) {
      float t = 0.f;
      for (int q = 0; q < step; ++q) t += red[q * lanes + (i >> 3)][i & 7];
      const int c = 8 * (int)blockIdx.x * lanes + i;
      if (gridDim.y > 1) {
        if (c < stride) a.work[(long)blockIdx.y * stride + c] = t;
      } else if (c < a.cols) {
        a.sums[c] = a.accumulate ? a.sums[c] + t : t;
      }
    }
  }
}

template <class E>
hipError_t launch(const DropoutArgs& a, hipStream_t s) {
  const bool sums = a.sums != nullptr, tail = a.cols % 8 != 0;
  const Grid g = grid_of(a.rows, a.cols, sums);
  const int stride = rows_pad(a.cols);
  const dim3 grid((unsigned)g.wide, (unsigned)g.deep);
#define DROPOUT(T, S) hipLaunchKernelGGL((dropout_k<E, T, S>), grid, dim3(NT), 0, s, a, g.lanes, g.rows, stride)
  if (tail && sums) DROPOUT(true, true);
  else if (tail) DROPOUT(true, false);
  else if (sums) DROPOUT(false, true);
  else DROPOUT(false, false);
#undef DROPOUT
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !sums || g.deep == 1) return e;
  return rows_finish(a.work, g.deep, 1, stride, a.cols, &a.sums, a.accumulate, s);
}

// Sums over partial rows: a workgroup takes 32 columns, eight threads across and
// 32 sets of rows down, which are added in order.
constexpr int FC = 32, FG = NT / (FC / 4);
struct FinishArgs {
  const float* part;
  int n, vectors, stride, cols, accumulate;
  float* out[ROWS_MAX_VECTORS];
};

__global__ __launch_bounds__(NT) void rows_finish_k(FinishArgs a) {
  __shared__ float4 red[FG][FC / 4];
  float* out = a.out[blockIdx.y];
  if (!out) return;
  const int cl = threadIdx.x % (FC / 4), rg = threadIdx.x / (FC / 4);
  const int c = (int)blockIdx.x * FC + 4 * cl;
  const float* src = a.part + (long)blockIdx.y * a.stride + c;
  const long step = (long)a.vectors * a.stride;
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < a.stride) {
    for (int r = rg; r < a.n; r += 8 * FG) {
      float4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (r + u * FG < a.n) v[u] = *(const float4*)(src + (r + u * FG) * step);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (r + u * FG < a.n) {
          t.x += v[u].x;
          t.y += v[u].y;
          t.z += v[u].z;
          t.w += v[u].w;
        }
    }
  }
  red[rg][cl] = t;
  __syncthreads();
  if (threadIdx.x < FC) {
    const int k = (int)blockIdx.x * FC + threadIdx.x;
    if (k < a.cols) {
      float sum = 0.f;
#pragma unroll
      for (int q = 0; q < FG; ++q) sum += ((const float*)&red[q][0])[threadIdx.x];
      out[k] = a.accumulate ? out[k] + sum : sum;
    }
  }
}

}  // namespace

hipError_t rows_finish(const float* part, int n, int vectors, int stride, int cols, float* const* outs, int accumulate,
                       hipStream_t s) {
  FinishArgs f{part, n, vectors, stride, cols, accumulate, {}};
  for (int i = 0; i < vectors; ++i) f.out[i] = outs[i];
  hipLaunchKernelGGL(rows_finish_k, dim3((unsigned)((cols + FC - 1) / FC), (unsigned)vectors), dim3(NT), 0, s, f);
  return hipGetLastError();
}

size_t dropout_work_bytes(long rows, int cols) {
  const int deep = grid_of(rows, cols, true).deep;
  return deep > 1 ? sizeof(float) * (size_t)deep * rows_pad(cols) : 0;
}

hipError_t dropout_rows(const DropoutArgs& a, int elt, hipStream_t s) {
  if (a.rows == 0 && !a.sums) return hipSuccess;
  return elt == 2 ? launch<bf16>(a, s) : launch<float>(a, s);
}
