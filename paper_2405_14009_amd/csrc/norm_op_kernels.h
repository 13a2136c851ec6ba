// Layer norm of total = residual + D(x + bias), forward and backward.
//
// Bound by memory.  LPR lanes share a row, CPL groups of eight columns each, so
// that a row is read once and stays in registers: the statistics (mean, then the
// squares around it) are sums of 32 bits over the lanes, by shuffles within a
// wave and through LDS between the waves of a row.  Rows of up to 128 columns
// share a wave, rows beyond 1024 take several.
//
// The backward pass goes over the rows with as many workgroups as fill the card
// and keeps the columns' sums (of dy xhat, dy and dx) in its lanes' registers; each
// workgroup stores one row of them, which a second launch adds in order.
#pragma once

#include <algorithm>

#include "rows_op_kernels.h"

namespace {

constexpr int block_of(int lpr) { return lpr > 256 ? lpr : 256; }

// Sums of N values over the LPR lanes of a row (every lane gets them).  red:
// two sets of [waves][N] floats, used in turn, so one barrier a call will do.
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red, int& turn) {
#pragma unroll
  for (int o = (LPR < 64 ? LPR : 64) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o, 64);
  if constexpr (LPR > 64) {
    constexpr int W = LPR / 64;
    float* r = red + turn * (W * N);
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) r[(threadIdx.x >> 6) * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += r[w * N + i];
  }
}

template <class E, int LPR, int CPL, bool TAIL>
__global__ __launch_bounds__(block_of(LPR)) void norm_fwd_k(NormArgs a) {
  typedef Columns<E, TAIL> C;
  constexpr int NT = block_of(LPR), RPW = NT / LPR;
  __shared__ float red[2 * (LPR > 64 ? LPR / 64 : 1)];
  const int lane = threadIdx.x % LPR;
  const bool add = a.total.data != nullptr;
  Philox rng;
  if (a.drop.on) rng.init(a.drop);
  int turn = 0;
  auto work = [&](long row) {
    Raw8<E> x[CPL], res[CPL];
    RawParams b[CPL], w[CPL], h[CPL];
  #pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = lane + LPR * q;
      if (8 * g < a.cols) {
        x[q] = C::load((const E*)a.x.data + row * a.x.stride, g, a.cols);
        if (a.residual.data) res[q] = C::load((const E*)a.residual.data + row * a.residual.stride, g, a.cols);
        if (a.bias) b[q] = load_params<TAIL>(a.bias, a.params_f32, g, a.cols);
        if (a.weight) w[q] = load_params<TAIL>(a.weight, a.params_f32, g, a.cols);
        if (a.shift) h[q] = load_params<TAIL>(a.shift, a.params_f32, g, a.cols);
      }
    }
    float f[CPL][8], s[1] = {0.f};
  #pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = lane + LPR * q;
  #pragma unroll
      for (int e = 0; e < 8; ++e) f[q][e] = 0.f;
      if (8 * g < a.cols) {
        C::floats(x[q], g, a.cols, f[q]);
        float t[8];
        if (a.bias) {
          param_floats<TAIL>(b[q], a.params_f32, g, a.cols, t);
  #pragma unroll
          for (int e = 0; e < 8; ++e) f[q][e] += t[e];
        }
        if (a.drop.on) drop8(rng, a.drop, g, row, f[q]);
        if (a.residual.data) {
          C::floats(res[q], g, a.cols, t);
  #pragma unroll
          for (int e = 0; e < 8; ++e) f[q][e] += t[e];
        }
        if (add) {
          C::store((E*)a.total.data + row * a.total.stride, g, a.cols, f[q]);
          // the norm is that of the stored total, which the backward pass reads
  #pragma unroll
          for (int e = 0; e < 8; ++e) f[q][e] = to_f32(from_f32<E>(f[q][e]));
        }
  #pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!TAIL || 8 * g + e < a.cols) s[0] += f[q][e];
      }
    }
    row_sums<LPR>(s, red, turn);
    const float mean = s[0] / a.cols;
    s[0] = 0.f;
  #pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = lane + LPR * q;
      if (8 * g < a.cols) {
  #pragma unroll
        for (int e = 0; e < 8; ++e) {
          f[q][e] -= mean;
          if (!TAIL || 8 * g + e < a.cols) s[0] += f[q][e] * f[q][e];
        }
      }
    }
    row_sums<LPR>(s, red, turn);
    const float rstd = 1.0f / sqrtf(s[0] / a.cols + a.eps);
  #pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = lane + LPR * q;
      if (8 * g < a.cols) {
        float t[8];
  #pragma unroll
        for (int e = 0; e < 8; ++e) f[q][e] *= rstd;
        if (a.weight) {
          param_floats<TAIL>(w[q], a.params_f32, g, a.cols, t);
  #pragma unroll
          for (int e = 0; e < 8; ++e) f[q][e] *= t[e];
        }
        if (a.shift) {
          param_floats<TAIL>(h[q], a.params_f32, g, a.cols, t);
  #pragma unroll
          for (int e = 0; e < 8; ++e) f[q][e] += t[e];
        }
        C::store((E*)a.y.data + row * a.y.stride, g, a.cols, f[q]);
      }
    }
    if (a.stats && lane == 0) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = rstd;
    }
  };
  // one set of rows a workgroup, but in the largest calls
  for (long k = (long)blockIdx.x * RPW; k < a.rows; k += (long)gridDim.x * RPW) {
    const long row = k + threadIdx.x / LPR;
    if (LPR > 64 || row < a.rows) work(row);   // (rows of several waves: one a workgroup)
  }
}

template <class E, int LPR, int CPL, bool TAIL>
__global__ __launch_bounds__(block_of(LPR)) void norm_bwd_k(NormArgs a, int stride) {
  typedef Columns<E, TAIL> C;
  constexpr int NT = block_of(LPR), RPW = NT / LPR;
  __shared__ float red[4 * (LPR > 64 ? LPR / 64 : 1)];
  const int lane = threadIdx.x % LPR;
  const long step = (long)gridDim.x * RPW;
  const bool sums = a.dweight || a.dshift || a.dbias, grads = a.dtotal.data || a.dx.data || a.dbias;
  Philox rng;
  if (a.drop.on) rng.init(a.drop);
  float wt[CPL][8], sw[CPL][8], sh[CPL][8], sb[CPL][8];
#pragma unroll
  for (int q = 0; q < CPL; ++q) {
    const int g = lane + LPR * q;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      wt[q][e] = 1.f;
      sw[q][e] = sh[q][e] = sb[q][e] = 0.f;
    }
    if (a.weight && 8 * g < a.cols)
      param_floats<TAIL>(load_params<TAIL>(a.weight, a.params_f32, g, a.cols), a.params_f32, g, a.cols, wt[q]);
  }
  struct Row {
    Raw8<E> dy[CPL], t[CPL], in[CPL];
    float mean, rstd;
  };
  auto fetch = [&](Row& r, long row) {
    if (row >= a.rows) return;
    r.mean = a.stats[row];
    r.rstd = a.stats[a.rows + row];
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = lane + LPR * q;
      if (8 * g < a.cols) {
        r.dy[q] = C::load((const E*)a.dy.data + row * a.dy.stride, g, a.cols);
        r.t[q] = C::load((const E*)a.total.data + row * a.total.stride, g, a.cols);
        if (a.dtotal_in.data && grads)
          r.in[q] = C::load((const E*)a.dtotal_in.data + row * a.dtotal_in.stride, g, a.cols);
      }
    }
  };
  int turn = 0;
  auto work = [&](const Row& r, long row) {
    if (LPR <= 64 && row >= a.rows) return;   // (wider rows: the whole workgroup is here or not)
    float d[CPL][8], xh[CPL][8], m[2] = {0.f, 0.f};
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = lane + LPR * q;
#pragma unroll
      for (int e = 0; e < 8; ++e) d[q][e] = xh[q][e] = 0.f;
      if (8 * g < a.cols) {
        C::floats(r.dy[q], g, a.cols, d[q]);
        C::floats(r.t[q], g, a.cols, xh[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          xh[q][e] = (xh[q][e] - r.mean) * r.rstd;
          if (!TAIL || 8 * g + e < a.cols) {
            sw[q][e] += d[q][e] * xh[q][e];
            sh[q][e] += d[q][e];
            d[q][e] *= wt[q][e];
            m[0] += d[q][e];
            m[1] += d[q][e] * xh[q][e];
          }
        }
      }
    }
    if (!grads) return;
    row_sums<LPR>(m, red, turn);
    const float m0 = m[0] / a.cols, m1 = m[1] / a.cols;
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = lane + LPR * q;
      if (8 * g < a.cols) {
#pragma unroll
        for (int e = 0; e < 8; ++e) d[q][e] = r.rstd * (d[q][e] - m0 - xh[q][e] * m1);
        if (a.dtotal_in.data) {
          float t[8];
          C::floats(r.in[q], g, a.cols, t);
#pragma unroll
          for (int e = 0; e < 8; ++e) d[q][e] += t[e];
        }
        if (a.dtotal.data) C::store((E*)a.dtotal.data + row * a.dtotal.stride, g, a.cols, d[q]);
        if (a.drop.on && (a.dx.data || a.dbias)) drop8(rng, a.drop, g, row, d[q]);
        if (a.dx.data) C::store((E*)a.dx.data + row * a.dx.stride, g, a.cols, d[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sb[q][e] += d[q][e];
      }
    }
  };
  const long first = (long)blockIdx.x * RPW + threadIdx.x / LPR;
  const long base = (long)blockIdx.x * RPW;   // workgroup uniform
  Row ra;
  if constexpr (LPR < 1024) {
    // the next row's loads are in flight while a row is worked on
    Row rb;
    fetch(ra, first);
    for (long k = 0; base + k < a.rows; k += 2 * step) {
      fetch(rb, first + k + step);
      work(ra, first + k);
      if (base + k + step < a.rows) {
        fetch(ra, first + k + 2 * step);
        work(rb, first + k + step);
      }
    }
  } else {   // (sixteen waves have no registers for that)
    for (long k = 0; base + k < a.rows; k += step) {
      fetch(ra, first + k);
      work(ra, first + k);
    }
  }
  if (!sums) return;
  // the row sets of the workgroup in order
  float* out = a.work + (long)blockIdx.x * ROWS_MAX_VECTORS * stride;
  if constexpr (RPW == 1) {
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = lane + LPR * q;
      if (8 * g < a.cols) {
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          *(float4*)(out + 8 * g + e) = make_float4(sw[q][e], sw[q][e + 1], sw[q][e + 2], sw[q][e + 3]);
          *(float4*)(out + stride + 8 * g + e) = make_float4(sh[q][e], sh[q][e + 1], sh[q][e + 2], sh[q][e + 3]);
          *(float4*)(out + 2 * stride + 8 * g + e) = make_float4(sb[q][e], sb[q][e + 1], sb[q][e + 2], sb[q][e + 3]);
        }
      }
    }
  } else {
    __shared__ float set[NT][9];
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
#pragma unroll
      for (int v = 0; v < 3; ++v) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) set[threadIdx.x][e] = v == 0 ? sw[q][e] : v == 1 ? sh[q][e] : sb[q][e];
        __syncthreads();
        for (int i = threadIdx.x; i < 8 * LPR; i += NT) {
          const int c = 8 * LPR * q + i;
          float t = 0.f;
          for (int k = 0; k < RPW; ++k) t += set[k * LPR + (i >> 3)][i & 7];
          if (c < stride) out[v * stride + c] = t;
        }
      }
    }
  }
}

// The lanes of a row and its groups a lane.
template <class E, template <class, int, int, bool> class K>
struct NormShapes {
  template <bool TAIL, class... A>
  static hipError_t run(int cols, A... args) {
    if (cols <= 32) return K<E, 4, 1, TAIL>::go(args...);
    if (cols <= 128) return K<E, 16, 1, TAIL>::go(args...);
    if (cols <= 512) return K<E, 64, 1, TAIL>::go(args...);
    if (cols <= 1024) return K<E, 64, 2, TAIL>::go(args...);
    if (cols <= 2048) return K<E, 256, 1, TAIL>::go(args...);
    if (cols <= 4096) return K<E, 256, 2, TAIL>::go(args...);
    if (cols <= 8192) return K<E, 512, 2, TAIL>::go(args...);
    return K<E, 1024, 2, TAIL>::go(args...);
  }
};

template <class E, int LPR, int CPL, bool TAIL>
struct NormForward {
  static hipError_t go(const NormArgs& a, hipStream_t s) {
    constexpr int RPW = block_of(LPR) / LPR;
    hipLaunchKernelGGL((norm_fwd_k<E, LPR, CPL, TAIL>), dim3((unsigned)std::min((a.rows + RPW - 1) / RPW, 1L << 20)),
                       dim3(block_of(LPR)), 0, s, a);
    return hipGetLastError();
  }
};

template <class E, int LPR, int CPL, bool TAIL>
struct NormBackward {
  static hipError_t go(const NormArgs& a, int groups, hipStream_t s) {
    hipLaunchKernelGGL((norm_bwd_k<E, LPR, CPL, TAIL>), dim3((unsigned)groups), dim3(block_of(LPR)), 0, s, a,
                       rows_pad(a.cols));
    return hipGetLastError();
  }
};

template <class E>
hipError_t norm_fwd(const NormArgs& a, hipStream_t s) {
  typedef NormShapes<E, NormForward> F;
  return a.cols % 8 ? F::template run<true, const NormArgs&, hipStream_t>(a.cols, a, s)
                    : F::template run<false, const NormArgs&, hipStream_t>(a.cols, a, s);
}
template <class E>
hipError_t norm_bwd(const NormArgs& a, int groups, hipStream_t s) {
  typedef NormShapes<E, NormBackward> B;
  return a.cols % 8 ? B::template run<true, const NormArgs&, int, hipStream_t>(a.cols, a, groups, s)
                    : B::template run<false, const NormArgs&, int, hipStream_t>(a.cols, a, groups, s);
}

}  // namespace

// one file each
hipError_t norm_fwd_bf16(const NormArgs& a, hipStream_t s);
hipError_t norm_fwd_f32(const NormArgs& a, hipStream_t s);
hipError_t norm_bwd_bf16(const NormArgs& a, int groups, hipStream_t s);
hipError_t norm_bwd_f32(const NormArgs& a, int groups, hipStream_t s);
