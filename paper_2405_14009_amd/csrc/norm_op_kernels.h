// Layer norm of total = residual + D(x + bias), forward and backward.
//
// Bound by memory.  The lanes of a row hold CPL groups of eight columns each, so
// that a row is read once and stays in registers: the statistics (mean, then the
// squares around it) are sums of 32 bits over the lanes, by moves within a
// wave and through LDS between the waves of a row.  Rows of up to 128 columns
// share a wave, rows beyond 1024 take as many waves as they fill: one group a lane
// (16384 x 5120 with bias, dropout and residual: 127 us, 671 MB, at the rate of a
// large copy; 265 with two groups in half the waves, whose registers leave room for
// fewer of them).  Workgroups walk over rows, the next row's loads in flight while a
// row is worked on.
//
// The backward pass keeps the columns' sums (of dy xhat, dy and dx) in its lanes'
// registers; each workgroup stores one row of them, which a second launch adds in
// order (the same size: 189 + 5 us, 839 MB; vector instructions issue in half the
// cycles).  So it has as many rows side by side in a workgroup, and as few
// workgroups, as fill the card.
#pragma once

#include <algorithm>

#include "rows_op_kernels.h"

namespace {

// The threads of a workgroup: LPR lanes a row (4, 16 or 64: 256 threads), or, LPR
// 0, `waves` whole waves a row and as many rows side by side as fit.
template <int LPR>
struct RowLanes {
  int lanes, lane, slot, slots, waves;
  __device__ __forceinline__ RowLanes(int w) {
    if constexpr (LPR > 0) {
      lanes = LPR;
      lane = threadIdx.x % LPR;
      slot = threadIdx.x / LPR;
      slots = 256 / LPR;
      waves = 1;
    } else {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      waves = w;
      lanes = 64 * w;
      slot = wave / w;
      lane = (wave - slot * w) * 64 + (threadIdx.x & 63);
      slots = blockDim.x / lanes;
    }
  }
};

// Sums of N values over the lanes of a row (every lane gets them).  red: two sets
// of 16 waves' N floats, used in turn, so one barrier a call will do.
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red, int& turn, const RowLanes<LPR>& at) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lane_sum<(LPR > 0 ? LPR : 64)>(v[i]);
  if constexpr (LPR == 0) {
    float* r = red + turn * (16 * N);
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) r[(threadIdx.x >> 6) * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    for (int w = at.slot * at.waves; w < (at.slot + 1) * at.waves; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += r[w * N + i];
  }
}

// Runs work(row data, row, next row) over the rows of a workgroup.  AHEAD: work
// fetches the next row's data as soon as it has this row's numbers, so that its
// loads are in flight during the rest.  All threads go through the same number of
// steps (work has barriers); rows beyond the last are the work's to leave out.
template <bool AHEAD, class Row, class Fetch, class Work>
__device__ __forceinline__ void walk_rows(long rows, int slot, int slots, Fetch fetch, Work work) {
  const long step = (long)gridDim.x * slots;
  long k = (long)blockIdx.x * slots;
  Row r;
  if (AHEAD) fetch(r, k + slot);
  for (; k < rows; k += step) {
    if (!AHEAD) fetch(r, k + slot);
    work(r, k + slot, k + step + slot);
  }
}
// Rows of more than 8192 columns hold two groups a lane in nine to sixteen waves,
// whose registers have no room for the next row's data (and, backward, the weight,
// which is read again from the caches).  Without it the backward pass still spills,
// its sums being two groups' whatever the caller asks for: beyond 12288 columns
// (128 registers a lane) 39 registers in bf16 and 79 in fp32, of counts that are no
// multiple of 8 65 and 207; up to 12288 none and 18, of such counts 16 and 37.  The
// forward spills for such counts alone: 32 and 42, up to 12288 none and 2.  With a
// residual sum, bf16 (in brackets at the copy's rate): 4096 x 12288 forward 101 us
// (82), backward 117 (103); 16384: 143 (110), 232 (137); 12289: 167, 283.
constexpr bool roomy(int lpr, int cpl) { return lpr > 0 || cpl == 1; }

template <class E, int LPR, int CPL, bool TAIL, int NT>
__global__ __launch_bounds__(NT) void norm_fwd_k(NormArgs a, int waves) {
  typedef Columns<E, TAIL> C;
  __shared__ float red[LPR == 0 ? 2 * 16 : 1];
  const RowLanes<LPR> at(waves);
  const bool add = a.total.data != nullptr;
  Philox rng;
  if (a.drop.on) rng.init(a.drop);
  // the vectors' values of a group (0 or 1 where there is none)
  auto vector = [&](const void* p, float none, int g, float(&f)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = none;
    if (p && 8 * g < a.cols) param_floats<TAIL>(load_params<TAIL>(p, a.params_f32, g, a.cols), a.params_f32, g, a.cols, f);
  };
  constexpr bool KEEP = roomy(LPR, CPL);
  constexpr int KEPT = KEEP ? CPL : 1;
  float ib[KEPT][8], wt[KEPT][8], sh[KEPT][8];
  if constexpr (KEEP) {
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      vector(a.bias, 0.f, g, ib[q]);
      vector(a.weight, 1.f, g, wt[q]);
      vector(a.shift, 0.f, g, sh[q]);
    }
  }
  struct Row {
    Raw8<E> x[CPL], res[CPL];
  };
  auto fetch = [&](Row& r, long row) {
    if (row >= a.rows) return;
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      if (8 * g < a.cols) {
        r.x[q] = C::load((const E*)a.x.data + row * a.x.stride, g, a.cols);
        if (a.residual.data) r.res[q] = C::load((const E*)a.residual.data + row * a.residual.stride, g, a.cols);
      }
    }
  };
  int turn = 0;
  auto work = [&](Row& r, long row, long next) {
    const bool here = row < a.rows;
    if (LPR > 0 && !here) return;
    float f[CPL][8], res[CPL][8], s[1] = {0.f};
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      C::floats(r.x[q], g, a.cols, f[q]);
      C::floats(r.res[q], g, a.cols, res[q]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (KEEP) fetch(r, next);
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      if (here && 8 * g < a.cols) {
        if (!KEEP) vector(a.bias, 0.f, g, ib[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[q][e] += ib[q % KEPT][e];
        if (a.drop.on) drop8(rng, a.drop, g, row, f[q]);
        if (a.residual.data) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[q][e] += res[q][e];
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
    row_sums<LPR>(s, red, turn, at);
    const float mean = s[0] / a.cols;
    s[0] = 0.f;
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      if (8 * g < a.cols) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f[q][e] -= mean;
          if (!TAIL || 8 * g + e < a.cols) s[0] += f[q][e] * f[q][e];
        }
      }
    }
    row_sums<LPR>(s, red, turn, at);
    const float rstd = 1.0f / sqrtf(s[0] / a.cols + a.eps);
    if (!here) return;
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      if (8 * g < a.cols) {
        if (!KEEP) {
          vector(a.weight, 1.f, g, wt[0]);
          vector(a.shift, 0.f, g, sh[0]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) f[q][e] = f[q][e] * rstd * wt[q % KEPT][e] + sh[q % KEPT][e];
        C::store((E*)a.y.data + row * a.y.stride, g, a.cols, f[q]);
      }
    }
    if (a.stats && at.lane == 0) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = rstd;
    }
  };
  walk_rows<roomy(LPR, CPL), Row>(a.rows, at.slot, at.slots, fetch, work);
}

template <class E, int LPR, int CPL, bool TAIL, int NT>
__global__ __launch_bounds__(NT) void norm_bwd_k(NormArgs a, int waves, int stride) {
  typedef Columns<E, TAIL> C;
  __shared__ float red[LPR == 0 ? 4 * 16 : 1];
  const RowLanes<LPR> at(waves);
  const bool sums = a.dweight || a.dshift || a.dbias, grads = a.dtotal.data || a.dx.data || a.dbias;
  Philox rng;
  if (a.drop.on) rng.init(a.drop);
  constexpr int KEPT = roomy(LPR, CPL) ? CPL : 1;
  float kept[KEPT][8], sw[CPL][8], sh[CPL][8], sb[CPL][8];
  auto weight = [&](int g, float(&f)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 1.f;
    if (a.weight && 8 * g < a.cols)
      param_floats<TAIL>(load_params<TAIL>(a.weight, a.params_f32, g, a.cols), a.params_f32, g, a.cols, f);
  };
#pragma unroll
  for (int q = 0; q < CPL; ++q) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sw[q][e] = sh[q][e] = sb[q][e] = 0.f;
    if (roomy(LPR, CPL)) weight(at.lane + at.lanes * q, kept[q % KEPT]);
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
      const int g = at.lane + at.lanes * q;
      if (8 * g < a.cols) {
        r.dy[q] = C::load((const E*)a.dy.data + row * a.dy.stride, g, a.cols);
        r.t[q] = C::load((const E*)a.total.data + row * a.total.stride, g, a.cols);
        if (a.dtotal_in.data && grads)
          r.in[q] = C::load((const E*)a.dtotal_in.data + row * a.dtotal_in.stride, g, a.cols);
      }
    }
  };
  int turn = 0;
  auto work = [&](Row& r, long row, long next) {
    const bool here = row < a.rows;
    if (LPR > 0 && !here) return;
    float d[CPL][8], xh[CPL][8], m[2] = {0.f, 0.f};
    Raw8<E> in[CPL];
    const float mean = r.mean, rstd = r.rstd;
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      C::floats(r.dy[q], g, a.cols, d[q]);
      C::floats(r.t[q], g, a.cols, xh[q]);
      in[q] = r.in[q];
    }
    __builtin_amdgcn_sched_barrier(0);
    if (roomy(LPR, CPL)) fetch(r, next);
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      if (here && 8 * g < a.cols) {
        if (!roomy(LPR, CPL)) weight(g, kept[0]);
        float(&wt)[8] = kept[q % KEPT];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          xh[q][e] = (xh[q][e] - mean) * rstd;
          if (!TAIL || 8 * g + e < a.cols) {
            sw[q][e] += d[q][e] * xh[q][e];
            sh[q][e] += d[q][e];
            d[q][e] *= wt[e];
            m[0] += d[q][e];
            m[1] += d[q][e] * xh[q][e];
          }
        }
      }
    }
    if (!grads) return;
    row_sums<LPR>(m, red, turn, at);
    if (!here) return;
    const float m0 = m[0] / a.cols, m1 = m[1] / a.cols;
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      if (8 * g < a.cols) {
#pragma unroll
        for (int e = 0; e < 8; ++e) d[q][e] = rstd * (d[q][e] - m0 - xh[q][e] * m1);
        if (a.dtotal_in.data) {
          float t[8];
          C::floats(in[q], g, a.cols, t);
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
  walk_rows<roomy(LPR, CPL), Row>(a.rows, at.slot, at.slots, fetch, work);
  if (!sums) return;
  // The row sets of the workgroup in order: into its row of partial sums, or, of the
  // only workgroup, to where they belong.
  const bool only = gridDim.x == 1;
  float* const part = a.work + (long)blockIdx.x * ROWS_MAX_VECTORS * stride;
  __shared__ float set[NT][9];
#pragma unroll
  for (int v = 0; v < 3; ++v) {
    float* const own = v == 0 ? a.dweight : v == 1 ? a.dshift : a.dbias;
    if (!own) continue;
#pragma unroll
    for (int q = 0; q < CPL; ++q) {
      const int g = at.lane + at.lanes * q;
      float(&t)[8] = v == 0 ? sw[q] : v == 1 ? sh[q] : sb[q];
      if (at.slots > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) set[threadIdx.x][e] = t[e];
        __syncthreads();
        for (int i = threadIdx.x; i < 8 * at.lanes; i += blockDim.x) {
          const int c = 8 * at.lanes * q + i;
          float sum = 0.f;
          for (int k = 0; k < at.slots; ++k) sum += set[k * at.lanes + (i >> 3)][i & 7];
          if (only && c < a.cols) own[c] = a.accumulate ? own[c] + sum : sum;
          if (!only && c < stride) part[v * stride + c] = sum;
        }
      } else if (only) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * g + e < a.cols) own[8 * g + e] = a.accumulate ? own[8 * g + e] + t[e] : t[e];
      } else if (8 * g < a.cols) {
#pragma unroll
        for (int e = 0; e < 8; e += 4) *(float4*)(part + v * stride + 8 * g + e) = make_float4(t[e], t[e + 1], t[e + 2], t[e + 3]);
      }
    }
  }
}

template <class E, bool TAIL, template <class, int, int, bool, int> class K, class... A>
hipError_t norm_run(const NormPlan& p, A... args) {
  switch (p.lpr) {
    case 4: return K<E, 4, 1, TAIL, 256>::go(p, args...);
    case 16: return K<E, 16, 1, TAIL, 256>::go(p, args...);
    case 64: return p.cpl == 1 ? K<E, 64, 1, TAIL, 256>::go(p, args...) : K<E, 64, 2, TAIL, 256>::go(p, args...);
    default: break;
  }
  if (p.cpl == 1) return p.threads <= 512 ? K<E, 0, 1, TAIL, 512>::go(p, args...) : K<E, 0, 1, TAIL, 1024>::go(p, args...);
  if (p.threads <= 768) return K<E, 0, 2, TAIL, 768>::go(p, args...);
  return K<E, 0, 2, TAIL, 1024>::go(p, args...);
}

template <class E, int LPR, int CPL, bool TAIL, int NT>
struct NormForward {
  static hipError_t go(const NormPlan& p, const NormArgs* a, hipStream_t s) {
    hipLaunchKernelGGL((norm_fwd_k<E, LPR, CPL, TAIL, NT>), dim3((unsigned)p.groups), dim3(p.threads), 0, s, *a, p.waves);
    return hipGetLastError();
  }
};

template <class E, int LPR, int CPL, bool TAIL, int NT>
struct NormBackward {
  static hipError_t go(const NormPlan& p, const NormArgs* a, hipStream_t s) {
    hipLaunchKernelGGL((norm_bwd_k<E, LPR, CPL, TAIL, NT>), dim3((unsigned)p.groups), dim3(p.threads), 0, s, *a, p.waves,
                       rows_pad(a->cols));
    return hipGetLastError();
  }
};

template <class E>
hipError_t norm_fwd(const NormPlan& p, const NormArgs& a, hipStream_t s) {
  return a.cols % 8 ? norm_run<E, true, NormForward>(p, &a, s) : norm_run<E, false, NormForward>(p, &a, s);
}
template <class E>
hipError_t norm_bwd(const NormPlan& p, const NormArgs& a, hipStream_t s) {
  return a.cols % 8 ? norm_run<E, true, NormBackward>(p, &a, s) : norm_run<E, false, NormBackward>(p, &a, s);
}

}  // namespace
