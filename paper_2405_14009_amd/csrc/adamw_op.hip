// One AdamW step over many tensors, with fp32 or 8-bit moments.
//
//   g = grad_scale grad;  m' = beta1 m + (1 - beta1) g;  v' = beta2 v + (1 - beta2) g^2
//   p' = p (1 - lr wd [decay]) - lr / (1 - beta1^t) m' / (sqrt(v' / (1 - beta2^t)) + eps)
//
// The work is one pass over the streams (28 bytes an element with fp32
// moments and gradients, 16 with 8-bit ones), so HBM bounds it.  The tensors'
// descriptors travel as kernel arguments, up to MAX of them a launch, and
// workgroups take chunks of elements of any tensor: a set of many small
// tensors is one launch, and no table has to be copied to the device.
//
// 8-bit moments.  Blocks of 128 elements of a tensor share a power of two per
// moment, the smallest with which the block's largest value fits:
//   m: e4m3 codes (largest 448), units of 2^(byte - 127);
//   v: unsigned codes of five exponent and three fraction bits: code c holds
//      c for c < 8 and (8 + c % 8) 2^(c / 8 - 1) otherwise (largest, 254:
//      1.75 2^33), units of 2^(byte - 160).  It spans 2^34 in v, as e4m3 would
//      in sqrt(v), at half of e4m3's error there, and needs no square root.
// Codes round to nearest, ties to even; a v above zero keeps at least the
// smallest code, so that no moment loses its denominator.  A moment that fp32
// does not hold (NaN, infinite) becomes the format's NaN, 0x7f and 255, and
// leaves its block's power of two alone.  Powers of two make every step from
// code to value and back exact but the one rounding, and the moments are
// formed in 64 bits (the vector units have the time: at 16 bytes an element
// HBM allows about 120 vector operations for each), so that the codes are
// those of the formulas and do not depend on how 32-bit sums round.  The
// update itself uses m' and v' before that rounding.
#include <cmath>

#include "adam.h"
#include "adamw_op.h"
#include "common.h"

namespace {

constexpr int NT = 256;
constexpr int MAX = 48;       // tensors a launch: their descriptors fill 3.4 of the 4 KB of arguments
// Elements that a workgroup takes: one turn of its threads, two where the
// moments are only read (us at one / two turns: 8-bit step of 4.0e8 parameters
// with bf16 gradients 1285 / 1395, fp32 step of 1.5e8 784 / 798, reading 8-bit
// moments of 4.0e8 1230 / 890, whose two output streams alternate more coarsely).
constexpr int CHUNK8 = 2048, CHUNK32 = 1024, CHUNK_READ = 4096;

struct Tensor {
  float* p;
  const void* g;
  void *m, *v;
  uint8_t *ms, *vs;
  bf16* copy;
  long n;
  int first;  // its first chunk
  int flags;
};
enum { DECAY = 1, GRAD_BF16 = 2, WIDE = 4 };  // WIDE: every pointer is aligned to its vector accesses

enum { IN_PLACE, BANKS, UNDO };  // where 8-bit moments go: where they were, `to` bytes on, nowhere

struct Args {
  AdamwHyper h;
  long to;
  int n;
  Tensor t[MAX];
};

// 8 bytes, streamed past the caches as the fp32 arrays are (adam.h).
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void load8_nt(void* to, const void* from) {
  *(u32x2*)to = __builtin_nontemporal_load((const u32x2*)from);
}
__device__ __forceinline__ void store8_nt(void* to, const void* from) {
  __builtin_nontemporal_store(*(const u32x2*)from, (u32x2*)to);
}

// N consecutive elements at i of a tensor, and their stores; scalar at its end
// or where the pointers are not aligned.
template <int N>
__device__ __forceinline__ void load_f32(float (&x)[N], const float* p, long i, int left, bool wide) {
  if (wide) {
#pragma unroll
    for (int k = 0; k < N; k += 4) {
      const float4 v = ld_nt((const float4*)(p + i + k));
      x[k] = v.x;
      x[k + 1] = v.y;
      x[k + 2] = v.z;
      x[k + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = k < left ? p[i + k] : 0.f;
  }
}
template <int N>
__device__ __forceinline__ void store_f32(const float (&x)[N], float* p, long i, int left, bool wide) {
  if (wide) {
#pragma unroll
    for (int k = 0; k < N; k += 4) st_nt((float4*)(p + i + k), make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]));
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < left) p[i + k] = x[k];
  }
}
template <int N>
__device__ __forceinline__ void load_grad(float (&x)[N], const Tensor& t, long i, int left, bool wide) {
  if (!(t.flags & GRAD_BF16)) return load_f32<N>(x, (const float*)t.g, i, left, wide);
  const bf16* g = (const bf16*)t.g;
  if (wide) {
    bf16 b[N];
#pragma unroll
    for (int k = 0; k < N; k += 4) load8_nt(b + k, g + i + k);
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = (float)b[k];
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = k < left ? (float)g[i + k] : 0.f;
  }
}
template <int N>
__device__ __forceinline__ void store_copy(const float (&x)[N], const Tensor& t, long i, int left, bool wide) {
  if (!t.copy) return;
  if (wide) {
#pragma unroll
    for (int k = 0; k < N; k += 4) store_bf16x4(t.copy + i + k, make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]));
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < left) t.copy[i + k] = (bf16)x[k];
  }
}

// Largest of 16 consecutive lanes, in all of them.
__device__ __forceinline__ int max16(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0xB1, 0xf, 0xf, false));   // lane ^ 1
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x4E, 0xf, 0xf, false));   // lane ^ 2
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x141, 0xf, 0xf, false));  // 7 - lane of 8
  return max(x, __builtin_amdgcn_update_dpp(x, x, 0x140, 0xf, 0xf, false));  // 15 - lane of 16
}

__device__ __forceinline__ bool fits(double x) { return fabs(x) <= 3.4028234663852886e38; }

// Smallest e with |x| <= 1.75 2^(e + most); far below every exponent for zero.
__device__ __forceinline__ int exponent_for(double x, int most) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x) & 0x7fffffffffffffffull;
  const int e = (int)(b >> 52) - 1023 - most + ((b & 0xfffffffffffffull) > 0xc000000000000ull);
  return b && fits(x) ? e : -100000;
}

// x 2^-e as fp32, rounded to odd: the low bit also stands for what is cut off, so
// that a further rounding to few bits is that of x.  (Values below 2^-126 become
// a number below every code.)
__device__ __forceinline__ float scaled_odd(double x, int e) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t hi = (uint32_t)(b >> 32), lo = (uint32_t)b;
  const int exp = (int)((hi >> 20) & 0x7ff) - 1023 - e;
  uint32_t f = (uint32_t)(exp + 127) << 23 | (hi & 0xfffff) << 3 | lo >> 29 | ((lo & 0x1fffffff) != 0);
  if (exp < -126) f = (hi << 1 | lo) != 0 ? 0x00800000u : 0u;
  return __uint_as_float(f | (hi & 0x80000000u));
}

__device__ __forceinline__ double power_of_two(int e) {
  return __builtin_bit_cast(double, (uint64_t)(e + 1023) << 52);
}

__device__ __forceinline__ int encode_v(float x) {
  const uint32_t b = __float_as_uint(x);
  const int high = (int)((b + 0x7ffff + ((b >> 20) & 1)) >> 20) - (129 << 3);
  const int c = x < 8.f ? (int)rintf(x) : high;
  return x > 0.f && c == 0 ? 1 : c;
}
__device__ __forceinline__ double decode_v(int c, double unit) {
  const int e = c >> 3, f = c & 7;
  const double x = e ? (double)(8 + f) * power_of_two(e - 1) : (double)f;
  return c == 255 ? __builtin_nan("") : x * unit;
}

// A thread takes 8 elements, 16 lanes a block of 128.
template <int MODE>
__device__ __forceinline__ void step8(const Tensor& t, const AdamwHyper& h, long i, long to) {
  const long left_l = t.n - i;
  const int left = left_l < 8 ? (left_l > 0 ? (int)left_l : 0) : 8;
  const bool wide = (t.flags & WIDE) && left == 8;
  float p[8], g[8];
  load_f32<8>(p, t.p, i, left, wide);
  load_grad<8>(g, t, i, left, wide);
  const uint8_t* const mc = (const uint8_t*)t.m + i;
  const uint8_t* const vc = (const uint8_t*)t.v + i;
  uint32_t mw[2] = {0, 0}, vw[2] = {0, 0};
  if (wide) {
    load8_nt(mw, mc);
    load8_nt(vw, vc);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) {
        mw[k >> 2] |= (uint32_t)mc[k] << (8 * (k & 3));
        vw[k >> 2] |= (uint32_t)vc[k] << (8 * (k & 3));
      }
  }
  const long blk = i / ADAMW_BLOCK;
  const double mu = left ? power_of_two((int)t.ms[blk] - 127) : 0.0;
  const double vu = left ? power_of_two((int)t.vs[blk] - 160) : 0.0;
  double m[8], v[8];
  int em = -100000, ev = -100000;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int word = mw[k >> 2];
    const float mf = (k & 3) == 0   ? __builtin_amdgcn_cvt_f32_fp8(word, 0)
                     : (k & 3) == 1 ? __builtin_amdgcn_cvt_f32_fp8(word, 1)
                     : (k & 3) == 2 ? __builtin_amdgcn_cvt_f32_fp8(word, 2)
                                    : __builtin_amdgcn_cvt_f32_fp8(word, 3);
    const double gd = (double)g[k] * h.grad_scale;
    m[k] = h.beta1 * ((double)mf * mu) + (1.0 - h.beta1) * gd;
    v[k] = h.beta2 * decode_v((vw[k >> 2] >> (8 * (k & 3))) & 255, vu) + (1.0 - h.beta2) * gd * gd;
    if (k < left) {
      em = max(em, exponent_for(m[k], 8));
      ev = max(ev, exponent_for(v[k], 33));
    }
  }
  em = max16(em);
  ev = max16(ev);
  // a block of zeros: byte 0
  em = max(em, -127);
  ev = max(ev, -160);
  if (!left) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float u = adam_update((float)m[k], (float)v[k], h.eps, h.step_size, h.inv_sqrt_bc2);
    const float shrink = 1.f - h.lr * h.weight_decay;
    if constexpr (MODE == UNDO) {
      p[k] += u;
      if (t.flags & DECAY) p[k] /= shrink;
    } else {
      if (t.flags & DECAY) p[k] *= shrink;
      p[k] -= u;
    }
  }
  store_f32<8>(p, t.p, i, left, wide);
  store_copy<8>(p, t, i, left, wide);
  if constexpr (MODE == UNDO) return;
  mw[0] = mw[1] = vw[0] = vw[1] = 0;
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    const bool a = fits(m[k]), b = fits(m[k + 1]);
    int two = __builtin_amdgcn_cvt_pk_fp8_f32(a ? scaled_odd(m[k], em) : 0.f, b ? scaled_odd(m[k + 1], em) : 0.f, 0, false);
    two = (two & 0xffff) | (a ? 0 : 0x7f) | (b ? 0 : 0x7f00);
    mw[k >> 2] |= (uint32_t)two << (8 * (k & 3));
    const int c0 = fits(v[k]) ? encode_v(scaled_odd(v[k], ev)) : 255;
    const int c1 = fits(v[k + 1]) ? encode_v(scaled_odd(v[k + 1], ev)) : 255;
    vw[k >> 2] |= (uint32_t)(c0 | c1 << 8) << (8 * (k & 3));
  }
  uint8_t* const mo = (uint8_t*)t.m + i + (MODE == BANKS ? to : 0);
  uint8_t* const vo = (uint8_t*)t.v + i + (MODE == BANKS ? to : 0);
  if (wide) {
    store8_nt(mo, mw);
    store8_nt(vo, vw);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) {
        mo[k] = (uint8_t)(mw[k >> 2] >> (8 * (k & 3)));
        vo[k] = (uint8_t)(vw[k >> 2] >> (8 * (k & 3)));
      }
  }
  if (i % ADAMW_BLOCK == 0) {
    t.ms[blk + (MODE == BANKS ? to : 0)] = (uint8_t)(em + 127);
    t.vs[blk + (MODE == BANKS ? to : 0)] = (uint8_t)(ev + 160);
  }
}

__device__ __forceinline__ void step32(const Tensor& t, const AdamwHyper& h, long i) {
  const long left_l = t.n - i;
  if (left_l <= 0) return;
  const int left = left_l < 4 ? (int)left_l : 4;
  const bool wide = (t.flags & WIDE) && left == 4;
  float p[4], g[4], m[4], v[4];
  load_f32<4>(p, t.p, i, left, wide);
  load_grad<4>(g, t, i, left, wide);
  load_f32<4>(m, (const float*)t.m, i, left, wide);
  load_f32<4>(v, (const float*)t.v, i, left, wide);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    p[k] = adam_one(p[k], g[k], m[k], v[k], t.flags & DECAY, h.lr, (float)h.beta1, (float)h.beta2, h.eps,
                    h.weight_decay, h.step_size, h.inv_sqrt_bc2, (float)h.grad_scale);
  store_f32<4>(p, t.p, i, left, wide);
  store_f32<4>(m, (float*)t.m, i, left, wide);
  store_f32<4>(v, (float*)t.v, i, left, wide);
  store_copy<4>(p, t, i, left, wide);
}

// The tensor of chunk c: the last one whose first chunk is not after it.
__device__ __forceinline__ const Tensor& tensor_of(const Args& a, int c) {
  int lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].first <= c)
      lo = mid;
    else
      hi = mid - 1;
  }
  return a.t[lo];
}

template <int BITS, int MODE>
__global__ __launch_bounds__(NT) void adamw_tensors_k(Args a) {
  const Tensor& t = tensor_of(a, blockIdx.x);
  constexpr int N = BITS == 8 ? 8 : 4, CHUNK = BITS == 8 ? CHUNK8 : CHUNK32;
  const long at = (long)((int)blockIdx.x - t.first) * CHUNK;
  for (int k = 0; k < CHUNK; k += NT * N) {
    const long i = at + k + (long)threadIdx.x * N;
    if constexpr (BITS == 8)
      step8<MODE>(t, a.h, i, a.to);
    else
      step32(t, a.h, i);
  }
}

// Moments as values: m and v of a tensor into p and g of its descriptor.
template <int BITS>
__global__ __launch_bounds__(NT) void adamw_read_k(Args a) {
  const Tensor& t = tensor_of(a, blockIdx.x);
  const long at = (long)((int)blockIdx.x - t.first) * CHUNK_READ;
  for (int k = 0; k < CHUNK_READ; k += NT * 8) {
    const long i = at + k + (long)threadIdx.x * 8, left_l = t.n - i;
    if (left_l <= 0) return;
    const int left = left_l < 8 ? (int)left_l : 8;
    const bool wide = (t.flags & WIDE) && left == 8;
    float m[8], v[8];
    if constexpr (BITS == 32) {
      load_f32<8>(m, (const float*)t.m, i, left, wide);
      load_f32<8>(v, (const float*)t.v, i, left, wide);
    } else {
      uint8_t mc[8], vc[8];
      if (wide) {
        *(uint2*)mc = *(const uint2*)((const uint8_t*)t.m + i);
        *(uint2*)vc = *(const uint2*)((const uint8_t*)t.v + i);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          mc[j] = j < left ? ((const uint8_t*)t.m)[i + j] : 0;
          vc[j] = j < left ? ((const uint8_t*)t.v)[i + j] : 0;
        }
      }
      const double mu = power_of_two((int)t.ms[i / ADAMW_BLOCK] - 127);
      const double vu = power_of_two((int)t.vs[i / ADAMW_BLOCK] - 160);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = (float)((double)__builtin_amdgcn_cvt_f32_fp8(mc[j], 0) * mu);
        v[j] = (float)decode_v(vc[j], vu);
      }
    }
    store_f32<8>(m, t.p, i, left, wide);
    store_f32<8>(v, (float*)t.g, i, left, wide);
  }
}

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// launch(args, chunks) for groups of up to MAX of the tensors, whose descriptors set(tensor, i) makes.
template <class Set, class Launch>
hipError_t in_groups(const rc_adamw_tensor* ts, int n, int chunk, Args& a, Set set, Launch launch) {
  for (int at = 0; at < n;) {
    long chunks = 0;
    a.n = 0;
    for (; at < n && a.n < MAX; ++at) {
      if (ts[at].count == 0) continue;
      const long own = (ts[at].count + chunk - 1) / chunk;
      if (a.n && chunks + own > ADAMW_MAX_GROUPS) break;
      Tensor& t = a.t[a.n++];
      t = set(ts[at], at);
      t.n = ts[at].count;
      t.first = (int)chunks;
      chunks += own;
    }
    if (!a.n) break;
    launch(dim3((unsigned)chunks));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

Tensor step_tensor(const rc_adamw_tensor& x, int bits) {
  const size_t moment = bits == 8 ? 8 : 16;
  const bool wide = aligned(x.param, 16) && aligned(x.grad, x.grad_dtype == RC_BF16 ? 8 : 16) &&
                    aligned(x.exp_avg, moment) && aligned(x.exp_avg_sq, moment) && aligned(x.copy, 8);
  Tensor t = {x.param, x.grad, x.exp_avg, x.exp_avg_sq, x.exp_avg_scale, x.exp_avg_sq_scale, (bf16*)x.copy, 0, 0, 0};
  t.flags = (x.decay ? DECAY : 0) | (x.grad_dtype == RC_BF16 ? GRAD_BF16 : 0) | (wide ? WIDE : 0);
  return t;
}

}  // namespace

AdamwHyper adamw_hyper(const rc_adam_config& a, int64_t step, float grad_scale) {
  AdamwHyper h;
  h.beta1 = a.beta1;
  h.beta2 = a.beta2;
  h.grad_scale = grad_scale;
  h.lr = a.lr;
  h.weight_decay = a.weight_decay;
  h.eps = a.eps;
  h.step_size = (float)(a.lr / (1.0 - std::pow(h.beta1, (double)step)));
  h.inv_sqrt_bc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(h.beta2, (double)step)));
  return h;
}

hipError_t adamw_tensors(const rc_adamw_tensor* ts, int n, int bits, const AdamwHyper& h, hipStream_t s) {
  Args a;
  a.h = h;
  a.to = 0;
  return in_groups(
      ts, n, bits == 8 ? CHUNK8 : CHUNK32, a, [&](const rc_adamw_tensor& x, int) { return step_tensor(x, bits); },
      [&](dim3 grid) {
        if (bits == 8)
          hipLaunchKernelGGL((adamw_tensors_k<8, IN_PLACE>), grid, dim3(NT), 0, s, a);
        else
          hipLaunchKernelGGL((adamw_tensors_k<32, IN_PLACE>), grid, dim3(NT), 0, s, a);
      });
}

hipError_t adamw_banks(const rc_adamw_tensor* ts, int n, const AdamwHyper& h, long to, bool undo, hipStream_t s) {
  Args a;
  a.h = h;
  a.to = to;
  return in_groups(
      ts, n, CHUNK8, a, [&](const rc_adamw_tensor& x, int) { return step_tensor(x, 8); },
      [&](dim3 grid) {
        if (undo)
          hipLaunchKernelGGL((adamw_tensors_k<8, UNDO>), grid, dim3(NT), 0, s, a);
        else
          hipLaunchKernelGGL((adamw_tensors_k<8, BANKS>), grid, dim3(NT), 0, s, a);
      });
}

hipError_t adamw_read(const rc_adamw_tensor* ts, int n, int bits, float* const* m, float* const* v, hipStream_t s) {
  Args a;
  a.h = {};
  a.to = 0;
  return in_groups(
      ts, n, CHUNK_READ, a,
      [&](const rc_adamw_tensor& x, int i) {
        const size_t moment = bits == 8 ? 8 : 16;
        const bool wide = aligned(m[i], 16) && aligned(v[i], 16) && aligned(x.exp_avg, moment) &&
                          aligned(x.exp_avg_sq, moment);
        return Tensor{m[i], v[i], x.exp_avg, x.exp_avg_sq, x.exp_avg_scale, x.exp_avg_sq_scale, nullptr, 0, 0,
                      wide ? WIDE : 0};
      },
      [&](dim3 grid) {
        if (bits == 8)
          hipLaunchKernelGGL(adamw_read_k<8>, grid, dim3(NT), 0, s, a);
        else
          hipLaunchKernelGGL(adamw_read_k<32>, grid, dim3(NT), 0, s, a);
      });
}

float adamw_decode_m(int code, int scale) {
  const int e = (code >> 3) & 15, f = code & 7;
  if ((code & 127) == 127) return NAN;
  const float x = e ? std::ldexp((float)(8 + f), e - 10) : std::ldexp((float)f, -9);
  return std::ldexp(code & 128 ? -x : x, scale - 127);
}

float adamw_decode_v(int code, int scale) {
  if (code == 255) return NAN;
  const double x = code < 8 ? code : std::ldexp((double)(8 + (code & 7)), (code >> 3) - 1);
  return (float)std::ldexp(x, scale - 160);
}
