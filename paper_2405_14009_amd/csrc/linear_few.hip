// The weight's gradient of few tokens: dW = x^T dy as a sum of at most 32 outer
// products, and the bias gradient with it.
//
// Bound by the writing of dW (fp32: 2 n operations of n tokens for 4 bytes).  A
// thread owns four neighbouring columns, holds their values of the right operand
// for every token in registers and walks down FEW_ROWS rows of dW; the left
// operand's values, which a workgroup shares, lie in LDS as fp32.  No matrix
// instructions: a tile kernel multiplies a whole k-tile of tokens whatever their
// number (2 tokens of 8752 x 15760: 332 us fp32 and 146 us bf16 over tiles).  The
// tokens are added in order.
#include <algorithm>

#include "common.h"
#include "linear_few.h"

namespace {

constexpr int NT = 256;

template <class E>
__device__ __forceinline__ void load4(const E* p, float (&f)[4]) {
  if constexpr (sizeof(E) == 2) {
    const uint2 u = *(const uint2*)p;
    f[0] = __uint_as_float(u.x << 16);
    f[1] = __uint_as_float(u.x & 0xffff0000u);
    f[2] = __uint_as_float(u.y << 16);
    f[3] = __uint_as_float(u.y & 0xffff0000u);
  } else {
    const float4 u = *(const float4*)p;
    f[0] = u.x;
    f[1] = u.y;
    f[2] = u.z;
    f[3] = u.w;
  }
}

// T: tokens held (the operands of those that are not there are zeros).  Both
// widths are multiples of 8 (a thread's four columns are there or not).
template <class E, int T>
__global__ __launch_bounds__(NT) void few_tokens_k(FewTokens a) {
  __shared__ float left[T][FEW_ROWS];
  const int i0 = (int)blockIdx.y * FEW_ROWS, rows = min(FEW_ROWS, a.m - i0);
  const int j = ((int)blockIdx.x * NT + (int)threadIdx.x) * 4;
  for (int k = threadIdx.x; k < T * (FEW_ROWS / 4); k += NT) {
    const int t = k / (FEW_ROWS / 4), i = 4 * (k % (FEW_ROWS / 4));
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    if (t < a.tokens && i < rows) load4((const E*)a.left.data + (long)t * a.left.stride + i0 + i, f);
    *(float4*)&left[t][i] = make_float4(f[0], f[1], f[2], f[3]);
  }
  float right[T][4];
#pragma unroll
  for (int t = 0; t < T; ++t) {
#pragma unroll
    for (int e = 0; e < 4; ++e) right[t][e] = 0.f;
    if (t < a.tokens && j < a.n) load4((const E*)a.right.data + (long)t * a.right.stride + j, right[t]);
  }
  __syncthreads();
  // column sums of the operand that is dy, once
  if (a.sums && a.sums_right && blockIdx.y == 0 && j < a.n) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float s = 0.f;
#pragma unroll
      for (int t = 0; t < T; ++t) s += right[t][e];
      a.sums[j + e] = a.accumulate ? a.sums[j + e] + s : s;
    }
  }
  if (a.sums && !a.sums_right && blockIdx.x == 0 && (int)threadIdx.x < rows) {
    float s = 0.f;
#pragma unroll
    for (int t = 0; t < T; ++t) s += left[t][threadIdx.x];
    const int c = i0 + threadIdx.x;
    a.sums[c] = a.accumulate ? a.sums[c] + s : s;
  }
  if (j >= a.n) return;
  float* out = a.out + (long)i0 * a.n + j;
  for (int i = 0; i < rows; i += 4) {   // (rows is a multiple of 8)
    float4 v[4];
    if (a.accumulate) {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *(const float4*)(out + (long)(i + u) * a.n);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float4 s[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const float4 l = *(const float4*)&left[t][i];
      const float ll[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        s[u].x += ll[u] * right[t][0];
        s[u].y += ll[u] * right[t][1];
        s[u].z += ll[u] * right[t][2];
        s[u].w += ll[u] * right[t][3];
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      *(float4*)(out + (long)(i + u) * a.n) = make_float4(v[u].x + s[u].x, v[u].y + s[u].y, v[u].z + s[u].z, v[u].w + s[u].w);
  }
}

template <class E>
hipError_t launch(const FewTokens& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n / 4 + NT - 1) / NT), (unsigned)((a.m + FEW_ROWS - 1) / FEW_ROWS));
  if (a.tokens <= 4) hipLaunchKernelGGL((few_tokens_k<E, 4>), grid, dim3(NT), 0, s, a);
  else if (a.tokens <= 8) hipLaunchKernelGGL((few_tokens_k<E, 8>), grid, dim3(NT), 0, s, a);
  else if constexpr (few_tokens_most(sizeof(E)) > 8) {
    if (a.tokens <= 16) hipLaunchKernelGGL((few_tokens_k<E, 16>), grid, dim3(NT), 0, s, a);
    else hipLaunchKernelGGL((few_tokens_k<E, 32>), grid, dim3(NT), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t few_tokens(const FewTokens& a, int elt, hipStream_t s) {
  if (a.tokens > few_tokens_most(elt) || a.m > FEW_MOST_ROWS) return hipErrorInvalidValue;
  return elt == 2 ? launch<bf16>(a, s) : launch<float>(a, s);
}
