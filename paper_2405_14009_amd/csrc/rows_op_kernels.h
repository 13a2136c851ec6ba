// Device helpers of the operators over rows: groups of eight columns, and the
// numbers that decide which of them dropout keeps.
#pragma once

#include "common.h"
#include "rows_op.h"

namespace {

// Eight elements as they are in memory.
template <class E>
struct Raw8 {
  uint4 v[sizeof(E) / 2];
};

__device__ __forceinline__ void to_floats(const Raw8<bf16>& r, float (&f)[8]) { unpack(r.v[0], (const bf16*)nullptr, f); }
__device__ __forceinline__ void to_floats(const Raw8<float>& r, float (&f)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f[4 * h] = __uint_as_float(r.v[h].x);
    f[4 * h + 1] = __uint_as_float(r.v[h].y);
    f[4 * h + 2] = __uint_as_float(r.v[h].z);
    f[4 * h + 3] = __uint_as_float(r.v[h].w);
  }
}

// Columns of a row in groups of eight.  Rows may start at any element: gfx950
// loads 16 bytes from any address.  TAIL: cols is no multiple of 8; the last
// group then is loaded eight columns before the row's end and moved down (so that
// all lanes of a wave run the same loads), or, in rows of fewer than eight
// columns, element by element; what lies behind the row is zero.
template <class E, bool TAIL>
struct Columns {
  __device__ __forceinline__ static Raw8<E> load(const E* row, int group, int cols) {
    Raw8<E> r;
    uint32_t c = 8u * (uint32_t)group;   // (32 bits, unsigned: a lane's offset from its row's address)
    if constexpr (TAIL) {
      if (cols < 8) {
        E t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = (int)c + e < cols ? row[c + e] : (E)0.f;
        __builtin_memcpy(&r, t, sizeof(r));
        return r;
      }
      c = min(c, (uint32_t)cols - 8u);
    }
    __builtin_memcpy(&r, (const char*)row + c * (uint32_t)sizeof(E), sizeof(r));
    return r;
  }
  // the loaded group as numbers
  __device__ __forceinline__ static void floats(const Raw8<E>& r, int group, int cols, float (&f)[8]) {
    to_floats(r, f);
    if constexpr (TAIL) {
      const int by = cols < 8 ? 0 : max(0, 8 * group + 8 - cols);
#pragma unroll
      for (int b = 4; b > 0; b >>= 1)
        if (by & b) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = e + b < 8 ? f[e + b] : 0.f;
        }
    }
  }
  __device__ __forceinline__ static void store(E* row, int group, int cols, const float (&f)[8]) {
    E t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = from_f32<E>(f[e]);
    if (!TAIL || 8 * group + 8 <= cols) {
      __builtin_memcpy((char*)row + 8u * (uint32_t)group * (uint32_t)sizeof(E), t, sizeof(t));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * group + e < cols) row[8 * group + e] = t[e];
    }
  }
};

// Eight values of a vector of parameters (fp32 or bf16), as loaded.
struct RawParams {
  uint4 v[2];
};
template <bool TAIL>
__device__ __forceinline__ RawParams load_params(const void* p, int f32, int group, int cols) {
  RawParams r;
  if (f32) {
    const Raw8<float> t = Columns<float, TAIL>::load((const float*)p, group, cols);
    r.v[0] = t.v[0];
    r.v[1] = t.v[1];
  } else {
    r.v[0] = r.v[1] = Columns<bf16, TAIL>::load((const bf16*)p, group, cols).v[0];
  }
  return r;
}
template <bool TAIL>
__device__ __forceinline__ void param_floats(const RawParams& r, int f32, int group, int cols, float (&f)[8]) {
  if (f32) {
    Raw8<float> t;
    t.v[0] = r.v[0];
    t.v[1] = r.v[1];
    Columns<float, TAIL>::floats(t, group, cols, f);
  } else {
    Raw8<bf16> t;
    t.v[0] = r.v[0];
    Columns<bf16, TAIL>::floats(t, group, cols, f);
  }
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", SC 2011): ten rounds of two 32 x 32-bit products over a counter of
// four words, here (group of columns, row, offset), under a key of two, the seed.
// One counter serves eight elements with 16 bits each (p is held to 2^-16), so an
// element costs about 10 integer operations.  Nothing is stored: the backward
// pass forms the same numbers again.
struct Philox {
  uint32_t k0, k1, c2, c3;
  __device__ __forceinline__ void init(const DropArgs& d) {
    uint64_t o = d.offset;
    if (d.step) o += *d.step;
    k0 = (uint32_t)d.seed;
    k1 = (uint32_t)(d.seed >> 32);
    c2 = (uint32_t)o;
    c3 = (uint32_t)(o >> 32);
  }
  // (one operation; 0x96 is the truth table of a ^ b ^ c)
  __device__ __forceinline__ static uint32_t xor3(uint32_t x, uint32_t y, uint32_t z) {
    return __builtin_amdgcn_bitop3_b32(x, y, z, 0x96);
  }
  __device__ __forceinline__ void words(uint32_t group, uint32_t row, uint32_t (&w)[4]) const {
    uint32_t x0 = group, x1 = row, x2 = c2, x3 = c3, a = k0, b = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t p = (uint64_t)x0 * 0xD2511F53u, q = (uint64_t)x2 * 0xCD9E8D57u;
      x0 = xor3((uint32_t)(q >> 32), x1, a);
      x1 = (uint32_t)q;
      x2 = xor3((uint32_t)(p >> 32), x3, b);
      x3 = (uint32_t)p;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
    w[0] = x0;
    w[1] = x1;
    w[2] = x2;
    w[3] = x3;
  }
};

// f = D(f) of one group of a row (dropped elements are 0 whatever they held).
__device__ __forceinline__ void drop8(const Philox& g, const DropArgs& d, int group, long row, float (&f)[8]) {
  uint32_t w[4];
  g.words((uint32_t)group, (uint32_t)row, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t n = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
    f[e] = n >= d.threshold ? f[e] * d.scale : 0.f;
  }
}

}  // namespace
