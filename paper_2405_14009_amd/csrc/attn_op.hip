// Host side of the attention operator: scratch memory, buckets, launches; and
// the sum of several calls' bias gradients.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#include "attn_op.h"
#include "common.h"

namespace {

// x^n as 32-bit words, lowest first.
std::vector<uint32_t> power(uint32_t x, int n, std::vector<uint32_t> r = {1}) {
  for (; n > 0; --n) {
    uint64_t carry = 0;
    for (uint32_t& w : r) {
      carry += (uint64_t)w * x;
      w = (uint32_t)carry;
      carry >>= 32;
    }
    if (carry) r.push_back((uint32_t)carry);
  }
  return r;
}

bool at_least(const std::vector<uint32_t>& a, const std::vector<uint32_t>& b) {
  if (a.size() != b.size()) return a.size() > b.size();
  for (size_t i = a.size(); i-- > 0;)
    if (a[i] != b[i]) return a[i] > b[i];
  return true;
}

// First distance of bucket exact + step, of k logarithmic buckets that start at
// `exact` and reach max_distance: the smallest n with
//   n^k >= exact^(k - step) max_distance^step,
// estimated by logarithms, which decide unless n is at the border to their rounding.
int border(int exact, int k, int max_distance, int step) {
  const double t = std::log((double)exact) + (double)step / k * std::log((double)max_distance / exact);
  const double x = std::exp(t);
  const int near = (int)std::lround(x);
  if (std::fabs(x - near) > 1e-6 * x) return (int)std::ceil(x);
  const auto want = power((uint32_t)max_distance, step, power((uint32_t)exact, k - step));
  return at_least(power((uint32_t)near, k), want) ? near : near + 1;
}

__global__ __launch_bounds__(256) void attn_op_add_dbias_k(AttnOpShares shares, int n, long count, float* out,
                                                           int accumulate) {
  const long i = blockIdx.x * 256L + threadIdx.x;
  if (i >= count) return;
  float t = accumulate ? out[i] : 0.f;
  for (int k = 0; k < n; ++k) t += shares.p[k][i];
  out[i] = t;
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

int columns(int d) { return (d + 31) / 32 * 32; }

size_t rows(const AttnOpArgs& a) { return (size_t)a.batch * a.heads * a.spad; }

// Work memory is the same for every form of the grid, so that its size does not
// depend on the device.
int sink_chunks(const AttnOpArgs& a) { return (a.s + a.chunk_len - 1) / a.chunk_len; }
size_t bias_bytes(const AttnOpArgs& a) {
  return align256(4 * (size_t)a.batch * a.heads * ((a.s + 31) / 32) * a.buckets);
}

size_t part_bytes(const AttnOpArgs& a) {
  return a.parts > 1 ? align256(4 * (size_t)a.batch * a.kv_heads * a.parts * 2 * a.part_rows * columns(a.d)) : 0;
}
size_t sink_bytes(const AttnOpArgs& a) {
  return a.sinks ? align256(4 * (size_t)a.batch * a.kv_heads * (1 + sink_chunks(a) * a.parts) * 2 * a.sink_rows *
                            columns(a.d))
                 : 0;
}

}  // namespace

// Fills what follows from the sizes: the window, buckets and the chunks of sink blocks.
void attn_op_plan(AttnOpArgs& a, int elt, int window, int max_distance) {
  const int far = 1 << 30;
  a.spad = (a.s + 63) / 64 * 64;
  a.group = a.heads / a.kv_heads;
  a.sl2 = a.scale * 1.4426950408889634f;
  if (window >= a.s) window = 0;
  a.left = window ? window - 1 : far;
  a.right = a.causal ? 0 : a.left;
  if (!window) a.sinks = 0;
  a.sinks = a.sinks < a.s ? a.sinks : a.s;
  const long seen = window ? (a.causal ? 1L : 2L) * window + a.sinks : a.s;
  a.seen = (int)(seen < a.s ? seen : a.s);
  if (a.buckets) {
    const int side = a.causal ? a.buckets : a.buckets / 2, exact = side / 2, k = side - exact;
    for (int c = 0; c < side; ++c)
      a.first[c] = (unsigned short)(c <= exact ? c : border(exact, k, max_distance, c - exact));
    a.far = a.first[side - 1];
    for (int n = 0, c = 0; n < a.far; ++n) {
      while (c + 1 < side && a.first[c + 1] <= n) ++c;
      a.bucket[n] = (unsigned char)c;
    }
  }
  const long cus = device_compute_units(), blocks = (a.s + 31) / 32 * (long)a.batch;
  a.split_q = elt == 4 || blocks * a.heads <= cus;
  a.split_f = elt == 4 || blocks * a.heads <= 2 * cus;
  a.split_k = elt == 4 || blocks * a.kv_heads <= cus;
  a.sink_rows = (a.sinks + 31) / 32 * 32;
  // (us of dk and dv: fp32, 4 sequences of 955, 16 / 4 heads of 96, window 6, 16 sinks: 185 by chunks
  // of 512, 122 by 128; bf16, 2 sequences of 2048, 16 heads of 128, window 512: 72 and 79)
  a.chunk_len = elt == 4 ? 128 : 512;
  while ((long)a.chunk_len * 64 < a.s) a.chunk_len *= 2;
  // Parts of the heads of a key head: a workgroup visits the queries of all of
  // them, and few workgroups leave compute units empty (256 of them; not the
  // device's number, as the memory depends on it).  us of dk and dv with and without
  // parts, a bias: blocks of 128 keys, 7 sequences of 4128, 4 / 1 heads of 40 (231 blocks):
  // 188, 465; 7 of 1827, 6 / 3 heads of 128 (315): 95, 144; 2 of 4096, 16 / 8 heads
  // of 128 (512): 434, 396.  Blocks of 32, 2 of 512, 8 / 1 heads of 64 (32): 15, 35;
  // 1 of 1024, 32 / 8 heads of 128, window 256 (256): 44, 31; fp32, 1 of 1604,
  // 4 / 1 heads of 96 (51): 103, 365.
  const bool whole = elt == 2 && blocks * a.kv_heads > 256;
  const long keys = whole ? 128 : 32, units = (a.s + keys - 1) / keys * a.batch * a.kv_heads;
  const long most = !whole ? (elt == 4 ? 512 : 256) : units < 384 ? 1024 : units;
  const long span = std::min((long)a.s, (long)a.left + a.right + keys);
  a.parts = span * a.group >= 512 ? (int)std::max(1L, std::min((long)a.group, most / units)) : 1;
  a.part_rows = (a.s + 127) / 128 * 128;
  // No more chunks than 1024 workgroups take: each writes a share of dk and dv of its
  // rows.  (us of dk and dv and their shares' sum, and bytes of work memory, with 16 chunks
  // whatever the sinks and so: 8192 tokens, 32 heads of 128, window 512, 512 sinks:
  // 737 and 0.29 GB, 502 and 0.05; 8000 sinks: 5767 and 4.46 GB, 2080 and 0.53.)
  const long sink_units = (long)a.sink_rows / 32 * a.batch * a.kv_heads * a.parts;
  while (a.chunk_len < a.s && sink_units * sink_chunks(a) > 1024) a.chunk_len *= 2;
  a.chunks = a.sinks && !(a.split_k && a.s <= a.chunk_len) ? sink_chunks(a) : 0;
}

size_t attn_op_saved_bytes(const AttnOpArgs& a, int elt) {
  return 2 * align256(4 * rows(a)) + (elt == 2 ? align256(2 * (size_t)a.batch * a.s * a.heads * a.d) : 0);
}

size_t attn_op_work_bytes(const AttnOpArgs& a) {
  return align256(4 * rows(a)) + bias_bytes(a) + sink_bytes(a) + part_bytes(a);
}

namespace {

void set_saved(AttnOpArgs& a, const void* saved) {
  char* p = (char*)saved;
  a.m = a.l = nullptr;
  a.rest = nullptr;
  if (!p) return;
  a.m = (float*)p;
  a.l = (float*)(p + align256(4 * rows(a)));
  a.rest = p + 2 * align256(4 * rows(a));
}

}  // namespace

hipError_t attn_op_forward(AttnOpArgs a, int elt, void* saved, hipStream_t st) {
  set_saved(a, saved);
  const int c = columns(a.d);
  if (elt == 4)
    return c == 32   ? attn_op_fwd_f32_32(a, st)
           : c == 64 ? attn_op_fwd_f32_64(a, st)
           : c == 96 ? attn_op_fwd_f32_96(a, st)
                     : attn_op_fwd_f32_128(a, st);
  return c == 32   ? attn_op_fwd_bf16_32(a, st)
         : c == 64 ? attn_op_fwd_bf16_64(a, st)
         : c == 96 ? attn_op_fwd_bf16_96(a, st)
                   : attn_op_fwd_bf16_128(a, st);
}

hipError_t attn_op_backward(AttnOpArgs a, int elt, const void* saved, void* work, hipStream_t st) {
  set_saved(a, saved);
  char* w = (char*)work;
  a.drow = (float*)w;
  w += align256(4 * rows(a));
  a.bpart = (float*)w;
  w += bias_bytes(a);
  a.spart = (float*)w;
  w += sink_bytes(a);
  a.gpart = (float*)w;
  const int c = columns(a.d);
  if (elt == 4)
    return c == 32   ? attn_op_bwd_f32_32(a, st)
           : c == 64 ? attn_op_bwd_f32_64(a, st)
           : c == 96 ? attn_op_bwd_f32_96(a, st)
                     : attn_op_bwd_f32_128(a, st);
  return c == 32   ? attn_op_bwd_bf16_32(a, st)
         : c == 64 ? attn_op_bwd_bf16_64(a, st)
         : c == 96 ? attn_op_bwd_bf16_96(a, st)
                   : attn_op_bwd_bf16_128(a, st);
}

hipError_t attn_op_add_dbias(const AttnOpShares& shares, int n, long count, float* out, int accumulate, hipStream_t st) {
  if (n < 1 || n > ATTN_OP_MAX_SHARES) return hipErrorInvalidValue;
  hipLaunchKernelGGL(attn_op_add_dbias_k, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, st, shares, n, count, out,
                     accumulate);
  return hipGetLastError();
}
